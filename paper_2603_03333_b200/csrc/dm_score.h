// Host-side declarations of the tensor-core score kernel (dm_score_sm100.cu), shared with the C ABI.
#pragma once
#include "dm_rows.cuh"

namespace dm {

constexpr int kScoreChunk = 512;   // hidden rows of one launch, and rows whose logits exist at a time

struct ScoreState;                 // how the vocabulary is cut, and the tensor maps of W
int score_create(ScoreState** out, const HeadDesc& head);   // bf16 heads of the tensor-core kernels
void score_destroy(ScoreState* st);
size_t score_workspace_bytes(const ScoreState* st, int rows, bool alternatives);   // for up to `rows` rows per launch

// rp: rows (at most kScoreChunk), tokens, n_top, temperature and outputs of dropmatch_logprobs.
int launch_score(const ScoreState* st, const HeadDesc& head, const void* H, const RowsParams& rp, unsigned char* ws, uint32_t* err,
                 long long wait_limit, bool allow_pdl, cudaStream_t stream);

}  // namespace dm
