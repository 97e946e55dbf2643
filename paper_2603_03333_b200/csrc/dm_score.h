// Host-side declarations of the tensor-core score kernel (dm_score_sm100.cu), shared with the C ABI.
#pragma once
#include "dm_rows.cuh"

namespace dm {

struct ScoreWorkspace { size_t off_tok, off_max, off_logits, bytes; };
constexpr int kScoreChunk = 512;   // hidden rows of one launch, and rows whose logits exist at a time

// Layout of the workspace for up to `rows` hidden rows per launch.
ScoreWorkspace score_workspace(const SliceGeometry& geo, int rows, bool alternatives);

// rp: rows (at most kScoreChunk), tokens, n_top, temperature and outputs of dropmatch_logprobs.
int launch_score(const FusedState* fs, const HeadDesc& head, const void* H, const RowsParams& rp, unsigned char* ws, uint32_t* err,
                 long long wait_limit, bool allow_pdl, cudaStream_t stream);

}  // namespace dm
