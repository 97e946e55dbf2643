// dropmatch_score on bf16 heads: l = H W^T on tcgen05 tensor cores, and of every row of l the
// log-sum-exp, the entropy, the given token's logit and the largest entries, without a second pass
// over the vocabulary.
//
//   z = l / T;  lse = log sum exp z;  log p(tok) = z[tok] - lse;  entropy = -sum p log p
//
// score_head_kernel.  The vocabulary is cut as in the verify kernel (one slice per CTA, equal tiles
// of at most 128 vocabulary rows, CTA pairs); a W tile is the M operand, the hidden rows are the N
// operand, up to two blocks of 256 of them against one W tile: W crosses the HBM interface once per
// 512 hidden rows, and of the bytes a CTA pair loads per step only half (one block) or two thirds
// (two blocks) are hidden rows.  Hidden rows come straight from the caller's array through a tensor
// map made for the call; rows past its end load as zeros.  Bounds: W from HBM up to some 200 rows,
// the tensor pipe above.
//
// Epilogue.  32 accumulator lanes (vocabulary rows) x 16 columns (hidden rows) at a time: the
// maximum of the 32, the sum of 2^((l - max) c) over the others (c = log2(e) / T) and the same times
// the exponent, each column reduced over the lanes by a halving exchange (16 exchanges for 16
// columns).  A warp merges its tiles into one record (maximum, rest, weighted sum) per column in
// shared memory; "rest" leaves the largest entry out, so that log(1 + rest) keeps its precision.
// If alternatives are asked for, the 32 logits and their maximum also go to global memory.
//
// score_finish_kernel.  One block per hidden row merges the records of all CTAs.  Alternatives: the
// k-th largest of the threads' maxima over the maxima of the groups of 32 is a lower bound on the
// k-th largest logit; only groups that reach it are read (about k of 4000).
#include <new>

#include "dm_internal.h"
#include "dm_ptx.cuh"
#include "dm_score.h"

namespace dm {

namespace {

constexpr int kThreads = 10 * 32;           // warp 0 TMA, warp 1 MMA, warps 2-9 epilogue
constexpr int kFirstEpiWarp = 2, kEpiWarps = 8;
constexpr int kBlockK = 64;                 // hidden-size elements per step (128 bytes of bf16)
constexpr int kTileM = 128;
constexpr int kWStageBytes = kTileM * kBlockK * 2;
constexpr int kTmemCols = 512;
constexpr int kMaxSteps = 12;
constexpr int kMaxBlock = 256;              // hidden rows of one MMA (UMMA N)
constexpr int kBarBytes = 512;
constexpr int kSmemLimit = 227 * 1024;
constexpr long long kWaitLimitCycles = 2000000000ll;
constexpr int kPollNs = 32, kIdlePollNs = 500;
constexpr float kFloorExp = -200.0f;
constexpr float kLn2 = 0.693147180559945309f;

struct ScoreParams {
    int d, V, rows;
    int kb_count, tiles_per_cta, tile_rows, slice_rows;
    int n_pad, n_blk, cols;      // hidden rows of a block (multiple of 32), blocks, accumulator columns of a tile
    int n_slots, n_steps;        // accumulator slots in TMEM; stages of the ring
    uint32_t step_bytes, b_bytes;   // bytes of a stage, and of one block's half of the hidden rows
    int pdl;
    long long wait_limit;
    float c;                     // log2(e) / T
    const int32_t* tokens;       // [rows] or null
    float* tok_logit;            // [rows]
    float4* records;             // [4 * CTAs][rows]
    float* group_max;            // [rows][groups] or null: no alternatives
    float* logits;               // [rows][groups][32]
    int n_groups;                // 4 * tiles_per_cta * CTAs
    uint32_t* err;
    uint32_t off_rec, off_tok, off_max, off_bar;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xFF800000u); }

struct Record { float m, rest, t; };   // maximum; sums over everything else (see dm_rows.cu)

__device__ __forceinline__ Record merge(const Record& a, const Record& b, float c) {
    const bool a_up = a.m >= b.m;
    const float m = a_up ? a.m : b.m, lo = a_up ? b.m : a.m;
    Record r{m, a_up ? a.rest : b.rest, a_up ? a.t : b.t};
    if (lo == neg_inf()) return r;
    const float d = fmaxf((lo - m) * c, kFloorExp), f = ex2(d);
    const float all = (a_up ? b.rest : a.rest) + 1.0f, t = a_up ? b.t : a.t;
    r.rest = fmaf(f, all, r.rest);
    r.t = fmaf(f, fmaf(d, all, t), r.t);
    return r;
}

// Reduce 16 columns over 32 lanes in 16 exchanges: each round hands half of the columns to the partner
// and keeps the other half; lanes 2x and 2x + 1 end up with column x.
template <typename Op>
__device__ __forceinline__ float halving16(const float (&x)[16], int lane, Op op) {
    float a[8], b[4], e[2], y;
    {
        const bool up = (lane & 16) != 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float give = up ? x[j] : x[j + 8], keep = up ? x[j + 8] : x[j];
            a[j] = op(keep, __shfl_xor_sync(0xFFFFFFFFu, give, 16));
        }
    }
    {
        const bool up = (lane & 8) != 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float give = up ? a[j] : a[j + 4], keep = up ? a[j + 4] : a[j];
            b[j] = op(keep, __shfl_xor_sync(0xFFFFFFFFu, give, 8));
        }
    }
    {
        const bool up = (lane & 4) != 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float give = up ? b[j] : b[j + 2], keep = up ? b[j + 2] : b[j];
            e[j] = op(keep, __shfl_xor_sync(0xFFFFFFFFu, give, 4));
        }
    }
    {
        const bool up = (lane & 2) != 0;
        const float give = up ? e[0] : e[1], keep = up ? e[1] : e[0];
        y = op(keep, __shfl_xor_sync(0xFFFFFFFFu, give, 2));
    }
    return op(y, __shfl_xor_sync(0xFFFFFFFFu, y, 1));
}
struct MaxOp { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct SumOp { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };

__global__ void __launch_bounds__(kThreads, 1)
score_head_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_h,
                  const ScoreParams P) {
    extern __shared__ unsigned char smem_dyn[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(
        (reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t smem_base = ptx::smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float* s_rec = reinterpret_cast<float*>(smem + P.off_rec);       // [3][4][cols]: maximum, rest, weighted sum
    int32_t* s_tok = reinterpret_cast<int32_t*>(smem + P.off_tok);   // [cols]
    float* s_max = reinterpret_cast<float*>(smem + P.off_max);       // [8 warps][16]
    uint64_t* s_bar = reinterpret_cast<uint64_t*>(smem + P.off_bar);
    // barriers: full[n_steps] empty[n_steps] acc_full[n_slots] acc_empty[n_slots] dealloc
    const uint32_t full = smem_base + P.off_bar, empty = full + 8 * P.n_steps;
    const uint32_t acc_full = empty + 8 * P.n_steps, acc_empty = acc_full + 8 * P.n_slots;
    const uint32_t dealloc_bar = acc_empty + 8 * P.n_slots;
    const int n_bars = 2 * P.n_steps + 2 * P.n_slots + 1;
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_bar + n_bars);
    volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
    volatile int* s_never = reinterpret_cast<volatile int*>(s_tmem + 2);
    const uint32_t rank = ptx::cluster_ctarank();

    if (threadIdx.x == 0) {
        ptx::prefetch_tensormap(&tmap_w);
        ptx::prefetch_tensormap(&tmap_h);
        for (int s = 0; s < P.n_steps; ++s) { ptx::mbar_init(full + 8 * s, 1); ptx::mbar_init(empty + 8 * s, 1); }
        for (int s = 0; s < P.n_slots; ++s) { ptx::mbar_init(acc_full + 8 * s, 1); ptx::mbar_init(acc_empty + 8 * s, 2 * kEpiWarps); }
        ptx::mbar_init(dealloc_bar, 1);
        *s_abort = 0;
        *s_never = 0;
        ptx::fence_mbar_init();
        ptx::fence_proxy_async_smem();
    }
    if (warp == kFirstEpiWarp) {
        ptx::tmem_alloc_pair(ptx::smem_u32(s_tmem), kTmemCols);
        ptx::tmem_relinquish_pair();
    }
    for (int i = threadIdx.x; i < 4 * P.cols; i += kThreads) s_rec[i] = neg_inf();
    for (int i = threadIdx.x; i < 8 * P.cols; i += kThreads) s_rec[4 * P.cols + i] = 0.0f;
    ptx::tc_fence_before();
    __syncthreads();
    ptx::cluster_sync_all();   // the other CTA's barriers are initialised before anyone signals them
    ptx::tc_fence_after();
    const uint32_t tmem_base = *s_tmem;
    if (P.pdl) ptx::griddep_launch_dependents();

    const int slice = (int)blockIdx.x, v_cta0 = slice * P.slice_rows;
    const int n_tiles = P.tiles_per_cta;   // both CTAs of a pair; rows past the end of W load as zeros and are never taken
    const uint32_t off_b = kWStageBytes;

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        if (lane != 0) return;
        const uint32_t step_tx = 2u * ((uint32_t)P.tile_rows * (kBlockK * 2) + (uint32_t)P.n_blk * P.b_bytes);   // both CTAs
        const uint64_t w_policy = ptx::l2_policy_evict_first();
        const int b_row0 = (int)rank * (P.n_pad / 2);
        const int total = n_tiles * P.kb_count;
        // W does not depend on the kernel ahead, the hidden rows may: the ring is first filled with W tiles
        const int ahead = P.pdl ? min(P.n_steps, total) : 0;
        int x = 0, v = v_cta0;
        for (int n = 0; n < ahead; ++n) {
            const uint32_t bar = full + 8 * n;
            if (rank == 0) ptx::mbar_arrive_expect_tx(bar, step_tx);
            ptx::tma_load_2d_pair_hint(smem_base + (uint32_t)n * P.step_bytes, &tmap_w, x, v, ptx::map_to_cta(bar, 0), w_policy);
            x += kBlockK;
            if (x == P.d) { x = 0; v += P.tile_rows; }
        }
        if (P.pdl) ptx::griddep_wait();
        x = 0;
        v = v_cta0;
        int stage = 0;
        uint32_t parity = 1, bar = full, bar_e = empty, dst = smem_base;
        for (int n = 0; n < total; ++n) {
            if (n >= ahead) {
                if (!ptx::mbar_wait<kPollNs>(bar_e, parity, s_abort, P.wait_limit)) {
                    atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_EMPTY);
                    return;
                }
                if (rank == 0) ptx::mbar_arrive_expect_tx(bar, step_tx);
                ptx::tma_load_2d_pair_hint(dst, &tmap_w, x, v, ptx::map_to_cta(bar, 0), w_policy);
            }
            for (int b = 0; b < P.n_blk; ++b)
                ptx::tma_load_2d_pair(dst + off_b + (uint32_t)b * P.b_bytes, &tmap_h, x, b * P.n_pad + b_row0, ptx::map_to_cta(bar, 0));
            x += kBlockK;
            if (x == P.d) { x = 0; v += P.tile_rows; }
            bar += 8; bar_e += 8; dst += P.step_bytes;
            if (++stage == P.n_steps) { stage = 0; parity ^= 1; bar = full; bar_e = empty; dst = smem_base; }
        }
        return;
    }
    if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        // (the whole warp stays converged; one elected lane issues: see the verify kernel)
        if (rank != 0) return;
        const uint32_t idesc = ptx::idesc_bf16_f32(2 * kTileM, P.n_pad);
        const uint64_t a_desc0 = ptx::smem_desc_sw128(smem_base), b_desc0 = ptx::smem_desc_sw128(smem_base + off_b);
        const uint32_t step_units = P.step_bytes >> 4, b_units = P.b_bytes >> 4;
        int stage = 0, slot = 0;
        uint32_t parity = 0, slot_parity = 1;
        uint64_t a_desc = a_desc0, b_desc = b_desc0;
        uint32_t bar_f = full, bar_e = empty;
        for (int tile = 0; tile < n_tiles; ++tile) {
            if (!ptx::mbar_wait_converged<kPollNs, true>(acc_empty + 8 * slot, slot_parity, s_abort, P.wait_limit)) {
                if (lane == 0) atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_ACC_EMPTY);
                return;
            }
            ptx::tc_fence_after();
            const uint32_t d_tmem = tmem_base + (uint32_t)(slot * P.cols);
            for (int kb = 0; kb < P.kb_count; ++kb) {
                if (!ptx::mbar_wait_converged<kPollNs, true>(bar_f, parity, s_abort, P.wait_limit)) {
                    if (lane == 0) atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_FULL);
                    return;
                }
                ptx::tc_fence_after();
                if (ptx::elect_one()) {
                    for (int b = 0; b < P.n_blk; ++b) {
#pragma unroll
                        for (int k = 0; k < kBlockK / 16; ++k)
                            ptx::mma_f16_pair(d_tmem + (uint32_t)(b * P.n_pad), a_desc + 2 * k, b_desc + (uint32_t)b * b_units + 2 * k, idesc,
                                              (kb | k) != 0);
                    }
                    ptx::mma_commit_pair(bar_e, 3);
                }
                __syncwarp();
                bar_f += 8; bar_e += 8; a_desc += step_units; b_desc += step_units;
                if (++stage == P.n_steps) { stage = 0; parity ^= 1; bar_f = full; bar_e = empty; a_desc = a_desc0; b_desc = b_desc0; }
            }
            if (ptx::elect_one()) ptx::mma_commit_pair(acc_full + 8 * slot, 3);
            __syncwarp();
            if (++slot == P.n_slots) { slot = 0; slot_parity ^= 1; }
        }
        return;
    }

    // ---------------------------------------------------------------------- epilogue
    if (P.pdl) ptx::griddep_wait();       // tokens may be the kernel ahead's; global writes only after it
    for (int i = threadIdx.x - kFirstEpiWarp * 32; i < P.cols; i += kEpiWarps * 32) {
        const int row = i;                // columns are hidden rows: block 0, then block 1
        s_tok[i] = P.tokens != nullptr && row < P.rows ? P.tokens[row] : -1;
    }
    ptx::bar_sync(2, kEpiWarps * 32);
    const int quarter = warp & 3, set = (warp - kFirstEpiWarp) >> 2;   // TMEM lanes 32 * quarter ..; columns are shared by two sets
    const int m_lane = quarter * 32 + lane;
    float* my_max = s_max + (warp - kFirstEpiWarp) * 16;
    const int n_cols = min(P.cols, (P.rows + 15) & ~15);
    bool alive = true;
    int slot = 0;
    uint32_t parity = 0;
    for (int tile = 0; tile < n_tiles; ++tile) {
        if (!ptx::mbar_wait_warp<kIdlePollNs>(acc_full + 8 * slot, parity, s_abort, P.wait_limit)) {
            atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_ACC_FULL);
            alive = false;
            break;
        }
        ptx::tc_fence_after();
        const int v = v_cta0 + tile * P.tile_rows + m_lane;
        const bool valid = m_lane < P.tile_rows && v < P.V;
        const int group = (slice * n_tiles + tile) * 4 + quarter;
#pragma unroll 1
        for (int n0 = 16 * set; n0 < n_cols; n0 += 32) {
            uint32_t acc[16];
            ptx::tmem_ld16(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(slot * P.cols + n0), acc);
            ptx::tmem_ld_wait();
            float x[16], y[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] = valid ? __uint_as_float(acc[j]) : neg_inf();
            if (P.tokens != nullptr && valid) {
                const int4* tk = reinterpret_cast<const int4*>(s_tok + n0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int4 t4 = tk[j];
                    if (t4.x == v) P.tok_logit[n0 + 4 * j] = x[4 * j];
                    if (t4.y == v) P.tok_logit[n0 + 4 * j + 1] = x[4 * j + 1];
                    if (t4.z == v) P.tok_logit[n0 + 4 * j + 2] = x[4 * j + 2];
                    if (t4.w == v) P.tok_logit[n0 + 4 * j + 3] = x[4 * j + 3];
                }
            }
            if (P.group_max != nullptr) {
                float* out = P.logits + ((size_t)n0 * P.n_groups + group) * 32 + lane;
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (n0 + j < P.rows) out[(size_t)j * P.n_groups * 32] = x[j];
            }
            const float gm = halving16(x, lane, MaxOp());    // lanes 2x, 2x+1: column x of the chunk
            if ((lane & 1) == 0) my_max[lane >> 1] = gm;
            __syncwarp();
            float mx[16];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 m4 = reinterpret_cast<const float4*>(my_max)[j];
                mx[4 * j] = m4.x; mx[4 * j + 1] = m4.y; mx[4 * j + 2] = m4.z; mx[4 * j + 3] = m4.w;
            }
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                // the first lane that holds the maximum is left out, further ones count as 1
                const float z = fmaxf((x[j] - mx[j]) * P.c, kFloorExp);
                const bool is_max = x[j] == mx[j];
                const unsigned int holders = __ballot_sync(0xFFFFFFFFu, is_max);
                const bool first = is_max && (holders & ((1u << lane) - 1u)) == 0u;
                x[j] = first || !valid ? 0.0f : ex2(z);
                y[j] = x[j] * (is_max ? 0.0f : z);
            }
            const float rest = halving16(x, lane, SumOp()), t = halving16(y, lane, SumOp());
            if ((lane & 1) == 0) {
                const int col = n0 + (lane >> 1), at = quarter * P.cols + col, plane = 4 * P.cols;
                const Record old{s_rec[at], s_rec[plane + at], s_rec[2 * plane + at]};
                const Record now = merge(old, Record{gm, rest, t}, P.c);
                s_rec[at] = now.m; s_rec[plane + at] = now.rest; s_rec[2 * plane + at] = now.t;
                if (P.group_max != nullptr && col < P.rows) P.group_max[(size_t)col * P.n_groups + group] = gm;
            }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) {   // the issuer's barrier is the leader's
            if (rank != 0) ptx::mbar_arrive_cluster(ptx::map_to_cta(acc_empty + 8 * slot, 0));
            else ptx::mbar_arrive(acc_empty + 8 * slot);
        }
        if (++slot == P.n_slots) { slot = 0; parity ^= 1; }
    }
    if (alive) {
        __syncwarp();
        for (int n0 = 16 * set; n0 < n_cols; n0 += 32) {   // the records this warp has built
            const int col = n0 + lane;
            if (lane < 16 && col < P.rows) {
                const int at = quarter * P.cols + col, plane = 4 * P.cols;
                P.records[(size_t)(slice * 4 + quarter) * P.rows + col] = make_float4(s_rec[at], s_rec[plane + at], s_rec[2 * plane + at], 0.0f);
            }
        }
    }
    // -------------------------------------------------------------------------- teardown
    // (as in the verify kernel: after an abandoned wait the other CTA of the pair is told, and copies and
    // MMAs that may still be in flight are given time to finish)
    ptx::tc_fence_before();
    ptx::bar_sync(2, kEpiWarps * 32);
    if (*s_abort) {
        if (threadIdx.x == kFirstEpiWarp * 32)
            ptx::st_cluster_u32(ptx::map_to_cta(ptx::smem_u32(const_cast<int*>(s_abort)), rank ^ 1u), 1u);
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
    ptx::bar_sync(2, kEpiWarps * 32);
    if (warp == kFirstEpiWarp) {
        ptx::tc_fence_after();
        // neither CTA may free TMEM, or leave, while the other still reads accumulators or sends signals here
        if (lane == 0) ptx::mbar_arrive_cluster(ptx::map_to_cta(dealloc_bar, rank ^ 1u));
        ptx::mbar_wait_warp<kPollNs>(dealloc_bar, 0, s_never, 2 * max(P.wait_limit, kWaitLimitCycles));
        ptx::tmem_dealloc_pair(tmem_base, kTmemCols);
    }
}

// ------------------------------------------------------------------------------------------ finish

constexpr int kFinThreads = 256, kFinWarps = kFinThreads / 32;
constexpr int kFinList = 1024;

struct FinishParams {
    int rows, V, n_records, n_groups, tiles_per_cta, tile_rows, slice_rows;
    float c, inv_temp;
    const float4* records;
    const float *tok_logit, *group_max, *logits;
    const int32_t* tokens;
    const uint32_t* err;
    int n_top;
    float *out_logprob, *out_lse, *out_entropy, *out_top_logprob;
    int32_t* out_top_ids;
};

__device__ __forceinline__ int group_first(const FinishParams& P, int group) {
    const int quarter = group & 3, tile = (group >> 2) % P.tiles_per_cta, slice = (group >> 2) / P.tiles_per_cta;
    return slice * P.slice_rows + tile * P.tile_rows + quarter * 32;
}

__global__ void __launch_bounds__(kFinThreads)
score_finish_kernel(const FinishParams P) {
    __shared__ Record s_part[kFinWarps];
    __shared__ Record s_all;
    __shared__ uint32_t s_key[kFinThreads];
    __shared__ uint32_t s_thr;
    __shared__ int s_n, s_groups;
    __shared__ unsigned long long s_list[kFinList];
    __shared__ unsigned long long s_sorted[DM_MAX_TOP];
    __shared__ int s_group[kFinList];
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool failed = *P.err != 0u;
    const float bad = __uint_as_float(0x7FC00000u);

    // the maxima of the groups and the records are fetched side by side
    const float* gm = P.group_max != nullptr ? P.group_max + (size_t)row * P.n_groups : nullptr;
    float thread_max = neg_inf();
    if (P.n_top > 0) {
#pragma unroll 8
        for (int g = tid; g < P.n_groups; g += kFinThreads) thread_max = fmaxf(thread_max, gm[g]);
        s_key[tid] = tid < P.n_groups ? float_key(thread_max) : 0u;
    }
    Record r{neg_inf(), 0.0f, 0.0f};
    for (int i = tid; i < P.n_records; i += kFinThreads) {
        const float4 q = P.records[(size_t)i * P.rows + row];
        r = merge(r, Record{q.x, q.y, q.z}, P.c);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const Record o{__shfl_xor_sync(0xFFFFFFFFu, r.m, off), __shfl_xor_sync(0xFFFFFFFFu, r.rest, off),
                       __shfl_xor_sync(0xFFFFFFFFu, r.t, off)};
        r = (lane & off) == 0 ? merge(r, o, P.c) : merge(o, r, P.c);   // the same order on both sides
    }
    if (lane == 0) s_part[warp] = r;
    if (tid == 0) { s_n = 0; s_groups = 0; }
    __syncthreads();
    if (warp == 0) {
        Record a = s_part[0];
        for (int w = 1; w < kFinWarps; ++w) a = merge(a, s_part[w], P.c);
        if (lane == 0) {
            s_all = a;
            const float log_total = log1pf(a.rest);
            const int tok = P.tokens != nullptr ? P.tokens[row] : -1;
            if (P.out_logprob != nullptr)
                P.out_logprob[row] = failed ? bad : tok < 0 || tok >= P.V ? 0.0f : fmaf(P.tok_logit[row] - a.m, P.inv_temp, -log_total);
            if (P.out_lse != nullptr) P.out_lse[row] = failed ? bad : fmaf(a.m, P.inv_temp, log_total);
            if (P.out_entropy != nullptr) P.out_entropy[row] = failed ? bad : fmaf(-kLn2 / (1.0f + a.rest), a.t, log_total);
        }
    }
    if (P.n_top == 0) return;
    const int k = P.n_top;
    if (warp == 1) {   // a key that k threads' maxima reach (0 if there are fewer than k groups)
        uint32_t key[kFinWarps];
#pragma unroll
        for (int i = 0; i < kFinWarps; ++i) key[i] = s_key[32 * i + lane];
        uint32_t t = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t c = t | (1u << bit);
            int n = 0;
#pragma unroll
            for (int i = 0; i < kFinWarps; ++i) n += __popc(__ballot_sync(0xFFFFFFFFu, key[i] >= c));
            if (n >= k) { t = c; if (n <= k + (k >> 1)) break; }
        }
        if (lane == 0) s_thr = t;
    }
    __syncthreads();
    const uint32_t thr = s_thr;
    const Record a = s_all;
    // groups that reach the key, then their entries, a warp per group
    if (float_key(thread_max) >= thr)
        for (int g = tid; g < P.n_groups; g += kFinThreads)
            if (float_key(gm[g]) >= thr) {
                const int at = atomicAdd(&s_groups, 1);
                if (at < kFinList) s_group[at] = g;
            }
    __syncthreads();
    const float* logits = P.logits + (size_t)row * P.n_groups * 32 + lane;
    const int n_near = min(s_groups, kFinList);
#pragma unroll 4
    for (int i = warp; i < n_near; i += kFinWarps) {
        const int g = s_group[i];
        const float x = logits[(size_t)g * 32];
        if (float_key(x) >= thr && x != neg_inf()) {   // (rows past the end of W were written as -inf)
            const int at = atomicAdd(&s_n, 1);
            if (at < kFinList) s_list[at] = pack_best(float_key(x), (uint32_t)(group_first(P, g) + lane));
        }
    }
    __syncthreads();
    int n = s_n;
    if (n > kFinList || s_groups > kFinList) {
        // too many entries reach that key (equal logits): the k-th largest packed word by bisection over
        // the row's logits; exactly k words reach it
        unsigned long long lo = 0ull;
        for (int bit = 63; bit >= -1; --bit) {
            const unsigned long long c = bit >= 0 ? lo | (1ull << bit) : lo;
            __syncthreads();
            if (tid == 0) s_n = 0;
            __syncthreads();
            for (int g = warp; g < P.n_groups; g += kFinWarps) {
                if (float_key(gm[g]) < (uint32_t)(c >> 32)) continue;
                const float x = logits[(size_t)g * 32];
                const unsigned long long word = pack_best(float_key(x), (uint32_t)(group_first(P, g) + lane));
                if (x != neg_inf() && word >= c) {
                    const int at = atomicAdd(&s_n, 1);
                    if (bit < 0 && at < kFinList) s_list[at] = word;
                }
            }
            __syncthreads();
            if (s_n >= k) lo = c;
        }
        n = k;
    }
    for (int i = tid; i < k; i += kFinThreads) s_sorted[i] = 0ull;
    __syncthreads();
    for (int i = tid; i < n; i += kFinThreads) {   // the packed words are all different: rank by counting
        const unsigned long long mine = s_list[i];
        int place = 0;
#pragma unroll 8
        for (int o = 0; o < n; ++o) place += s_list[o] > mine ? 1 : 0;
        if (place < k) s_sorted[place] = mine;
    }
    __syncthreads();
    const float log_total = log1pf(a.rest);
    for (int i = tid; i < k; i += kFinThreads) {
        const unsigned long long word = s_sorted[i];
        const float x = key_float((uint32_t)(word >> 32));
        P.out_top_ids[(size_t)row * k + i] = failed || word == 0ull ? -1 : (int32_t)best_index(word);
        P.out_top_logprob[(size_t)row * k + i] = failed || word == 0ull ? bad : fmaf(x - a.m, P.inv_temp, -log_total);
    }
}

bool plan(int rows, ScoreParams* P) {
    const int half = rows > kMaxBlock ? 2 : 1;
    P->n_blk = half;
    P->n_pad = ((rows + half - 1) / half + 31) & ~31;
    if (P->n_pad < 64) P->n_pad = 64;   // narrower pair MMAs are no faster
    P->cols = P->n_blk * P->n_pad;
    P->n_slots = kTmemCols / P->cols;
    if (P->n_slots > 4) P->n_slots = 4;
    P->b_bytes = (uint32_t)(P->n_pad / 2) * (kBlockK * 2);
    P->step_bytes = kWStageBytes + (uint32_t)P->n_blk * P->b_bytes;
    const uint32_t fixed = 12u * P->cols * 4u + 4u * P->cols + kEpiWarps * 16u * 4u + kBarBytes;
    P->n_steps = (int)((kSmemLimit - 1024 - fixed) / P->step_bytes);
    if (P->n_steps > kMaxSteps) P->n_steps = kMaxSteps;
    P->off_rec = (uint32_t)P->n_steps * P->step_bytes;
    P->off_tok = P->off_rec + 12u * P->cols * 4u;
    P->off_max = P->off_tok + 4u * P->cols;
    P->off_bar = P->off_max + kEpiWarps * 16u * 4u;
    return P->n_steps >= 2 && P->n_slots >= 1;
}

}  // namespace

int score_groups(const SliceGeometry& geo) { return 4 * geo.tiles_per_cta * ((geo.n_ctas + 1) & ~1); }

ScoreWorkspace score_workspace(const SliceGeometry& geo, int rows, bool alternatives) {
    // records | token logits | maxima of groups | logits, each 256-byte aligned
    const auto up = [](size_t n) { return (n + 255) & ~static_cast<size_t>(255); };
    const size_t groups = (size_t)score_groups(geo), records = 4 * (size_t)((geo.n_ctas + 1) & ~1);
    ScoreWorkspace w{};
    w.off_tok = up(records * rows * sizeof(float4));
    w.off_max = w.off_tok + up((size_t)rows * sizeof(float));
    w.off_logits = w.off_max + (alternatives ? up((size_t)rows * groups * sizeof(float)) : 0);
    w.bytes = w.off_logits + (alternatives ? (size_t)rows * groups * 32 * sizeof(float) : 0);
    return w;
}

int launch_score(const FusedState* fs, const HeadDesc& head, const void* H, const RowsParams& rp, unsigned char* ws, uint32_t* err,
                 long long wait_limit, bool allow_pdl, cudaStream_t stream) {
    const SliceGeometry& geo = fused_slices(fs);
    ScoreParams P{};
    P.d = head.d; P.V = head.V; P.rows = rp.rows;
    if (!plan(rp.rows, &P)) return DM_EUNSUPPORTED;
    P.kb_count = head.d / kBlockK;
    P.tiles_per_cta = geo.tiles_per_cta; P.tile_rows = geo.tile_rows; P.slice_rows = geo.slice_rows;
    P.pdl = allow_pdl ? 1 : 0;
    P.wait_limit = wait_limit > 0 ? wait_limit : kWaitLimitCycles;
    P.c = rp.c;
    const int ctas = (geo.n_ctas + 1) & ~1;
    P.n_groups = score_groups(geo);
    const ScoreWorkspace w = score_workspace(geo, rp.rows, rp.n_top > 0);
    P.tokens = rp.tokens;
    P.records = reinterpret_cast<float4*>(ws);
    P.tok_logit = reinterpret_cast<float*>(ws + w.off_tok);
    if (rp.n_top > 0) {
        P.group_max = reinterpret_cast<float*>(ws + w.off_max);
        P.logits = reinterpret_cast<float*>(ws + w.off_logits);
    }
    P.err = err;
    CUtensorMap tmap_h;
    if (!tensor_map_bf16(&tmap_h, H, rp.rows, head.d, P.n_pad / 2)) return DM_ECUDA;
    const size_t smem = P.off_bar + kBarBytes + 1024;
    if (cudaFuncSetAttribute(score_head_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) != cudaSuccess) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attrs[2]{};
    attrs[0].id = cudaLaunchAttributeClusterDimension;
    attrs[0].val.clusterDim.x = 2; attrs[0].val.clusterDim.y = 1; attrs[0].val.clusterDim.z = 1;
    attrs[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attrs;
    cfg.numAttrs = allow_pdl ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, score_head_kernel, geo.tmap_w, tmap_h, P) != cudaSuccess || cudaGetLastError() != cudaSuccess) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    FinishParams F{};
    F.rows = rp.rows; F.V = head.V; F.n_records = 4 * ctas; F.n_groups = P.n_groups;
    F.tiles_per_cta = geo.tiles_per_cta; F.tile_rows = geo.tile_rows; F.slice_rows = geo.slice_rows;
    F.c = rp.c; F.inv_temp = rp.inv_temp;
    F.records = P.records; F.tok_logit = P.tok_logit; F.group_max = P.group_max; F.logits = P.logits;
    F.tokens = rp.tokens; F.err = err;
    F.n_top = rp.n_top;
    F.out_logprob = rp.out_logprob; F.out_lse = rp.out_lse; F.out_entropy = rp.out_entropy;
    F.out_top_ids = rp.out_top_ids; F.out_top_logprob = rp.out_top_logprob;
    cudaLaunchConfig_t fin{};
    fin.gridDim = dim3((unsigned)rp.rows);
    fin.blockDim = dim3(kFinThreads);
    fin.stream = stream;
    fin.attrs = attrs + 1;
    fin.numAttrs = 1;   // (what it reads it waits for: griddep_wait)
    if (cudaLaunchKernelEx(&fin, score_finish_kernel, F) != cudaSuccess || cudaGetLastError() != cudaSuccess) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    return DM_OK;
}

}  // namespace dm
