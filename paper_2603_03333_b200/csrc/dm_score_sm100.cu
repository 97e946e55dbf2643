// dropmatch_score on bf16 heads: l = H W^T on tcgen05 tensor cores, and of every row of l the
// log-sum-exp, the entropy, the given token's logit and the largest entries, without a second pass
// over the vocabulary.
//
//   z = l / T;  lse = log sum exp z;  log p(tok) = z[tok] - lse;  entropy = -sum p log p
//
// score_head_kernel.  The hidden rows are the M operand, a tile of up to 256 vocabulary rows is the N
// operand: accumulator lane = hidden row, column = vocabulary entry, so that an epilogue thread owns a
// row and runs its softmax statistics in registers, without exchanges between lanes.  (With the
// operands the other way round, as in the verify kernel, the reductions over lanes took 31 us per tile
// of 512 rows.)  The vocabulary is cut into one slice per CTA (up to 128 rows: M = 128, N = 256) or per
// CTA pair (above: cta_group::2, M = 256, each CTA its 128 hidden rows and half of the W tile; above 256
// two blocks of hidden rows against one W tile, which fill TMEM), W crosses the HBM interface once per
// 512 hidden rows.  Hidden rows come straight from the caller's array through a tensor map made for the
// call; rows past its end load as zeros.  Bounds: W from HBM up to some 200 rows, the tensor pipe above.
// Measured: one row against 128256 x 4096 with 5 alternatives 161-171 us (1.05 GB: 6.1-6.5 TB/s), 61 rows
// against 151936 x 4096 191-208 us (1.24 GB: 6.0-6.5 TB/s), 509 rows against 128256 x 8192 with 32
// alternatives 835-895 us (1.07 PFLOP: 1.19-1.28 PFLOP/s, 0.9 of what a GEMM sustains under the power cap;
// the tensor pipe is busy 85 % of the cycles).
//
// Epilogue.  32 columns at a time: their maximum, the sum of 2^((l - max) c) over the others
// (c = log2(e) / T) and the same times the exponent, merged into the thread's record (maximum, rest,
// weighted sum).  "rest" leaves the largest entry out, so that log(1 + rest) keeps its precision.  If
// alternatives are asked for, the 32 logits and their maximum also go to global memory.
//
// score_finish_kernel.  One block per hidden row merges the records of all slices.  Alternatives: the
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
constexpr int kRowsM = 128;                 // hidden rows of a CTA's operand tile
constexpr int kHBytes = kRowsM * kBlockK * 2;
constexpr int kTmemCols = 512;
constexpr int kMaxSteps = 12;
constexpr int kTileN = 256;                 // most vocabulary entries of a tile (UMMA N), accumulator columns of one
constexpr int kDirectRows = 64;             // up to this many rows logits are stored without turning tiles around
constexpr int kBarBytes = 512;
constexpr int kSmemLimit = 227 * 1024;
constexpr long long kWaitLimitCycles = 2000000000ll;
constexpr int kPollNs = 32, kIdlePollNs = 500;
constexpr float kFloorExp = -200.0f;
constexpr float kLn2 = 0.693147180559945309f;

struct ScoreParams {
    int d, V, rows;
    int kb_count;
    int slice, n_tiles, tile_n, last_n;  // vocabulary entries of a slice, tiles in it, entries of a tile and of the last one (multiples of 16)
    int n_blk;                   // blocks of 256 hidden rows (pairs only)
    int n_slots, n_steps;        // accumulator slots in TMEM; stages of the ring
    uint32_t step_bytes, w_bytes, h_bytes;   // bytes of a stage, of its W part, and that one load of hidden rows brings
    int pdl;
    long long wait_limit;
    float c;                     // log2(e) / T
    const int32_t* tokens;       // [rows] or null
    float* tok_logit;            // [rows]
    float4* records;             // [2 * slices][rows]
    float* group_max;            // [rows][groups] or null: no alternatives
    float* logits;               // [rows][groups][32]
    int groups_per_tile, groups_per_slice, n_groups;
    uint32_t* err;
    uint32_t off_out, off_bar;   // alternatives: 4 KB per epilogue warp to turn a tile of logits around in
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

// Record of 32 logits of one row (at least one of them a number): relative to their maximum.
__device__ __forceinline__ Record group_record(const float (&x)[32], float gm, float c) {
    float2 s = make_float2(0.0f, 0.0f), t = s, ties = s;
    const float2 m2 = make_float2(-gm, -gm), c2 = make_float2(c, c);
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
        float2 z = __fmul2_rn(__fadd2_rn(make_float2(x[j], x[j + 1]), m2), c2);
        z.x = fmaxf(z.x, kFloorExp);      // (-inf past the end of the vocabulary)
        z.y = fmaxf(z.y, kFloorExp);
        // an entry equal to the maximum has z = 0 and e = 1 exactly: counted, not summed
        const float2 top = make_float2(z.x == 0.0f ? -1.0f : 0.0f, z.y == 0.0f ? -1.0f : 0.0f);
        const float2 e = make_float2(ex2(z.x), ex2(z.y));
        s = __fadd2_rn(s, __fadd2_rn(e, top));
        ties = __fadd2_rn(ties, top);
        t = __ffma2_rn(e, z, t);
    }
    return Record{gm, (s.x + s.y) - (ties.x + ties.y) - 1.0f, t.x + t.y};
}

// x[i] by five rounds of selection: an array indexed by a register would live in local memory.
__device__ __forceinline__ float pick32(const float (&x)[32], uint32_t i) {
    float a[16], b[8], c[4], d[2];
#pragma unroll
    for (int j = 0; j < 16; ++j) a[j] = (i & 16u) ? x[j + 16] : x[j];
#pragma unroll
    for (int j = 0; j < 8; ++j) b[j] = (i & 8u) ? a[j + 8] : a[j];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = (i & 4u) ? b[j + 4] : b[j];
#pragma unroll
    for (int j = 0; j < 2; ++j) d[j] = (i & 2u) ? c[j + 2] : c[j];
    return (i & 1u) ? d[1] : d[0];
}

// kPair: clusters of two CTAs; the leader (cluster rank 0) issues cta_group::2 MMAs over both CTAs'
// hidden rows and both halves of the W tile.  Barriers that the issuer waits on live in the leader,
// those that it signals exist in both CTAs.
template <bool kPair>
__global__ void __launch_bounds__(kThreads, 1)
score_head_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_w_last,
                  const __grid_constant__ CUtensorMap tmap_h, const ScoreParams P) {
    extern __shared__ unsigned char smem_dyn[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(
        (reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t smem_base = ptx::smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t* s_bar = reinterpret_cast<uint64_t*>(smem + P.off_bar);
    // barriers: full[n_steps] empty[n_steps] acc_full[n_slots] acc_empty[n_slots] dealloc
    const uint32_t full = smem_base + P.off_bar, empty = full + 8 * P.n_steps;
    const uint32_t acc_full = empty + 8 * P.n_steps, acc_empty = acc_full + 8 * P.n_slots;
    const uint32_t dealloc_bar = acc_empty + 8 * P.n_slots;
    const int n_bars = 2 * P.n_steps + 2 * P.n_slots + 1;
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_bar + n_bars);
    volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
    volatile int* s_never = reinterpret_cast<volatile int*>(s_tmem + 2);
    const uint32_t rank = kPair ? ptx::cluster_ctarank() : 0u;
    constexpr int kCtas = kPair ? 2 : 1;

    if (threadIdx.x == 0) {
        ptx::prefetch_tensormap(&tmap_w);
        ptx::prefetch_tensormap(&tmap_w_last);
        ptx::prefetch_tensormap(&tmap_h);
        for (int s = 0; s < P.n_steps; ++s) { ptx::mbar_init(full + 8 * s, 1); ptx::mbar_init(empty + 8 * s, 1); }
        for (int s = 0; s < P.n_slots; ++s) { ptx::mbar_init(acc_full + 8 * s, 1); ptx::mbar_init(acc_empty + 8 * s, kCtas * kEpiWarps); }
        ptx::mbar_init(dealloc_bar, 1);
        *s_abort = 0;
        *s_never = 0;
        ptx::fence_mbar_init();
        ptx::fence_proxy_async_smem();
    }
    if (warp == kFirstEpiWarp) {
        if (kPair) { ptx::tmem_alloc_pair(ptx::smem_u32(s_tmem), kTmemCols); ptx::tmem_relinquish_pair(); }
        else { ptx::tmem_alloc(ptx::smem_u32(s_tmem), kTmemCols); ptx::tmem_relinquish(); }
    }
    if (P.h_bytes < kHBytes) {   // operand rows that no load fills stay zero
        const int per_stage = (int)(kHBytes - P.h_bytes) / 16;
        for (int i = threadIdx.x; i < P.n_steps * per_stage; i += kThreads)
            *reinterpret_cast<uint4*>(smem + (uint32_t)(i / per_stage) * P.step_bytes + P.w_bytes + P.h_bytes + (uint32_t)(i % per_stage) * 16) =
                make_uint4(0u, 0u, 0u, 0u);
        ptx::fence_proxy_async_smem();
    }
    ptx::tc_fence_before();
    __syncthreads();
    if (kPair) ptx::cluster_sync_all();   // the other CTA's barriers are initialised before anyone signals them
    ptx::tc_fence_after();
    const uint32_t tmem_base = *s_tmem;
    if (P.pdl) ptx::griddep_launch_dependents();

    const int slice = (int)blockIdx.x / kCtas, v_slice = slice * P.slice;
    const int n_tiles = P.n_tiles;   // entries past the end of W load as zeros and are never taken

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        if (lane != 0) return;
        const uint64_t w_policy = ptx::l2_policy_evict_first();
        const int total = n_tiles * P.kb_count;
        const uint32_t h_tx = (uint32_t)(kCtas * P.n_blk) * P.h_bytes;                       // all CTAs of the cluster
        const uint32_t bar_map = kPair ? ptx::map_to_cta(full, 0) : full;                  // the leader's barriers
        // cursor over (tile, hidden-size block) of the W loads
        int x = 0, tile = 0;
        auto load_w = [&](int stage) {
            const bool last = tile == n_tiles - 1;
            const int n = last ? P.last_n : P.tile_n;
            const CUtensorMap* map = last ? &tmap_w_last : &tmap_w;
            const int v = v_slice + tile * P.tile_n + (int)rank * (n / 2);
            const uint32_t dst = smem_base + (uint32_t)stage * P.step_bytes;
            if (rank == 0) ptx::mbar_arrive_expect_tx(full + 8 * stage, (uint32_t)n * (kBlockK * 2) + h_tx);
            if (kPair) ptx::tma_load_2d_pair_hint(dst, map, x, v, bar_map + 8 * stage, w_policy);
            else ptx::tma_load_2d_hint(dst, map, x, v, full + 8 * stage, w_policy);
            x += kBlockK;
            if (x == P.d) { x = 0; ++tile; }
        };
        // W does not depend on the kernel ahead, the hidden rows may: the ring is first filled with W tiles
        const int ahead = P.pdl ? min(P.n_steps, total) : 0;
        for (int n = 0; n < ahead; ++n) load_w(n);
        if (P.pdl) ptx::griddep_wait();
        int stage = 0, hx = 0;
        uint32_t parity = 1;
        for (int n = 0; n < total; ++n) {
            if (n >= ahead) {
                if (!ptx::mbar_wait<kPollNs>(empty + 8 * stage, parity, s_abort, P.wait_limit)) {
                    atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_EMPTY);
                    return;
                }
                load_w(stage);
            }
            const uint32_t dst = smem_base + (uint32_t)stage * P.step_bytes + P.w_bytes;
            if (kPair) {
                for (int b = 0; b < P.n_blk; ++b)
                    ptx::tma_load_2d_pair(dst + (uint32_t)b * kHBytes, &tmap_h, hx, (2 * b + (int)rank) * kRowsM, bar_map + 8 * stage);
            } else {
                ptx::tma_load_2d(dst, &tmap_h, hx, 0, full + 8 * stage);
            }
            hx += kBlockK;
            if (hx == P.d) hx = 0;
            if (++stage == P.n_steps) { stage = 0; parity ^= 1; }
        }
        return;
    }
    if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        // (the whole warp stays converged; one elected lane issues: see the verify kernel)
        if (rank != 0) return;
        const uint64_t w_desc0 = ptx::smem_desc_sw128(smem_base), h_desc0 = ptx::smem_desc_sw128(smem_base + P.w_bytes);
        const uint32_t step_units = P.step_bytes >> 4;
        int stage = 0, slot = 0;
        uint32_t parity = 0, slot_parity = 1;
        uint64_t w_desc = w_desc0, h_desc = h_desc0;
        uint32_t bar_f = full, bar_e = empty;
        for (int tile = 0; tile < n_tiles; ++tile) {
            const uint32_t idesc = ptx::idesc_bf16_f32(kCtas * kRowsM, tile == n_tiles - 1 ? P.last_n : P.tile_n);
            if (!ptx::mbar_wait_converged<kPollNs, true>(acc_empty + 8 * slot, slot_parity, s_abort, P.wait_limit)) {
                if (lane == 0) atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_ACC_EMPTY);
                return;
            }
            ptx::tc_fence_after();
            const uint32_t d_tmem = tmem_base + (uint32_t)(slot * P.n_blk * kTileN);
            for (int kb = 0; kb < P.kb_count; ++kb) {
                if (!ptx::mbar_wait_converged<kPollNs, true>(bar_f, parity, s_abort, P.wait_limit)) {
                    if (lane == 0) atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_FULL);
                    return;
                }
                ptx::tc_fence_after();
                if (ptx::elect_one()) {
                    for (int b = 0; b < P.n_blk; ++b) {
                        const uint64_t a_desc = h_desc + (uint32_t)b * (kHBytes >> 4);
#pragma unroll
                        for (int k = 0; k < kBlockK / 16; ++k)   // 16 elements = 32 bytes = 2 descriptor units
                            if (kPair) ptx::mma_f16_pair(d_tmem + (uint32_t)(b * kTileN), a_desc + 2 * k, w_desc + 2 * k, idesc, (kb | k) != 0);
                            else ptx::mma_f16(d_tmem, a_desc + 2 * k, w_desc + 2 * k, idesc, (kb | k) != 0);
                    }
                    if (kPair) ptx::mma_commit_pair(bar_e, 3); else ptx::mma_commit(bar_e);
                }
                __syncwarp();
                bar_f += 8; bar_e += 8; w_desc += step_units; h_desc += step_units;
                if (++stage == P.n_steps) { stage = 0; parity ^= 1; bar_f = full; bar_e = empty; w_desc = w_desc0; h_desc = h_desc0; }
            }
            if (ptx::elect_one()) { if (kPair) ptx::mma_commit_pair(acc_full + 8 * slot, 3); else ptx::mma_commit(acc_full + 8 * slot); }
            __syncwarp();
            if (++slot == P.n_slots) { slot = 0; slot_parity ^= 1; }
        }
        return;
    }

    // ---------------------------------------------------------------------- epilogue
    if (P.pdl) ptx::griddep_wait();       // tokens may be the kernel ahead's; global writes only after it
    const int quarter = warp & 3, set = (warp - kFirstEpiWarp) >> 2;   // TMEM lanes 32 * quarter ..; a set takes every other group of 32 columns
    const int v_end = min(P.V, v_slice + P.slice);
    float4* turn = reinterpret_cast<float4*>(smem + P.off_out) + (warp - kFirstEpiWarp) * 256;
    Record rec[2];
    int row[2], tok[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        row[b] = (2 * b + (int)rank) * kRowsM + quarter * 32 + lane;
        rec[b] = Record{neg_inf(), 0.0f, 0.0f};
        tok[b] = P.tokens != nullptr && b < P.n_blk && row[b] < P.rows ? P.tokens[row[b]] : -1;
    }
    int slot = 0;
    uint32_t parity = 0;
    for (int tile = 0; tile < n_tiles; ++tile) {
        if (!ptx::mbar_wait_warp<kIdlePollNs>(acc_full + 8 * slot, parity, s_abort, P.wait_limit)) {
            atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_ACC_FULL);
            break;
        }
        ptx::tc_fence_after();
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (b >= P.n_blk || row[b] - lane >= P.rows) continue;     // (the same for the whole warp)
            const int n_here = min(tile == n_tiles - 1 ? P.last_n : P.tile_n, v_end - (v_slice + tile * P.tile_n));
            int n0 = 32 * set;
#pragma unroll 1
            for (; n0 < n_here; n0 += 64) {
                uint32_t acc[32];
                ptx::tmem_ld32(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)((slot * P.n_blk + b) * kTileN + n0), acc);
                ptx::tmem_ld_wait();
                const int v0 = v_slice + tile * P.tile_n + n0;
                float x[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) x[j] = __uint_as_float(acc[j]);
                if (n_here - n0 < 32) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) x[j] = n0 + j < n_here ? x[j] : neg_inf();
                }
                float gm = x[0];
#pragma unroll
                for (int j = 1; j < 32; ++j) gm = fmaxf(gm, x[j]);
                if ((unsigned)(tok[b] - v0) < (unsigned)min(32, n_here - n0)) {   // (the rest is the next tile's)
                    P.tok_logit[row[b]] = pick32(x, (uint32_t)(tok[b] - v0));
                }
                if (P.group_max != nullptr) {
                    const size_t g = (size_t)slice * P.groups_per_slice + tile * P.groups_per_tile + (n0 >> 5);
                    if (row[b] < P.rows) P.group_max[(size_t)row[b] * P.n_groups + g] = gm;
                    if (P.off_out == P.off_bar) {
                        // few rows: each thread stores its own line, and the ring has a stage more (1 to 61 rows on
                        // the Llama-3-8B head: 161-172 us against 167-178 us)
                        if (row[b] < P.rows) {
                            float4* out = reinterpret_cast<float4*>(P.logits + ((size_t)row[b] * P.n_groups + g) * 32);
#pragma unroll
                            for (int j = 0; j < 8; ++j) out[j] = make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
                        }
                    } else {
                        // the warp's 32 x 32 logits go through shared memory (16-byte chunks at c ^ (row mod 8)) so that
                        // a store covers four whole lines instead of a piece of 32 (509 rows: 432 against 775 us)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            turn[lane * 8 + (j ^ (lane & 7))] = make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int r = 4 * i + (lane >> 3), q = row[b] - lane + r;
                            if (q < P.rows)
                                reinterpret_cast<float4*>(P.logits + ((size_t)q * P.n_groups + g) * 32)[lane & 7] = turn[r * 8 + ((lane & 7) ^ (r & 7))];
                        }
                        __syncwarp();
                    }
                }
                rec[b] = merge(rec[b], group_record(x, gm, P.c), P.c);
                __syncwarp();
            }
            // groups that hold nothing (a last tile shorter than the others, the end of the vocabulary) say so
            if (P.group_max != nullptr && row[b] < P.rows) {
                for (; n0 < 32 * P.groups_per_tile; n0 += 64)
                    P.group_max[(size_t)row[b] * P.n_groups + (size_t)slice * P.groups_per_slice + tile * P.groups_per_tile + (n0 >> 5)] = neg_inf();
            }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) {   // the issuer's barrier is the leader's
            if (kPair && rank != 0) ptx::mbar_arrive_cluster(ptx::map_to_cta(acc_empty + 8 * slot, 0));
            else ptx::mbar_arrive(acc_empty + 8 * slot);
        }
        if (++slot == P.n_slots) { slot = 0; parity ^= 1; }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
        if (b < P.n_blk && row[b] < P.rows)
            P.records[(size_t)(slice * 2 + set) * P.rows + row[b]] = make_float4(rec[b].m, rec[b].rest, rec[b].t, 0.0f);
    // -------------------------------------------------------------------------- teardown
    // (as in the verify kernel: after an abandoned wait the other CTA of a pair is told, and copies and
    // MMAs that may still be in flight are given time to finish)
    ptx::tc_fence_before();
    ptx::bar_sync(2, kEpiWarps * 32);
    if (*s_abort) {
        if (kPair && threadIdx.x == kFirstEpiWarp * 32)
            ptx::st_cluster_u32(ptx::map_to_cta(ptx::smem_u32(const_cast<int*>(s_abort)), rank ^ 1u), 1u);
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
    ptx::bar_sync(2, kEpiWarps * 32);
    if (warp == kFirstEpiWarp) {
        ptx::tc_fence_after();
        if (kPair) {
            // neither CTA may free TMEM, or leave, while the other still reads accumulators or sends signals here
            if (lane == 0) ptx::mbar_arrive_cluster(ptx::map_to_cta(dealloc_bar, rank ^ 1u));
            ptx::mbar_wait_warp<kPollNs>(dealloc_bar, 0, s_never, 2 * max(P.wait_limit, kWaitLimitCycles));
            ptx::tmem_dealloc_pair(tmem_base, kTmemCols);
        } else {
            ptx::tmem_dealloc(tmem_base, kTmemCols);
        }
    }
}

// ------------------------------------------------------------------------------------------ finish

constexpr int kFinThreads = 256, kFinWarps = kFinThreads / 32;
constexpr int kFinList = 1024;
constexpr int kFinOwn = 20;     // maxima of groups a thread keeps in registers (more are read twice)

struct FinishParams {
    int rows, V, n_records, groups_per_tile, n_tiles, slice, tile_n;
    int n_groups;              // per row; a maximum of -inf: nothing in it, its logits are not written
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
    const int tile = group / P.groups_per_tile, slice = tile / P.n_tiles;
    return slice * P.slice + (tile - slice * P.n_tiles) * P.tile_n + (group - tile * P.groups_per_tile) * 32;
}

__global__ void __launch_bounds__(kFinThreads)
score_finish_kernel(const FinishParams P) {
    __shared__ Record s_part[kFinWarps];
    __shared__ Record s_all;
    __shared__ __align__(16) uint32_t s_key[kFinThreads];
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
    float own[kFinOwn];
    float thread_max = neg_inf();
    if (P.n_top > 0) {
#pragma unroll
        for (int i = 0; i < kFinOwn; ++i) own[i] = i * kFinThreads + tid < P.n_groups ? gm[i * kFinThreads + tid] : neg_inf();
#pragma unroll
        for (int i = 0; i < kFinOwn; ++i) thread_max = fmaxf(thread_max, own[i]);
#pragma unroll 4
        for (int g = kFinOwn * kFinThreads + tid; g < P.n_groups; g += kFinThreads) thread_max = fmaxf(thread_max, gm[g]);
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
    if (tid == 0) { s_n = 0; s_groups = 0; s_thr = 0u; }
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
    {   // the k-th largest of the threads' maxima (0 if fewer threads have one)
        const uint32_t mine = s_key[tid];
        int reach = 0;
#pragma unroll 8
        for (int i = 0; i < kFinThreads / 4; ++i) {
            const uint4 o = reinterpret_cast<const uint4*>(s_key)[i];
            reach += (o.x >= mine) + (o.y >= mine) + (o.z >= mine) + (o.w >= mine);
        }
        if (reach >= k && mine != 0u) atomicMax(&s_thr, mine);
    }
    __syncthreads();
    const uint32_t thr = s_thr;
    const Record a = s_all;
    // groups that reach the key, then their entries, a warp per group
    if (float_key(thread_max) >= thr) {
        const auto take = [&](int g) {
            const int at = atomicAdd(&s_groups, 1);
            if (at < kFinList) s_group[at] = g;
        };
#pragma unroll
        for (int i = 0; i < kFinOwn; ++i)
            if (own[i] > neg_inf() && float_key(own[i]) >= thr) take(i * kFinThreads + tid);
        for (int g = kFinOwn * kFinThreads + tid; g < P.n_groups; g += kFinThreads)
            if (gm[g] > neg_inf() && float_key(gm[g]) >= thr) take(g);
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
                if (!(gm[g] > neg_inf()) || float_key(gm[g]) < (uint32_t)(c >> 32)) continue;
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

}  // namespace

// How the vocabulary is cut: [0] a slice per CTA, [1] a slice per CTA pair.
struct ScoreState {
    struct Cut {
        CUtensorMap w, w_last;      // boxes of a full and of a slice's last tile (a CTA's part of it)
        int slice, n_tiles, tile_n, last_n, n_slices, groups_per_tile;
        int groups_per_slice() const { return n_tiles * groups_per_tile; }
    } cut[2];
};

int score_create(ScoreState** out, const HeadDesc& head) {
    *out = nullptr;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 2) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    ScoreState* st = new (std::nothrow) ScoreState();
    if (st == nullptr) return DM_ECUDA;
    for (int p = 0; p < 2; ++p) {
        ScoreState::Cut& cut = st->cut[p];
        const int units = p ? sms / 2 : sms;
        cut.slice = ((head.V + units - 1) / units + 15) & ~15;      // UMMA N is a multiple of 16
        cut.n_tiles = (cut.slice + kTileN - 1) / kTileN;
        cut.tile_n = ((cut.slice + cut.n_tiles - 1) / cut.n_tiles + 15) & ~15;   // (a short last tile would leave the ring idle)
        cut.n_tiles = (cut.slice + cut.tile_n - 1) / cut.tile_n;
        cut.last_n = cut.slice - (cut.n_tiles - 1) * cut.tile_n;
        cut.n_slices = (head.V + cut.slice - 1) / cut.slice;
        cut.groups_per_tile = (cut.tile_n + 31) / 32;
        if (!tensor_map_bf16(&cut.w, head.W, head.V, head.d, cut.tile_n >> p) ||
            !tensor_map_bf16(&cut.w_last, head.W, head.V, head.d, cut.last_n >> p)) {
            delete st;
            return DM_ECUDA;
        }
    }
    if (cudaFuncSetAttribute(score_head_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) != cudaSuccess ||
        cudaFuncSetAttribute(score_head_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) != cudaSuccess) {
        cudaGetLastError();
        delete st;
        return DM_ECUDA;
    }
    *out = st;
    return DM_OK;
}

void score_destroy(ScoreState* st) { delete st; }

namespace {

struct Workspace { size_t off_tok, off_max, off_logits, bytes; };

// records | token logits | maxima of groups | logits, each 256-byte aligned
Workspace workspace(const ScoreState::Cut& cut, int rows, bool alternatives) {
    const auto up = [](size_t n) { return (n + 255) & ~static_cast<size_t>(255); };
    const size_t groups = (size_t)cut.n_slices * cut.groups_per_slice();
    Workspace w{};
    w.off_tok = up(2 * (size_t)cut.n_slices * rows * sizeof(float4));
    w.off_max = w.off_tok + up((size_t)rows * sizeof(float));
    w.off_logits = w.off_max + (alternatives ? up((size_t)rows * groups * sizeof(float)) : 0);
    w.bytes = w.off_logits + (alternatives ? (size_t)rows * groups * 32 * sizeof(float) : 0);
    return w;
}

}  // namespace

size_t score_workspace_bytes(const ScoreState* st, int rows, bool alternatives) {
    // calls of fewer rows may use the other cut
    const size_t one = workspace(st->cut[0], rows < kRowsM ? rows : kRowsM, alternatives).bytes;
    const size_t two = rows > kRowsM ? workspace(st->cut[1], rows, alternatives).bytes : 0;
    return one > two ? one : two;
}

int launch_score(const ScoreState* st, const HeadDesc& head, const void* H, const RowsParams& rp, unsigned char* ws, uint32_t* err,
                 long long wait_limit, bool allow_pdl, cudaStream_t stream) {
    if (rp.rows > kScoreChunk) return DM_EUNSUPPORTED;
    const bool pair = rp.rows > kRowsM;
    const ScoreState::Cut& cut = st->cut[pair];
    ScoreParams P{};
    P.d = head.d; P.V = head.V; P.rows = rp.rows;
    P.kb_count = head.d / kBlockK;
    P.slice = cut.slice; P.n_tiles = cut.n_tiles; P.tile_n = cut.tile_n; P.last_n = cut.last_n;
    P.n_blk = rp.rows > 2 * kRowsM ? 2 : 1;
    P.n_slots = kTmemCols / (P.n_blk * kTileN);
    P.w_bytes = ((uint32_t)(cut.tile_n >> pair) * (kBlockK * 2) + 1023u) & ~1023u;   // swizzle atoms start on 1024-byte boundaries
    P.step_bytes = P.w_bytes + (uint32_t)P.n_blk * kHBytes;
    const int box = pair ? kRowsM : (rp.rows + 7) & ~7;
    P.h_bytes = (uint32_t)box * (kBlockK * 2);
    const uint32_t out_bytes = rp.n_top > 0 && rp.rows > kDirectRows ? kEpiWarps * 4096u : 0u;
    P.n_steps = (int)((kSmemLimit - 1024 - kBarBytes - out_bytes) / P.step_bytes);
    if (P.n_steps > kMaxSteps) P.n_steps = kMaxSteps;
    P.off_out = (uint32_t)P.n_steps * P.step_bytes;
    P.off_bar = P.off_out + out_bytes;
    P.pdl = allow_pdl ? 1 : 0;
    P.wait_limit = wait_limit > 0 ? wait_limit : kWaitLimitCycles;
    P.c = rp.c;
    P.groups_per_tile = cut.groups_per_tile;
    P.groups_per_slice = cut.groups_per_slice();
    P.n_groups = cut.n_slices * P.groups_per_slice;
    const Workspace w = workspace(cut, rp.rows, rp.n_top > 0);
    P.tokens = rp.tokens;
    P.records = reinterpret_cast<float4*>(ws);
    P.tok_logit = reinterpret_cast<float*>(ws + w.off_tok);
    if (rp.n_top > 0) {
        P.group_max = reinterpret_cast<float*>(ws + w.off_max);
        P.logits = reinterpret_cast<float*>(ws + w.off_logits);
    }
    P.err = err;
    CUtensorMap tmap_h;
    if (!tensor_map_bf16(&tmap_h, H, rp.rows, head.d, box)) return DM_ECUDA;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(cut.n_slices << pair));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = P.off_bar + kBarBytes + 1024;
    cfg.stream = stream;
    cudaLaunchAttribute attrs[2]{};
    int n_attrs = 0;
    if (allow_pdl) {
        attrs[n_attrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attrs[n_attrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (pair) {
        attrs[n_attrs].id = cudaLaunchAttributeClusterDimension;
        attrs[n_attrs].val.clusterDim.x = 2; attrs[n_attrs].val.clusterDim.y = 1; attrs[n_attrs++].val.clusterDim.z = 1;
    }
    cfg.attrs = attrs;
    cfg.numAttrs = n_attrs;
    const cudaError_t launched = pair ? cudaLaunchKernelEx(&cfg, score_head_kernel<true>, cut.w, cut.w_last, tmap_h, P)
                                      : cudaLaunchKernelEx(&cfg, score_head_kernel<false>, cut.w, cut.w_last, tmap_h, P);
    if (launched != cudaSuccess || cudaGetLastError() != cudaSuccess) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    FinishParams F{};
    F.rows = rp.rows; F.V = head.V; F.n_records = 2 * cut.n_slices; F.n_groups = P.n_groups;
    F.groups_per_tile = cut.groups_per_tile; F.n_tiles = cut.n_tiles; F.slice = cut.slice; F.tile_n = cut.tile_n;
    F.c = rp.c; F.inv_temp = rp.inv_temp;
    F.records = P.records; F.tok_logit = P.tok_logit; F.group_max = P.group_max; F.logits = P.logits;
    F.tokens = rp.tokens; F.err = err;
    F.n_top = rp.n_top;
    F.out_logprob = rp.out_logprob; F.out_lse = rp.out_lse; F.out_entropy = rp.out_entropy;
    F.out_top_ids = rp.out_top_ids; F.out_top_logprob = rp.out_top_logprob;
    cudaLaunchAttribute behind{};   // (what the kernel reads it waits for: griddep_wait)
    behind.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    behind.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t fin{};
    fin.gridDim = dim3((unsigned)rp.rows);
    fin.blockDim = dim3(kFinThreads);
    fin.stream = stream;
    fin.attrs = &behind;
    fin.numAttrs = 1;
    if (cudaLaunchKernelEx(&fin, score_finish_kernel, F) != cudaSuccess || cudaGetLastError() != cudaSuccess) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    return DM_OK;
}

}  // namespace dm
