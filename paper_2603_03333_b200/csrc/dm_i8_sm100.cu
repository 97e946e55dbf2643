// dropmatch_quantize_i8, dropmatch_matmul_i8, dropmatch_linear_i8: products through a head (or any projection) held in
// 8-bit integers, with a scale for each row of either matrix.
//
//   quantise:  scale[r] = max(max_j |x[r,j]| / 127, 2^-126),  q[r,j] = round_to_even(x[r,j] / scale[r])
//   product:   out[r,v] = a_scale[r] w_scale[v] sum_j a[r,j] w[v,j]       (the sum exact, in 32-bit integers)
//
// matmul_i8_kernel.  Rows of W are the M operand (128 of a CTA, 256 of a CTA pair), up to 256 tokens the N operand, so that an
// epilogue thread owns a vocabulary entry and a warp's store of one token's outputs is contiguous as it comes out of
// TMEM.  CTAs (pairs) walk over tiles, the token tiles of one piece of W next to each other, with the accumulator of the
// next tile filling while one is read out.  Bounds: HBM's stream of W for up to some 200 tokens, the tensor pipe above, and
// under sustained load the power cap in either case (integers of full range toggle every bit of what is streamed).
// Measured, quantisation included: one token against 128256 x 4096 90-96 us (525 MB, a bare read of which takes 78-86), 61
// tokens against 151936 x 4096 117-120 us (622 MB; 130-135 back to back), 2047 against 128256 x 8192 1.54-1.6 ms
// (2.7-2.8 PFLOP/s; back to back 1.78-1.86 ms, 2.3-2.4 PFLOP/s, 0.85 of twice what a bf16 GEMM sustains).
// Tried: two blocks of 256 tokens per piece of W, filling TMEM (a quarter less traffic into shared memory, but read-out that
// the next tile does not hide: 978 against 826 us at d = 4096, the same at 8192); pairs for few tokens, steps that start at
// another depth in every CTA (no difference).
#include <atomic>

#include "dm_i8.h"
#include "dm_ptx.cuh"

namespace dm {

namespace {

// ------------------------------------------------------------------------------------------ quantise

constexpr int kQThreads = 256;

__device__ __forceinline__ float entry_f32(const float* x, long long j) { return x[j]; }
__device__ __forceinline__ float entry_f32(const __nv_bfloat16* x, long long j) { return __bfloat162float(x[j]); }

// Sixteen entries from j on: 16-byte loads where the row allows them, what lies past the end as 0.
template <typename T, bool VEC>
__device__ __forceinline__ void load16(const T* row, int j, int n, float (&v)[16]) {
    constexpr int kN = 16 / sizeof(T);
    if (VEC && n - j >= 16) {
#pragma unroll
        for (int i = 0; i < 16 / kN; ++i) {
            alignas(16) T part[kN];
            *reinterpret_cast<uint4*>(part) = reinterpret_cast<const uint4*>(row + j)[i];
#pragma unroll
            for (int k = 0; k < kN; ++k) v[i * kN + k] = entry_f32(part, k);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = n - j > i ? entry_f32(row, j + i) : 0.0f;
    }
}

// x / scale in fp32, rounded to the nearest whole number, ties to even: in the low byte.  The product with the reciprocal is off
// by less than 127 (2^-24 + 2^-24 + 2^-47) from the quotient, the fp32 quotient by 127 2^-24: only within 2^-15 of a
// half, one entry in 16 thousand, can they round apart, and there the division decides (all entries by division: 22 us
// instead of 17 for 2047 rows of 8192 bf16).
__device__ __forceinline__ uint32_t rounded(float x, float scale, float inverse) {
    const float shift = 12582912.0f;       // 1.5 2^23: the sum's low bits hold the rounded value
    const float t = x * inverse;
    float k = t + shift;
    if (!(fabsf(t - (k - shift)) <= 0.5f - 3.0517578125e-5f)) k = __fdiv_rn(x, scale) + shift;
    return __float_as_uint(k);
}

// WARPS warps per row.  The row is read twice (the second time from L1): once for its largest magnitude, once to round it.
template <typename T, bool VEC, int WARPS>
__global__ void __launch_bounds__(kQThreads)
quantize_kernel(const QuantizeParams P) {
    __shared__ float s_max[kQThreads / 32];
    ptx::griddep_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long r = (long long)blockIdx.x * (kQThreads / 32 / WARPS) + warp / WARPS;
    if (r >= P.n_rows) return;               // (whole blocks with WARPS = 8, whole warps without a barrier else)
    const T* x = static_cast<const T*>(P.x) + r * P.ld;
    const int first = 16 * ((warp % WARPS) * 32 + lane);
    constexpr int kStep = 16 * 32 * WARPS;
    float top = 0.0f;
    bool bad = false;
    for (int j = first; j < P.n; j += kStep) {
        float v[16];
        load16<T, VEC>(x, j, P.n, v);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            top = fmaxf(top, fabsf(v[i]));
            bad |= !(fabsf(v[i]) <= 3.4028234663852886e38f);      // NaN, +-inf
        }
    }
    if (bad) top = __uint_as_float(0x7F800000u);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, off));
    if (WARPS > 1) {
        if (lane == 0) s_max[warp] = top;
        __syncthreads();
        for (int w = 0; w < WARPS; ++w) top = fmaxf(top, s_max[w]);
    }
    bad = top > 3.4028234663852886e38f;
    const float scale = fmaxf(__fdiv_rn(top, 127.0f), 1.17549435082228751e-38f);
    if (first == 0) P.scale[r] = bad ? __uint_as_float(0x7FC00000u) : scale;
    const float inverse = bad ? 0.0f : __fdiv_rn(1.0f, scale);
    int8_t* q = P.q + r * P.ld_q;
    for (int j = first; j < P.n; j += kStep) {
        float v[16];
        load16<T, VEC>(x, j, P.n, v);
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t low = __byte_perm(rounded(v[4 * i], scale, inverse), rounded(v[4 * i + 1], scale, inverse), 0x0040);
            const uint32_t high = __byte_perm(rounded(v[4 * i + 2], scale, inverse), rounded(v[4 * i + 3], scale, inverse), 0x0040);
            o[i] = bad ? 0u : __byte_perm(low, high, 0x5410);
        }
        if (P.n - j >= 16) {
            *reinterpret_cast<uint4*>(q + j) = make_uint4(o[0], o[1], o[2], o[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (P.n - j > i) q[j + i] = (int8_t)(o[i / 4] >> (8 * (i % 4)));
        }
    }
}

template <typename T>
int launch_quantize(const QuantizeParams& P, cudaStream_t stream) {
    const bool vec = ((reinterpret_cast<uintptr_t>(P.x) | (uintptr_t)(P.ld * (long long)sizeof(T))) & 15u) == 0;
    const bool wide = P.n > 1024;       // (a warp takes up to two steps of 512 entries on its own)
    const long long blocks = wide ? P.n_rows : (P.n_rows + 7) / 8;
    if (blocks > 0x7FFFFFFFll) return DM_EUNSUPPORTED;
    const unsigned grid = (unsigned)blocks;
    if (wide) {
        if (vec) quantize_kernel<T, true, 8><<<grid, kQThreads, 0, stream>>>(P);
        else quantize_kernel<T, false, 8><<<grid, kQThreads, 0, stream>>>(P);
    } else {
        if (vec) quantize_kernel<T, true, 1><<<grid, kQThreads, 0, stream>>>(P);
        else quantize_kernel<T, false, 1><<<grid, kQThreads, 0, stream>>>(P);
    }
    return cudaGetLastError() == cudaSuccess ? DM_OK : DM_ECUDA;
}

// ------------------------------------------------------------------------------------------ product

constexpr int kThreads = 10 * 32;           // warp 0 TMA, warp 1 MMA, warps 2-9 epilogue
constexpr int kFirstEpiWarp = 2, kEpiWarps = 8;
constexpr int kBlockK = 128;                // entries (bytes) of a row per step: one swizzle width
constexpr int kTileM = 128;                 // rows of W of a CTA's tile
constexpr int kWBytes = kTileM * kBlockK;
constexpr int kTileN = 256;                 // most tokens of a tile; accumulator columns of a slot
constexpr int kSlots = 2;
constexpr int kTmemCols = 512;
constexpr int kMaxSteps = 12;
constexpr int kBarBytes = 512;
constexpr int kSmemLimit = 227 * 1024;
constexpr long long kWaitLimitCycles = 2000000000ll;
constexpr int kPollNs = 32, kIdlePollNs = 200;

struct I8Params {
    int V, rows;
    int kb_count;
    int tile_m;                          // rows of W that a CTA's tile takes up (the operand always has kTileM; what no load fills is not stored)
    int tile_n, n_tiles_n, n_tiles;      // tokens of a tile (a multiple of 32), tiles along the tokens, tiles in all
    int n_steps;
    uint32_t step_bytes, off_bar;
    int early, once;                     // W may be fetched ahead of the kernel in front; W is read once
    long long wait_limit;
    const float *a_scale, *w_scale;
    void* out;
    long long ld_out;
    uint32_t* err;
};

// Instruction descriptor: signed 8-bit x signed 8-bit -> 32-bit integer, both operands K-major, M x N tile.
__host__ __device__ constexpr uint32_t idesc_i8_s32(int M, int N) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// D[tmem] (+)= A[smem desc] * B[smem desc]^T, 32 entries deep; one thread issues (of the pair's leader for kPair).
template <bool kPair>
__device__ __forceinline__ void mma_i8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    if (kPair)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

__device__ __forceinline__ void put(float* out, float x) { *out = x; }
__device__ __forceinline__ void put(__nv_bfloat16* out, float x) { *out = __float2bfloat16_rn(x); }

// kPair: clusters of two CTAs; the leader (cluster rank 0) issues cta_group::2 MMAs over both CTAs' rows of W and both
// halves of the tokens.  Barriers that the issuer waits on live in the leader, those that it signals exist in both CTAs.
template <bool kPair, typename OUT>
__global__ void __launch_bounds__(kThreads, 1)
matmul_i8_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_a, const I8Params P) {
    extern __shared__ unsigned char smem_dyn[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(
        (reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~static_cast<uintptr_t>(1023));
    const uint32_t smem_base = ptx::smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t* s_bar = reinterpret_cast<uint64_t*>(smem + P.off_bar);
    // barriers: full[n_steps] empty[n_steps] acc_full[kSlots] acc_empty[kSlots] dealloc
    const uint32_t full = smem_base + P.off_bar, empty = full + 8 * P.n_steps;
    const uint32_t acc_full = empty + 8 * P.n_steps, acc_empty = acc_full + 8 * kSlots;
    const uint32_t dealloc_bar = acc_empty + 8 * kSlots;
    const int n_bars = 2 * P.n_steps + 2 * kSlots + 1;
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_bar + n_bars);
    volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
    volatile int* s_never = reinterpret_cast<volatile int*>(s_tmem + 2);
    const uint32_t rank = kPair ? ptx::cluster_ctarank() : 0u;
    constexpr int kCtas = kPair ? 2 : 1;

    if (threadIdx.x == 0) {
        ptx::prefetch_tensormap(&tmap_w);
        ptx::prefetch_tensormap(&tmap_a);
        for (int s = 0; s < P.n_steps; ++s) { ptx::mbar_init(full + 8 * s, 1); ptx::mbar_init(empty + 8 * s, 1); }
        for (int s = 0; s < kSlots; ++s) { ptx::mbar_init(acc_full + 8 * s, 1); ptx::mbar_init(acc_empty + 8 * s, kCtas * kEpiWarps); }
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
    ptx::tc_fence_before();
    __syncthreads();
    if (kPair) ptx::cluster_sync_all();   // the other CTA's barriers are initialised before anyone signals them
    ptx::tc_fence_after();
    const uint32_t tmem_base = *s_tmem;

    const int unit = (int)blockIdx.x / kCtas, units = (int)gridDim.x / kCtas;

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        if (lane != 0) return;
        const uint64_t w_policy = P.once ? ptx::l2_policy_evict_first() : ptx::l2_policy_evict_normal();
        const int a_rows = P.tile_n / kCtas;
        const uint32_t tx = (uint32_t)((kCtas * P.tile_m + P.tile_n) * kBlockK);              // of all CTAs of the cluster
        const uint32_t bar_map = kPair ? ptx::map_to_cta(full, 0) : full;                  // the leader's barriers
        const int my_tiles = unit < P.n_tiles ? (P.n_tiles - unit + units - 1) / units : 0;
        const int total = my_tiles * P.kb_count;
        // cursors over (tile, step) of the loads of W and of the tokens
        int w_tile = unit, w_kb = 0, a_tile = unit, a_kb = 0;
        auto load_w = [&](int stage) {
            if (rank == 0) ptx::mbar_arrive_expect_tx(full + 8 * stage, tx);
            const uint32_t dst = smem_base + (uint32_t)stage * P.step_bytes;
            const int y = ((w_tile / P.n_tiles_n) * kCtas + (int)rank) * P.tile_m;
            if (kPair) ptx::tma_load_2d_pair_hint(dst, &tmap_w, w_kb * kBlockK, y, bar_map + 8 * stage, w_policy);
            else ptx::tma_load_2d_hint(dst, &tmap_w, w_kb * kBlockK, y, full + 8 * stage, w_policy);
            if (++w_kb == P.kb_count) { w_kb = 0; w_tile += units; }
        };
        auto load_a = [&](int stage) {
            const uint32_t dst = smem_base + (uint32_t)stage * P.step_bytes + kWBytes;
            const int y = (a_tile % P.n_tiles_n) * P.tile_n + (int)rank * a_rows;
            if (kPair) ptx::tma_load_2d_pair(dst, &tmap_a, a_kb * kBlockK, y, bar_map + 8 * stage);
            else ptx::tma_load_2d(dst, &tmap_a, a_kb * kBlockK, y, full + 8 * stage);
            if (++a_kb == P.kb_count) { a_kb = 0; a_tile += units; }
        };
        // W does not depend on the kernel ahead, the tokens do: the ring is first filled with pieces of W
        const int ahead = P.early ? min(P.n_steps, total) : 0;
        for (int n = 0; n < ahead; ++n) load_w(n);
        if (P.early) ptx::griddep_wait();
        int stage = 0;
        uint32_t parity = 1;
        for (int n = 0; n < total; ++n) {
            if (n >= ahead) {
                if (!ptx::mbar_wait<kPollNs>(empty + 8 * stage, parity, s_abort, P.wait_limit)) {
                    atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_EMPTY);
                    return;
                }
                load_w(stage);
            }
            load_a(stage);
            if (++stage == P.n_steps) { stage = 0; parity ^= 1; }
        }
        return;
    }
    if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        // (the whole warp stays converged; one elected lane issues: see the verify kernel)
        if (rank != 0) return;
        const uint64_t w_desc0 = ptx::smem_desc_sw128(smem_base), a_desc0 = ptx::smem_desc_sw128(smem_base + kWBytes);
        const uint32_t step_units = P.step_bytes >> 4;
        const uint32_t idesc = idesc_i8_s32(kCtas * kTileM, P.tile_n);
        int stage = 0, slot = 0;
        uint32_t parity = 0, slot_parity = 1;
        uint64_t w_desc = w_desc0, a_desc = a_desc0;
        uint32_t bar_f = full, bar_e = empty;
        for (int tile = unit; tile < P.n_tiles; tile += units) {
            if (!ptx::mbar_wait_converged<kPollNs, true>(acc_empty + 8 * slot, slot_parity, s_abort, P.wait_limit)) {
                if (lane == 0) atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_ACC_EMPTY);
                return;
            }
            ptx::tc_fence_after();
            const uint32_t d_tmem = tmem_base + (uint32_t)(slot * kTileN);
            for (int kb = 0; kb < P.kb_count; ++kb) {
                if (!ptx::mbar_wait_converged<kPollNs, true>(bar_f, parity, s_abort, P.wait_limit)) {
                    if (lane == 0) atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_FULL);
                    return;
                }
                ptx::tc_fence_after();
                if (ptx::elect_one()) {
#pragma unroll
                    for (int k = 0; k < kBlockK / 32; ++k)   // 32 entries = 32 bytes = 2 descriptor units
                        mma_i8<kPair>(d_tmem, w_desc + 2 * k, a_desc + 2 * k, idesc, (kb | k) != 0);
                    if (kPair) ptx::mma_commit_pair(bar_e, 3); else ptx::mma_commit(bar_e);
                }
                __syncwarp();
                bar_f += 8; bar_e += 8; w_desc += step_units; a_desc += step_units;
                if (++stage == P.n_steps) { stage = 0; parity ^= 1; bar_f = full; bar_e = empty; w_desc = w_desc0; a_desc = a_desc0; }
            }
            if (ptx::elect_one()) { if (kPair) ptx::mma_commit_pair(acc_full + 8 * slot, 3); else ptx::mma_commit(acc_full + 8 * slot); }
            __syncwarp();
            if (++slot == kSlots) { slot = 0; slot_parity ^= 1; }
        }
        return;
    }

    // ---------------------------------------------------------------------- epilogue
    if (P.early) ptx::griddep_wait();     // the tokens' scales are the kernel ahead's
    const int quarter = warp & 3, set = (warp - kFirstEpiWarp) >> 2;   // TMEM lanes 32 * quarter ..; a set takes every other group of 32 tokens
    const float nan = __uint_as_float(0x7FC00000u);
    OUT* const out = static_cast<OUT*>(P.out);
    bool dead = false;                    // a wait ran out: what is left of this CTA's outputs is NaN
    int slot = 0;
    uint32_t parity = 0;
    for (int tile = unit; tile < P.n_tiles; tile += units) {
        const int tile_m = tile / P.n_tiles_n;
        const int m = quarter * 32 + lane, v = m < P.tile_m ? (tile_m * kCtas + (int)rank) * P.tile_m + m : P.V;
        const int n_first = (tile - tile_m * P.n_tiles_n) * P.tile_n, n_here = min(P.tile_n, P.rows - n_first);
        const float w_scale = v < P.V ? P.w_scale[v] : 0.0f;
        if (!dead && !ptx::mbar_wait_warp<kIdlePollNs>(acc_full + 8 * slot, parity, s_abort, P.wait_limit)) {
            if (lane == 0) atomicCAS(P.err, 0u, (uint32_t)ERR_WAIT_ACC_FULL);
            dead = true;
        }
        ptx::tc_fence_after();
#pragma unroll 1
        for (int n0 = 32 * set; n0 < n_here; n0 += 64) {
            uint32_t acc[32];
            if (!dead) {
                ptx::tmem_ld32(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(slot * kTileN + n0), acc);
                ptx::tmem_ld_wait();
            }
            const int n = n_first + n0, count = min(32, n_here - n0);
            const float a_scale = lane < count ? P.a_scale[n + lane] : 0.0f;
            OUT* o = out + (long long)n * P.ld_out + v;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const float s = __shfl_sync(0xFFFFFFFFu, a_scale, j);
                if (j < count && v < P.V) put(o + (long long)j * P.ld_out, dead ? nan : (float)(int)acc[j] * w_scale * s);
            }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) {   // the issuer's barrier is the leader's
            if (kPair && rank != 0) ptx::mbar_arrive_cluster(ptx::map_to_cta(acc_empty + 8 * slot, 0));
            else ptx::mbar_arrive(acc_empty + 8 * slot);
        }
        if (++slot == kSlots) { slot = 0; parity ^= 1; }
    }
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

template <bool kPair, typename OUT>
int launch(const I8Args& A, I8Params& P, int sms, cudaStream_t stream) {
    constexpr int kCtas = kPair ? 2 : 1;
    const int all = sms / kCtas;
    int tiles_m = (A.V + kCtas * kTileM - 1) / (kCtas * kTileM);
    P.tile_m = kTileM;
    P.n_tiles_n = (A.n_rows + kTileN - 1) / kTileN;
    P.tile_n = ((A.n_rows + P.n_tiles_n - 1) / P.n_tiles_n + 31) & ~31;      // (UMMA N: steps of 32 for a pair)
    P.n_tiles_n = (A.n_rows + P.tile_n - 1) / P.tile_n;
    P.once = P.n_tiles_n == 1;
    if (P.once && tiles_m > all) {
        // W is read once and bounds the call: the same number of rows for everybody, in equal tiles (one token against
        // 128256 x 4096, 6.8 tiles of 128 rows for each CTA: 90 us in 7 tiles of 124, 92 in up to 7 of 128)
        const int rounds = (tiles_m + all - 1) / all;
        const long long share = (long long)all * kCtas * rounds;
        P.tile_m = (int)((((long long)A.V + share - 1) / share + 3) & ~3ll);
        tiles_m = (int)(((long long)A.V + kCtas * P.tile_m - 1) / (kCtas * P.tile_m));
    }
    if ((long long)tiles_m * P.n_tiles_n > 0x3FFFFFFFll) return DM_EUNSUPPORTED;
    P.n_tiles = tiles_m * P.n_tiles_n;
    P.step_bytes = (uint32_t)(kWBytes + P.tile_n / kCtas * kBlockK);
    P.n_steps = (int)((kSmemLimit - 1024 - kBarBytes) / P.step_bytes);
    if (P.n_steps > kMaxSteps) P.n_steps = kMaxSteps;
    P.off_bar = (uint32_t)P.n_steps * P.step_bytes;
    CUtensorMap tmap_w, tmap_a;
    if (!tensor_map_u8(&tmap_w, A.w, A.V, A.d, A.ld_w, P.tile_m) || !tensor_map_u8(&tmap_a, A.a, A.n_rows, A.d, A.ld_a, P.tile_n / kCtas))
        return DM_ECUDA;
    static std::atomic<uint64_t> allowed{0};      // devices on which this kernel may have that much shared memory
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return DM_ECUDA;
    if (dev >= 64 || !(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
        if (cudaFuncSetAttribute(matmul_i8_kernel<kPair, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit) != cudaSuccess) {
            cudaGetLastError();
            return DM_ECUDA;
        }
        if (dev < 64) allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    const int units = P.n_tiles < all ? P.n_tiles : all;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(units * kCtas));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = P.off_bar + kBarBytes + 1024;
    cfg.stream = stream;
    cudaLaunchAttribute attrs[2]{};
    int n_attrs = 0;
    if (P.early) {
        attrs[n_attrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attrs[n_attrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (kPair) {
        attrs[n_attrs].id = cudaLaunchAttributeClusterDimension;
        attrs[n_attrs].val.clusterDim.x = 2; attrs[n_attrs].val.clusterDim.y = 1; attrs[n_attrs++].val.clusterDim.z = 1;
    }
    cfg.attrs = attrs;
    cfg.numAttrs = n_attrs;
    if (cudaLaunchKernelEx(&cfg, matmul_i8_kernel<kPair, OUT>, tmap_w, tmap_a, P) != cudaSuccess || cudaGetLastError() != cudaSuccess) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    return DM_OK;
}

}  // namespace

int launch_quantize_i8(const QuantizeParams& P, int dtype, cudaStream_t stream) {
    return dtype == DM_F32 ? launch_quantize<float>(P, stream) : launch_quantize<__nv_bfloat16>(P, stream);
}

int launch_matmul_i8(const I8Args& A, cudaStream_t stream) {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 2) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    I8Params P{};
    P.V = A.V; P.rows = A.n_rows;
    P.kb_count = (A.d + kBlockK - 1) / kBlockK;
    P.early = A.behind_quantize ? 1 : 0;
    P.wait_limit = A.wait_limit > 0 ? A.wait_limit : kWaitLimitCycles;
    P.a_scale = A.a_scale; P.w_scale = A.w_scale;
    P.out = A.out; P.ld_out = A.ld_out;
    P.err = A.err;
    const bool pair = A.n_rows > 128;
    if (A.out_dtype == DM_F32) return pair ? launch<true, float>(A, P, sms, stream) : launch<false, float>(A, P, sms, stream);
    return pair ? launch<true, __nv_bfloat16>(A, P, sms, stream) : launch<false, __nv_bfloat16>(A, P, sms, stream);
}

}  // namespace dm
