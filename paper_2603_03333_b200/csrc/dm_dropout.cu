// dropmatch_dropout and its gradient: Eq. 1 and Eq. 2 as operators on rows in memory.
//
//   out[q,i,j]  = keep(q,i,j) x[q,j] / (1 - p)          dx[q,j] = sum_i keep(q,i,j) g[q,i,j] / (1 - p)
//
// with keep(q,i,j) = word (j mod 4) of Philox4x32-10 at the counter (j/4, i, t, s) >= floor(p 2^32), the masks of
// the verify calls.  No mask is read or written: forward and backward generate it.
//
// A warp takes a chunk of one hidden row (128 entries of fp32, 256 of bf16: 16 bytes per lane) through a run of
// paths, so that x crosses the memory interface once (forward) and the sums over paths stay in registers
// (backward).  A lane generates whole quads of the generator; rows that start on 16-byte boundaries are
// read and written by the lane that owns the quad, others entry by entry with neighbouring lanes on
// neighbouring entries, the flags handed over by shuffles (a quad that straddles two vectors would
// otherwise be generated twice).
//
// What bounds it: HBM and the generator alike.  Ten rounds are 20 widening multiplies per quad; in a loop over paths
// five of them stay the same (see PhiloxQuad), which leaves about 43 instructions per 8 bytes of bf16.
#include "dm_dropout.h"

namespace dm {

namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr uint32_t kMulA = 0xD2511F53u, kMulB = 0xCD9E8D57u, kKeyA = 0x9E3779B9u, kKeyB = 0xBB67AE85u;

__device__ __forceinline__ void mul_wide(uint32_t a, uint32_t b, uint32_t& hi, uint32_t& lo) {
    const unsigned long long p = (unsigned long long)a * b;
    hi = (uint32_t)(p >> 32);
    lo = (uint32_t)p;
}

// Philox4x32-10 at the counter (quad, path, t, s), cut at what does not change from path to path.
// Round r maps (x, y, z, w) to (hi(B z) ^ y ^ k0, lo(B z), hi(A x) ^ w ^ k1, lo(A x)).  The path index is in y only:
// after round 1 it is in x alone, after round 2 in z and w, so the product B z of round 2 and A x of round 3
// are the quad's, and A x of round 2 is the path's.
struct PhiloxPath {       // the same for all quads of a row
    uint32_t hi2, lo2;    // A x of round 2
    __device__ __forceinline__ PhiloxPath(uint32_t path, uint32_t t, uint32_t k0) {
        uint32_t hi, lo;
        mul_wide(kMulB, t, hi, lo);
        mul_wide(kMulA, hi ^ path ^ k0, hi2, lo2);
    }
};
struct PhiloxQuad {       // the same for all paths
    uint32_t z2, y2, z3, w3;
    __device__ __forceinline__ PhiloxQuad() {}
    __device__ __forceinline__ PhiloxQuad(uint32_t quad, uint32_t t, uint32_t s, uint32_t k0, uint32_t k1) {
        uint32_t hi_t, lo_t, hi, w1, x2;
        mul_wide(kMulB, t, hi_t, lo_t);
        mul_wide(kMulA, quad, hi, w1);
        mul_wide(kMulB, hi ^ s ^ k1, x2, y2);
        x2 ^= lo_t ^ (k0 + kKeyA);
        z2 = w1 ^ (k1 + kKeyB);
        mul_wide(kMulA, x2, z3, w3);
        z3 ^= k1 + 2 * kKeyB;
        y2 ^= k0 + 2 * kKeyA;
    }
    __device__ __forceinline__ uint4 words(const PhiloxPath& p, uint32_t k0, uint32_t k1) const {
        uint4 c;
        mul_wide(kMulB, p.hi2 ^ z2, c.x, c.y);      // round 3
        c.x ^= y2;
        c.z = z3 ^ p.lo2;
        c.w = w3;
#pragma unroll
        for (uint32_t r = 3; r < 10; ++r) {
            uint32_t hi_a, lo_a, hi_b, lo_b;
            mul_wide(kMulA, c.x, hi_a, lo_a);
            mul_wide(kMulB, c.z, hi_b, lo_b);
            c = make_uint4(hi_b ^ c.y ^ (k0 + r * kKeyA), lo_b, hi_a ^ c.w ^ (k1 + r * kKeyB), lo_a);
        }
        return c;
    }
    __device__ __forceinline__ uint32_t keep(const PhiloxPath& p, uint32_t k0, uint32_t k1, uint32_t thr) const {
        const uint4 w = words(p, k0, k1);
        return (w.x >= thr ? 1u : 0u) | (w.y >= thr ? 2u : 0u) | (w.z >= thr ? 4u : 0u) | (w.w >= thr ? 8u : 0u);
    }
};

// Where a warp stands: hidden row, first quad of its chunk, its paths.
template <int Q>   // quads of a lane
struct Place {
    long long row;
    int first;          // first entry of the chunk
    int path0, path1;
    uint32_t t, s;
    __device__ __forceinline__ Place(const DropoutParams& P, long long task) {
        const int chunk = (int)(task % P.n_chunks);
        const long long rest = task / P.n_chunks;
        const int group = (int)(rest % P.n_groups);
        row = rest / P.n_groups;
        first = chunk * (32 * 4 * Q);
        path0 = group * P.group_paths;
        path1 = min(P.K, path0 + P.group_paths);
        const long long b = row / P.T;
        t = P.shared_masks ? 0u : (uint32_t)(row - b * P.T);
        s = P.seq_base_lo + (uint32_t)b;
    }
};

// The same value in every lane, and known to be: what follows from it stays out of the lanes' registers and pipes.
__device__ __forceinline__ int warp_index() { return __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0); }

// Four entries of a lane's vector, kept or zero, as words of two or one entries.
__device__ __forceinline__ void keep_words(const uint32_t* v, const uint4& w, uint32_t thr, uint32_t* o, float) {
    o[0] = w.x >= thr ? v[0] : 0u;
    o[1] = w.y >= thr ? v[1] : 0u;
    o[2] = w.z >= thr ? v[2] : 0u;
    o[3] = w.w >= thr ? v[3] : 0u;
}
__device__ __forceinline__ void keep_words(const uint32_t* v, const uint4& w, uint32_t thr, uint32_t* o, __nv_bfloat16) {
    o[0] = w.x >= thr ? v[0] & 0xFFFFu : 0u;
    if (w.y >= thr) o[0] |= v[0] & 0xFFFF0000u;
    o[1] = w.z >= thr ? v[1] & 0xFFFFu : 0u;
    if (w.w >= thr) o[1] |= v[1] & 0xFFFF0000u;
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void round_to(float x, float* out) { *out = x; }
__device__ __forceinline__ void round_to(float x, __nv_bfloat16* out) { *out = __float2bfloat16_rn(x); }

// T: storage type.  VEC: every row starts on a 16-byte boundary (entries past the last whole vector of a row
// are then read and written one by one by the same lane).
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(const DropoutParams P) {
    constexpr int Q = sizeof(T) == 2 ? 2 : 1, E = 4 * Q;     // quads and entries of a lane
    const long long task = (long long)blockIdx.x * kWarps + warp_index();
    if (task >= P.n_tasks) return;                           // (the same for the whole warp)
    const Place<Q> at(P, task);
    const int lane = threadIdx.x & 31;
    const T* x = static_cast<const T*>(P.in) + at.row * P.ld_in;
    T* out = static_cast<T*>(P.out) + (at.row * P.K + at.path0) * P.ld_out;
    PhiloxQuad quad[Q];
    const uint32_t quad0 = (uint32_t)at.first / 4;
#pragma unroll
    for (int r = 0; r < Q; ++r)
        quad[r] = PhiloxQuad(quad0 + (VEC ? Q * lane + r : 32 * r + lane), at.t, at.s, P.key0, P.key1);
    alignas(16) T v[E];      // x / (1 - p), rounded once; entry n of the lane's own vector, or entry 32 n + lane of the chunk
    const int own = at.first + E * lane;
    if (VEC && own + E <= P.d) {
        *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(x + own);
    } else {
#pragma unroll
        for (int n = 0; n < E; ++n) {
            const int j = VEC ? own + n : at.first + 32 * n + lane;
            round_to(0.0f, &v[n]);
            if (j < P.d) v[n] = x[j];
        }
    }
#pragma unroll
    for (int n = 0; n < E; ++n) round_to(to_float(v[n]) * P.scale, &v[n]);
    T zero;
    round_to(0.0f, &zero);
#pragma unroll 2
    for (int i = at.path0; i < at.path1; ++i, out += P.ld_out) {
        const PhiloxPath path((uint32_t)i, at.t, P.key0);
        if (VEC) {
            uint32_t o[4];
#pragma unroll
            for (int r = 0; r < Q; ++r)
                keep_words(reinterpret_cast<const uint32_t*>(v) + 4 / Q * r, quad[r].words(path, P.key0, P.key1), P.thr, o + 4 / Q * r, zero);
            if (own + E <= P.d) {
                *reinterpret_cast<uint4*>(out + own) = make_uint4(o[0], o[1], o[2], o[3]);
            } else {
#pragma unroll
                for (int n = 0; n < E; ++n)
                    if (own + n < P.d) out[own + n] = reinterpret_cast<const T*>(o)[n];
            }
        } else {
#pragma unroll
            for (int r = 0; r < Q; ++r) {
                const uint32_t flags = quad[r].keep(path, P.key0, P.key1, P.thr);
#pragma unroll
                for (int n = 0; n < 4; ++n) {      // entries 128 r + 32 n + lane: quad 8 n + lane / 4 of the 32
                    const uint32_t f = __shfl_sync(0xFFFFFFFFu, flags, 8 * n + (lane >> 2));
                    const int j = at.first + 128 * r + 32 * n + lane;
                    if (j < P.d) out[j] = (f >> (lane & 3)) & 1u ? v[4 * r + n] : zero;
                }
            }
        }
    }
}

// Sums over the paths: fp32, paths in order within a run of them; long sums are cut into P.n_groups runs that
// neighbouring warps of a block take and the first of them joins in order.  The cut follows from K alone, so that
// a row's result does not depend on the others.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads)
dropout_grad_kernel(const DropoutParams P) {
    constexpr int Q = sizeof(T) == 2 ? 2 : 1, E = 4 * Q;
    __shared__ float s_part[kWarps][E * 32];
    const int warp = warp_index(), lane = threadIdx.x & 31;
    const int group = warp & (P.n_groups - 1);               // (a power of two, at most kWarps)
    // tasks count chunks of all runs; a block takes kWarps / n_groups chunks
    const long long chunk_id = (long long)blockIdx.x * (kWarps / P.n_groups) + warp / P.n_groups;
    const bool live = chunk_id < P.n_tasks;
    const long long row = live ? chunk_id / P.n_chunks : 0;
    const int first = live ? (int)(chunk_id - row * P.n_chunks) * (32 * E) : 0;
    const int path0 = min(P.K, group * P.group_paths), path1 = live ? min(P.K, path0 + P.group_paths) : path0;
    const long long b = row / P.T;
    const uint32_t t = P.shared_masks ? 0u : (uint32_t)(row - b * P.T), s = P.seq_base_lo + (uint32_t)b;
    PhiloxQuad quad[Q];
#pragma unroll
    for (int r = 0; r < Q; ++r)
        quad[r] = PhiloxQuad((uint32_t)first / 4 + (VEC ? Q * lane + r : 32 * r + lane), t, s, P.key0, P.key1);
    const T* g = static_cast<const T*>(P.in) + (row * P.K + path0) * P.ld_in;
    const int own = first + E * lane;
    const bool whole = VEC && own + E <= P.d;
    float sum[E];
#pragma unroll
    for (int n = 0; n < E; ++n) sum[n] = 0.0f;
    constexpr int kAhead = 2;
#pragma unroll 1
    for (int i0 = path0; i0 < path1; i0 += kAhead) {
        alignas(16) T v[kAhead][E];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            if (i0 + a >= path1) break;
            const T* gi = g + (long long)(i0 - path0 + a) * P.ld_in;
            if (whole) {
                *reinterpret_cast<uint4*>(v[a]) = *reinterpret_cast<const uint4*>(gi + own);
            } else {
#pragma unroll
                for (int n = 0; n < E; ++n) {
                    const int j = VEC ? own + n : first + 32 * n + lane;
                    round_to(0.0f, &v[a][n]);
                    if (j < P.d) v[a][n] = gi[j];
                }
            }
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            if (i0 + a >= path1) break;
            const PhiloxPath path((uint32_t)(i0 + a), t, P.key0);
#pragma unroll
            for (int r = 0; r < Q; ++r) {
                const uint32_t flags = quad[r].keep(path, P.key0, P.key1, P.thr);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const uint32_t f = VEC ? flags >> n : __shfl_sync(0xFFFFFFFFu, flags, 8 * n + (lane >> 2)) >> (lane & 3);
                    if (f & 1u) sum[4 * r + n] += to_float(v[a][4 * r + n]);    // (a dropped NaN stays out)
                }
            }
        }
    }
    if (P.n_groups > 1) {
#pragma unroll
        for (int n = 0; n < E; ++n) s_part[warp][32 * n + lane] = sum[n];
        __syncthreads();
        if (group != 0) return;
        for (int w = 1; w < P.n_groups; ++w)
#pragma unroll
            for (int n = 0; n < E; ++n) sum[n] += s_part[warp + w][32 * n + lane];
    }
    if (!live) return;
    alignas(16) T o[E];
#pragma unroll
    for (int n = 0; n < E; ++n) round_to(sum[n] * P.scale, &o[n]);
    T* out = static_cast<T*>(P.out) + row * P.ld_out;
    if (whole) {
        *reinterpret_cast<uint4*>(out + own) = *reinterpret_cast<const uint4*>(o);
    } else {
#pragma unroll
        for (int n = 0; n < E; ++n) {
            const int j = VEC ? own + n : first + 32 * n + lane;
            if (j < P.d) out[j] = o[n];
        }
    }
}

bool aligned_rows(const void* p, long long ld, int elem) {
    return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * elem)) & 15u) == 0;
}

template <typename T>
int launch(DropoutParams& P, bool grad, cudaStream_t stream) {
    constexpr int kEntries = 32 * 4 * (sizeof(T) == 2 ? 2 : 1);      // of a warp's chunk
    const bool vec = aligned_rows(P.in, P.ld_in, sizeof(T)) && aligned_rows(P.out, P.ld_out, sizeof(T));
    P.n_chunks = (P.d + kEntries - 1) / kEntries;
    long long blocks;
    if (grad) {
        // runs of at least eight paths: what a warp adds up in one go
        P.n_groups = P.K >= 64 ? 8 : P.K >= 32 ? 4 : P.K >= 16 ? 2 : 1;
        P.group_paths = (P.K + P.n_groups - 1) / P.n_groups;
        P.n_tasks = P.rows * P.n_chunks;
        const int per_block = kWarps / P.n_groups;
        blocks = (P.n_tasks + per_block - 1) / per_block;
    } else {
        // a warp takes all paths of its chunk unless that leaves the GPU short of warps (some 16 on each of its SMs)
        const long long chunks = P.rows * P.n_chunks;
        P.group_paths = P.K;
        while (P.group_paths > 1 && chunks * ((P.K + P.group_paths - 1) / P.group_paths) < 2368) P.group_paths = (P.group_paths + 1) / 2;
        P.n_groups = (P.K + P.group_paths - 1) / P.group_paths;
        P.n_tasks = chunks * P.n_groups;
        blocks = (P.n_tasks + kWarps - 1) / kWarps;
    }
    if (blocks > 0x7FFFFFFFll) return DM_EUNSUPPORTED;
    const unsigned grid = (unsigned)blocks;
    if (grad) {
        if (vec) dropout_grad_kernel<T, true><<<grid, kThreads, 0, stream>>>(P);
        else dropout_grad_kernel<T, false><<<grid, kThreads, 0, stream>>>(P);
    } else {
        if (vec) dropout_kernel<T, true><<<grid, kThreads, 0, stream>>>(P);
        else dropout_kernel<T, false><<<grid, kThreads, 0, stream>>>(P);
    }
    return cudaGetLastError() == cudaSuccess ? DM_OK : DM_ECUDA;
}

}  // namespace

int launch_dropout(DropoutParams P, int dtype, bool grad, cudaStream_t stream) {
    return dtype == DM_F32 ? launch<float>(P, grad, stream) : launch<__nv_bfloat16>(P, grad, stream);
}

}  // namespace dm
