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
// What bounds it: the generator, then HBM.  Ten rounds are 20 widening multiplies per quad, at a quarter of the issue rate; in a
// loop over paths a quarter of them stays the same (see PhiloxQuad).  What is left keeps that pipe 72 % and the ALU 57 % busy,
// and takes more: timed alone, the seven rounds are 58 cycles per quad, warp and quarter of an SM, and each integer
// instruction beside them (comparison, selection, address) 2, as if multiplier and ALU were fed through one port.  A quad here has
// some 49 of both: 97 cycles, as many as measured.
// Measured: 4096 rows of 4096 bf16 under 8 paths (302 MB) 92-94 us, where the multiplies alone take 58 and HBM 46;
// the gradient of 976 x 16 rows of 8192 bf16 (272 MB) 98 us; 4084 rows of 5003 fp32 (163 MB, rows off 16-byte boundaries) 39-41 us.
// Round keys as constants, two vectors a lane, divisions by multiplication: 103, 107 and 56 us before.
#include "dm_dropout.h"
namespace dm {

namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr uint32_t kMulA = 0xD2511F53u, kMulB = 0xCD9E8D57u;

__device__ __forceinline__ void mul_wide(uint32_t a, uint32_t b, uint32_t& hi, uint32_t& lo) {
    asm("{\n\t.reg .u64 p;\n\tmul.wide.u32 p, %2, %3;\n\tmov.b64 {%0, %1}, p;\n\t}" : "=r"(lo), "=r"(hi) : "r"(a), "r"(b));
}

// Philox4x32-10 at the counter (quad, path, t, s), cut at what does not change from path to path.
// Round r maps (x, y, z, w) to (hi(B z) ^ y ^ k0, lo(B z), hi(A x) ^ w ^ k1, lo(A x)).  The path index is in y only:
// after round 1 it is in x alone, after round 2 in z and w, so the product B z of round 2 and A x of round 3
// are the quad's, and A x of round 2 is the path's.
struct PhiloxPath {       // the same for all quads of a row
    uint32_t hi2, lo2;    // A x of round 2
    __device__ __forceinline__ PhiloxPath(uint32_t path, uint32_t t, const DropoutParams& P) {
        uint32_t hi, lo;
        mul_wide(kMulB, t, hi, lo);
        mul_wide(kMulA, hi ^ path ^ P.key[0][0], hi2, lo2);
    }
};
struct PhiloxQuad {       // the same for all paths
    uint32_t z2, y2, z3, w3;
    __device__ __forceinline__ PhiloxQuad() {}
    __device__ __forceinline__ PhiloxQuad(uint32_t quad, uint32_t t, uint32_t s, const DropoutParams& P) {
        uint32_t hi_t, lo_t, hi, w1, x2;
        mul_wide(kMulB, t, hi_t, lo_t);
        mul_wide(kMulA, quad, hi, w1);
        mul_wide(kMulB, hi ^ s ^ P.key[0][1], x2, y2);
        x2 ^= lo_t ^ P.key[1][0];
        z2 = w1 ^ P.key[1][1];
        mul_wide(kMulA, x2, z3, w3);
        z3 ^= P.key[2][1];
        y2 ^= P.key[2][0];
    }
    __device__ __forceinline__ uint4 words(const PhiloxPath& p, const DropoutParams& P) const {
        uint4 c;
        mul_wide(kMulB, p.hi2 ^ z2, c.x, c.y);      // round 3
        c.x ^= y2;
        c.z = z3 ^ p.lo2;
        c.w = w3;
#pragma unroll
        for (int r = 3; r < 10; ++r) {
            uint32_t hi_a, lo_a, hi_b, lo_b;
            mul_wide(kMulA, c.x, hi_a, lo_a);
            mul_wide(kMulB, c.z, hi_b, lo_b);
            c = make_uint4(hi_b ^ c.y ^ P.key[r][0], lo_b, hi_a ^ c.w ^ P.key[r][1], lo_a);
        }
        return c;
    }
    __device__ __forceinline__ uint32_t keep(const PhiloxPath& p, const DropoutParams& P) const {
        const uint4 w = words(p, P);
        const uint32_t thr = P.thr;
        return (w.x >= thr ? 1u : 0u) | (w.y >= thr ? 2u : 0u) | (w.z >= thr ? 4u : 0u) | (w.w >= thr ? 8u : 0u);
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
__device__ __forceinline__ void add_to(float& sum, float x) { sum += x; }
__device__ __forceinline__ void add_to(float& sum, __nv_bfloat16 x) {
    asm("add.rn.f32.bf16 %0, %1, %0;" : "+f"(sum) : "h"(__bfloat16_as_ushort(x)));      // (exact conversion, one rounding)
}
__device__ __forceinline__ void round_to(float x, float* out) { *out = x; }
__device__ __forceinline__ void round_to(float x, __nv_bfloat16* out) { *out = __float2bfloat16_rn(x); }

// Quads and entries of a lane: NV vectors of 16 bytes.
template <typename T, int NV> constexpr int kQuads = NV * 4 / (int)sizeof(T);
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);

// T: storage type.  VEC: every row starts on a 16-byte boundary; lane l's vector i is the chunk's vector 32 i + l (entries past
// the last whole vector of a row are then read and written one by one by the same lane).  Otherwise lane l generates the
// quads 32 r + l and reads and writes the entries 32 n + l.
template <typename T, bool VEC, int NV>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(const __grid_constant__ DropoutParams P) {
    constexpr int Q = kQuads<T, NV>, E = 4 * Q, V = kVec<T>;
    const uint32_t task = blockIdx.x * kWarps + warp_index();
    if (task >= P.n_tasks) return;                           // (the same for the whole warp)
    const uint32_t run = P.by_chunks.div(task), row = P.by_groups.div(run), b = P.by_T.div(row);
    const int first = (int)(task - run * P.by_chunks.d) * (32 * E), path0 = (int)(run - row * P.by_groups.d) * P.group_paths;
    const int path1 = min(P.K, path0 + P.group_paths), lane = threadIdx.x & 31;
    const uint32_t t = P.shared_masks ? 0u : row - b * P.by_T.d, s = P.seq_base_lo + b;
    const T* x = static_cast<const T*>(P.in) + row * P.ld_in;
    T* out = static_cast<T*>(P.out) + ((long long)row * P.K + path0) * P.ld_out;
    PhiloxQuad quad[Q];
#pragma unroll
    for (int r = 0; r < Q; ++r)
        quad[r] = PhiloxQuad((uint32_t)first / 4 + (VEC ? (32 * (r / (V / 4)) + lane) * (V / 4) + r % (V / 4) : 32 * r + lane), t, s, P);
    alignas(16) T v[E];      // x / (1 - p), rounded once
    const auto at = [&](int n) { return VEC ? first + V * (32 * (n / V) + lane) + n % V : first + 32 * n + lane; };      // of the lane's entry n
#pragma unroll
    for (int n = 0; n < E; n += V) {
        if (VEC && at(n) + V <= P.d) {
            *reinterpret_cast<uint4*>(v + n) = *reinterpret_cast<const uint4*>(x + at(n));
        } else {
#pragma unroll
            for (int k = n; k < n + V; ++k) {
                round_to(0.0f, &v[k]);
                if (at(k) < P.d) v[k] = x[at(k)];
            }
        }
    }
#pragma unroll
    for (int n = 0; n < E; ++n) round_to(to_float(v[n]) * P.scale, &v[n]);
    T zero;
    round_to(0.0f, &zero);
#pragma unroll 1
    for (int i = path0; i < path1; ++i, out += P.ld_out) {
        const PhiloxPath path((uint32_t)i, t, P);
        if (VEC) {
            alignas(16) uint32_t o[E * sizeof(T) / 4];
#pragma unroll
            for (int r = 0; r < Q; ++r)
                keep_words(reinterpret_cast<const uint32_t*>(v) + sizeof(T) * r, quad[r].words(path, P), P.thr, o + sizeof(T) * r, zero);
#pragma unroll
            for (int n = 0; n < E; n += V) {
                if (at(n) + V <= P.d) {
                    *reinterpret_cast<uint4*>(out + at(n)) = reinterpret_cast<const uint4*>(o)[n / V];
                } else {
#pragma unroll
                    for (int k = n; k < n + V; ++k)
                        if (at(k) < P.d) out[at(k)] = reinterpret_cast<const T*>(o)[k];
                }
            }
        } else {
#pragma unroll
            for (int r = 0; r < Q; ++r) {
                const uint32_t flags = quad[r].keep(path, P);
#pragma unroll
                for (int n = 0; n < 4; ++n) {      // entries 128 r + 32 n + lane: quad 8 n + lane / 4 of the 32
                    const uint32_t f = __shfl_sync(0xFFFFFFFFu, flags, 8 * n + (lane >> 2));
                    if (at(4 * r + n) < P.d) out[at(4 * r + n)] = (f >> (lane & 3)) & 1u ? v[4 * r + n] : zero;
                }
            }
        }
    }
}

// Sums over the paths: fp32, paths in order within a run of them; long sums are cut into n_groups runs that
// neighbouring warps of a block take and the first of them joins in order.  The cut follows from K alone, so that
// a row's result does not depend on the others.
template <typename T, bool VEC, int NV>
__global__ void __launch_bounds__(kThreads, 3)
dropout_grad_kernel(const __grid_constant__ DropoutParams P) {
    constexpr int Q = kQuads<T, NV>, E = 4 * Q, V = kVec<T>;
    __shared__ float s_part[kWarps][E * 32];
    const int warp = warp_index(), lane = threadIdx.x & 31, n_groups = (int)P.by_groups.d;
    const int group = warp & (n_groups - 1);                 // (a power of two, at most kWarps)
    const uint32_t task = blockIdx.x * (uint32_t)(kWarps / n_groups) + P.by_groups.div(warp);
    const bool live = task < P.n_tasks;
    const uint32_t row = live ? P.by_chunks.div(task) : 0u, b = P.by_T.div(row);
    const int first = live ? (int)(task - row * P.by_chunks.d) * (32 * E) : 0;
    const int path0 = min(P.K, group * P.group_paths), path1 = live ? min(P.K, path0 + P.group_paths) : path0;
    const uint32_t t = P.shared_masks ? 0u : row - b * P.by_T.d, s = P.seq_base_lo + b;
    PhiloxQuad quad[Q];
#pragma unroll
    for (int r = 0; r < Q; ++r)
        quad[r] = PhiloxQuad((uint32_t)first / 4 + (VEC ? (32 * (r / (V / 4)) + lane) * (V / 4) + r % (V / 4) : 32 * r + lane), t, s, P);
    const T* g = static_cast<const T*>(P.in) + ((long long)row * P.K + path0) * P.ld_in;
    const auto at = [&](int n) { return VEC ? first + V * (32 * (n / V) + lane) + n % V : first + 32 * n + lane; };
    float sum[E];
#pragma unroll
    for (int n = 0; n < E; ++n) sum[n] = 0.0f;
    alignas(16) T v[2][E];       // the next path's entries are on their way while one is added
    const auto load = [&](T (&to)[E]) {
#pragma unroll
        for (int n = 0; n < E; n += V) {
            if (VEC && at(n) + V <= P.d) {
                *reinterpret_cast<uint4*>(to + n) = *reinterpret_cast<const uint4*>(g + at(n));
            } else {
#pragma unroll
                for (int k = n; k < n + V; ++k) {
                    round_to(0.0f, &to[k]);
                    if (at(k) < P.d) to[k] = g[at(k)];
                }
            }
        }
        g += P.ld_in;
    };
    const auto add = [&](int i, const T (&from)[E]) {
        const PhiloxPath path((uint32_t)i, t, P);
#pragma unroll
        for (int r = 0; r < Q; ++r) {
            if (VEC) {
                const uint4 w = quad[r].words(path, P);
                if (w.x >= P.thr) add_to(sum[4 * r + 0], from[4 * r + 0]);      // (a dropped NaN stays out)
                if (w.y >= P.thr) add_to(sum[4 * r + 1], from[4 * r + 1]);
                if (w.z >= P.thr) add_to(sum[4 * r + 2], from[4 * r + 2]);
                if (w.w >= P.thr) add_to(sum[4 * r + 3], from[4 * r + 3]);
            } else {
                const uint32_t flags = quad[r].keep(path, P);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const uint32_t f = __shfl_sync(0xFFFFFFFFu, flags, 8 * n + (lane >> 2));
                    if ((f >> (lane & 3)) & 1u) add_to(sum[4 * r + n], from[4 * r + n]);
                }
            }
        }
    };
    if (path0 < path1) load(v[0]);
#pragma unroll 1
    for (int i = path0; i < path1; i += 2) {
        if (i + 1 < path1) load(v[1]);
        add(i, v[0]);
        if (i + 2 < path1) load(v[0]);
        if (i + 1 < path1) add(i + 1, v[1]);
    }
    if (n_groups > 1) {
#pragma unroll
        for (int n = 0; n < E; ++n) s_part[warp][32 * n + lane] = sum[n];
        __syncthreads();
        if (group != 0) return;
        for (int w = 1; w < n_groups; ++w)
#pragma unroll
            for (int n = 0; n < E; ++n) sum[n] += s_part[warp + w][32 * n + lane];
    }
    if (!live) return;
    alignas(16) T o[E];
#pragma unroll
    for (int n = 0; n < E; ++n) round_to(sum[n] * P.scale, &o[n]);
    T* out = static_cast<T*>(P.out) + row * P.ld_out;
#pragma unroll
    for (int n = 0; n < E; n += V) {
        if (VEC && at(n) + V <= P.d) {
            *reinterpret_cast<uint4*>(out + at(n)) = *reinterpret_cast<const uint4*>(o + n);
        } else {
#pragma unroll
            for (int k = n; k < n + V; ++k)
                if (at(k) < P.d) out[at(k)] = o[k];
        }
    }
}

bool aligned_rows(const void* p, long long ld, int elem) {
    return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * elem)) & 15u) == 0;
}

template <typename T, int NV>
int launch(DropoutParams& P, bool grad, cudaStream_t stream) {
    constexpr int kEntries = 32 * 4 * kQuads<T, NV>;      // of a warp's chunk
    const bool vec = aligned_rows(P.in, P.ld_in, sizeof(T)) && aligned_rows(P.out, P.ld_out, sizeof(T));
    const long long n_chunks = (P.d + kEntries - 1) / kEntries, chunks = P.rows * n_chunks;
    int n_groups;
    long long tasks, blocks;
    if (grad) {
        // runs of at least eight paths: what a warp adds up in one go
        n_groups = P.K >= 64 ? 8 : P.K >= 32 ? 4 : P.K >= 16 ? 2 : 1;
        P.group_paths = (P.K + n_groups - 1) / n_groups;
        tasks = chunks;
        const int per_block = kWarps / n_groups;
        blocks = (tasks + per_block - 1) / per_block;
    } else {
        // a warp takes all paths of its chunk unless that leaves the GPU short of warps (some 16 on each of its SMs)
        P.group_paths = P.K;
        while (P.group_paths > 1 && chunks * ((P.K + P.group_paths - 1) / P.group_paths) < 2368) P.group_paths = (P.group_paths + 1) / 2;
        n_groups = (P.K + P.group_paths - 1) / P.group_paths;
        tasks = chunks * n_groups;
        blocks = (tasks + kWarps - 1) / kWarps;
    }
    if (tasks > 0x7FFFFFF0ll) return DM_EUNSUPPORTED;
    P.n_tasks = (uint32_t)tasks;
    P.by_chunks = Divisor((uint32_t)n_chunks);
    P.by_groups = Divisor((uint32_t)n_groups);
    P.by_T = Divisor((uint32_t)P.T);
    const unsigned grid = (unsigned)blocks;
    if (grad) {
        if (vec) dropout_grad_kernel<T, true, NV><<<grid, kThreads, 0, stream>>>(P);
        else dropout_grad_kernel<T, false, NV><<<grid, kThreads, 0, stream>>>(P);
    } else {
        if (vec) dropout_kernel<T, true, NV><<<grid, kThreads, 0, stream>>>(P);
        else dropout_kernel<T, false, NV><<<grid, kThreads, 0, stream>>>(P);
    }
    return cudaGetLastError() == cudaSuccess ? DM_OK : DM_ECUDA;
}

template <typename T>
int launch_wide(DropoutParams& P, bool grad, cudaStream_t stream) {
    // two vectors a lane share the paths' part of the generator and the keys; short rows would leave lanes idle, small calls warps
    const long long chunks = P.rows * ((P.d + 64 * kVec<T> - 1) / (64 * kVec<T>));
    const bool wide = P.d >= 64 * kVec<T> && chunks >= 2368;
    return wide ? launch<T, 2>(P, grad, stream) : launch<T, 1>(P, grad, stream);
}

}  // namespace

int launch_dropout(DropoutParams P, const MaskKey& mk, int dtype, bool grad, cudaStream_t stream) {
    P.thr = mk.thr;
    P.scale = mk.scale;
    for (uint32_t r = 0; r < 10; ++r) {
        P.key[r][0] = mk.key0 + r * 0x9E3779B9u;
        P.key[r][1] = mk.key1 + r * 0xBB67AE85u;
    }
    return dtype == DM_F32 ? launch_wide<float>(P, grad, stream) : launch_wide<__nv_bfloat16>(P, grad, stream);
}

}  // namespace dm
