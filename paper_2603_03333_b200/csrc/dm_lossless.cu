// dropmatch_verify_lossless: drafted tokens against the target's distribution, from given random numbers.
//
//   p_t = Softmax(target[t] / T),  q_t = Softmax(draft[t] / T_d)  (or all of q_t on the drafted token x_t)
//   accept x_t  <=>  u_t q_t(x_t) < p_t(x_t);   n = length of the accepted prefix
//   next ~ max(p_n - q_n, 0) / sum  (n < drafted)  or  p_n  (all accepted),  by inverse CDF in token order:
//   the first v with  sum_{w <= v} r(w) > u_next sum r
//
// Two kernels, no workspace.
// ratio_kernel: a cluster per drafted position reads both rows once (sums of fp32 exponentials against a running reference)
// and leaves min(1, p / q) in out_accept_prob.  Bounds: HBM, with the exponentials close behind (16 per cycle and SM).
// next_kernel: a cluster per sequence finds n and draws from row n.  Bounds: the fp64 exponentials of one row of each model.
// Decisions and the place in the cumulative sum are those of 64-bit arithmetic: a position whose u_t lies within 2^-15 of the fp32 ratio (more than that
// can be off, see kBand) is decided again from fp64 sums, and all sums over row n are fp64 with exponentials good to
// 2^-42 (see weight).  In fp32 a token of the flat tail of 100 thousand would come out one place off in about a
// draw of ten, and two engines with equal random numbers would drift apart.
// Measured: 96 sequences of 7 tokens, 151936 bf16 entries, both models (408 MB) 150 us (135 back to back in a graph): 73 + 74,
// where HBM takes 62; one sequence of 5 tokens of 128256 18-20 us (14 in a graph), 4 tokens of 4096 fp32 14 (9).  Rows through registers instead of the ring, per-thread joins and
// two fp64 passes took 396 and 89; ratios and draws in one kernel, a cluster going through its sequence's rows, 160 and 22.
#include <math.h>
#include <string.h>

#include <atomic>

#include "dm_lossless.h"
#include "dm_ptx.cuh"

namespace dm {

namespace {

constexpr int kMaxCluster = 16;      // (more than 8 has to be asked for)
constexpr int kRatioThreads = 256, kRatioWarps = kRatioThreads / 32;
// The fp32 ratio is p / q with the sums of two rows.  A term 2^w, w = (x - m) c, has a relative error of at most
// 2 |w| ln 2 2^-24 (two roundings) + 2^-24 |w| ln 2 (c) + 2^-22 (the instruction); the mean of |w| ln 2 under the
// row's own distribution is at most ln V + 20 ln 2 <= 35 (m lies up to 20 powers of two below the maximum), a batch adds 7
// roundings, each of three joins an instruction and at most 5: (105 + 4 + 7 + 30) 2^-24 < 2^-16, for two rows and with u and
// the ratio rounded still within 2^-15.
constexpr float kBand = 1.0f / 32768.0f;

__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xFF800000u); }
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void st_cluster_f64(uint32_t addr, double v) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory");
}

__device__ __forceinline__ float entry(const float* row, long long j) { return row[j]; }
__device__ __forceinline__ float entry(const __nv_bfloat16* row, long long j) { return __bfloat162float(row[j]); }

// ---------------------------------------------------------------------------------------- ratios

template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int kN = 4;
    static constexpr uint32_t kNone = 0xFF800000u;      // -inf
    __device__ static void unpack(const uint4& v, float* x) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
    template <int N> __device__ static float max(const uint4 (&v)[N]) {
        float m = neg_inf();
#pragma unroll
        for (int i = 0; i < N; ++i)
            m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(v[i].x), __uint_as_float(v[i].y)), fmaxf(__uint_as_float(v[i].z), __uint_as_float(v[i].w))));
        return m;
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int kN = 8;
    static constexpr uint32_t kNone = 0xFF80FF80u;
    __device__ static void unpack(const uint4& v, float* x) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
    template <int N> __device__ static float max(const uint4 (&v)[N]) {      // two entries per instruction
        uint32_t m = kNone;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[k]));
        }
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    }
};

// Sum of exp((x - m) / T) over some entries of a row, with what additions have lost of it (Kahan: a thread's share of a row may
// be any number of batches).  m is an entry of which no other exceeds the 2^20-fold: it moves only beyond that, so that a
// row in ascending order does not round its sum anew with every batch.  A NaN, and +inf, make the sum a NaN.
struct Sum {
    float m = neg_inf(), s = 0.0f, lost = 0.0f;

    template <int N>
    __device__ __forceinline__ void add(const float (&x)[N], float bm, float c) {      // N entries whose maximum is bm
        if ((bm - m) * c > 20.0f) {
            const float f = ex2((m - bm) * c);       // (0 at the first batch; a NaN stays)
            s *= f;
            lost *= f;
            m = bm;
        }
        const float ref = m == neg_inf() ? 0.0f : m;      // nothing but -inf so far: every term 0
        const float2 m2 = make_float2(-ref, -ref), c2 = make_float2(c, c);
        float2 t[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float2 z = __fmul2_rn(__fadd2_rn(make_float2(x[i], x[i + 1]), m2), c2);
            t[(i >> 1) & 1] = __fadd2_rn(t[(i >> 1) & 1], make_float2(ex2(z.x), ex2(z.y)));
        }
        const float y = ((t[0].x + t[0].y) + (t[1].x + t[1].y)) - lost, sum = s + y;
        lost = (sum - s) - y;
        s = sum;
    }
};

// Entries [lo, hi) of a row: 16-byte vectors, and the ragged ends entry by entry.
template <typename T>
struct Share {
    static constexpr int kN = Vec<T>::kN;
    const T* row;
    const uint4* body;
    int lo, head, vecs, tail, hi;     // entries [lo, head) and [tail, hi) lie outside the vectors: at most kN - 1 each
    __device__ __forceinline__ Share(const T* r, int l, int h) : row(r), lo(l), hi(h) {
        const int off = (int)((reinterpret_cast<uintptr_t>(r + l) & 15u) / sizeof(T));
        head = min(h, l + (off == 0 ? 0 : kN - off));
        vecs = (h - head) / kN;
        tail = head + vecs * kN;
        body = reinterpret_cast<const uint4*>(r + head);
    }
    template <int N>
    __device__ __forceinline__ static void add(Sum& a, const uint4 (&v)[N], float c) {
        float x[N * kN];
#pragma unroll
        for (int i = 0; i < N; ++i) Vec<T>::unpack(v[i], x + i * kN);
        a.add(x, Vec<T>::max(v), c);
    }
    __device__ __forceinline__ void add_ends(Sum& a, float c) const {
        if (threadIdx.x >= 2 * kN) return;
        const int j = threadIdx.x < kN ? lo + (int)threadIdx.x : tail + (int)threadIdx.x - kN;
        const bool have = threadIdx.x < kN ? j < head : j < hi;
        const float x[2] = {have ? entry(row, j) : neg_inf(), neg_inf()};
        a.add(x, x[0], c);
    }
};

// Sum of exp relative to a maximum above the thread's or warp's own.
__device__ __forceinline__ float rescaled(float m, float s, float to, float c) { return m == to ? s : s * ex2((m - to) * c); }
__device__ __forceinline__ float warp_max(float x) {
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));      // (leaves a NaN out)
    return y;
}
// Largest reference and sum over the lanes of a warp, the same bits in every lane.
__device__ __forceinline__ float2 join_lanes(float m, float s, float c) {
    const float top = warp_max(m);
    s = rescaled(m, s, top, c);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, off);
    return make_float2(top, s);
}
// ... over n <= 32 parts in shared memory, `stride` apart.
__device__ __forceinline__ float2 join_parts(const float2* part, int n, int stride, float c) {
    const int lane = threadIdx.x & 31;
    const float2 p = lane < n ? part[lane * stride] : make_float2(neg_inf(), 0.0f);
    return join_lanes(p.x, p.y, c);
}

__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Every thread streams its vectors of the rows through its own slots of a ring in shared memory (no barrier: nobody
// else reads them), kStages batches ahead.
template <bool HAS_Q> constexpr int kVecs = HAS_Q ? 2 : 4;       // vectors of a row in a batch
constexpr int kStages = 4;      // (three or six: 3 to 8 % slower)
constexpr int kRatioSmem = kStages * 4 * kRatioThreads * 16;

template <typename TP, typename TQ, bool HAS_Q>
__global__ void __launch_bounds__(kRatioThreads)
ratio_kernel(const __grid_constant__ LosslessParams P, int cluster) {
    extern __shared__ __align__(16) unsigned char s_ring[];
    __shared__ __align__(16) float2 s_warp[kRatioWarps][2];     // maximum and sum of the target's row, of the draft's
    __shared__ __align__(16) float2 s_part[kMaxCluster][2];     // of every CTA, written by it into the first
    ptx::griddep_launch_dependents();
    const int pos = (int)(blockIdx.x / (unsigned)cluster), rank = (int)(blockIdx.x % (unsigned)cluster);
    const int b = pos / P.T, t = pos - b * P.T;
    if (P.draft_len != nullptr && t >= P.draft_len[b]) {       // (the same for the whole cluster)
        if (rank == 0 && threadIdx.x == 0) P.out_accept_prob[pos] = 0.0f;
        return;
    }
    // (arrives; whoever has waited may write to the other CTAs' shared memory)
    if (cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const TP* row_p = static_cast<const TP*>(P.target) + ((long long)b * (P.T + P.bonus) + t) * P.ld_target;
    const TQ* row_q = static_cast<const TQ*>(P.draft_logits) + (long long)pos * P.ld_draft;
    const int lo = (int)min((long long)P.V, (long long)rank * P.share), hi = (int)min((long long)P.V, (long long)lo + P.share);
    const Share<TP> sp(row_p, lo, hi);
    const Share<TQ> sq(row_q, lo, HAS_Q ? hi : lo);

    constexpr int kV = kVecs<HAS_Q>, kRows = HAS_Q ? 2 : 1;
    const uint4* slots = reinterpret_cast<const uint4*>(s_ring) + threadIdx.x;       // [stage][row][vector][thread]
    const uint32_t slots_smem = ptx::smem_u32(slots);
    const auto fetch = [&](int batch) {      // (an empty group past the end keeps the count)
        const uint32_t to = slots_smem + (uint32_t)(batch % kStages) * (kRows * kV * kRatioThreads * 16);
        const int v0 = batch * kV * kRatioThreads + (int)threadIdx.x;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const int v = v0 + i * kRatioThreads;
            if (v < sp.vecs) copy_async(to + i * kRatioThreads * 16, sp.body + v);
            if (HAS_Q && v < sq.vecs) copy_async(to + (kV + i) * kRatioThreads * 16, sq.body + v);
        }
        copies_commit();
    };
    const int both = HAS_Q ? min(sp.vecs, sq.vecs) : sp.vecs, most = max(sp.vecs, sq.vecs);
    const int n_batches = (most + kV * kRatioThreads - 1) / (kV * kRatioThreads);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(i);
    const int tok = P.draft[pos];
    const bool in_range = (unsigned)tok < (unsigned)P.V;
    float xp = 0.0f, xq = 0.0f;
    if (rank == 0 && threadIdx.x == 0 && in_range) {
        xp = entry(row_p, tok);
        if (HAS_Q) xq = entry(row_q, tok);
    }
    Sum p, q;
    sp.add_ends(p, P.c);
    if (HAS_Q) sq.add_ends(q, P.c_draft);
#pragma unroll 1
    for (int batch = 0; batch < n_batches; ++batch) {
        fetch(batch + kStages - 1);
        copies_wait<kStages - 1>();
        const uint4* at = slots + (batch % kStages) * (kRows * kV * kRatioThreads);
        const int v0 = batch * kV * kRatioThreads + (int)threadIdx.x;
        if (v0 + (kV - 1) * kRatioThreads < both) {
            uint4 v[kV];
#pragma unroll
            for (int i = 0; i < kV; ++i) v[i] = at[i * kRatioThreads];
            sp.add(p, v, P.c);
            if (HAS_Q) {
#pragma unroll
                for (int i = 0; i < kV; ++i) v[i] = at[(kV + i) * kRatioThreads];
                sq.add(q, v, P.c_draft);
            }
        } else {      // the last batch, and of rows of different types the half of the wider one that has no counterpart
#pragma unroll 1
            for (int i = 0; i < kV; ++i) {
                if (v0 + i * kRatioThreads < sp.vecs) {
                    const uint4 v[1] = {at[i * kRatioThreads]};
                    sp.add(p, v, P.c);
                }
                if (HAS_Q && v0 + i * kRatioThreads < sq.vecs) {
                    const uint4 v[1] = {at[(kV + i) * kRatioThreads]};
                    sq.add(q, v, P.c_draft);
                }
            }
        }
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float2 wp = join_lanes(p.m, p.s, P.c), wq = HAS_Q ? join_lanes(q.m, q.s, P.c_draft) : make_float2(0.0f, 1.0f);
    if (lane == 0) { s_warp[warp][0] = wp; s_warp[warp][1] = wq; }
    __syncthreads();
    // warp 0 takes the target's parts, warp 1 the draft's
    float2 all = make_float2(0.0f, 1.0f);
    const bool mine = warp < kRows;
    const float c = warp == 0 ? P.c : P.c_draft;
    if (mine) all = join_parts(&s_warp[0][warp], kRatioWarps, 2, c);
    if (cluster > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        if (mine && lane == 0) {
            const uint32_t to = ptx::map_to_cta(ptx::smem_u32(&s_part[rank][warp]), 0);
            ptx::st_cluster_u32(to, __float_as_uint(all.x));
            ptx::st_cluster_u32(to + 4, __float_as_uint(all.y));
        }
        __syncwarp();
        ptx::cluster_sync_all();
        if (rank != 0) return;
        if (mine) all = join_parts(&s_part[0][warp], cluster, 2, c);
    }
    if (HAS_Q) {
        __syncthreads();
        if (warp == 1 && lane == 0) s_warp[0][1] = all;
        __syncthreads();
    }
    if (threadIdx.x != 0) return;
    const float2 other = HAS_Q ? s_warp[0][1] : make_float2(0.0f, 1.0f);
    float ratio = 0.0f;
    if (isnan(all.y) || isnan(other.y)) {
        ratio = __uint_as_float(0x7FC00000u);
    } else if (in_range && xp > neg_inf()) {          // (a row of nothing but -inf has no such entry)
        double l = ((double)xp - (double)all.x) * P.inv_temp - log((double)all.y);
        if (HAS_Q) l -= ((double)xq - (double)other.x) * P.inv_draft_temp - log((double)other.y);
        ratio = HAS_Q && xq == neg_inf() ? 1.0f : fminf((float)exp(l), 1.0f);
    }
    P.out_accept_prob[pos] = ratio;
}

// ------------------------------------------------------------------------------------------ next

// exp((x - m) / T) for x <= m in fp64, up to a factor that is the same for all entries of a row, straight through: with
// k = round(16 log2(e) x / T) and r = x - k T ln2/16 it is 2^((k - k0)/16) e^(r/T), k0 the row's (that of its maximum), so that
// 2^((k - k0)/16) = 2^e table[j], j the low four bits of k - k0; e^(r/T) by its Taylor polynomial, the powers of
// 1/T and the factorials in the coefficients: table-driven reduction after Tang, ACM TOMS 15 (1989).  |r/T| <= ln2/32, so
// what the polynomial leaves out is below 2^-42 of the value.  Twenty instructions, eight of them fp64; with a
// polynomial for |r/T| <= ln2/2 that needs no table, three fp64 instructions more.  Sixteen doubles lie in as many pairs of banks: lanes never
// conflict.  Where k would be beyond 2^17, x - m takes x's place: fp32 holds it exactly for every entry that counts.
// x = -inf, and what lies below e^-700 of the reference: 0.  A NaN, or +inf (then m is +inf too): NaN.
struct Row64 {
    float ref, bias;      // m or 0; 1.5 2^23 - k0
    double offset;        // 2^52 + (bits of 1.5 2^23) - k0
    double base;          // the x of weight 1
    __device__ __forceinline__ Row64() {}
    __device__ __forceinline__ Row64(float m, const Exp64& E) {
        const bool far = fabsf(m) * E.c16 >= 131072.0f, none = m == neg_inf();
        ref = far && !none ? m : 0.0f;
        const float k0 = far ? 0.0f : rintf(m * E.c16);
        bias = 12582912.0f - k0;
        offset = 4503599627370496.0 + 1262485504.0 - (double)k0;
        base = (double)ref + (double)k0 * E.step;
    }
};
__device__ __forceinline__ double weight(float x, const Row64& R, const Exp64& E, const double* table) {
    const float d = x - R.ref, kf = fmaf(d, E.c16, R.bias);      // 1.5 2^23 + (k - k0): rounded to whole numbers, in the low bits
    const int bits = __float_as_int(fmaxf(kf, 12582912.0f - 16300.0f));
    const double k = __hiloint2double(0x43300000, bits) - R.offset;
    const double r = fma(-k, E.step, (double)d);
    double e = fma(r, E.a[4], E.a[3]);
    e = fma(r, e, E.a[2]);
    e = fma(r, e, E.a[1]);
    e = fma(r, e, E.a[0]);
    e = fma(r, e, 1.0);
    const double t = table[bits & 15];       // (its high word is less j 2^16, so that adding all of k - k0 there adds the exponent)
    e *= __hiloint2double((int)((uint32_t)__double2hiint(t) + ((uint32_t)bits << 16)), __double2loint(t));
    return kf < 12582912.0f - 16160.0f ? 0.0 : e;
}
// Is a row's largest entry far from fp64's ends, measured from the row's reference, so that nothing of it can have been lost?
__device__ __forceinline__ bool in_reach(float top, const Row64& R, const Exp64& E) {
    const float kf = fmaf(top - R.ref, E.c16, R.bias);
    return kf > 12582912.0f - 500.0f && kf < 12582912.0f + 15000.0f;
}
// A reference for a row's weights that need not be its maximum.
__device__ __forceinline__ bool near_zero(float x, const Exp64& E) { return fabsf(x) * E.c16 < 131072.0f; }

// Which of the lanes' parts (of a CTA, of a warp) holds the place `at` of their cumulative weight; `at` becomes the place
// within it.  Where rounding (or a random number of 1) leaves none, the last part with any weight, and no place in it is reached.
__device__ __forceinline__ int part_of(double& at, double w) {
    const int lane = threadIdx.x & 31;
    const bool any = w > 0.0;
    double sum = any ? w : 0.0;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const double o = __shfl_up_sync(0xFFFFFFFFu, sum, off);
        if (lane >= off) sum += o;
    }
    double before = __shfl_up_sync(0xFFFFFFFFu, sum, 1);
    if (lane == 0) before = 0.0;
    const uint32_t with = __ballot_sync(0xFFFFFFFFu, any), reached = __ballot_sync(0xFFFFFFFFu, any && at < sum);
    if (reached == 0) {
        at = __longlong_as_double(0x7FF0000000000000ll);
        return with == 0 ? 0 : 31 - __clz(with);
    }
    const int pick = __ffs(reached) - 1;
    at -= __shfl_sync(0xFFFFFFFFu, before, pick);
    return pick;
}

constexpr int kNone = 0x7FFFFFFF;
constexpr double kAbove = 1.0 + 9.094947017729282e-13;     // 1 + 2^-40: what p has to exceed q by for the difference to count

template <int kNextWarps>
struct NextShared {
    double table[16];
    float2 warp_sum[kNextWarps][2];
    double warp_part[kNextWarps][4];
    float2 warp_top[kNextWarps], top[2][kMaxCluster];
    int warp_closest[kNextWarps], closest[2][kMaxCluster];
    double part[2][kMaxCluster][4];     // of every CTA, written by it; two sets in turn, so that one barrier per exchange does
    double scan[kNextWarps];
    int found, last;
    int tok[32];                        // of 32 positions: drafted token, random number, logits
    float u[32], x[32], y[32], ratio[32];
    float behind, u_next;
};

// Lane i of warp 0 hands v, top and closest to CTA i of the cluster: everybody's numbers for everybody.
template <typename S_>
__device__ __forceinline__ void exchange(S_& S, int set, int rank, int cluster, const double (&v)[4], float2 top, int closest) {
    if (threadIdx.x < (unsigned)cluster) {
        const uint32_t at = ptx::map_to_cta(ptx::smem_u32(&S.top[set][rank]), threadIdx.x);
        ptx::st_cluster_u32(at, __float_as_uint(top.x));
        ptx::st_cluster_u32(at + 4, __float_as_uint(top.y));
        ptx::st_cluster_u32(ptx::map_to_cta(ptx::smem_u32(&S.closest[set][rank]), threadIdx.x), (uint32_t)closest);
        const uint32_t to = ptx::map_to_cta(ptx::smem_u32(&S.part[set][rank][0]), threadIdx.x);
#pragma unroll
        for (int i = 0; i < 4; ++i) st_cluster_f64(to + 8 * i, v[i]);
    }
    __syncwarp();
    ptx::cluster_sync_all();
}
// a += t and d += q where t > 0, by predicate: a branch would part the exponentials, a selection costs four instructions.
__device__ __forceinline__ void add_if_above(double t, double q, double& a, double& d) {
    asm("{\n\t.reg .pred more;\n\t"
        "setp.gt.f64 more, %2, 0d0000000000000000;\n\t"
        "@more add.rn.f64 %0, %0, %2;\n\t"
        "@more add.rn.f64 %1, %1, %3;\n\t}"
        : "+d"(a), "+d"(d) : "d"(t), "d"(q));
}
// Sums over the lanes, the same bits in every lane.
__device__ __forceinline__ void add_lanes(double (&a)[4]) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] += __shfl_xor_sync(0xFFFFFFFFu, a[i], off);
}

// The row that a token is drawn from.  Weights of entry v, in units of 1 / sum p:
//   p(v) = exp(x / T) up to a factor (see Row64),  q(v) likewise,  r(v) = max(p(v) - rho q(v), 0)  with rho = sum p / sum q.
// A difference of less than 2^-40 p counts as 0: next to a token that both are certain of it would be rounding (the
// exponentials are good to 2^-42), and outweigh a rest of 1e-90 that is not.  So entry v counts where
// t(v) = p(v) - border q(v) > 0, border = rho (1 + 2^-40).
// Sums over r need rho, which needs the sums over p and q: one pass takes all of them, with a border from an fp32
// rho (off by some 2^-22) that the first kernel, or a quick pass over the row, has left behind.  With sums A of t and D of q over
// the entries that counted, sum r = A + (border - rho) D for the rho that came out, if the same entries count against
// the right border.  An entry changes sides only if the border is off by |t| / q or more, so the pass also notes the entry
// that comes closest to it: the largest difference of the high words of p and |t|, taken as whole numbers, which are logarithms to
// within 0.0861 + 2^-19, in 2^-20 of a power of two (see nearest).  Where the border was off by as much as that, an entry of any weight
// may have been on the wrong side - most of the row, if the draft agrees with the target on most of the vocabulary - and
// the pass is done once more, with the right border (3 of 1183 rows of 151936 bf16 entries, the draft's noise 0.5).
// (Two passes in any case, the first for rho, took 40 % longer.)

// How far, at least, every entry of a row is from `border`, as a difference of borders: |t| >= g p, and p = t + border q, give
// |t| / q >= border g / (1 + g).
__device__ __forceinline__ double nearest(double border, int closest) {
    const float g = exp2f(-9.5367431640625e-7f * (float)closest - 0.0875f);
    return border * (double)g / (1.0 + (double)g);
}
__device__ __forceinline__ int closeness(double p, double t) { return __double2hiint(p) + ~(__double2hiint(t) & 0x7FFFFFFF); }

// THREADS: 256, three CTAs per SM, or 512 where there are fewer CTAs than SMs.
template <typename TP, typename TQ, bool HAS_Q, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 3 : 1)
next_kernel(const __grid_constant__ LosslessParams P, int cluster) {
    constexpr int kNextThreads = THREADS, kNextWarps = THREADS / 32;
    __shared__ NextShared<kNextWarps> S;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = (int)(blockIdx.x / (unsigned)cluster), rank = (int)(blockIdx.x % (unsigned)cluster);
    if (threadIdx.x < 16) S.table[threadIdx.x] = P.table[threadIdx.x];
    if (threadIdx.x == 0) { S.found = kNone; S.last = -1; }
    const int len = P.draft_len == nullptr ? P.T : min(P.T, max(0, P.draft_len[b]));
    // the CTA's part of a row, and the warp's part of that, both in token order
    const int lo = (int)min((long long)P.V, (long long)rank * P.share), hi = (int)min((long long)P.V, (long long)lo + P.share);
    const int per_warp = ((hi - lo + kNextWarps - 1) / kNextWarps + 31) & ~31;
    const int w_lo = (int)min((long long)hi, (long long)lo + (long long)warp * per_warp), w_hi = (int)min((long long)hi, (long long)w_lo + per_warp);
    const TP* target = static_cast<const TP*>(P.target) + (long long)b * (P.T + P.bonus) * P.ld_target;
    const TQ* draft_rows = static_cast<const TQ*>(P.draft_logits) + (long long)b * P.T * P.ld_draft;
    int set = 0;

    // What every thread of the cluster knows about a row.
    Row64 at_p, at_q;
    double border = 0.0, rho = 0.0, sum_p = 0.0, sum_q = 0.0, sum_t = 0.0, sum_d = 0.0;
    int closest = 0;
    const TP* row_p = target;
    const TQ* row_q = draft_rows;

    // fp64 sums over the row; entry `skip` of p counts as masked.  The warps' and CTAs' sums of p, q, t, D stay in warp_part
    // and part[set ^ 1].  Are the weights in reach of their reference?
    auto sums = [&](bool with_q, int skip) {
        double a[4] = {};
        closest = 0;
        float2 top = make_float2(neg_inf(), neg_inf());
        const auto add = [&](auto& x, auto& y) {      // (all the exponentials side by side, without a branch between them)
            constexpr int N = sizeof(x) / sizeof(x[0]);
            double p[N], q[N];
#pragma unroll
            for (int i = 0; i < N; ++i) p[i] = weight(x[i], at_p, P.e, S.table);
#pragma unroll
            for (int i = 0; i < N; i += 2) top.x = fmaxf(top.x, fmaxf(x[i], x[i + 1 < N ? i + 1 : i]));
            if (HAS_Q && with_q) {
#pragma unroll
                for (int i = 0; i < N; ++i) q[i] = weight(y[i], at_q, P.e_draft, S.table);
#pragma unroll
                for (int i = 0; i < N; i += 2) top.y = fmaxf(top.y, fmaxf(y[i], y[i + 1 < N ? i + 1 : i]));
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const double t = fma(-border, q[i], p[i]);
                    a[1] += q[i];
                    add_if_above(t, q[i], a[2], a[3]);
                    closest = max(closest, closeness(p[i], t));
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) a[0] += p[i];
        };
        constexpr int kAhead = 8;
        const TP* at_x = row_p + w_lo + lane;
        const TQ* at_y = row_q + w_lo + lane;
        int left = w_hi - w_lo - lane, off = skip - w_lo - lane;      // entries from the lane's on; where the one to skip is
        const auto load = [&](float (&x)[kAhead], float (&y)[kAhead]) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                x[i] = entry(at_x, 32 * i);
                if (HAS_Q && with_q) y[i] = entry(at_y, 32 * i);
                else if (off == 32 * i) x[i] = neg_inf();
            }
            at_x += 32 * kAhead;
            at_y += 32 * kAhead;
            left -= 32 * kAhead;
            off -= 32 * kAhead;
        };
#pragma unroll 1
        while (left > 32 * (kAhead - 1)) {
            float x[kAhead], y[kAhead] = {};
            load(x, y);
            add(x, y);
        }
#pragma unroll 1
        for (; left > 0; left -= 32, off -= 32, at_x += 32, at_y += 32) {
            const float x1[1] = {off == 0 ? neg_inf() : entry(at_x, 0)}, y1[1] = {HAS_Q && with_q ? entry(at_y, 0) : 0.0f};
            add(x1, y1);
        }
        __syncwarp();
        add_lanes(a);
        top = make_float2(warp_max(top.x), warp_max(top.y));
        closest = __reduce_max_sync(0xFFFFFFFFu, closest);
        if (lane < 4) S.warp_part[warp][lane] = lane == 0 ? a[0] : lane == 1 ? a[1] : lane == 2 ? a[2] : a[3];
        if (lane == 0) { S.warp_top[warp] = top; S.warp_closest[warp] = closest; }
        __syncthreads();
        if (warp == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = lane < kNextWarps ? S.warp_part[lane][i] : 0.0;
            add_lanes(a);
            top = S.warp_top[lane < kNextWarps ? lane : 0];
            top = make_float2(warp_max(top.x), warp_max(top.y));
            closest = __reduce_max_sync(0xFFFFFFFFu, S.warp_closest[lane < kNextWarps ? lane : 0]);
        }
        exchange(S, set, rank, cluster, a, top, closest);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = lane < cluster ? S.part[set][lane][i] : 0.0;
        add_lanes(a);
        sum_p = a[0]; sum_q = a[1]; sum_t = a[2]; sum_d = a[3];
        top = S.top[set][lane < cluster ? lane : 0];
        top = make_float2(warp_max(top.x), warp_max(top.y));
        closest = __reduce_max_sync(0xFFFFFFFFu, S.closest[set][lane < cluster ? lane : 0]);
        set ^= 1;
        return in_reach(top.x, at_p, P.e) && (!(HAS_Q && with_q) || in_reach(top.y, at_q, P.e_draft));
    };
    // 32 positions' drafted tokens, random numbers and logits (by warp 0), of the first 32, and of what follows the draft,
    // ahead of the ratios.
    int window = 0;
    const auto open_window = [&]() {
        const int t = window + lane;
        if (warp != 0 || t >= len) return;
        const int tok = P.draft[(long long)b * P.T + t];
        S.tok[lane] = tok;
        S.u[lane] = P.u_accept[(long long)b * P.T + t];
        if ((unsigned)tok < (unsigned)P.V) {
            S.x[lane] = entry(target + (long long)t * P.ld_target, tok);
            if (HAS_Q) S.y[lane] = entry(draft_rows + (long long)t * P.ld_draft, tok);
        }
    };
    open_window();
    if (warp == 1) {
        const float behind = len < P.T + P.bonus ? warp_max(entry(target + (long long)len * P.ld_target, (long long)lane * P.V / 32)) : 0.0f;
        if (lane == 0) { S.behind = behind; S.u_next = P.u_next[b]; }
    }
    __syncwarp();
    ptx::cluster_sync_all();      // (the other CTAs have started: their shared memory may be written)
    ptx::griddep_wait();
    const auto ratios = [&]() {
        if (warp == 0 && window + lane < len) S.ratio[lane] = P.out_accept_prob[(long long)b * P.T + window + lane];
        __syncthreads();
    };
    ratios();

    // Row n, and whether a token was rejected there: known at once, or after a look at the row in 64 bits.
    int n = 0, skip = -1;
    bool decided = false, against_q = false;
    double total = 0.0;
    // (one loop, so that there is one copy of the sums in the code: a single sequence's draw waits for instructions, too)
#pragma unroll 1
    for (;;) {
        // the accepted prefix: up to the first position that is not surely accepted
        while (!decided) {
            if (n >= len) { decided = true; break; }
            if (n >= window + 32) {
                __syncthreads();
                window += 32;
                open_window();
                ratios();
            }
            const int t = window + lane;
            const uint32_t open = __ballot_sync(0xFFFFFFFFu, t >= n && t < len && !(S.u[lane] < S.ratio[lane] * (1.0f - kBand)));
            if (open == 0) { n = min(len, window + 32); continue; }
            const int first = __ffs(open) - 1;
            n = window + first;
            decided = S.u[first] > S.ratio[first] * (1.0f + kBand) || (unsigned)S.tok[first] >= (unsigned)P.V;
            break;
        }
        if (n >= P.T + P.bonus) {      // every drafted token accepted and no row behind them
            if (rank == 0 && threadIdx.x == 0) { P.out_accept_len[b] = n; P.out_next[b] = -1; }
            return;
        }
        const bool drafted = n < len;
        const int tok = drafted ? S.tok[n - window] : -1;
        const float ratio = drafted ? S.ratio[n - window] : 0.0f;
        const bool token = (unsigned)tok < (unsigned)P.V;
        against_q = HAS_Q && drafted;
        skip = !HAS_Q && decided && token ? tok : -1;

        // The drafted token's logits are a reference as good as the rows' maxima, as a rule, and with them its ratio (from the
        // first kernel) says what rho is, but for the rounding; without a token some entry of the row is.  Where they are not (no such token, a
        // ratio of nothing, logits too far apart for fp64), a quick pass over the rows finds maxima and rho first.
        row_p = target + (long long)n * P.ld_target;
        row_q = draft_rows + (long long)n * P.ld_draft;
        const float x = drafted ? S.x[n - window] : S.behind, y = HAS_Q && drafted ? S.y[n - window] : 0.0f;      // (of a token that does not exist: not used)
        enum { kQuick, kCareful, kExact } how = kCareful;
        bool accepted = false, again = false;
        if (drafted == token && near_zero(x, P.e) && (!against_q || (near_zero(y, P.e_draft) && ratio > 1e-30f))) {      // (false for a NaN)
            how = kQuick;
            at_p = Row64(x, P.e);
            at_q = Row64(y, P.e_draft);
            border = against_q ? kAbove * weight(x, at_p, P.e, S.table) / (weight(y, at_q, P.e_draft, S.table) * (double)ratio) : 0.0;
        }
#pragma unroll 1
        for (;;) {
            if (how == kCareful) {
                const bool two = against_q;
                Sum p, q;
                const Share<TP> sp(row_p, lo, hi);
                const Share<TQ> sq(row_q, lo, two ? hi : lo);
#pragma unroll 1
                for (int v0 = threadIdx.x; v0 < max(sp.vecs, sq.vecs); v0 += kNextThreads) {
                    uint4 v[1] = {make_uint4(Vec<TP>::kNone, Vec<TP>::kNone, Vec<TP>::kNone, Vec<TP>::kNone)};
                    uint4 w[1] = {make_uint4(Vec<TQ>::kNone, Vec<TQ>::kNone, Vec<TQ>::kNone, Vec<TQ>::kNone)};
                    if (v0 < sp.vecs) v[0] = sp.body[v0];
                    if (v0 < sq.vecs) w[0] = sq.body[v0];
                    sp.add(p, v, P.c);
                    if (two) sq.add(q, w, P.c_draft);
                }
                sp.add_ends(p, P.c);
                if (two) sq.add_ends(q, P.c_draft);
                __syncwarp();
                const float2 wp = join_lanes(p.m, p.s, P.c), wq = join_lanes(q.m, q.s, P.c_draft);
                if (lane == 0) { S.warp_sum[warp][0] = wp; S.warp_sum[warp][1] = wq; }
                __syncthreads();
                double v[4] = {};
                if (warp == 0) {
                    const float2 cp = join_parts(&S.warp_sum[0][0], kNextWarps, 2, P.c), cq = join_parts(&S.warp_sum[0][1], kNextWarps, 2, P.c_draft);
                    v[0] = cp.x; v[1] = cp.y; v[2] = cq.x; v[3] = cq.y;
                }
                exchange(S, set, rank, cluster, v, make_float2(0.0f, 0.0f), 0);
                const double* part = S.part[set][lane < cluster ? lane : 0];
                const float2 ap = join_lanes((float)part[0], lane < cluster ? (float)part[1] : 0.0f, P.c);
                const float2 aq = join_lanes((float)part[2], lane < cluster ? (float)part[3] : 0.0f, P.c_draft);
                at_p = Row64(ap.x, P.e);
                at_q = Row64(aq.x, P.e_draft);
                border = aq.y > 0.0f ? kAbove * (double)ap.y * weight(ap.x, at_p, P.e, S.table) / ((double)aq.y * weight(aq.x, at_q, P.e_draft, S.table)) : 0.0;
                set ^= 1;
            }
            if (!sums(against_q, skip) && how == kQuick) { how = kCareful; continue; }
            total = sum_p;
            if (!decided) {
                // is this position's token accepted?  (p(x) = 0, or a NaN or +inf in a row: no)
                accepted = x > neg_inf() && sum_p > 0.0 && (!HAS_Q || sum_q >= 0.0);
                if (accepted && (!HAS_Q || y > neg_inf())) {      // (q(x) = 0 otherwise: yes)
                    // by logarithms: p(x) and q(x) may both lie below fp64's range
                    double l = ((double)x - at_p.base) * P.inv_temp - log(sum_p);
                    if (HAS_Q) l -= ((double)y - at_q.base) * P.inv_draft_temp - log(sum_q);
                    const float u = S.u[n - window];
                    accepted = u <= 0.0f || (double)u < exp(l);
                }
                if (accepted) break;
                decided = true;
                again = !HAS_Q;       // (without a draft's distribution the sums have to leave the token out)
            }
            if (against_q) {
                rho = sum_q > 0.0 ? sum_p / sum_q : 0.0;
                total = fma(border - rho, sum_d, sum_t);
                const double right = rho * kAbove;
                // (a NaN comes here once; of weights near fp64's lower end the high words are no logarithms)
                if (how != kExact && right != border && !(fabs(right - border) < nearest(border, closest) && total > 1e-270)) {
                    how = kExact;
                    border = right;
                    continue;
                }
            }
            break;
        }
        if (accepted) { ++n; continue; }
        if (!again) break;
    }
    if (rank == 0 && threadIdx.x == 0) P.out_accept_len[b] = n;
    if (skip >= 0 && total == 0.0) {      // nothing but the rejected token
        if (rank == 0 && threadIdx.x == 0) P.out_next[b] = entry(row_p, skip) > neg_inf() ? skip : -1;
        return;
    }
    const bool from_q = against_q;
    if (against_q && total == 0.0) {       // p - q leaves nothing: p
        against_q = false;
        total = sum_p;
    }
    // (no CTA writes to another from here on: each may leave when it is done)
    if (!(sum_p > 0.0) || !(total > 0.0) || (from_q && !(sum_q >= 0.0))) {      // nothing to draw from, or a NaN or +inf in a row
        if (rank == 0 && threadIdx.x == 0) P.out_next[b] = -1;
        return;
    }
    const auto entry_weight = [&](int j) {
        const double p = j == skip ? 0.0 : weight(entry(row_p, j), at_p, P.e, S.table);
        if (!HAS_Q || !against_q) return p;
        const double q = weight(entry(row_q, j), at_q, P.e_draft, S.table), t = fma(-border, q, p);
        return t > 0.0 ? fma(border - rho, q, t) : 0.0;
    };
    const auto part_weight = [&](const double* part) { return against_q ? fma(border - rho, part[3], part[2]) : part[0]; };
    // the part that holds the place u_next * total: a CTA's, then a warp's
    double place = (double)S.u_next * total;
    if (part_of(place, lane < cluster ? part_weight(S.part[set ^ 1][lane]) : 0.0) != rank) return;
    const int pick = part_of(place, lane < kNextWarps ? part_weight(S.warp_part[lane]) : 0.0);
    // the entry within that: the whole block, a run of four entries per thread
    const int p_lo = (int)min((long long)hi, (long long)lo + (long long)pick * per_warp), p_hi = (int)min((long long)hi, (long long)p_lo + per_warp);
    double base = 0.0;
#pragma unroll 1
    for (int j0 = p_lo; j0 < p_hi; j0 += 4 * kNextThreads) {
        double r[4], run = 0.0;
        int last = -1;
        const int first = j0 + 4 * (int)threadIdx.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r[i] = first + i < p_hi ? entry_weight(first + i) : 0.0;
            run += r[i];
            if (r[i] > 0.0) last = first + i;
        }
        double incl = run;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const double o = __shfl_up_sync(0xFFFFFFFFu, incl, off);
            if (lane >= off) incl += o;
        }
        if (lane == 31) S.scan[warp] = incl;
        __syncthreads();
        double cum = base + (incl - run);
#pragma unroll 1
        for (int w = 0; w < kNextWarps; ++w) {
            if (w < warp) cum += S.scan[w];
            base += S.scan[w];
        }
        int found = kNone;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            cum += r[i];
            if (found == kNone && r[i] > 0.0 && cum > place) found = first + i;
        }
        found = __reduce_min_sync(0xFFFFFFFFu, found);
        last = __reduce_max_sync(0xFFFFFFFFu, last);
        if (lane == 0) { atomicMin(&S.found, found); atomicMax(&S.last, last); }
        __syncthreads();
        if (S.found != kNone) break;
    }
    if (threadIdx.x == 0) P.out_next[b] = S.found != kNone ? S.found : S.last;
}

// Largest dynamic shared memory and cluster, once for each kernel and device.
template <auto KERNEL>
bool allow(int smem) {
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return true;
    if ((smem > 0 && cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) ||
        cudaFuncSetAttribute(KERNEL, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

cudaLaunchConfig_t launch_config(cudaLaunchAttribute (&attrs)[2], int clusters, int cluster, int threads, int smem, bool behind, cudaStream_t stream) {
    attrs[0].id = cudaLaunchAttributeClusterDimension;
    attrs[0].val.clusterDim.x = (unsigned)cluster; attrs[0].val.clusterDim.y = 1; attrs[0].val.clusterDim.z = 1;
    attrs[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)clusters * (unsigned)cluster);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cfg.attrs = attrs;
    cfg.numAttrs = behind ? 2 : 1;
    return cfg;
}

// Clusters of this size that the device runs at a time (looked up once for each kernel, device and size).
template <auto KERNEL>
int clusters_at_once(int cluster, int threads, int smem) {
    constexpr int kDevices = 16;
    static std::atomic<int> known[kDevices][kMaxCluster + 1];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev < kDevices && (n = known[dev][cluster].load(std::memory_order_relaxed)) > 0) return n;
    cudaLaunchAttribute attrs[2]{};
    const cudaLaunchConfig_t cfg = launch_config(attrs, 1, cluster, threads, smem, false, nullptr);
    if (cudaOccupancyMaxActiveClusters(&n, KERNEL, &cfg) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    if (dev < kDevices) known[dev][cluster].store(n, std::memory_order_relaxed);
    return n;
}

template <typename TP, typename TQ, bool HAS_Q>
int launch(LosslessParams& P, cudaStream_t stream) {
    const auto enough = [&](int cluster) { return P.V / cluster >= 2048; };       // entries for a CTA
    const auto run = [&](auto* kernel, int clusters, int cluster, int threads, int smem, bool behind) {
        P.share = ((P.V + cluster - 1) / cluster + 7) & ~7;      // (whole 16-byte vectors)
        cudaLaunchAttribute attrs[2]{};
        const cudaLaunchConfig_t cfg = launch_config(attrs, clusters, cluster, threads, smem, behind, stream);
        if (cudaLaunchKernelEx(&cfg, kernel, P, cluster) != cudaSuccess || cudaGetLastError() != cudaSuccess) {
            cudaGetLastError();
            return DM_ECUDA;
        }
        return DM_OK;
    };
    if (P.T > 0) {
        // (96 x 7 rows of 151936 over 2 CTAs each: 73 us, 4: 79, 8: 96; the 5 of one sequence: 16 are the fastest)
        int cluster = 1;
        while (cluster < kMaxCluster && enough(2 * cluster) && 2ll * P.B * P.T * cluster <= 1400) cluster *= 2;
        if (!allow<ratio_kernel<TP, TQ, HAS_Q>>(kRatioSmem)) return DM_ECUDA;
        // (a part of a GPU may have no room for the largest clusters)
        while (cluster > 1 && clusters_at_once<ratio_kernel<TP, TQ, HAS_Q>>(cluster, kRatioThreads, kRatioSmem) == 0) cluster /= 2;
        const int st = run(ratio_kernel<TP, TQ, HAS_Q>, P.B * P.T, cluster, kRatioThreads, kRatioSmem, false);
        if (st != DM_OK) return st;
    }
    // The largest clusters with which all sequences are drawn side by side: of 512 threads where that gives each sequence
    // at least four CTAs, else of 256 (three on an SM); beyond that, in turns of six.  (Of 128256 entries, in all: 32
    // sequences 53 us with 4 x 512, 61 with 3 x 512, 55 with 8 x 256; 64: 84 with 6 x 256, 88 with 2 x 512, 96 with
    // 8 x 256; 128: 141 with 6 x 256, 147 with 3 x 256.)
    if (!allow<next_kernel<TP, TQ, HAS_Q, 512>>(0) || !allow<next_kernel<TP, TQ, HAS_Q, 256>>(0)) return DM_ECUDA;
    const auto largest = [&](auto at_once, int threads, int least) {
        for (int cluster = kMaxCluster; cluster >= least; --cluster)
            if (enough(cluster) && at_once(cluster, threads, 0) >= P.B) return cluster;
        return 0;
    };
    // Behind the ratios the kernel starts early and reads inputs before it waits for them.  out_accept_prob is all that the
    // kernel ahead writes, and that one must itself be launched without overlap: what came before both is then complete.
    int most = 1;
    while (most < kMaxCluster && enough(most + 1)) ++most;
    int cluster = largest(clusters_at_once<next_kernel<TP, TQ, HAS_Q, 512>>, 512, (most < 4 ? most : 4));
    if (cluster > 0) return run(next_kernel<TP, TQ, HAS_Q, 512>, P.B, cluster, 512, 0, P.T > 0);
    cluster = largest(clusters_at_once<next_kernel<TP, TQ, HAS_Q, 256>>, 256, (most < 4 ? most : 4));
    if (cluster == 0) {
        cluster = (most < 6 ? most : 6);
        while (cluster > 1 && clusters_at_once<next_kernel<TP, TQ, HAS_Q, 256>>(cluster, 256, 0) == 0) --cluster;
    }
    return run(next_kernel<TP, TQ, HAS_Q, 256>, P.B, cluster, 256, 0, P.T > 0);
}

template <typename TP>
int launch_target(LosslessParams& P, int draft_dtype, cudaStream_t stream) {
    if (P.draft_logits == nullptr) return launch<TP, TP, false>(P, stream);
    if (draft_dtype == DM_F32) return launch<TP, float, true>(P, stream);
    return launch<TP, __nv_bfloat16, true>(P, stream);
}

}  // namespace

int launch_lossless(LosslessParams P, int dtype, int draft_dtype, cudaStream_t stream) {
    const auto constants = [](double inv_temp) {
        Exp64 e{};
        e.c16 = (float)(16.0 * 1.4426950408889634074 * inv_temp);
        e.step = 0.69314718055994530942 / 16.0 / inv_temp;
        double a = 1.0;
        for (int n = 1; n <= 5; ++n) e.a[n - 1] = a *= inv_temp / n;
        return e;
    };
    P.e = constants(P.inv_temp);
    if (P.draft_logits != nullptr) P.e_draft = constants(P.inv_draft_temp);
    for (int j = 0; j < 16; ++j) {
        const double t = exp2(j / 16.0);
        uint64_t bits;
        memcpy(&bits, &t, sizeof bits);
        bits -= (uint64_t)j << 48;
        memcpy(&P.table[j], &bits, sizeof bits);
    }
    if (dtype == DM_F32) return launch_target<float>(P, draft_dtype, stream);
    return launch_target<__nv_bfloat16>(P, draft_dtype, stream);
}

}  // namespace dm
