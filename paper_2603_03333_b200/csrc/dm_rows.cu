// Operators on rows of logits x[N][V] in global memory (fp32 or bf16, any row stride):
//   logprobs       z = x / temperature;  lse = log sum_v exp z_v;  log-probability of a given token
//                  z_tok - lse;  entropy -sum_v p_v log p_v;  the n_top largest entries
//   logprobs_grad  gradient of g_lp * logprob + g_H * entropy with respect to x:
//                  (1/T) [ g_lp (1[v = tok] - p_v) - g_H p_v (log p_v + H) ]
//   distill        KL(teacher || student) for a teacher known by its top tokens, and its gradient
//                  (see distill_teacher below)
//
// A row belongs to one thread-block cluster; its CTAs take contiguous shares of the row, cut at
// 16-byte boundaries.  One pass over the share keeps, per warp, the exact maximum m so far (five
// shuffles per 1024 entries) and, per lane, the sum of e = 2^((x - m) log2(e) / T) and of e times its
// exponent (entropy) over the entries below m; entries equal to m are counted.  A batch whose maximum
// stays below m takes the short path: seven or eight instructions per entry.  Warps meet in the
// block, CTAs through distributed shared memory.  Sums never contain the row's largest entry, so that
// log(1 + rest) keeps its precision next to a near-certain token.
//
// Bound: memory, one read of x (and one write of the gradient).  The gradient kernels keep as much
// of a CTA's share as fits in shared memory, so that x is read once; what does not fit is read again.
#include <cooperative_groups.h>

#include <atomic>

#include "dm_internal.h"
#include "dm_rows.cuh"

namespace dm {

#ifndef DM_ROWS_THREADS
#define DM_ROWS_THREADS 256
#endif
#ifndef DM_ROWS_MINB
#define DM_ROWS_MINB 4
#endif
#ifndef DM_ROWS_RING
#define DM_ROWS_RING 2
#endif
#ifndef DM_ROWS_MINR
#define DM_ROWS_MINR 3
#endif

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = DM_ROWS_THREADS;
constexpr int kWarps = kThreads / 32;
constexpr int kUnroll = 4;             // vectors of a batch: 16-byte loads in flight per thread
constexpr int kRing = DM_ROWS_RING;    // batches in flight where rows stream
constexpr int kCandCap = 1024;         // candidates for the top entries of a CTA's share
constexpr int kHitCap = 2048;          // batches that hold them
constexpr int kMaxSlots = 16;          // maxima a thread keeps of its batches (for finding the top entries again)
constexpr float kFloorExp = -200.0f;   // exponents are clamped here: 2^-200 is 0 in fp32, and 0 * clamp stays 0
constexpr int kStashVecs = 4096;       // share of a gradient kernel's CTA up to which a row is cut: 64 KB, three CTAs per SM
constexpr size_t kRowsSmemLimit = 216 * 1024;
constexpr float kLn2 = 0.693147180559945309f;

enum { OP_LOGPROBS = 0, OP_GRAD = 1, OP_DISTILL = 2 };

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {   // a NaN on either side stays
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// Two entries per instruction: sm_100 has packed fp32 arithmetic.
typedef float2 f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) { return make_float2(lo, hi); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float sum2(f32x2 p) { return p.x + p.y; }
__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xFF800000u); }

// Ordered key of a logit; NaN sorts above everything.  Keys of numbers are never 0.
__device__ __forceinline__ uint32_t logit_key(float x) { return x != x ? 0xFFFFFFFFu : float_key(x); }

template <typename T> struct RowVec;
template <> struct RowVec<float> {
    static constexpr int N = 4;
    __device__ static void unpack(const uint4& v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y);
        x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
    __device__ static uint4 pack(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __device__ static void pairs(const uint4& v, f32x2 (&x)[2]) {
        x[0] = pair(__uint_as_float(v.x), __uint_as_float(v.y));
        x[1] = pair(__uint_as_float(v.z), __uint_as_float(v.w));
    }
    __device__ static uint4 pack_pairs(const f32x2 (&x)[2]) {
        return make_uint4(__float_as_uint(x[0].x), __float_as_uint(x[0].y), __float_as_uint(x[1].x), __float_as_uint(x[1].y));
    }
    static constexpr bool kFloorsEntries = false;   // exponents are clamped one by one
    __device__ static uint32_t floor_word(float) { return 0u; }
    __device__ static void raise(uint4&, uint32_t) {}
    __device__ static float vmax(const uint4 (&v)[kUnroll]) {
        float m = neg_inf();
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            m = max_nan(m, max_nan(max_nan(__uint_as_float(v[u].x), __uint_as_float(v[u].y)),
                                   max_nan(__uint_as_float(v[u].z), __uint_as_float(v[u].w))));
        return m;
    }
    __device__ static uint4 masked() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }
    // Which entries equal m (one bit each); they become -inf.
    __device__ static uint32_t take(uint4& v, float m) {
        uint32_t eq = 0;
        if (__uint_as_float(v.x) == m) { eq |= 1u; v.x = 0xFF800000u; }
        if (__uint_as_float(v.y) == m) { eq |= 2u; v.y = 0xFF800000u; }
        if (__uint_as_float(v.z) == m) { eq |= 4u; v.z = 0xFF800000u; }
        if (__uint_as_float(v.w) == m) { eq |= 8u; v.w = 0xFF800000u; }
        return eq;
    }
    __device__ static float get(const float* p) { return *p; }
    __device__ static void put(float* p, float x) { *p = x; }
};
template <> struct RowVec<__nv_bfloat16> {
    static constexpr int N = 8;
    __device__ static void unpack(const uint4& v, float (&x)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            x[2 * n] = __uint_as_float(w[n] << 16);
            x[2 * n + 1] = __uint_as_float(w[n] & 0xFFFF0000u);
        }
    }
    __device__ static uint4 pack(const float (&x)[8]) {   // the one rounding of a bf16 gradient, to nearest
        uint32_t w[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * n], x[2 * n + 1]);
            w[n] = *reinterpret_cast<const uint32_t*>(&b);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ static void pairs(const uint4& v, f32x2 (&x)[4]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int n = 0; n < 4; ++n) x[n] = pair(__uint_as_float(w[n] << 16), __uint_as_float(w[n] & 0xFFFF0000u));
    }
    __device__ static uint4 pack_pairs(const f32x2 (&x)[4]) {   // the one rounding of a bf16 gradient, to nearest
        uint32_t w[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const __nv_bfloat162 b = __float22bfloat162_rn(x[n]);
            w[n] = *reinterpret_cast<const uint32_t*>(&b);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static constexpr bool kFloorsEntries = true;    // entries are raised to a floor, two per instruction, before they are unpacked
    __device__ static uint32_t floor_word(float x) {
        const __nv_bfloat16 f = __float2bfloat16_rd(fmaxf(x, -3.3e38f));
        return (uint32_t)*reinterpret_cast<const unsigned short*>(&f) * 0x10001u;
    }
    __device__ static void raise(uint4& v, uint32_t floor2) {
        asm("max.bf16x2 %0, %0, %1;" : "+r"(v.x) : "r"(floor2));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(v.y) : "r"(floor2));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(v.z) : "r"(floor2));
        asm("max.bf16x2 %0, %0, %1;" : "+r"(v.w) : "r"(floor2));
    }
    __device__ static float vmax(const uint4 (&v)[kUnroll]) {   // two entries per instruction, NaN kept
        uint32_t m = 0xFF80FF80u;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            m = max2(m, max2(max2(v[u].x, v[u].y), max2(v[u].z, v[u].w)));
        }
        return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    }
    __device__ static uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t y;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
        return y;
    }
    __device__ static uint4 masked() { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }
    __device__ static uint32_t take_pair(uint32_t& v, uint32_t mm) {
        uint32_t eq;   // all ones in the halves that compare equal
        asm("set.eq.u32.bf16x2 %0, %1, %2;" : "=r"(eq) : "r"(v), "r"(mm));
        v = (v & ~eq) | (0xFF80FF80u & eq);
        return (eq & 1u) | ((eq >> 15) & 2u);
    }
    __device__ static uint32_t take(uint4& v, float m) {   // m is a bf16 value
        const uint32_t mm = (__float_as_uint(m) >> 16) * 0x10001u;
        return take_pair(v.x, mm) | (take_pair(v.y, mm) << 2) | (take_pair(v.z, mm) << 4) | (take_pair(v.w, mm) << 6);
    }
    __device__ static float get(const __nv_bfloat16* p) {
        return __uint_as_float((uint32_t)*reinterpret_cast<const unsigned short*>(p) << 16);
    }
    __device__ static void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
};

// Asynchronous 16-byte copies global -> shared memory, one group per batch; a thread waits for its own.
__device__ __forceinline__ void copy_async(uint4* dst, const uint4* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait(int newer) {   // all but the `newer` latest groups have landed (or more)
    if (newer <= 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else if (newer == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (newer == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (newer == 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else asm volatile("cp.async.wait_group 4;" ::: "memory");
}

// A CTA's share of a row: 16-byte vectors [first, last) of the row, vector j holding entries
// j*N - phase .. j*N - phase + N-1 (phase: entries between the 16-byte boundary below the row's
// start and that start).  Entries outside [0, V) read as -inf and are never written.
template <typename T> struct Share {
    const T* row;
    int V, phase, first, last;
    int whole_lo, whole_hi;   // vectors of the row that hold N of its entries
    __device__ __forceinline__ int entry0(int j) const { return j * RowVec<T>::N - phase; }
    __device__ __forceinline__ bool whole(int j) const { return j >= whole_lo && j < whole_hi; }
    __device__ __forceinline__ const uint4* vectors() const { return reinterpret_cast<const uint4*>(row - phase); }
    // Loads go to L2 (ld.global.cg): the row may be overwritten in place by this very kernel, each
    // entry by the thread that read it.
    __device__ __forceinline__ uint4 load(int j) const {
        constexpr int N = RowVec<T>::N;
        if (whole(j)) return __ldcg(vectors() + j);
        float x[N];
        const int i0 = entry0(j);
#pragma unroll
        for (int n = 0; n < N; ++n) x[n] = (i0 + n >= 0 && i0 + n < V) ? RowVec<T>::get(row + i0 + n) : neg_inf();
        return RowVec<T>::pack(x);
    }
    // Sends one batch (vectors b0 + u * kThreads + thread) on its way to the thread's slots of shared
    // memory; slots past the end of the share are filled with masked entries.
    __device__ __forceinline__ void fetch_batch(int b0, uint4* slot) const {
        const int j = b0 + (int)threadIdx.x;
        if (b0 >= whole_lo && b0 + kUnroll * kThreads <= min(last, whole_hi)) {
            const uint4* p = vectors() + j;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) copy_async(slot + u * kThreads, p + u * kThreads);
        } else {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int i = j + u * kThreads;
                if (i < last && whole(i)) copy_async(slot + u * kThreads, vectors() + i);
                else slot[u * kThreads] = i < last ? load(i) : RowVec<T>::masked();
            }
        }
        copy_commit();
    }
};

// Running statistics of a warp's entries.  Exponents are taken against rc, the rounded product m * c:
// w(x) = fma(x, ce, -rc) is then off by one rounding only; finish() moves the sums to m itself.  Where
// |m| c is beyond 1e37 (a row of nothing but the type's lowest value, say) every other entry is
// thousands of powers of two below m and adds nothing: ce = 0 says so.
struct Stats {
    float m, rc, ce;          // the warp's maximum (all lanes alike), and how exponents are taken
    uint32_t floor2;          // bf16: entries below this are raised to it (250 powers of two below m)
    float s, t, tail;         // this lane's sums over entries below m: 2^w, w 2^w; and 2^w outside the teacher's tokens (m included)
    int cnt;                  // this lane's entries equal to m
    __device__ __forceinline__ void init() {
        m = neg_inf(); rc = ce = 0.0f; s = t = tail = 0.0f; cnt = 0; floor2 = 0u;
    }
    __device__ __forceinline__ float of_maximum() const { return ce != 0.0f ? ex2(fmaf(m, ce, -rc)) : 1.0f; }

    // Exponents are taken against `top` from here on (the sums are not moved).
    template <typename T> __device__ __forceinline__ void set_maximum(float top, float c) {
        m = top;
        rc = top * c;
        ce = fabsf(rc) <= 1e37f ? c : 0.0f;
        floor2 = RowVec<T>::floor_word(top - 250.0f / c);
        cnt = 0;
    }
    // Entries equal to the maximum are counted and taken out of the batch.
    template <typename T, bool kTail>
    __device__ __forceinline__ void take(uint4 (&v)[kUnroll], const uint32_t (&top_bits)[kUnroll]) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const uint32_t eq = RowVec<T>::take(v[u], m);
            cnt += __popc(eq);
            if (kTail) tail = fmaf((float)__popc(eq & ~top_bits[u]), of_maximum(), tail);
        }
    }
    // A batch of entries below the maximum.
    template <typename T, bool kEntropy, bool kTail>
    __device__ __forceinline__ void sum(uint4 (&v)[kUnroll], const uint32_t (&top_bits)[kUnroll]) {
        constexpr int N = RowVec<T>::N;
        const f32x2 c2 = pair(ce, ce), rc2 = pair(-rc, -rc);
        f32x2 bs = pair(0.0f, 0.0f), bt = bs;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (kEntropy) RowVec<T>::raise(v[u], floor2);
            f32x2 x[N / 2], vs = pair(0.0f, 0.0f);
            RowVec<T>::pairs(v[u], x);
#pragma unroll
            for (int n = 0; n < N / 2; ++n) {
                f32x2 w = fma2(x[n], c2, rc2);
                if (kEntropy && !RowVec<T>::kFloorsEntries) { w.x = fmaxf(w.x, kFloorExp); w.y = fmaxf(w.y, kFloorExp); }
                const f32x2 e = pair(ex2(w.x), ex2(w.y));
                if (kTail) { vs = add2(vs, e); x[n] = e; } else { bs = add2(bs, e); }
                if (kEntropy) bt = fma2(e, w, bt);   // (a masked entry: 0 * a finite exponent)
            }
            if (kTail) {
                bs = add2(bs, vs);
                tail += top_bits[u] == 0u ? sum2(vs) : outside<N>(x, top_bits[u]);
            }
        }
        s += sum2(bs);
        t += sum2(bt);
    }
    // A batch of whatever entries, with the maximum so far kept exactly.
    template <typename T, bool kEntropy, bool kTail>
    __device__ __forceinline__ void add(uint4 (&v)[kUnroll], float lane_max, float c, const uint32_t (&top_bits)[kUnroll]) {
        float wm = lane_max;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) wm = max_nan(wm, __shfl_xor_sync(0xFFFFFFFFu, wm, off));
        if (!(wm < m && ce != 0.0f)) {
            if (wm == neg_inf()) return;   // nothing but masked entries so far
            if (!(wm <= m)) {              // a new maximum: the old one becomes an entry like the others
                const Stats old = *this;
                set_maximum<T>(wm, c);
                if (old.ce != 0.0f && ce != 0.0f) {
                    const float d = fmaxf(old.rc - rc, kFloorExp), f = ex2(d);
                    const float w = fmaxf(fmaf(old.m, c, -rc), kFloorExp), e = (float)old.cnt * ex2(w);
                    t = fmaf(f, fmaf(d, s, t), e * w);
                    s = fmaf(f, s, e);
                    tail *= f;
                } else {
                    s = t = tail = 0.0f;
                }
            }
            take<T, kTail>(v, top_bits);
            if (ce == 0.0f) return;
        }
        sum<T, kEntropy, kTail>(v, top_bits);
    }
    template <int N> __device__ __forceinline__ static float outside(const f32x2 (&e)[N / 2], uint32_t bits) {
        float sum = 0.0f;
#pragma unroll
        for (int n = 0; n < N / 2; ++n) {
            sum += ((bits >> (2 * n)) & 1u) ? 0.0f : e[n].x;
            sum += ((bits >> (2 * n + 1)) & 1u) ? 0.0f : e[n].y;
        }
        return sum;
    }
    __device__ __forceinline__ void finish() {
        if (ce == 0.0f) return;
        const float d = fminf(fmaxf(fmaf(m, ce, -rc), -100.0f), 100.0f), f = ex2(-d);   // rounding of rc: tiny, either sign
        t = f * fmaf(-d, s, t);
        s *= f;
        tail *= f;
    }
};

struct Merged { float m, rest, t, tail; };   // maximum; sums relative to it, `rest` without one maximal entry

// Cluster barrier in two halves; every thread of every CTA takes both.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, off);
    return x;
}

struct RowsShared {
    float w_m[kWarps], w_s[kWarps], w_t[kWarps], w_tail[kWarps];
    int w_cnt[kWarps];
    Merged part[kRowsMaxCluster];   // every CTA's statistics, each written by its CTA
    Merged all;                  // the row's
    float log_total, inv_total;  // log(1 + rest), 1 / (1 + rest)
    int cand_n, hit_n;
    uint32_t threshold;
    unsigned int scan[kWarps];
    // teacher (distill): warps 0..3 hold its entries, one per thread
    int t_id[kRowsMaxTop];
    float t_q[kRowsMaxTop];
    float t_max[kRowsMaxTop / 32];
    double t_sum[kRowsMaxTop / 32];
    float t_loss[kRowsMaxTop / 32];
    int t_distinct, t_repeated;
};

// The block's statistics from its warps', written to every CTA of the cluster (complete behind the
// next cluster barrier: nobody reads another CTA's shared memory, so nobody waits for anybody to leave).
__device__ void block_merge(Stats& st, float c, RowsShared& ss, cg::cluster_group& cluster, int n_cta, int rank) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    st.finish();
    const float s = warp_sum(st.s), t = warp_sum(st.t), tail = warp_sum(st.tail);
    int cnt = st.cnt;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) cnt += __shfl_xor_sync(0xFFFFFFFFu, cnt, off);
    if (lane == 0) { ss.w_m[warp] = st.m; ss.w_s[warp] = s; ss.w_t[warp] = t; ss.w_tail[warp] = tail; ss.w_cnt[warp] = cnt; }
    __syncthreads();
    if (warp != 0) return;
    const bool have = lane < kWarps;
    const float wm = have ? ss.w_m[lane] : neg_inf();
    float m = wm;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, off));
    Merged r{m, 0.0f, 0.0f, 0.0f};
    cnt = 0;
    if (have && wm != neg_inf()) {
        const float ws = ss.w_s[lane], wt = ss.w_t[lane];
        if (wm == m) {
            r.rest = ws; r.t = wt; r.tail = ss.w_tail[lane]; cnt = ss.w_cnt[lane];
        } else {
            const float d = fmaxf((wm - m) * c, kFloorExp), f = ex2(d), all = ws + (float)ss.w_cnt[lane];
            r.rest = f * all; r.t = f * fmaf(d, all, wt); r.tail = f * ss.w_tail[lane];
        }
    }
    r.rest = warp_sum(r.rest); r.t = warp_sum(r.t); r.tail = warp_sum(r.tail);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) cnt += __shfl_xor_sync(0xFFFFFFFFu, cnt, off);
    if (cnt > 1) r.rest += (float)(cnt - 1);
    if (!(m < __uint_as_float(0x7F800000u))) r.rest = r.t = r.tail = __uint_as_float(0x7FC00000u);   // NaN or +inf: no distribution
    if (n_cta == 1) {
        if (lane == 0) ss.part[0] = r;
    } else if (lane < n_cta) {
        cluster.map_shared_rank(&ss, lane)->part[rank] = r;
    }
}

// The row's statistics from its CTAs', by one warp whose lanes all do the same: a few dozen dependent
// instructions, where shuffles among lanes that have come apart cost 250 cycles each.
__device__ void cluster_merge(RowsShared& ss, int n_cta, float c) {
    Merged a = ss.part[0];
#pragma unroll 1
    for (int r = 1; r < n_cta; ++r) {
        const Merged p = ss.part[r];
        const bool up = !(p.m <= a.m);                     // (a NaN on either side ends up as the maximum)
        const Merged hi = up && a.m == a.m ? p : a, lo = up && a.m == a.m ? a : p;
        const float d = fmaxf((lo.m - hi.m) * c, kFloorExp), f = lo.m == neg_inf() ? 0.0f : ex2(d), all = lo.rest + 1.0f;
        a.m = hi.m;
        a.rest = fmaf(f, all, hi.rest);
        a.t = fmaf(f, fmaf(d, all, lo.t), hi.t);
        a.tail = fmaf(f, lo.tail, hi.tail);
    }
    if ((threadIdx.x & 31) == 0) {
        ss.all = a;
        ss.log_total = log1pf(a.rest);
        ss.inv_total = 1.0f / (1.0f + a.rest);
    }
}

// ---------------------------------------------------------------------------- the largest entries
// Entries of the share with a key of at least `key_min` go to the candidate list.  Each thread looks
// at the maxima it kept of its batches; those that pass go to a list of hits, and the vectors behind
// the hits are read again by all threads, one vector each (read by the thread that owned them, one
// after the other, they took 8 to 25 thousand cycles).  More hits than the list takes count as an
// overflow of the candidate list.
template <typename T>
__device__ int collect(const Share<T>& sh, uint32_t my_key, uint32_t key_min, const uint32_t* slots, int slot_batches,
                       RowsShared& ss, int* hits, unsigned long long* cand) {
    constexpr int N = RowVec<T>::N;
    if (threadIdx.x == 0) ss.cand_n = ss.hit_n = 0;
    __syncthreads();
    const int per_slot = kUnroll * slot_batches, n_slots = (sh.last - sh.first + per_slot * kThreads - 1) / (per_slot * kThreads);
    if (my_key >= key_min) {
        for (int slot = 0; slot < n_slots; ++slot)
            if (slots[slot * kThreads + threadIdx.x] >= key_min) {
                const int at = atomicAdd(&ss.hit_n, 1);
                if (at < kHitCap) hits[at] = slot * per_slot * kThreads + (int)threadIdx.x;   // first vector of the slot, within the share
            }
    }
    __syncthreads();
    const int n_hits = min(ss.hit_n, kHitCap);
#pragma unroll 2
    for (int i = threadIdx.x; i < n_hits * per_slot; i += kThreads) {
        const int h = i / per_slot, j = sh.first + hits[h] + (i - h * per_slot) * kThreads;
        if (j >= sh.last) continue;
        float x[N];
        RowVec<T>::unpack(sh.load(j), x);
        const int i0 = sh.entry0(j);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t key = logit_key(x[n]);
            if (key >= key_min && i0 + n >= 0 && i0 + n < sh.V) {
                const int at = atomicAdd(&ss.cand_n, 1);
                if (at < kCandCap) cand[at] = pack_best(key, (uint32_t)(i0 + n));
            }
        }
    }
    __syncthreads();
    const int n = ss.hit_n > kHitCap ? kCandCap + 1 : ss.cand_n;
    __syncthreads();
    return n;
}
// Entries with a key above `key_min` (fewer than a list takes), read again by threads that hold one.
template <typename T>
__device__ int collect_above(const Share<T>& sh, uint32_t my_key, uint32_t key_min, RowsShared& ss, unsigned long long* cand) {
    constexpr int N = RowVec<T>::N;
    if (threadIdx.x == 0) ss.cand_n = 0;
    __syncthreads();
    if (my_key > key_min) {
#pragma unroll 4
        for (int j = sh.first + (int)threadIdx.x; j < sh.last; j += kThreads) {
            float x[N];
            RowVec<T>::unpack(sh.load(j), x);
            const int i0 = sh.entry0(j);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const uint32_t key = logit_key(x[n]);
                if (key > key_min && i0 + n >= 0 && i0 + n < sh.V) cand[atomicAdd(&ss.cand_n, 1)] = pack_best(key, (uint32_t)(i0 + n));
            }
        }
    }
    __syncthreads();
    const int n = ss.cand_n;
    __syncthreads();
    return n;
}

template <typename T>
__device__ int count_at_least(const Share<T>& sh, uint32_t key_min, RowsShared& ss) {
    constexpr int N = RowVec<T>::N;
    if (threadIdx.x == 0) ss.cand_n = 0;
    __syncthreads();
    int n_mine = 0;
#pragma unroll 4
    for (int j = sh.first + (int)threadIdx.x; j < sh.last; j += kThreads) {
        float x[N];
        RowVec<T>::unpack(sh.load(j), x);
        const int i0 = sh.entry0(j);
#pragma unroll
        for (int n = 0; n < N; ++n) n_mine += (logit_key(x[n]) >= key_min && i0 + n >= 0 && i0 + n < sh.V) ? 1 : 0;
    }
    if (n_mine) atomicAdd(&ss.cand_n, n_mine);
    __syncthreads();
    const int n = ss.cand_n;
    __syncthreads();
    return n;
}

// The first `need` entries (by id) whose key equals `key`, appended to the candidate list at `at`.
template <typename T>
__device__ void collect_ties(const Share<T>& sh, uint32_t key, int need, int at, RowsShared& ss, unsigned long long* cand) {
    constexpr int N = RowVec<T>::N;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int found = 0;
    for (int j0 = sh.first; j0 < sh.last && found < need; j0 += kThreads) {
        const int j = j0 + (int)threadIdx.x;
        uint32_t bits = 0;
        if (j < sh.last) {
            float x[N];
            RowVec<T>::unpack(sh.load(j), x);
            const int i0 = sh.entry0(j);
#pragma unroll
            for (int n = 0; n < N; ++n) bits |= (logit_key(x[n]) == key && i0 + n >= 0 && i0 + n < sh.V) ? 1u << n : 0u;
        }
        const unsigned int mine = __popc(bits);
        unsigned int incl = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const unsigned int o = __shfl_up_sync(0xFFFFFFFFu, incl, off);
            if (lane >= off) incl += o;
        }
        if (lane == 31) ss.scan[warp] = incl;
        __syncthreads();
        unsigned int before = 0, total = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) { if (w < warp) before += ss.scan[w]; total += ss.scan[w]; }
        int pos = found + (int)(before + incl - mine);
        for (int n = 0; n < N; ++n)
            if ((bits >> n) & 1u) {
                if (pos < need) cand[at + pos] = pack_best(key, (uint32_t)(sh.entry0(j) + n));
                ++pos;
            }
        found += (int)total;
        __syncthreads();
    }
}

// The k largest entries of the share (equal entries: lower id first), sorted, as packed words in
// `sorted` (0 where the share has fewer than k entries).  The k-th largest of the threads' maxima
// is a lower bound on the k-th largest entry, because k threads hold an entry that large: only
// entries above it are collected, a few more than k as a rule.  Where that overflows the list (many
// equal entries, or k large ones in few threads) the k-th largest key is found exactly.
template <typename T>
__device__ void top_of_share(const Share<T>& sh, float thread_max, int k, const uint32_t* slots, int slot_batches,
                             RowsShared& ss, int* hits, unsigned long long* cand, unsigned long long* sorted) {
    // a thread without an entry has key 0; padding and masked entries have the key of -inf
    const bool any = sh.first + (int)threadIdx.x < sh.last;
    const uint32_t my_key = any ? logit_key(thread_max) : 0u;
    // The k-th largest of the maxima of groups of threads: k groups hold an entry that large (0 if fewer
    // have one).  At least twice as many groups as entries are wanted: a close bound at the least work.
    const int group = k <= 16 ? 8 : k <= 32 ? 4 : k <= 64 ? 2 : 1, n_groups = kThreads / group;
    uint32_t* keys = reinterpret_cast<uint32_t*>(cand);   // (not yet in use)
    uint32_t mine = my_key;
    for (int off = group >> 1; off > 0; off >>= 1) mine = max(mine, __shfl_xor_sync(0xFFFFFFFFu, mine, off));
    if ((int)threadIdx.x % group == 0) keys[threadIdx.x / group] = mine;
    if (threadIdx.x == 0) ss.threshold = 0u;
    __syncthreads();
    if ((int)threadIdx.x < n_groups) {
        mine = keys[threadIdx.x];
        int reach = 0;
#pragma unroll 8
        for (int i = 0; i < n_groups / 4; ++i) {
            const uint4 o = reinterpret_cast<const uint4*>(keys)[i];
            reach += (o.x >= mine) + (o.y >= mine) + (o.z >= mine) + (o.w >= mine);
        }
        if (reach >= k && mine != 0u) atomicMax(&ss.threshold, mine);
    }
    __syncthreads();
    const uint32_t thr = ss.threshold;
    int n = collect(sh, my_key, thr, slots, slot_batches, ss, hits, cand);
    if (n > kCandCap) {
        // exact: the k-th largest key of the share.  First guess: the exact k-th largest thread
        // maximum, which is it whenever fewer than k entries lie above (a row full of equal entries).
        uint32_t kth = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t c = kth | (1u << bit);
            if (__syncthreads_count(my_key >= c) >= k) kth = c;
        }
        if (kth != 0xFFFFFFFFu && count_at_least(sh, kth + 1u, ss) >= k) {
            uint32_t lo = kth + 1u;        // at least k entries have a key >= lo
            for (uint32_t hi = 0xFFFFFFFFu; lo < hi;) {
                const uint32_t mid = lo + (hi - lo) / 2u + 1u;
                if (count_at_least(sh, mid, ss) >= k) lo = mid; else hi = mid - 1u;
            }
            kth = lo;
        }
        n = kth == 0xFFFFFFFFu ? 0 : collect_above(sh, my_key, kth, ss, cand);   // fewer than k
        collect_ties(sh, kth, k - n, n, ss, cand);
        n = k;
        __syncthreads();
    }
    for (int i = threadIdx.x; i < k; i += kThreads) sorted[i] = 0ull;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {   // the packed words are all different: rank by counting
        const unsigned long long mine = cand[i];
        int rank = 0;
#pragma unroll 4
        for (int o = 0; o < n; ++o) rank += cand[o] > mine ? 1 : 0;
        if (rank < k) sorted[rank] = mine;
    }
    __syncthreads();
}

// ---------------------------------------------------------------------------------- the teacher
// The teacher of a row is known by k tokens and values v (an id outside [0,V) is an absent entry):
//   renorm  q = Softmax(v) over the present entries:  L = sum q (log q - log p)
//   bucket  q = exp(v), the rest of the mass q_t = max(0, 1 - sum q) against the student's mass
//           p_t outside the teacher's tokens:          L = sum q (log q - log p) + q_t (log q_t - log p_t)
//   dL/dz_j = M p_j - q_j - [j is no teacher token] (q_t / p_t) p_j,   M = sum q + q_t;   dL/dx = dL/dz / T.
// One thread per entry.  q is computed and summed in fp64: 1 - sum q then keeps what the fp32 values
// carry.  A bitmap of the share's teacher tokens serves the sum of the tail (p_t would lose its
// precision as a difference) and tells entries that name the same token apart.
struct TeacherEntry { int id; float v, x; bool first; double q; };

// ------------------------------------------------------------------------------------ the kernel
// kResident: the row's gradient is wanted and a share fits in shared memory.  All of it is fetched at
// once by asynchronous copies (each thread waits for its own); one pass over shared memory finds the
// maximum, one sums, one writes the gradient.  Otherwise batches stream through registers.
template <typename T, int kOp, bool kResident>
__global__ void __launch_bounds__(kThreads, kResident ? DM_ROWS_MINR : DM_ROWS_MINB)
rows_kernel(const RowsParams P) {
    constexpr int N = RowVec<T>::N;
    constexpr bool kEntropy = kOp != OP_DISTILL, kTail = kOp == OP_DISTILL;
    constexpr int kBatch = kUnroll * kThreads;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowsShared ss;
    cg::cluster_group cluster = cg::this_cluster();
    const int n_cta = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    if (n_cta > 1) cluster_arrive();   // (waited for before anything is written to another CTA's shared memory)
    uint4* stash = reinterpret_cast<uint4*>(smem);                                      // [stash_vecs], vector first + x
    unsigned char* bitmap = reinterpret_cast<unsigned char*>(stash + P.stash_vecs);     // distill: teacher tokens of the share, a byte per vector
    // logprobs: behind the ring what is kept while the row streams, in the ring's place what comes after
    unsigned long long* merged = reinterpret_cast<unsigned long long*>(stash + kRing * kBatch);   // rank 0: every CTA's sorted list
    uint32_t* slots = reinterpret_cast<uint32_t*>(merged + (n_cta > 1 ? n_cta * P.n_top : 0));    // maxima of the threads' batches
    unsigned long long* cand = reinterpret_cast<unsigned long long*>(smem);             // candidates
    unsigned long long* sorted = cand + kCandCap;                                       // the largest of the share, sorted
    int* hits = reinterpret_cast<int*>(sorted + kRowsMaxTop);                           // [kHitCap]

    const int row = (int)(blockIdx.x / (unsigned)n_cta), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float c = P.c;

    Share<T> sh;
    sh.row = static_cast<const T*>(P.logits) + (long long)row * P.ld;
    sh.V = P.V;
    sh.phase = (int)((reinterpret_cast<uintptr_t>(sh.row) & 15u) / sizeof(T));
    const int n_vec = (sh.phase + P.V + N - 1) / N, per = (n_vec + n_cta - 1) / n_cta;
    sh.first = min(n_vec, rank * per);
    sh.last = min(n_vec, sh.first + per);
    sh.whole_lo = sh.phase != 0 ? 1 : 0;
    sh.whole_hi = (sh.phase + P.V) / N;
    T* grad_row = kOp != OP_LOGPROBS && P.out_grad != nullptr ? static_cast<T*>(P.out_grad) + (long long)row * P.ld_grad : nullptr;

    const int n_share = sh.last - sh.first, n_batches = (n_share + kBatch - 1) / kBatch;
    // on its way before anything else is looked at: the share, or its first batches
    for (int b = 0; b < (kResident ? n_batches : kRing); ++b) sh.fetch_batch(sh.first + b * kBatch, stash + b * kBatch + tid);

    float w = P.inv_temp;   // factor of the gradient
    int tok = -1;
    float tok_x = neg_inf();
    if (kOp != OP_DISTILL && P.tokens != nullptr) {
        tok = P.tokens[row];
        if (tok < 0 || tok >= P.V) tok = -1;
        if (tok >= 0) tok_x = RowVec<T>::get(sh.row + tok);
    }
    float g_lp = 0.0f, g_h = 0.0f;
    bool zero_grad = false;
    if (kOp == OP_GRAD) {
        g_lp = P.g_logprob != nullptr && tok >= 0 ? P.g_logprob[row] : 0.0f;
        g_h = P.g_entropy != nullptr ? P.g_entropy[row] : 0.0f;
        zero_grad = g_lp == 0.0f && g_h == 0.0f;
    }
    const bool use_bits = kOp == OP_DISTILL && (P.tail == DM_TAIL_BUCKET || grad_row != nullptr);
    TeacherEntry te{-1, neg_inf(), neg_inf(), false, 0.0};
    if (kOp == OP_DISTILL) {
        if (P.weight != nullptr) { const float wt = P.weight[row]; zero_grad = wt == 0.0f; w *= wt; }
        if (tid < P.k) {
            te.id = P.t_ids[(long long)row * P.k + tid];
            te.v = P.t_logprob[(long long)row * P.k + tid];
            if (te.id < 0 || te.id >= P.V) te.id = -1;
            if (te.id >= 0) te.x = RowVec<T>::get(sh.row + te.id);
            ss.t_id[tid] = te.id;
        }
        if (tid == 0) { ss.t_distinct = 0; ss.t_repeated = 0; }
        if (use_bits)
            for (int i = tid; i < n_batches * kBatch / 4; i += kThreads) reinterpret_cast<uint32_t*>(bitmap)[i] = 0u;
        if (warp < kRowsMaxTop / 32) {
            float vm = te.id >= 0 ? te.v : neg_inf();
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) vm = fmaxf(vm, __shfl_xor_sync(0xFFFFFFFFu, vm, off));
            if (lane == 0) ss.t_max[warp] = vm;
        }
        __syncthreads();
        if (use_bits && te.id >= 0) {
            const int at = (te.id + sh.phase) / N - sh.first;   // vector within the share
            if (at >= 0 && at < sh.last - sh.first) {
                const uint32_t bit = 1u << (8 * (at & 3) + (te.id + sh.phase) % N);
                te.first = (atomicOr(reinterpret_cast<uint32_t*>(bitmap) + (at >> 2), bit) & bit) == 0u;
                if (te.first) atomicAdd(&ss.t_distinct, 1); else ss.t_repeated = 1;
            }
        }
        __syncthreads();
        if (warp < kRowsMaxTop / 32) {
            float vm = ss.t_max[0];
#pragma unroll
            for (int i = 1; i < kRowsMaxTop / 32; ++i) vm = fmaxf(vm, ss.t_max[i]);
            const double shift = P.tail == DM_TAIL_RENORM && vm > neg_inf() ? (double)vm : 0.0;
            if (te.id >= 0) te.q = exp((double)te.v - shift);
            double sum = te.q;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
            if (lane == 0) ss.t_sum[warp] = sum;      // read behind the barriers below
        }
    }

    // A row whose gradient is zero whatever it holds is not looked at (unless its loss is wanted).
    const bool need_stats = !(zero_grad && (kOp == OP_GRAD || P.out_loss == nullptr));
    if (need_stats) {
        Stats st;
        st.init();
        const bool bucket = kTail && P.tail == DM_TAIL_BUCKET;
        float thread_max = neg_inf();
        if (kResident) {
            for (int b = 0; b < n_batches; ++b) {
                uint4 v[kUnroll];
                copy_wait(n_batches - 1 - b);
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) v[u] = stash[b * kBatch + u * kThreads + tid];
                thread_max = max_nan(thread_max, RowVec<T>::vmax(v));
            }
            float m = thread_max;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, off));
            if (lane == 0) ss.w_m[warp] = m;
            __syncthreads();
            m = ss.w_m[0];
#pragma unroll
            for (int i = 1; i < kWarps; ++i) m = max_nan(m, ss.w_m[i]);
            st.set_maximum<T>(m, c);
            const bool holder = __any_sync(0xFFFFFFFFu, thread_max == m && m != neg_inf());
            __syncthreads();   // (w_m is written again below)
            for (int b = 0; b < n_batches && (holder || st.ce != 0.0f); ++b) {
                uint4 v[kUnroll];
                uint32_t bits[kUnroll];
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    v[u] = stash[b * kBatch + u * kThreads + tid];
                    bits[u] = bucket ? bitmap[b * kBatch + u * kThreads + tid] : 0u;
                }
                if (holder) st.take<T, kTail>(v, bits);
                if (st.ce != 0.0f) st.sum<T, kEntropy, kTail>(v, bits);
            }
        } else {
            uint32_t* slot = slots + tid;
            uint32_t slot_key = 0u;
            int in_slot = 0;
            uint4* ring = stash + tid;
            for (int b = 0; b < n_batches; ++b) {   // the same for the whole block; kRing batches in flight
                uint4 v[kUnroll];
                uint32_t bits[kUnroll];
                copy_wait(kRing - 1);
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    v[u] = ring[u * kThreads];
                    bits[u] = bucket ? bitmap[b * kBatch + u * kThreads + tid] : 0u;
                }
                sh.fetch_batch(sh.first + (b + kRing) * kBatch, ring);
                ring = ring == stash + tid + (kRing - 1) * kBatch ? stash + tid : ring + kBatch;
                const float lane_max = RowVec<T>::vmax(v);
                if (kOp == OP_LOGPROBS && P.n_top > 0) {
                    thread_max = max_nan(thread_max, lane_max);
                    slot_key = max(slot_key, logit_key(lane_max));
                    if (++in_slot == P.slot_batches || b == n_batches - 1) {
                        *slot = slot_key;
                        slot += kThreads;
                        slot_key = 0u;
                        in_slot = 0;
                    }
                }
                st.add<T, kEntropy, kTail>(v, lane_max, c, bits);
            }
        }
        if (!kResident) copy_wait(0);   // (what is still in flight are empty batches)
        if (n_cta > 1) cluster_wait();
        block_merge(st, c, ss, cluster, n_cta, rank);
        if (kOp == OP_LOGPROBS && P.n_top > 0) {
            top_of_share(sh, thread_max, P.n_top, slots, P.slot_batches, ss, hits, cand, sorted);
            if (n_cta > 1)
                for (int i = tid; i < P.n_top; i += kThreads) cluster.map_shared_rank(merged, 0)[rank * P.n_top + i] = sorted[i];
        }
        if (n_cta > 1) {
            __syncwarp();
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
        if (warp == 0) cluster_merge(ss, n_cta, c);
    } else {
        copy_wait(0);
        if (n_cta > 1) cluster_wait();
        if (tid == 0) {
            ss.all = Merged{0.0f, 0.0f, 0.0f, 0.0f};
            ss.log_total = ss.inv_total = 0.0f;
        }
    }
    __syncthreads();
    const Merged a = ss.all;
    const bool dead = a.m == neg_inf();                 // every entry masked: no distribution
    const float log_total = ss.log_total, inv_total = ss.inv_total;
    const float entropy = dead ? 0.0f : fmaf(-kLn2 * inv_total, a.t, log_total);

    if (kOp == OP_LOGPROBS) {
        // fail-safe: a kernel ahead that produced these logits gave up on a wait
        const bool failed = P.err != nullptr && *P.err != 0u;
        const float bad = __uint_as_float(0x7FC00000u);
        if (rank == 0 && tid == 0) {
            if (P.out_logprob != nullptr)
                P.out_logprob[row] = failed ? bad : tok < 0 ? 0.0f : tok_x == neg_inf() && a.rest == a.rest ? neg_inf() : fmaf(tok_x - a.m, P.inv_temp, -log_total);
            if (P.out_lse != nullptr) P.out_lse[row] = failed ? bad : dead ? neg_inf() : fmaf(a.m, P.inv_temp, log_total);
            if (P.out_entropy != nullptr) P.out_entropy[row] = failed ? bad : entropy;
        }
        if (P.n_top > 0 && rank == 0) {
            // merge of sorted lists: the rank of an entry is its place in its own list plus the number
            // of larger ones in each other list
            const int k = P.n_top;
            const unsigned long long* lists = n_cta > 1 ? merged : sorted;
            for (int i = tid; i < n_cta * k; i += kThreads) {
                const unsigned long long mine = lists[i];
                if (mine == 0ull) continue;
                int place = i % k;
                for (int r = 0; r < n_cta && place < k; ++r) {
                    if (r == i / k) continue;
                    int lo = 0, hi = k;       // entries of list r that are larger
                    while (lo < hi) {
                        const int mid = (lo + hi) >> 1;
                        if (lists[r * k + mid] > mine) lo = mid + 1; else hi = mid;
                    }
                    place += lo;
                }
                if (place < k) {
                    const uint32_t key = (uint32_t)(mine >> 32);
                    const float x = key == 0xFFFFFFFFu ? bad : key_float(key);
                    P.out_top_ids[(long long)row * k + place] = failed ? -1 : (int32_t)best_index(mine);
                    P.out_top_logprob[(long long)row * k + place] =
                        failed ? bad : x == neg_inf() && a.rest == a.rest ? neg_inf() : fmaf(x - a.m, P.inv_temp, -log_total);
                }
            }
        }
    }

    float mass = 0.0f, rest = 0.0f;   // sum of the teacher's q, mass of its bucket (0: no bucket)
    if (kOp == OP_DISTILL) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < kRowsMaxTop / 32; ++i) sum += ss.t_sum[i];
        const double scale = P.tail == DM_TAIL_RENORM ? (sum != 0.0 ? 1.0 / sum : 0.0) : 1.0;
        mass = (float)(sum * scale);
        // tokens outside the teacher's exist unless k reaches V (such a row is one CTA's)
        if (P.tail == DM_TAIL_BUCKET && (P.k < P.V || ss.t_distinct < P.V)) rest = 1.0 - sum > 0.0 || sum != sum ? (float)(1.0 - sum) : 0.0f;
        if (warp < kRowsMaxTop / 32) {
            const float q = (float)(te.q * scale);
            if (tid < P.k) ss.t_q[tid] = q;
            if (rank == 0 && P.out_loss != nullptr) {
                // log q = v - shift - log(sum): no logarithm per entry
                float vm = ss.t_max[0];
#pragma unroll
                for (int i = 1; i < kRowsMaxTop / 32; ++i) vm = fmaxf(vm, ss.t_max[i]);
                const float log_sum = P.tail == DM_TAIL_RENORM && sum > 0.0 ? logf((float)sum) : 0.0f;
                const double base = P.tail == DM_TAIL_RENORM && vm > neg_inf() ? (double)vm + (double)log_sum : 0.0;
                float term = 0.0f;
                if (te.id >= 0 && !(q == 0.0f)) {
                    const double logp = dead || te.x == neg_inf() ? -INFINITY : ((double)te.x - (double)a.m) * P.inv_temp_d - (double)log_total;
                    term = (float)((double)q * (((double)te.v - base) - logp));
                }
                term = warp_sum(term);
                if (lane == 0) ss.t_loss[warp] = term;
            }
        }
        __syncthreads();
        if (rank == 0 && tid == 0 && P.out_loss != nullptr) {
            float loss = 0.0f;
#pragma unroll
            for (int i = 0; i < kRowsMaxTop / 32; ++i) loss += ss.t_loss[i];
            if (rest != 0.0f && !(dead && mass == 0.0f)) loss += rest * (logf(rest) - (logf(a.tail) - log_total));
            P.out_loss[row] = loss;
        }
    }

    if (kOp != OP_LOGPROBS && grad_row != nullptr) {
        // with w = (x - m) c in powers of two:  logprobs  dx = 2^w (A + B w);  distill  dx = 2^w A, A taking
        // the bucket's share off every entry (the teacher's tokens are written over below)
        const bool none = zero_grad || dead;
        float A, B = 0.0f, A_top = 0.0f;
        if (kOp == OP_GRAD) {
            A = -w * inv_total * fmaf(g_h, entropy - log_total, g_lp);
            B = -w * inv_total * g_h * kLn2;
        } else {
            const float tail_factor = rest > 0.0f && a.tail > 0.0f ? rest / a.tail : 0.0f;   // q_t / (sum of the tail's exponentials)
            A_top = w * (mass + rest) * inv_total;
            A = w * fmaf(mass + rest, inv_total, -tail_factor);
        }
        const bool same_phase = (int)((reinterpret_cast<uintptr_t>(grad_row) & 15u) / sizeof(T)) == sh.phase;
        const f32x2 m2 = pair(-a.m, -a.m), c2 = pair(c, c), A2 = pair(A, A), B2 = pair(B, B);
        const auto convert = [&](uint4 v) {
            f32x2 x[N / 2];
            RowVec<T>::pairs(v, x);
#pragma unroll
            for (int n = 0; n < N / 2; ++n) {
                f32x2 z = mul2(add2(x[n], m2), c2);
                if (kOp == OP_GRAD) {
                    z.x = fmaxf(z.x, kFloorExp);
                    z.y = fmaxf(z.y, kFloorExp);
                    x[n] = mul2(pair(ex2(z.x), ex2(z.y)), fma2(B2, z, A2));
                } else {
                    x[n] = mul2(pair(ex2(z.x), ex2(z.y)), A2);
                }
            }
            return RowVec<T>::pack_pairs(x);
        };
        // whole vectors that are in the stash and land on a 16-byte boundary: the bulk of a row
        int j = sh.first + tid;
        if (same_phase && !none) {
            if (j < sh.whole_lo) j += kThreads;
            const int end = kResident ? min(sh.last, sh.whole_hi) : j;
            uint4* dst = reinterpret_cast<uint4*>(grad_row - sh.phase);
#pragma unroll 4
            for (; j < end; j += kThreads) __stcs(dst + j, convert(stash[j - sh.first]));
        }
        for (int edge = same_phase && !none && sh.first + tid < sh.whole_lo; edge >= 0; --edge) {   // ... and what is left
            for (int i = edge ? sh.first + tid : j; i < (edge ? sh.whole_lo : sh.last); i += kThreads) {
                const uint4 v = none ? make_uint4(0u, 0u, 0u, 0u)
                                     : convert(kResident ? stash[i - sh.first] : sh.load(i));
                const int i0 = sh.entry0(i);
                if (sh.whole(i) && same_phase) {
                    __stcs(reinterpret_cast<uint4*>(grad_row + i0), v);
                } else {
                    float x[N];
                    RowVec<T>::unpack(v, x);
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        if (i0 + n >= 0 && i0 + n < P.V) RowVec<T>::put(grad_row + i0 + n, x[n]);
                }
            }
        }
        __syncthreads();   // the entries that differ are written over by one thread each
        if (!none) {
            const int lo = sh.entry0(sh.first), hi = sh.entry0(sh.last);   // this share's entries
            if (kOp == OP_GRAD) {
                if (tid == 0 && tok >= 0 && tok >= lo && tok < hi) {   // (entries below 0 are the padding of the first vector)
                    const float z = fmaxf((tok_x - a.m) * c, kFloorExp), e = ex2(z);
                    // 1 - p of the largest entry is rest / total, without cancellation
                    const float one_less = tok_x == a.m ? a.rest * inv_total : 1.0f - e * inv_total;
                    const float by_entropy = -w * g_h * inv_total * e * fmaf(kLn2, z, entropy - log_total);
                    RowVec<T>::put(grad_row + tok, fmaf(w * g_lp, one_less, by_entropy));
                }
            } else if (te.first) {                       // (set only for tokens of this share)
                float q = ss.t_q[tid];
                if (ss.t_repeated) {
                    q = 0.0f;
                    for (int o = 0; o < P.k; ++o) q += ss.t_id[o] == te.id ? ss.t_q[o] : 0.0f;
                }
                const float e = ex2((te.x - a.m) * c);
                RowVec<T>::put(grad_row + te.id, fmaf(A_top, e, -w * q));
            }
        }
    }
}

template <typename T, int kOp, bool kResident>
int launch_kernel(const RowsParams& P, int dev, int cluster, size_t smem, cudaStream_t stream);

template <typename T, int kOp>
int launch_rows(RowsParams P, cudaStream_t stream) {
    constexpr int N = RowVec<T>::N, kBatch = kUnroll * kThreads;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    const bool grad = kOp != OP_LOGPROBS && P.out_grad != nullptr;
    const int n_vec = (P.V + 2 * N - 2) / N;          // at most, whatever the row's alignment
    // CTAs per row: as many as run at once where rows are few, not less than one batch each; gradient kernels cut a row until three shares fit an SM's shared memory.
    int cluster = 1;
    while (cluster < kRowsMaxCluster && 2ll * P.rows * cluster <= (grad ? 3ll : 4ll) * sms && n_vec > cluster * kBatch) cluster *= 2;
    if (grad)
        while (cluster < kRowsMaxCluster && (n_vec + cluster - 1) / cluster > kStashVecs) cluster *= 2;
    const int per = (n_vec + cluster - 1) / cluster, batches = (per + kBatch - 1) / kBatch;
    const size_t bits = kOp == OP_DISTILL && (P.tail == DM_TAIL_BUCKET || grad) ? (size_t)batches * kBatch : 0;
    const bool resident = grad && (size_t)batches * kBatch * 16 + bits <= kRowsSmemLimit;
    P.stash_vecs = (resident ? batches : kRing) * kBatch;
    size_t smem = (size_t)P.stash_vecs * 16 + bits;
    if (kOp == OP_LOGPROBS && P.n_top > 0) {
        P.slot_batches = (batches + kMaxSlots - 1) / kMaxSlots;
        const int n_slots = (batches + P.slot_batches - 1) / P.slot_batches;
        smem += (size_t)n_slots * kThreads * sizeof(uint32_t);
        if (cluster > 1) smem += (size_t)cluster * P.n_top * sizeof(unsigned long long);
        static_assert((kCandCap + kRowsMaxTop) * sizeof(unsigned long long) + kHitCap * sizeof(int) <= (size_t)kRing * kBatch * 16, "the lists fit the ring");
    }
    if (smem > kRowsSmemLimit) return DM_EUNSUPPORTED;
    if (kOp != OP_LOGPROBS && resident) return launch_kernel<T, kOp, kOp != OP_LOGPROBS>(P, dev, cluster, smem, stream);
    return launch_kernel<T, kOp, false>(P, dev, cluster, smem, stream);
}

template <typename T, int kOp, bool kResident>
int launch_kernel(const RowsParams& P, int dev, int cluster, size_t smem, cudaStream_t stream) {
    auto kern = rows_kernel<T, kOp, kResident>;
    static std::atomic<unsigned long long> prepared{0};   // devices whose limit has been raised, one bit each
    if (dev >= 64 || !((prepared.load() >> dev) & 1ull)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRowsSmemLimit) != cudaSuccess) {
            cudaGetLastError();
            return DM_ECUDA;
        }
        if (dev < 64) prepared.fetch_or(1ull << dev);
    }
    if ((long long)P.rows * cluster > 0x7FFFFFFFll) return DM_EUNSUPPORTED;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(P.rows * cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)cluster; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = cluster > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kern, P) != cudaSuccess || cudaGetLastError() != cudaSuccess) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    return DM_OK;
}

}  // namespace

int launch_rows_logprobs(const RowsParams& P, int dtype, cudaStream_t stream) {
    return dtype == DM_F32 ? launch_rows<float, OP_LOGPROBS>(P, stream) : launch_rows<__nv_bfloat16, OP_LOGPROBS>(P, stream);
}
int launch_rows_grad(const RowsParams& P, int dtype, cudaStream_t stream) {
    return dtype == DM_F32 ? launch_rows<float, OP_GRAD>(P, stream) : launch_rows<__nv_bfloat16, OP_GRAD>(P, stream);
}
int launch_rows_distill(const RowsParams& P, int dtype, cudaStream_t stream) {
    return dtype == DM_F32 ? launch_rows<float, OP_DISTILL>(P, stream) : launch_rows<__nv_bfloat16, OP_DISTILL>(P, stream);
}

}  // namespace dm
