// Device code shared by the kernels on rows of logits (dm_rows.cu, dm_rows_grad.cu): 16-byte vectors of
// a row, a CTA's share of it, and the running softmax statistics.
#pragma once
#include <atomic>

#include "dm_internal.h"
#include "dm_ptx.cuh"
#include "dm_rows.cuh"

namespace dm {
namespace rows {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kUnroll = 4;             // vectors of a batch: 16-byte loads in flight per thread
constexpr float kFloorExp = -200.0f;   // exponents are clamped here: 2^-200 is 0 in fp32, and 0 * clamp stays 0
// Exponents are taken against the rounded product m c while that is below this: its rounding error is then
// at most 64, half a step of fp32.  From here on the next number below m lies 2^-24 |m| or more away, 128
// powers of two: nothing next to m.
constexpr float kExactShift = 2147483648.0f;   // 2^31
constexpr float kSmallShift = 16777216.0f;     // 2^24: the error is at most half a power of two, and may scale any factor
// A tail of less than this, times the entries of the row, is summed anew, 2^64 times as large: 2^-126 of the
// row's mass may consist of entries far below fp32's range.  (Entries below 2^-126 are dropped by the first sum:
// at most 2^-32 of a larger tail.)
constexpr float kTailSmall = 5.0487097934144756e-29f;   // 2^-94
constexpr float kTailUp = 64.0f, kTailInv = 5.421010862427522e-20f;   // 2^-64
constexpr long long kRowsWaitCycles = 2000000000ll;   // about one second
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
// Maximum over the warp, in every lane: one instruction on sm_100a.  A NaN in any lane stays.
__device__ __forceinline__ float warp_max_nan(float x) {
    float y;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float warp_max(float x) {   // ... of numbers
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
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
    // ... counted only
    __device__ static void take_count(uint4& v, float m, uint32_t& n) { n += __popc(take(v, m)); }
    __device__ static int counted(uint32_t n) { return (int)n; }
    __device__ static float get(const float* p) { return *p; }
    // ... issued here and now, though the value is needed only at the end of the row
    __device__ static float get_early(const float* p) {
        float x;
        asm volatile("ld.global.f32 %0, [%1];" : "=f"(x) : "l"(p));
        return x;
    }
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
    // ... counted only, in the two halves of a word
    __device__ static void take_count_pair(uint32_t& v, uint32_t mm, uint32_t& n) {
        uint32_t eq;
        asm("set.eq.u32.bf16x2 %0, %1, %2;" : "=r"(eq) : "r"(v), "r"(mm));
        v = (v & ~eq) | (0xFF80FF80u & eq);
        n += eq & 0x00010001u;
    }
    __device__ static void take_count(uint4& v, float m, uint32_t& n) {
        const uint32_t mm = (__float_as_uint(m) >> 16) * 0x10001u;
        take_count_pair(v.x, mm, n); take_count_pair(v.y, mm, n); take_count_pair(v.z, mm, n); take_count_pair(v.w, mm, n);
    }
    __device__ static int counted(uint32_t n) { return (int)((n & 0xFFFFu) + (n >> 16)); }
    __device__ static float get(const __nv_bfloat16* p) {
        return __uint_as_float((uint32_t)*reinterpret_cast<const unsigned short*>(p) << 16);
    }
    __device__ static float get_early(const __nv_bfloat16* p) {
        unsigned short x;
        asm volatile("ld.global.u16 %0, [%1];" : "=h"(x) : "l"(p));
        return __uint_as_float((uint32_t)x << 16);
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
    int whole_end;            // ... and of the share: the smaller of last and whole_hi
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
    __device__ __forceinline__ bool whole_batch(int b0) const { return b0 >= whole_lo && b0 + kUnroll * kThreads <= whole_end; }
    // Sends one batch (vectors b0 + u * kThreads + thread) on its way to the thread's slots of shared
    // memory; slots past the end of the share are filled with masked entries.
    __device__ __forceinline__ void fetch_batch(int b0, uint4* slot) const {
        const uint4* p = vectors() + b0 + (int)threadIdx.x;
        if (whole_batch(b0)) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) copy_async(slot + u * kThreads, p + u * kThreads);
        } else {
            const int j = b0 + (int)threadIdx.x, n = whole_end - j, lo = whole_lo - j;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (u * kThreads < n && u * kThreads >= lo) copy_async(slot + u * kThreads, p + u * kThreads);
                else slot[u * kThreads] = RowVec<T>::masked();
            }
            if (j < whole_lo && j < last) *slot = load(j);   // the row's first vector, where it is not whole
            const int e = last - 1 - j;                      // ... and its last
            if (last > whole_hi && e >= 0 && e < kUnroll * kThreads && e % kThreads == 0) slot[e] = load(last - 1);
        }
        copy_commit();
    }
};

// Running statistics of a warp's entries.  Exponents are taken against rc, the rounded product m * c:
// w(x) = fma(x, ce, -rc) is then off by one rounding only; finish() moves the sums to m itself.  Where
// |m| c reaches kExactShift (rows filled with -1e10 or the type's lowest value, temperatures near 0) every
// other entry is nothing next to m: ce = 0 says so.
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
    template <typename T> __device__ __forceinline__ void set_maximum(float top, float c, float gap) {
        m = top;
        rc = top * c;
        ce = fabsf(rc) < kExactShift ? c : 0.0f;
        floor2 = RowVec<T>::floor_word(top - gap);
        cnt = 0;
    }
    // Entries equal to the maximum are counted and taken out of the batch.
    template <typename T, bool kTail>
    __device__ __forceinline__ void take(uint4 (&v)[kUnroll], uint32_t marks) {
        if constexpr (kTail) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const uint32_t eq = RowVec<T>::take(v[u], m);
                cnt += __popc(eq);
                tail = fmaf((float)__popc(eq & ~(marks >> (8 * u))), of_maximum(), tail);
            }
        } else {
            uint32_t n = 0u;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) RowVec<T>::take_count(v[u], m, n);
            cnt += RowVec<T>::counted(n);
        }
    }
    // A batch of entries below the maximum.  marks: the teacher's tokens in it (see mark_word); most warps
    // see none in a batch.
    template <typename T, bool kEntropy, bool kTail>
    __device__ __forceinline__ void sum(uint4 (&v)[kUnroll], uint32_t marks) {
        if (kTail && __any_sync(0xFFFFFFFFu, marks != 0u)) sum_marked<T>(v, marks);
        else sum_plain<T, kEntropy, kTail>(v);
    }
    template <typename T, bool kEntropy, bool kTail>
    __device__ __forceinline__ void sum_plain(uint4 (&v)[kUnroll]) {
        constexpr int N = RowVec<T>::N;
        const f32x2 c2 = pair(ce, ce), rc2 = pair(-rc, -rc);
        f32x2 bs = pair(0.0f, 0.0f), bt = bs;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (kEntropy) RowVec<T>::raise(v[u], floor2);
            f32x2 x[N / 2];
            RowVec<T>::pairs(v[u], x);
#pragma unroll
            for (int n = 0; n < N / 2; ++n) {
                f32x2 w = fma2(x[n], c2, rc2);
                if (kEntropy && !RowVec<T>::kFloorsEntries) { w.x = fmaxf(w.x, kFloorExp); w.y = fmaxf(w.y, kFloorExp); }
                const f32x2 e = pair(ex2(w.x), ex2(w.y));
                bs = add2(bs, e);
                if (kEntropy) bt = fma2(e, w, bt);   // (a masked entry: 0 * a finite exponent)
            }
        }
        const float all = sum2(bs);
        s += all;
        if (kTail) tail += all;
        if (kEntropy) t += sum2(bt);
    }
    template <typename T>
    __device__ __forceinline__ void sum_marked(const uint4 (&v)[kUnroll], uint32_t marks) {
        constexpr int N = RowVec<T>::N;
        const f32x2 c2 = pair(ce, ce), rc2 = pair(-rc, -rc);
        f32x2 in = pair(0.0f, 0.0f), out = in;     // the teacher's tokens, the others
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            f32x2 x[N / 2];
            RowVec<T>::pairs(v[u], x);
#pragma unroll
            for (int n = 0; n < N / 2; ++n) {
                const f32x2 w = fma2(x[n], c2, rc2), e = pair(ex2(w.x), ex2(w.y));
                const bool lo = (marks >> (8 * u + 2 * n)) & 1u, hi = (marks >> (8 * u + 2 * n + 1)) & 1u;
                out = add2(out, pair(lo ? 0.0f : e.x, hi ? 0.0f : e.y));
                in = add2(in, pair(lo ? e.x : 0.0f, hi ? e.y : 0.0f));
            }
        }
        const float rest = sum2(out);
        s += rest + sum2(in);
        tail += rest;
    }
    // A batch of whatever entries, with the maximum so far kept exactly.
    template <typename T, bool kEntropy, bool kTail>
    __device__ __forceinline__ void add(uint4 (&v)[kUnroll], float lane_max, float c, float gap, uint32_t marks) {
        const float wm = warp_max_nan(lane_max);
        if (!(wm < m && ce != 0.0f)) {
            if (wm == neg_inf()) return;   // nothing but masked entries so far
            if (m == m && !(wm <= m)) {    // a new maximum (a NaN stays one): the old one becomes an entry like the others
                const Stats old = *this;
                set_maximum<T>(wm, c, gap);
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
            take<T, kTail>(v, marks);
            if (ce == 0.0f) return;
        }
        sum<T, kEntropy, kTail>(v, marks);
    }
    __device__ __forceinline__ void finish() {
        if (ce == 0.0f) return;
        const float d = fmaf(m, ce, -rc), f = ex2(-d);   // rounding of rc, either sign: at most 64
        t = f * fmaf(-d, s, t);
        s *= f;
        tail *= f;
    }
};

struct Merged { float m, rest, t, tail; };   // maximum; sums relative to it, `rest` without one maximal entry

// Two parts of a row joined: relative to the larger maximum, whose holder alone stays left out.
__device__ __forceinline__ Merged join(const Merged& a, const Merged& p, float c) {
    const bool up = !(p.m <= a.m) && a.m == a.m;           // (a NaN on either side ends up as the maximum)
    const Merged hi = up ? p : a, lo = up ? a : p;
    const float d = fmaxf((lo.m - hi.m) * c, kFloorExp), f = lo.m == neg_inf() ? 0.0f : ex2(d), all = lo.rest + 1.0f;
    return Merged{hi.m, fmaf(f, all, hi.rest), fmaf(f, fmaf(d, all, lo.t), hi.t), fmaf(f, lo.tail, hi.tail)};
}

// Cluster barrier in two halves; every thread of every CTA takes both.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, off);
    return x;
}

// A vector's part of a small tail (entries that the teacher's tokens, marked, leave), 2^64 times as large.
template <typename T>
__device__ __forceinline__ float raised_sum(const uint4& v, uint32_t marks, float m, float c) {
    constexpr int N = RowVec<T>::N;
    float x[N], sum = 0.0f;
    RowVec<T>::unpack(v, x);
#pragma unroll
    for (int n = 0; n < N; ++n) sum += (marks >> n) & 1u ? 0.0f : ex2(fmaf(x[n] - m, c, kTailUp));
    return sum;
}
// Is the row's tail to be summed anew?  (The same in all CTAs of the cluster.)
__device__ __forceinline__ bool small_tail(const Merged& a, int V) { return a.tail < kTailSmall * (float)V && a.m != neg_inf(); }

// Less than 2^-126 of the row's mass counts as nothing.
__device__ __forceinline__ float counted_tail(float raised, float inv_total) {
    return raised * inv_total < 2.168404344971009e-19f ? 0.0f : raised;   // 2^(64 - 126)
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

// The largest value of a teacher's entries that are present, by one warp.
__device__ __forceinline__ float largest_value(const int* id, const float* v, int k) {
    float vm = neg_inf();
    for (int i = (int)(threadIdx.x & 31); i < k; i += 32) vm = fmaxf(vm, id[i] >= 0 ? v[i] : neg_inf());
    __syncwarp();
    return warp_max(vm);
}

// The loss of a row, by one warp.  fp64: it is a small difference of logarithms that are not small, and
// there are only k of them.  mass, rest: of the teacher's tokens and of its bucket (0: no bucket).
__device__ __forceinline__ float teacher_loss(const RowsParams& P, const Merged& a, const int* id, const float* v, const float* x,
                                              const float* q, double q_sum, double mass, double rest) {
    const int lane = threadIdx.x & 31;
    const bool dead = a.m == neg_inf();
    const float all_v = largest_value(id, v, P.k);
    // four logarithms at once, a lane each: of the student's total, the teacher's sum, its bucket, the tail
    const double of = lane == 0 ? 1.0 + (double)a.rest : lane == 1 ? q_sum : lane == 2 ? rest : (double)a.tail;
    const double logs = lane < 4 ? log(of) : 0.0;
    const double log_total = __shfl_sync(0xFFFFFFFFu, logs, 0), log_q = __shfl_sync(0xFFFFFFFFu, logs, 1);
    const double log_rest = __shfl_sync(0xFFFFFFFFu, logs, 2), log_tail = __shfl_sync(0xFFFFFFFFu, logs, 3);
    // log q = v - base: the teacher's normaliser
    const double base = P.tail == DM_TAIL_RENORM && all_v > neg_inf() ? (double)all_v + log_q : 0.0;
    double loss = 0.0, taken = 0.0;
    for (int i = lane; i < P.k; i += 32) {
        if (id[i] < 0 || q[i] == 0.0f) continue;
        const double logp = dead || x[i] == neg_inf() ? -INFINITY : ((double)x[i] - (double)a.m) * P.inv_temp_d - log_total;
        loss += (double)q[i] * (((double)v[i] - base) - logp);
        taken += (double)q[i];
    }
    __syncwarp();
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        loss += __shfl_xor_sync(0xFFFFFFFFu, loss, off);
        taken += __shfl_xor_sync(0xFFFFFFFFu, taken, off);
    }
    // the q's rounded to fp32 do not add up to the mass: log p of -3.4e38 (a mask) would become -inf
    if (taken > 0.0) loss *= mass / taken;
    if (rest != 0.0 && !(dead && mass == 0.0)) loss += rest * (log_rest - (log_tail - log_total));
    return (float)loss;
}

// Factors of a gradient, from the row's statistics: with w = (x - m) c in powers of two, every entry's
// gradient is 2^w (A + B w) (logprobs) or 2^(w + up) A (distill, where the teacher's tokens differ: top).
struct GradFactors { float A, B, top, up; };
__device__ __forceinline__ GradFactors logprob_factors(float w, float g_lp, float g_h, float entropy, float log_total, float inv_total) {
    return GradFactors{-w * inv_total * fmaf(g_h, entropy - log_total, g_lp), -w * inv_total * g_h * kLn2, 0.0f, 0.0f};
}
// mass: sum of the teacher's q; rest: mass of its bucket (0: no bucket), taken off every entry's share by
// q_t / (sum of the tail's exponentials)
__device__ __forceinline__ GradFactors distill_factors(float w, float mass, float rest, float tail, float inv_total) {
    const float share = rest > 0.0f && tail > 0.0f ? rest / tail : 0.0f;
    return GradFactors{w * fmaf(mass + rest, inv_total, -share), 0.0f, w * (mass + rest) * inv_total, 0.0f};
}
// The same for a tail that was summed anew, or where the factor overflows (a weight over a temperature of 1e20):
// `raised`, the tail 2^64 times as large; 0 if it counts as nothing.  The factor is 2^64 times too small and the exponents are raised, so that neither leaves fp32's range.
__device__ __forceinline__ GradFactors raised_factors(float w, float mass, float rest, float raised, float inv_total) {
    if (raised == 0.0f) return distill_factors(w, mass, rest, 0.0f, inv_total);
    float A = w * fmaf((mass + rest) * kTailInv, inv_total, -rest / raised);
    if (A == neg_inf()) A = -3.4028234e38f;   // (0 for a masked entry all the same)
    return GradFactors{A, 0.0f, w * (mass + rest) * inv_total, kTailUp};
}
// Gradient at the given token.  1 - p of the largest entry is rest / total, without cancellation.
__device__ __forceinline__ float token_grad(float x, const Merged& a, float c, float w, float g_lp, float g_h, float entropy,
                                            float log_total, float inv_total) {
    const float z = fmaxf((x - a.m) * c, kFloorExp), e = ex2(z);
    const float one_less = x == a.m ? a.rest * inv_total : 1.0f - e * inv_total;
    const float by_entropy = -w * g_h * inv_total * e * fmaf(kLn2, z, entropy - log_total);
    return fmaf(w * g_lp, one_less, by_entropy);
}
// A vector of the row -> the same vector of its gradient.  shift: the rounded product m c, whose rounding
// error `factors_against` has moved into the factors; where m c reaches kSmallShift, and for raised exponents,
// they are taken of differences (kPlain).
struct GradShift { float rc; uint32_t floor2; };
template <typename T, int kOp, bool kPlain = false>
__device__ __forceinline__ uint4 grad_vector(uint4 v, float m, float c, const GradShift& g, const GradFactors& f) {
    constexpr int N = RowVec<T>::N;
    const f32x2 m2 = kPlain ? pair(-m, -m) : pair(-g.rc, -g.rc), c2 = pair(c, c), A2 = pair(f.A, f.A), B2 = pair(f.B, f.B),
                up2 = pair(f.up, f.up);
    constexpr bool kClamp = kOp == OP_GRAD && (kPlain || !RowVec<T>::kFloorsEntries);   // (a masked entry: 0 * a finite exponent)
    if (kOp == OP_GRAD && !kClamp) RowVec<T>::raise(v, g.floor2);
    f32x2 x[N / 2];
    RowVec<T>::pairs(v, x);
#pragma unroll
    for (int n = 0; n < N / 2; ++n) {
        f32x2 z = kPlain ? kOp == OP_GRAD ? mul2(add2(x[n], m2), c2) : fma2(add2(x[n], m2), c2, up2) : fma2(x[n], c2, m2);
        if (kClamp) {
            z.x = fmaxf(z.x, kFloorExp);
            z.y = fmaxf(z.y, kFloorExp);
        }
        x[n] = mul2(pair(ex2(z.x), ex2(z.y)), kOp == OP_GRAD ? fma2(B2, z, A2) : A2);
    }
    return RowVec<T>::pack_pairs(x);
}
// With z' = z + d for every entry (d = m c - rc, at most 1/2 either way): 2^z (A + B z) = 2^z' 2^-d (A - B d + B z').
__device__ __forceinline__ GradFactors factors_against(const GradFactors& f, float d) {
    const float scale = ex2(-d);
    return GradFactors{scale * fmaf(-d, f.B, f.A), scale * f.B, f.top, 0.0f};
}
// ... and its way to the gradient's row (which may have another alignment).
template <typename T>
__device__ __forceinline__ void store_vector(T* grad_row, const Share<T>& sh, int j, bool same_phase, const uint4& v) {
    constexpr int N = RowVec<T>::N;
    const int i0 = sh.entry0(j);
    if (sh.whole(j) && same_phase) {
        __stcs(reinterpret_cast<uint4*>(grad_row + i0), v);
    } else {
        float x[N];
        RowVec<T>::unpack(v, x);
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (i0 + n >= 0 && i0 + n < sh.V) RowVec<T>::put(grad_row + i0 + n, x[n]);
    }
}
template <typename T>
__device__ __forceinline__ Share<T> share_of(const RowsParams& P, int row, int n_cta, int rank) {
    constexpr int N = RowVec<T>::N;
    Share<T> sh;
    sh.row = static_cast<const T*>(P.logits) + (long long)row * P.ld;
    sh.V = P.V;
    sh.phase = (int)((reinterpret_cast<uintptr_t>(sh.row) & 15u) / sizeof(T));
    const int n_vec = (sh.phase + P.V + N - 1) / N, per = (n_vec + n_cta - 1) >> (__ffs(n_cta) - 1);   // (a power of two)
    sh.first = min(n_vec, rank * per);
    sh.last = min(n_vec, sh.first + per);
    sh.whole_lo = sh.phase != 0 ? 1 : 0;
    sh.whole_hi = (sh.phase + P.V) / N;
    sh.whole_end = min(sh.last, sh.whole_hi);
    return sh;
}
// Marks of a share's teacher tokens: a byte per vector, the bytes of a thread's batch in one word.
__device__ __forceinline__ uint32_t* mark_word(unsigned char* marks, int at) {   // at: vector within the share
    return reinterpret_cast<uint32_t*>(marks) + at / (kUnroll * kThreads) * kThreads + at % kThreads;
}
__device__ __forceinline__ uint32_t mark_bit(int at, int entry) { return 1u << (8 * (at / kThreads % kUnroll) + entry); }
static_assert(kUnroll == 4, "the marks of a batch fill a word");

template <typename T>
__device__ __forceinline__ bool phase_of(const T* p, int phase) {
    return (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T)) == phase;
}

// The answer to a request for another row, by the thread that made it: the granted cluster's first CTA, or -1.
// An answer that comes after the limit is reported and used all the same: it lands in this CTA's shared memory,
// and the row that it grants is nobody else's.  (A limit of one cycle, which only dm_debug_set_wait_limit
// gives, has run out before the first look.)
__device__ __forceinline__ int granted_row(const RowsParams& P, uint32_t answer, uint32_t bar, uint32_t parity) {
    const long long t0 = clock64();
    bool late = P.wait_limit <= 1, came = true;
    while (came && !ptx::mbar_try_wait(bar, parity)) {
        __nanosleep(32);
        const long long waited = clock64() - t0;
        late = late || waited > P.wait_limit;
        came = waited <= P.wait_limit + kRowsWaitCycles;
    }
    if (late) atomicCAS(P.err_out, 0u, (uint32_t)ERR_WAIT_ROW);
    if (!came) return -1;
    const int next = ptx::granted_cluster(answer);
    ptx::fence_proxy_async_smem();   // read before the next request writes it
    return next;
}

// `prepared`: devices on which the kernel's shared-memory limit has been raised, one bit each.
template <typename Kernel>
bool raise_smem_limit(Kernel kern, std::atomic<unsigned long long>& prepared, int dev) {
    if (dev < 64 && ((prepared.load() >> dev) & 1ull)) return true;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRowsSmemLimit) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    if (dev < 64) prepared.fetch_or(1ull << dev);
    return true;
}
// Launches `ctas` CTAs in clusters.
template <typename Kernel>
int launch_clusters(Kernel kern, std::atomic<unsigned long long>& prepared, int dev, const RowsParams& P, long long ctas, int cluster,
                    size_t smem, cudaStream_t stream) {
    if (!raise_smem_limit(kern, prepared, dev)) return DM_ECUDA;
    if (ctas > 0x7FFFFFFFll) return DM_EUNSUPPORTED;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ctas);
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

}  // namespace rows
}  // namespace dm
