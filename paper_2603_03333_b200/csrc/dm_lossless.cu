// dropmatch_verify_lossless: drafted tokens against the target's distribution, from given random numbers.
//
//   p_t = Softmax(target[t] / T),  q_t = Softmax(draft[t] / T_d)  (or all of q_t on the drafted token x_t)
//   accept x_t  <=>  u_t q_t(x_t) < p_t(x_t);   n = length of the accepted prefix
//   next ~ max(p_n - q_n, 0) / sum  (n < drafted)  or  p_n  (all accepted),  by inverse CDF in token order:
//   the first v with  sum_{w <= v} r(w) > u_next sum r
//
// Two kernels, no workspace.
// ratio_kernel: a cluster per drafted position reads both rows once (running maximum and sum of each, fp32
// exponentials, sums of batches joined in fp64) and leaves min(1, p / q) in out_accept_prob.  Bounds: HBM.
// next_kernel: a cluster per sequence finds n and draws from row n.  Decisions and the place in the cumulative sum
// are those of 64-bit arithmetic: a position whose u_t lies within 2^-16 of the fp32 ratio (far more than that
// is off, see kBand) is decided again from fp64 sums, and all sums over row n are fp64 with exponentials good to
// some 2^-50 (see exp_neg).  In fp32 a token of the flat tail of 100 thousand would come out one place off in about a
// draw of ten, and two engines with equal random numbers would drift apart.
#include "dm_lossless.h"
#include "dm_ptx.cuh"

namespace dm {

namespace {

constexpr int kMaxCluster = 8;
constexpr int kRatioThreads = 256, kRatioWarps = kRatioThreads / 32;
constexpr int kNextThreads = 512, kNextWarps = kNextThreads / 32;
// The fp32 ratio is p / q with the sums of two rows.  A term 2^w, w = (x - m) c, has a relative error of at most
// 2 |w| ln 2 2^-24 (two roundings) + 2^-24 |w| ln 2 (c) + 2^-22 (the instruction); the mean of |w| ln 2 under the
// row's own distribution is at most ln V <= 21, batches add 7 roundings: below 2^-16 / 4 for each row.
constexpr float kBand = 1.0f / 65536.0f;
constexpr double kFloor = -700.0;        // exponents below count as -infinity (e^-700 = 1e-304)

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

// Maximum m of some entries of a row and the sum of exp((x - m) / T) over them.  A NaN, and +inf, make s a NaN.
struct Sum { float m; double s; };

// ---------------------------------------------------------------------------------------- ratios

__device__ __forceinline__ Sum join(const Sum& a, const Sum& b, float c) {
    const float m = fmaxf(a.m, b.m);
    const double fa = a.m == m ? 1.0 : (double)ex2((a.m - m) * c), fb = b.m == m ? 1.0 : (double)ex2((b.m - m) * c);
    return Sum{m, a.s * fa + b.s * fb};
}

template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int kN = 4;
    __device__ static void unpack(const uint4& v, float* x) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int kN = 8;
    __device__ static void unpack(const uint4& v, float* x) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
};

template <int N>
__device__ __forceinline__ void add_batch(Sum& a, const float (&x)[N], float c) {
    float bm = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) bm = fmaxf(bm, x[i]);
    if (bm > a.m) {
        a.s *= (double)ex2((a.m - bm) * c);     // (0 * 0 at the first batch; a NaN stays)
        a.m = bm;
    }
    const float ref = a.m == neg_inf() ? 0.0f : a.m;      // nothing but -inf so far: every term 0
    const float2 m2 = make_float2(-ref, -ref), c2 = make_float2(c, c);
    float2 s[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 z = __fmul2_rn(__fadd2_rn(make_float2(x[i], x[i + 1]), m2), c2);
        s[(i >> 1) & 1] = __fadd2_rn(s[(i >> 1) & 1], make_float2(ex2(z.x), ex2(z.y)));
    }
    a.s += (double)((s[0].x + s[0].y) + (s[1].x + s[1].y));
}

// Entries [lo, hi) of a row by the CTA's threads: 16-byte vectors, and the ragged ends entry by entry.
template <typename T>
__device__ __forceinline__ Sum thread_sum(const T* row, int lo, int hi, float c) {
    constexpr int kN = Vec<T>::kN, kBatch = 4;
    Sum a{neg_inf(), 0.0};
    const int off = (int)((reinterpret_cast<uintptr_t>(row + lo) & 15u) / sizeof(T));
    int head = off == 0 ? 0 : kN - off;
    head = min(head, hi - lo);
    const int vecs = (hi - lo - head) / kN, tail = lo + head + vecs * kN;
    if (threadIdx.x < 2 * kN) {     // at most kN - 1 entries on either side
        const int j = threadIdx.x < kN ? lo + (int)threadIdx.x : tail + (int)threadIdx.x - kN;
        const bool have = threadIdx.x < kN ? j < lo + head : j < hi;
        const float x[2] = {have ? entry(row, j) : neg_inf(), neg_inf()};
        add_batch(a, x, c);
    }
    const uint4* body = reinterpret_cast<const uint4*>(row + lo + head);
    const uint32_t none = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;      // -inf
#pragma unroll 1
    for (int v0 = threadIdx.x; v0 < vecs; v0 += kBatch * kRatioThreads) {
        uint4 v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            v[i] = make_uint4(none, none, none, none);
            if (v0 + i * kRatioThreads < vecs) v[i] = __ldg(body + v0 + i * kRatioThreads);
        }
        float x[kBatch * kN];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) Vec<T>::unpack(v[i], x + i * kN);
        add_batch(a, x, c);
    }
    return a;
}

__device__ __forceinline__ Sum block_sum(Sum a, float c, Sum* s_warp) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const Sum o{__shfl_xor_sync(0xFFFFFFFFu, a.m, off), __shfl_xor_sync(0xFFFFFFFFu, a.s, off)};
        a = (threadIdx.x & off) == 0 ? join(a, o, c) : join(o, a, c);
    }
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = a;
    __syncthreads();
    a = s_warp[0];
    for (int w = 1; w < kRatioWarps; ++w) a = join(a, s_warp[w], c);
    return a;
}

template <typename TP, typename TQ, bool HAS_Q>
__global__ void __launch_bounds__(kRatioThreads)
ratio_kernel(const LosslessParams P, int cluster) {
    __shared__ Sum s_warp[2][kRatioWarps];
    __shared__ __align__(16) double s_part[kMaxCluster][4];     // of every CTA: m and s of the target's row, of the draft's
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
    const int tok = P.draft[pos];
    const bool in_range = (unsigned)tok < (unsigned)P.V;
    float xp = 0.0f, xq = 0.0f;
    if (rank == 0 && threadIdx.x == 0 && in_range) {
        xp = entry(row_p, tok);
        if (HAS_Q) xq = entry(row_q, tok);
    }
    Sum p = thread_sum(row_p, lo, hi, P.c), q{0.0f, 1.0};
    if (HAS_Q) q = thread_sum(row_q, lo, hi, P.c_draft);
    p = block_sum(p, P.c, s_warp[0]);
    if (HAS_Q) q = block_sum(q, P.c_draft, s_warp[1]);
    if (cluster > 1) {
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        if (threadIdx.x == 0) {
            const uint32_t to = ptx::map_to_cta(ptx::smem_u32(&s_part[rank][0]), 0);
            st_cluster_f64(to, (double)p.m);
            st_cluster_f64(to + 8, p.s);
            st_cluster_f64(to + 16, (double)q.m);
            st_cluster_f64(to + 24, q.s);
        }
        ptx::cluster_sync_all();
        if (rank != 0 || threadIdx.x != 0) return;
        for (int r = 1; r < cluster; ++r) {
            p = join(p, Sum{(float)s_part[r][0], s_part[r][1]}, P.c);
            if (HAS_Q) q = join(q, Sum{(float)s_part[r][2], s_part[r][3]}, P.c_draft);
        }
    }
    if (threadIdx.x != 0) return;
    float ratio = 0.0f;
    if (isnan(p.s) || isnan(q.s)) {
        ratio = __uint_as_float(0x7FC00000u);
    } else if (in_range && xp > neg_inf()) {          // (a row of nothing but -inf has no such entry)
        const double lp = ((double)xp - (double)p.m) * P.inv_temp - log(p.s);
        if (!HAS_Q) ratio = (float)exp(lp);
        else if (xq == neg_inf()) ratio = 1.0f;
        else ratio = (float)exp(lp - (((double)xq - (double)q.m) * P.inv_draft_temp - log(q.s)));
        ratio = fminf(ratio, 1.0f);
    }
    P.out_accept_prob[pos] = ratio;
}

// ------------------------------------------------------------------------------------------ next

// exp(z) for z <= 0 (0 below kFloor; a NaN stays): z = n ln2/16 + r, |r| <= ln2/32, exp(z) = 2^(n div 16) table[n mod 16] e^r
// with e^r by its Taylor polynomial (r^7/7! < 2^-51): table-driven reduction after Tang, ACM TOMS 15 (1989).  Sixteen
// doubles lie in as many pairs of banks: lanes never conflict.
__device__ __forceinline__ double exp_neg(double z, const double* table) {
    const double shift = 6755399441055744.0;        // 1.5 2^52: the sum's low word holds the rounded quotient
    const double k = fma(z, 23.083120654223414, shift);
    const int n = __double2loint(k);
    const double r = fma(k - shift, -0.043321698784996581, z);
    double e = fma(r, 1.0 / 720.0, 1.0 / 120.0);
    e = fma(r, e, 1.0 / 24.0);
    e = fma(r, e, 1.0 / 6.0);
    e = fma(r, e, 0.5);
    e = fma(r, e, 1.0);
    e = fma(r, e, 1.0) * table[n & 15];
    e = __hiloint2double(__double2hiint(e) + (n >> 4) * 1048576, __double2loint(e));
    return z < kFloor ? 0.0 : e;
}

__device__ __forceinline__ Sum join64(const Sum& a, const Sum& b, double inv_temp, const double* table) {
    const float m = fmaxf(a.m, b.m);
    const double fa = a.m == m ? 1.0 : exp_neg(((double)a.m - (double)m) * inv_temp, table);
    const double fb = b.m == m ? 1.0 : exp_neg(((double)b.m - (double)m) * inv_temp, table);
    return Sum{m, a.s * fa + b.s * fb};
}

// exp((x - m) / T); m = -inf (a row of nothing else): 0.  x = +inf or NaN: NaN.
__device__ __forceinline__ double weight(float x, float m, double inv_temp, const double* table) {
    if (!(x > neg_inf()) && x == x) return 0.0;
    const double e = exp_neg(((double)x - (double)m) * inv_temp, table);
    return x == x && x < -neg_inf() ? e : __longlong_as_double(0x7FF8000000000000ll);
}

// Sum over entries [lo, hi) by a warp, lanes on neighbouring entries.
template <typename T>
__device__ __forceinline__ Sum warp_sum64(const T* row, int lo, int hi, double inv_temp, const double* table) {
    constexpr int kBatch = 8;
    const int lane = threadIdx.x & 31;
    Sum a{neg_inf(), 0.0};
#pragma unroll 1
    for (int j0 = lo; j0 < hi; j0 += 32 * kBatch) {
        float x[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) x[i] = hi - j0 > 32 * i + lane ? entry(row, j0 + 32 * i + lane) : neg_inf();
        float bm = x[0];
#pragma unroll
        for (int i = 1; i < kBatch; ++i) bm = fmaxf(bm, x[i]);
        if (bm > a.m) {
            a.s = a.s == 0.0 ? 0.0 : a.s * exp_neg(((double)a.m - (double)bm) * inv_temp, table);
            a.m = bm;
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) a.s += weight(x[i], a.m, inv_temp, table);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const Sum o{__shfl_xor_sync(0xFFFFFFFFu, a.m, off), __shfl_xor_sync(0xFFFFFFFFu, a.s, off)};
        a = (lane & off) == 0 ? join64(a, o, inv_temp, table) : join64(o, a, inv_temp, table);
    }
    return a;
}

// Which of `count` parts holds the place `at` of their cumulative weight; `at` becomes the place within it.  Where
// rounding (or a random number of 1) leaves none, the last part with any weight, and no place in it is reached.
template <typename F>
__device__ __forceinline__ int part_of(double& at, int count, F weight_of) {
    double sum = 0.0;
    int last = 0;
    for (int i = 0; i < count; ++i) {
        const double w = weight_of(i);
        if (!(w > 0.0)) continue;
        if (at < sum + w) {
            at -= sum;
            return i;
        }
        sum += w;
        last = i;
    }
    at = __longlong_as_double(0x7FF0000000000000ll);
    return last;
}

constexpr int kNone = 0x7FFFFFFF;

struct NextShared {
    double table[16];
    double warp_part[kNextWarps][4];
    double part[2][kMaxCluster][4];     // of every CTA, written by it; two sets in turn, so that one barrier per exchange does
    double scan[kNextWarps];
    int found, last;
};

// Everybody's four numbers for everybody: CTA `rank` writes v into set `set` of all CTAs of the cluster.
__device__ __forceinline__ void exchange(NextShared& S, int set, int rank, int cluster, const double (&v)[4]) {
    if (threadIdx.x < (unsigned)cluster) {
        const uint32_t to = ptx::map_to_cta(ptx::smem_u32(&S.part[set][rank][0]), threadIdx.x);
#pragma unroll
        for (int i = 0; i < 4; ++i) st_cluster_f64(to + 8 * i, v[i]);
    }
    ptx::cluster_sync_all();
}

template <typename TP, typename TQ, bool HAS_Q>
__global__ void __launch_bounds__(kNextThreads)
next_kernel(const LosslessParams P, int cluster) {
    __shared__ NextShared S;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = (int)(blockIdx.x / (unsigned)cluster), rank = (int)(blockIdx.x % (unsigned)cluster);
    if (threadIdx.x < 16) S.table[threadIdx.x] = exp2((double)threadIdx.x / 16.0);
    if (threadIdx.x == 0) { S.found = kNone; S.last = -1; }
    ptx::cluster_sync_all();      // (the other CTAs have started: their shared memory may be written)
    ptx::griddep_wait();

    const int len = P.draft_len == nullptr ? P.T : min(P.T, max(0, P.draft_len[b]));
    // the CTA's part of a row, and the warp's part of that, both in token order
    const int lo = (int)min((long long)P.V, (long long)rank * P.share), hi = (int)min((long long)P.V, (long long)lo + P.share);
    const int per_warp = ((hi - lo + kNextWarps - 1) / kNextWarps + 31) & ~31;
    const int w_lo = (int)min((long long)hi, (long long)lo + (long long)warp * per_warp), w_hi = (int)min((long long)hi, (long long)w_lo + per_warp);
    const TP* target = static_cast<const TP*>(P.target) + (long long)b * (P.T + P.bonus) * P.ld_target;
    const TQ* draft_rows = static_cast<const TQ*>(P.draft_logits) + (long long)b * P.T * P.ld_draft;
    int set = 0;

    Sum p{neg_inf(), 0.0}, q{neg_inf(), 0.0};
    auto sums = [&](int t, bool with_q) {       // fp64 sums of row t of both models, known to every thread of the cluster
        Sum a = warp_sum64(target + (long long)t * P.ld_target, w_lo, w_hi, P.inv_temp, S.table), o{neg_inf(), 0.0};
        if (HAS_Q && with_q) o = warp_sum64(draft_rows + (long long)t * P.ld_draft, w_lo, w_hi, P.inv_draft_temp, S.table);
        if (lane == 0) { S.warp_part[warp][0] = a.m; S.warp_part[warp][1] = a.s; S.warp_part[warp][2] = o.m; S.warp_part[warp][3] = o.s; }
        __syncthreads();
        p = q = Sum{neg_inf(), 0.0};
        for (int w = 0; w < kNextWarps; ++w) {
            p = join64(p, Sum{(float)S.warp_part[w][0], S.warp_part[w][1]}, P.inv_temp, S.table);
            if (HAS_Q && with_q) q = join64(q, Sum{(float)S.warp_part[w][2], S.warp_part[w][3]}, P.inv_draft_temp, S.table);
        }
        const double v[4] = {(double)p.m, p.s, (double)q.m, q.s};
        exchange(S, set, rank, cluster, v);
        p = q = Sum{neg_inf(), 0.0};
        for (int r = 0; r < cluster; ++r) {
            const double* o4 = S.part[set][r];
            p = join64(p, Sum{(float)o4[0], o4[1]}, P.inv_temp, S.table);
            if (HAS_Q && with_q) q = join64(q, Sum{(float)o4[2], o4[3]}, P.inv_draft_temp, S.table);
        }
        set ^= 1;
    };

    // the accepted prefix: the first position that is not surely accepted, decided in 64 bits if it may be
    int n = 0, known = -1;       // known: the row whose sums are in p and q
    while (n < len) {
        const int t = n + lane;
        float a = 1.0f, u = 0.0f;
        if (t < len) { a = P.out_accept_prob[(long long)b * P.T + t]; u = P.u_accept[(long long)b * P.T + t]; }
        const uint32_t open = __ballot_sync(0xFFFFFFFFu, !(u < a * (1.0f - kBand)));
        if (open == 0) { n = min(len, n + 32); continue; }
        const int first = __ffs(open) - 1;
        n += first;
        a = __shfl_sync(0xFFFFFFFFu, a, first);
        u = __shfl_sync(0xFFFFFFFFu, u, first);
        if (u > a * (1.0f + kBand)) break;
        const int tok = P.draft[(long long)b * P.T + n];
        if ((unsigned)tok >= (unsigned)P.V) break;
        sums(n, true);
        known = n;
        const float xp = entry(target + (long long)n * P.ld_target, tok), xq = HAS_Q ? entry(draft_rows + (long long)n * P.ld_draft, tok) : 0.0f;
        if (!(xp > neg_inf()) || !(p.s > 0.0) || !(HAS_Q ? q.s >= 0.0 : true)) break;     // p(x) = 0, or a NaN or +inf in a row
        if (!HAS_Q || xq > neg_inf()) {      // (q(x) = 0 otherwise)
            // by logarithms: p(x) and q(x) may both lie below fp64's range
            double l = ((double)xp - (double)p.m) * P.inv_temp - log(p.s);
            if (HAS_Q) l -= ((double)xq - (double)q.m) * P.inv_draft_temp - log(q.s);
            if (!(u <= 0.0f || (double)u < exp(l))) break;
        }
        ++n;
    }
    if (rank == 0 && threadIdx.x == 0) P.out_accept_len[b] = n;
    if (n >= P.T + P.bonus) {      // every drafted token accepted and no row behind them
        if (rank == 0 && threadIdx.x == 0) P.out_next[b] = -1;
        return;
    }

    // weights of row n: r = max(p - q, 0) if a token was rejected there, else p; p too, where r leaves nothing
    const bool rejected = n < len;
    if (known != n) sums(n, rejected);
    const int tok = rejected ? P.draft[(long long)b * P.T + n] : -1;
    const TP* row_p = target + (long long)n * P.ld_target;
    const TQ* row_q = draft_rows + (long long)n * P.ld_draft;
    const double inv_p = 1.0 / p.s, inv_q = HAS_Q && rejected && q.s != 0.0 ? 1.0 / q.s : 0.0;
    auto weights = [&](int j, double& all, double& rest) {
        all = weight(entry(row_p, j), p.m, P.inv_temp, S.table) * inv_p;
        rest = all;
        if (!rejected) return;
        if (HAS_Q) {
            const double other = weight(entry(row_q, j), q.m, P.inv_draft_temp, S.table) * inv_q;
            rest = other >= all ? 0.0 : all - other;      // (a NaN in either stays)
        } else if (j == tok) {
            rest = 0.0;
        }
    };
    double sum_all = 0.0, sum_rest = 0.0;
#pragma unroll 4
    for (int j = w_lo + lane; j < w_hi; j += 32) {
        double all, rest;
        weights(j, all, rest);
        sum_all += all;
        sum_rest += rest;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        sum_all += __shfl_xor_sync(0xFFFFFFFFu, sum_all, off);
        sum_rest += __shfl_xor_sync(0xFFFFFFFFu, sum_rest, off);
    }
    if (lane == 0) { S.warp_part[warp][0] = sum_all; S.warp_part[warp][1] = sum_rest; }
    __syncthreads();
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    for (int w = 0; w < kNextWarps; ++w) { v[0] += S.warp_part[w][0]; v[1] += S.warp_part[w][1]; }
    exchange(S, set, rank, cluster, v);
    double total[2] = {0.0, 0.0};
    for (int r = 0; r < cluster; ++r) { total[0] += S.part[set][r][0]; total[1] += S.part[set][r][1]; }
    // (no CTA writes to another from here on: each may leave when it is done)
    const int use = total[1] > 0.0 ? 1 : 0;
    if (!(total[use] > 0.0)) {      // nothing to draw from, or a NaN or +inf in a row
        if (rank == 0 && threadIdx.x == 0) P.out_next[b] = -1;
        return;
    }
    // the part that holds the place u_next * total: a CTA's, then a warp's
    double place = (double)P.u_next[b] * total[use];
    if (part_of(place, cluster, [&](int r) { return S.part[set][r][use]; }) != rank) return;
    const int pick = part_of(place, kNextWarps, [&](int w) { return S.warp_part[w][use]; });
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
            double all = 0.0, rest = 0.0;
            if (first + i < p_hi) weights(first + i, all, rest);
            r[i] = use ? rest : all;
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
        for (int w = 0; w < warp; ++w) cum += S.scan[w];
        for (int w = 0; w < kNextWarps; ++w) base += S.scan[w];
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

template <typename TP, typename TQ, bool HAS_Q>
int launch(LosslessParams& P, cudaStream_t stream) {
    const auto config = [&](cudaLaunchAttribute* attrs, int positions, int cluster, int threads, bool behind) {
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)positions * (unsigned)cluster);
        cfg.blockDim = dim3((unsigned)threads);
        cfg.stream = stream;
        cfg.attrs = attrs;
        attrs[0].id = cudaLaunchAttributeClusterDimension;
        attrs[0].val.clusterDim.x = (unsigned)cluster; attrs[0].val.clusterDim.y = 1; attrs[0].val.clusterDim.z = 1;
        attrs[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attrs[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.numAttrs = behind ? 2 : 1;
        return cfg;
    };
    // CTAs of a row: as many as have at least 2048 entries each, whole 16-byte vectors
    const auto cut = [&](int least) {
        int cluster = kMaxCluster;
        while (cluster > 1 && P.V / cluster < least) cluster /= 2;
        P.share = ((P.V + cluster - 1) / cluster + 7) & ~7;
        return cluster;
    };
    cudaLaunchAttribute attrs[2]{};
    if (P.T > 0) {
        const int cluster = cut(2048);
        const cudaLaunchConfig_t cfg = config(attrs, P.B * P.T, cluster, kRatioThreads, false);
        if (cudaLaunchKernelEx(&cfg, ratio_kernel<TP, TQ, HAS_Q>, P, cluster) != cudaSuccess) { cudaGetLastError(); return DM_ECUDA; }
    }
    const int cluster = cut(2048);
    // (behind the ratios: the kernel waits for them before it reads anything)
    const cudaLaunchConfig_t cfg = config(attrs, P.B, cluster, kNextThreads, P.T > 0);
    if (cudaLaunchKernelEx(&cfg, next_kernel<TP, TQ, HAS_Q>, P, cluster) != cudaSuccess) { cudaGetLastError(); return DM_ECUDA; }
    return cudaGetLastError() == cudaSuccess ? DM_OK : DM_ECUDA;
}

template <typename TP>
int launch_target(LosslessParams& P, int draft_dtype, cudaStream_t stream) {
    if (P.draft_logits == nullptr) return launch<TP, TP, false>(P, stream);
    if (draft_dtype == DM_F32) return launch<TP, float, true>(P, stream);
    return launch<TP, __nv_bfloat16, true>(P, stream);
}

}  // namespace

int launch_lossless(LosslessParams P, int dtype, int draft_dtype, cudaStream_t stream) {
    if (dtype == DM_F32) return launch_target<float>(P, draft_dtype, stream);
    return launch_target<__nv_bfloat16>(P, draft_dtype, stream);
}

}  // namespace dm
