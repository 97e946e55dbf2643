// Operators on rows of logits x[N][V] in global memory (fp32 or bf16, any row stride):
//   logprobs       z = x / temperature;  lse = log sum_v exp z_v;  log-probability of a given token
//                  z_tok - lse;  entropy -sum_v p_v log p_v;  the n_top largest entries
//   logprobs_grad  gradient of g_lp * logprob + g_H * entropy with respect to x:
//                  (1/T) [ g_lp (1[v = tok] - p_v) - g_H p_v (log p_v + H) ]
//   distill        KL(teacher || student) for a teacher known by its top tokens, and its gradient
//                  (see distill_teacher below)
//
// A row belongs to one thread-block cluster; its CTAs take contiguous shares of the row, cut at
// 16-byte boundaries.  One pass over the share keeps, per thread, a running reference, the sum of
// 2^((x - ref) c) with c = log2(e) / T, the sum of those times their exponents (entropy) and the
// exact maximum.  Threads meet in the block, CTAs through distributed shared memory; the sums are
// kept WITHOUT the row's largest entry (its holder goes over its entries once more), so that
// log(1 + rest) keeps its precision next to a near-certain token.
//
// Bound: memory, one read of x (and one write of the gradient).  The gradient kernels keep as much
// of a CTA's share as fits in shared memory, so that x is read once; what does not fit is read again.
#include <cooperative_groups.h>

#include <atomic>

#include "dm_internal.h"
#include "dm_rows.cuh"

namespace dm {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kUnroll = 4;             // 16-byte loads in flight per thread
constexpr int kCandCap = 1024;         // candidates for the top entries of a CTA's share
constexpr float kSlack = 20.0f;        // how far (in powers of two) an entry may lie above the running reference
constexpr float kFloorExp = -200.0f;   // exponents are clamped here: 2^-200 is 0 in fp32, and 0 * clamp stays 0
constexpr int kStashVecs = 4352;       // 68 KB: three CTAs of a gradient kernel per SM
constexpr size_t kRowsSmemLimit = 200 * 1024;
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
    __device__ static float get(const __nv_bfloat16* p) {
        return __uint_as_float((uint32_t)*reinterpret_cast<const unsigned short*>(p) << 16);
    }
    __device__ static void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
};

// A CTA's share of a row: 16-byte vectors [first, last) of the row, vector j holding entries
// j*N - phase .. j*N - phase + N-1 (phase: entries between the 16-byte boundary below the row's
// start and that start).  Entries outside [0, V) read as -inf and are never written.
template <typename T> struct Share {
    const T* row;
    int V, phase, first, last;
    __device__ __forceinline__ int entry0(int j) const { return j * RowVec<T>::N - phase; }
    __device__ __forceinline__ bool whole(int j) const {
        const int i0 = entry0(j);
        return i0 >= 0 && i0 + RowVec<T>::N <= V;
    }
    // Loads go to L2 (ld.global.cg): the row may be overwritten in place by this very kernel, each
    // entry by the thread that read it.
    __device__ __forceinline__ uint4 load(int j) const {
        constexpr int N = RowVec<T>::N;
        if (whole(j)) return __ldcg(reinterpret_cast<const uint4*>(row + (long long)j * N - phase));
        float x[N];
        const int i0 = entry0(j);
#pragma unroll
        for (int n = 0; n < N; ++n) x[n] = (i0 + n >= 0 && i0 + n < V) ? RowVec<T>::get(row + i0 + n) : neg_inf();
        return RowVec<T>::pack(x);
    }
};

// Running statistics of a thread's entries, all relative to `ref` (<= mx): s = sum 2^z, t = sum z 2^z.
struct Stats {
    float ref, mx, s, t, tail;
    __device__ __forceinline__ void init() { ref = mx = neg_inf(); s = t = tail = 0.0f; }
    template <int N, bool kEntropy, bool kTail>
    __device__ __forceinline__ void add(const float (&x)[N], float c, uint32_t top_bits) {
        float vm = x[0];
#pragma unroll
        for (int n = 1; n < N; ++n) vm = max_nan(vm, x[n]);
        mx = max_nan(mx, vm);
        if (vm == neg_inf()) return;             // nothing but masked entries
        if (!((vm - ref) * c <= kSlack)) {       // rare: the first entries, or a far larger one (or NaN)
            const float d = max_nan((ref - vm) * c, kFloorExp), f = ref == neg_inf() ? 0.0f : ex2(d);
            t = f * fmaf(d, s, t);
            s *= f;
            tail *= f;
            ref = vm;
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float z = max_nan((x[n] - ref) * c, kFloorExp);
            const float e = ex2(z);
            s += e;
            if (kEntropy) t = fmaf(e, z, t);
            if (kTail) tail += ((top_bits >> n) & 1u) ? 0.0f : e;
        }
    }
};

struct Merged { float m, rest, t, tail; };   // maximum; sums relative to it, `rest` without one maximal entry

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, off);
    return x;
}

struct RowsShared {
    float red[3][kThreads / 32];
    int red_cnt[kThreads / 32];
    Merged mine;                 // this CTA's statistics, read by the others of the cluster
    int cand_n, thr_hits;
    unsigned int scan[kThreads / 32];
    // teacher (distill)
    int t_id[kRowsMaxTop];
    float t_q[kRowsMaxTop], t_x[kRowsMaxTop];
    unsigned char t_first[kRowsMaxTop];
    float t_mass, t_rest;        // sum of q, mass of the bucket (0: no bucket)
};

// The block's statistics from its threads'.  Holders of the block's maximum go over their entries
// once more and leave entries equal to it out of their sum, counting them instead.
template <typename T, bool kEntropy>
__device__ Merged block_merge(const Stats& st, const Share<T>& sh, float c, RowsShared& ss) {
    constexpr int N = RowVec<T>::N;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float m = st.mx;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, off));
    if (lane == 0) ss.red[0][warp] = m;
    __syncthreads();
    m = ss.red[0][0];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) m = max_nan(m, ss.red[0][w]);
    __syncthreads();
    float s = 0.0f, t = 0.0f, tail = 0.0f;
    int cnt = 0;
    if (st.ref != neg_inf()) {
        const float d = max_nan((st.ref - m) * c, kFloorExp), f = ex2(d);
        s = st.s * f;
        t = f * fmaf(d, st.s, st.t);
        tail = st.tail * f;
    }
    if (st.mx == m && m != neg_inf()) {
        s = t = 0.0f;
        for (int j = sh.first + (int)threadIdx.x; j < sh.last; j += kThreads) {
            float x[N];
            RowVec<T>::unpack(sh.load(j), x);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const float z = max_nan((x[n] - m) * c, kFloorExp), e = ex2(z);
                if (x[n] == m) ++cnt;
                else { s += e; if (kEntropy) t = fmaf(e, z, t); }
            }
        }
    }
    s = warp_sum(s);
    if (kEntropy) t = warp_sum(t);
    tail = warp_sum(tail);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) cnt += __shfl_xor_sync(0xFFFFFFFFu, cnt, off);
    if (lane == 0) { ss.red[0][warp] = s; ss.red[1][warp] = t; ss.red[2][warp] = tail; ss.red_cnt[warp] = cnt; }
    __syncthreads();
    Merged r{m, 0.0f, 0.0f, 0.0f};
    cnt = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        r.rest += ss.red[0][w]; r.t += ss.red[1][w]; r.tail += ss.red[2][w]; cnt += ss.red_cnt[w];
    }
    if (cnt > 1) r.rest += (float)(cnt - 1);
    if (m == __uint_as_float(0x7F800000u)) r.rest = r.t = r.tail = __uint_as_float(0x7FC00000u);   // +inf: no distribution
    return r;
}

// The cluster's statistics from its CTAs' (already published and synchronised).
__device__ Merged cluster_merge(cg::cluster_group& cluster, RowsShared& ss, int n_cta, float c) {
    if (n_cta == 1) return ss.mine;
    Merged part[kRowsMaxCluster];
    float m = neg_inf();
    int base = 0;
#pragma unroll 1
    for (int r = 0; r < n_cta; ++r) {
        part[r] = *cluster.map_shared_rank(&ss.mine, r);
        if (m == m && !(part[r].m <= m)) { m = part[r].m; base = r; }   // a NaN stays
    }
    Merged a{m, part[base].rest, part[base].t, part[base].tail};
    if (m != m) { a.rest = m; return a; }
#pragma unroll 1
    for (int r = 0; r < n_cta; ++r) {
        if (r == base || part[r].m == neg_inf()) continue;
        const float d = max_nan((part[r].m - m) * c, kFloorExp), f = ex2(d), s = part[r].rest + 1.0f;
        a.rest = fmaf(f, s, a.rest);
        a.t = fmaf(f, fmaf(d, s, part[r].t), a.t);
        a.tail = fmaf(f, part[r].tail, a.tail);
    }
    return a;
}

// ---------------------------------------------------------------------------- the largest entries
// Entries of the share with a key above `floor_key` (or not below it, with `or_equal`) go to the
// candidate list; only threads whose maximum passes look at their entries again.
template <typename T>
__device__ int collect(const Share<T>& sh, uint32_t my_key, uint32_t floor_key, bool or_equal, RowsShared& ss,
                       unsigned long long* cand) {
    constexpr int N = RowVec<T>::N;
    if (threadIdx.x == 0) ss.cand_n = 0;
    __syncthreads();
    if (my_key > floor_key || (or_equal && my_key == floor_key)) {
        for (int j = sh.first + (int)threadIdx.x; j < sh.last; j += kThreads) {
            float x[N];
            RowVec<T>::unpack(sh.load(j), x);
            const int i0 = sh.entry0(j);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const uint32_t key = logit_key(x[n]);
                if ((key > floor_key || (or_equal && key == floor_key)) && i0 + n >= 0 && i0 + n < sh.V) {
                    const int at = atomicAdd(&ss.cand_n, 1);
                    if (at < kCandCap) cand[at] = pack_best(key, (uint32_t)(i0 + n));
                }
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
        for (int w = 0; w < kThreads / 32; ++w) { if (w < warp) before += ss.scan[w]; total += ss.scan[w]; }
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
__device__ void top_of_share(const Share<T>& sh, float thread_max, int k, RowsShared& ss, unsigned long long* cand,
                             unsigned long long* sorted) {
    // a thread without an entry has key 0; padding and masked entries have the key of -inf
    const bool any = sh.first + (int)threadIdx.x < sh.last;
    const uint32_t my_key = any ? logit_key(thread_max) : 0u;
    uint32_t thr = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t c = thr | (1u << bit);
        const int n = __syncthreads_count(my_key >= c);
        if (n >= k) { thr = c; if (n <= 2 * k) break; }
    }
    int n = collect(sh, my_key, thr, true, ss, cand);
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
        n = kth == 0xFFFFFFFFu ? 0 : collect(sh, my_key, kth, false, ss, cand);   // fewer than k
        collect_ties(sh, kth, k - n, n, ss, cand);
        n = k;
        __syncthreads();
    }
    for (int i = threadIdx.x; i < k; i += kThreads) sorted[i] = 0ull;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {   // the packed words are all different: rank by counting
        const unsigned long long mine = cand[i];
        int rank = 0;
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
// k values per row: fp64 throughout, so that 1 - sum q keeps what fp32 values carry.
__device__ void distill_teacher(const RowsParams& P, int row, RowsShared& ss) {
    const int lane = threadIdx.x & 31;
    if (threadIdx.x < 32) {
        double vmax = -INFINITY;
        for (int i = lane; i < P.k; i += 32) {
            const bool have = ss.t_id[i] >= 0;
            if (have) vmax = fmax(vmax, (double)P.t_logprob[(long long)row * P.k + i]);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) vmax = fmax(vmax, __shfl_xor_sync(0xFFFFFFFFu, vmax, off));
        const double shift = P.tail == DM_TAIL_RENORM && vmax > -INFINITY ? vmax : 0.0;
        double e[kRowsMaxTop / 32], sum = 0.0;
        int distinct = 0;
#pragma unroll
        for (int u = 0; u < kRowsMaxTop / 32; ++u) {
            const int i = lane + 32 * u;
            e[u] = 0.0;
            if (i < P.k && ss.t_id[i] >= 0) {
                e[u] = exp((double)P.t_logprob[(long long)row * P.k + i] - shift);
                sum += e[u];
                bool first = true;
                for (int o = 0; o < i; ++o) first = first && ss.t_id[o] != ss.t_id[i];
                ss.t_first[i] = first;
                distinct += first;
            } else if (i < P.k) {
                ss.t_first[i] = 0;
            }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
            distinct += __shfl_xor_sync(0xFFFFFFFFu, distinct, off);
        }
        const double scale = P.tail == DM_TAIL_RENORM ? (sum != 0.0 ? 1.0 / sum : 0.0) : 1.0;
#pragma unroll
        for (int u = 0; u < kRowsMaxTop / 32; ++u)
            if (lane + 32 * u < P.k) ss.t_q[lane + 32 * u] = (float)(e[u] * scale);
        if (lane == 0) {
            ss.t_mass = (float)(sum * scale);
            const double rest = 1.0 - sum;
            ss.t_rest = P.tail == DM_TAIL_BUCKET && distinct < P.V ? (rest < 0.0 ? 0.0f : (float)rest) : 0.0f;
        }
    }
}

// ------------------------------------------------------------------------------------ the kernel
template <typename T, int kOp>
__global__ void __launch_bounds__(kThreads)
rows_kernel(const RowsParams P) {
    constexpr int N = RowVec<T>::N;
    constexpr bool kEntropy = kOp != OP_DISTILL, kTail = kOp == OP_DISTILL;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ RowsShared ss;
    uint4* stash = reinterpret_cast<uint4*>(smem);                                      // [stash_vecs], vector first + x
    uint32_t* bitmap = reinterpret_cast<uint32_t*>(stash + P.stash_vecs);               // distill: teacher tokens of the share
    unsigned long long* cand = reinterpret_cast<unsigned long long*>(smem);             // logprobs: candidates, then the sorted list
    unsigned long long* sorted = cand + kCandCap;
    unsigned long long* merged = sorted + kRowsMaxTop;                                  // rank 0: every CTA's list

    cg::cluster_group cluster = cg::this_cluster();
    const int n_cta = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = (int)(blockIdx.x / (unsigned)n_cta), tid = threadIdx.x;
    const float c = P.c;

    Share<T> sh;
    sh.row = static_cast<const T*>(P.logits) + (long long)row * P.ld;
    sh.V = P.V;
    sh.phase = (int)((reinterpret_cast<uintptr_t>(sh.row) & 15u) / sizeof(T));
    const int n_vec = (sh.phase + P.V + N - 1) / N, per = (n_vec + n_cta - 1) / n_cta;
    sh.first = min(n_vec, rank * per);
    sh.last = min(n_vec, sh.first + per);
    T* grad_row = kOp != OP_LOGPROBS && P.out_grad != nullptr ? static_cast<T*>(P.out_grad) + (long long)row * P.ld_grad : nullptr;

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
    if (kOp == OP_DISTILL) {
        if (P.weight != nullptr) { const float wt = P.weight[row]; zero_grad = wt == 0.0f; w *= wt; }
        for (int i = tid; i < P.k; i += kThreads) {
            int id = P.t_ids[(long long)row * P.k + i];
            if (id < 0 || id >= P.V) id = -1;
            ss.t_id[i] = id;
            ss.t_x[i] = id >= 0 ? RowVec<T>::get(sh.row + id) : neg_inf();
        }
        if (P.tail == DM_TAIL_BUCKET) {
            const int n_words = (per * N + 31) / 32;
            for (int i = tid; i < n_words; i += kThreads) bitmap[i] = 0u;
        }
        __syncthreads();
        distill_teacher(P, row, ss);
        if (P.tail == DM_TAIL_BUCKET) {
            for (int i = tid; i < P.k; i += kThreads) {
                const int u = ss.t_id[i] + sh.phase - sh.first * N;     // position within the share
                if (ss.t_id[i] >= 0 && u >= 0 && u < (sh.last - sh.first) * N) atomicOr(&bitmap[u >> 5], 1u << (u & 31));
            }
        }
        __syncthreads();
    }

    // A row whose gradient is zero whatever it holds is not read (unless its loss is wanted).
    const bool need_stats = !(zero_grad && (kOp == OP_GRAD || P.out_loss == nullptr));
    Merged a{0.0f, 0.0f, 0.0f, 0.0f};
    if (need_stats) {
        Stats st;
        st.init();
        for (int j0 = sh.first + tid; j0 < sh.last; j0 += kUnroll * kThreads) {
            uint4 v[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
                if (j0 + u * kThreads < sh.last) v[u] = sh.load(j0 + u * kThreads);
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int j = j0 + u * kThreads;
                if (j >= sh.last) break;
                if (kOp != OP_LOGPROBS && j - sh.first < P.stash_vecs) stash[j - sh.first] = v[u];
                float x[N];
                RowVec<T>::unpack(v[u], x);
                uint32_t top_bits = 0;
                if (kTail && P.tail == DM_TAIL_BUCKET) {
                    const int at = (j - sh.first) * N;
                    top_bits = bitmap[at >> 5] >> (at & 31);
                }
                st.add<N, kEntropy, kTail>(x, c, top_bits);
            }
        }
        const Merged mine = block_merge<T, kEntropy>(st, sh, c, ss);
        if (tid == 0) ss.mine = mine;
        if (kOp == OP_LOGPROBS && P.n_top > 0) top_of_share(sh, st.mx, P.n_top, ss, cand, sorted);
        if (n_cta > 1) cluster.sync(); else __syncthreads();
        a = cluster_merge(cluster, ss, n_cta, c);
    }
    const bool dead = a.m == neg_inf();                 // every entry masked: no distribution
    const float log_total = log1pf(a.rest), inv_total = 1.0f / (1.0f + a.rest);
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
            for (int i = tid; i < n_cta * k; i += kThreads) {
                const unsigned long long* theirs = n_cta == 1 ? sorted : cluster.map_shared_rank(sorted, i / k);
                merged[i] = theirs[i % k];
            }
            __syncthreads();
            for (int i = tid; i < n_cta * k; i += kThreads) {
                const unsigned long long mine = merged[i];
                if (mine == 0ull) continue;
                int place = i % k;
                for (int r = 0; r < n_cta && place < k; ++r) {
                    if (r == i / k) continue;
                    int lo = 0, hi = k;       // entries of list r that are larger
                    while (lo < hi) {
                        const int mid = (lo + hi) >> 1;
                        if (merged[r * k + mid] > mine) lo = mid + 1; else hi = mid;
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

    float tail_factor = 0.0f;   // q_t / (sum of the tail's exponentials)
    if (kOp == OP_DISTILL) {
        if (ss.t_rest > 0.0f && a.tail > 0.0f) tail_factor = ss.t_rest / a.tail;
        if (rank == 0 && P.out_loss != nullptr && tid < 32) {
            double loss = 0.0;
            const double log_tot = log1p((double)a.rest);
            for (int i = tid; i < P.k; i += 32) {
                const float q = ss.t_q[i];
                if (ss.t_id[i] < 0 || q == 0.0f) continue;
                const float x = ss.t_x[i];
                const double logp = dead || x == neg_inf() ? -INFINITY : ((double)x - (double)a.m) * P.inv_temp_d - log_tot;
                loss += (double)q * (log((double)q) - logp);
            }
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) loss += __shfl_xor_sync(0xFFFFFFFFu, loss, off);
            if (tid == 0) {
                const double qt = ss.t_rest;
                if (qt > 0.0 && !(dead && ss.t_mass == 0.0f)) loss += qt * (log(qt) - (log((double)a.tail) - log_tot));
                P.out_loss[row] = (float)loss;
            }
        }
    }

    if (kOp != OP_LOGPROBS && grad_row != nullptr) {
        // logprobs: dx = p (A + B z), z in powers of two;  distill: dx = p A, less the bucket's share outside the top
        float A = 0.0f, B = 0.0f, A_top = 0.0f;
        const bool none = zero_grad || dead;
        if (kOp == OP_GRAD) {
            A = -w * inv_total * fmaf(g_h, entropy - log_total, g_lp);
            B = -w * inv_total * g_h * kLn2;
        } else {
            const float mass = ss.t_mass + ss.t_rest;
            A_top = w * mass * inv_total;
            A = w * fmaf(mass, inv_total, -tail_factor);
        }
        const bool same_phase = (int)((reinterpret_cast<uintptr_t>(grad_row) & 15u) / sizeof(T)) == sh.phase;
        for (int j = sh.first + tid; j < sh.last; j += kThreads) {
            float x[N];
            if (!none) RowVec<T>::unpack(j - sh.first < P.stash_vecs ? stash[j - sh.first] : sh.load(j), x);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (none) { x[n] = 0.0f; continue; }
                const float z = max_nan((x[n] - a.m) * c, kFloorExp);
                x[n] = kOp == OP_GRAD ? ex2(z) * fmaf(B, z, A) : ex2(z) * A;
            }
            const int i0 = sh.entry0(j);
            if (sh.whole(j) && same_phase) {
                *reinterpret_cast<uint4*>(grad_row + i0) = RowVec<T>::pack(x);
            } else {
#pragma unroll
                for (int n = 0; n < N; ++n)
                    if (i0 + n >= 0 && i0 + n < P.V) RowVec<T>::put(grad_row + i0 + n, x[n]);
            }
        }
        __syncthreads();   // the entries that differ are written over by one thread each
        if (!none) {
            const int lo = sh.entry0(sh.first), hi = sh.entry0(sh.last);   // this share's entries
            if (kOp == OP_GRAD) {
                if (tid == 0 && tok >= 0 && tok >= lo && tok < hi) {   // (entries below 0 are the padding of the first vector)
                    const float z = max_nan((tok_x - a.m) * c, kFloorExp), e = ex2(z);
                    // 1 - p of the largest entry is rest / total, without cancellation
                    const float one_less = tok_x == a.m ? a.rest * inv_total : 1.0f - e * inv_total;
                    const float by_entropy = -w * g_h * inv_total * e * fmaf(kLn2, z, entropy - log_total);
                    RowVec<T>::put(grad_row + tok, fmaf(w * g_lp, one_less, by_entropy));
                }
            } else {
                for (int i = tid; i < P.k; i += kThreads) {
                    const int id = ss.t_id[i];
                    if (id < 0 || id < lo || id >= hi || !ss.t_first[i]) continue;
                    float q = 0.0f;
                    for (int o = i; o < P.k; ++o) q += ss.t_id[o] == id ? ss.t_q[o] : 0.0f;
                    const float e = ex2(max_nan((ss.t_x[i] - a.m) * c, kFloorExp));
                    RowVec<T>::put(grad_row + id, fmaf(A_top, e, -w * q));
                }
            }
        }
    }
    if (n_cta > 1) cluster.sync();   // nobody leaves while another CTA may still read its shared memory
}

template <typename T, int kOp>
int launch_rows(RowsParams P, cudaStream_t stream) {
    constexpr int N = RowVec<T>::N;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    const bool grad = kOp != OP_LOGPROBS && P.out_grad != nullptr;
    const int n_vec = (P.V + 2 * N - 2) / N;          // at most, whatever the row's alignment
    // CTAs per row: enough of them to fill the GPU where rows are few, not less than one vector per
    // thread; gradient kernels cut a row until a share fits their part of shared memory.
    int cluster = 1;
    while (cluster < kRowsMaxCluster && (long long)P.rows * cluster < 4ll * sms && n_vec > cluster * kThreads) cluster *= 2;
    if (grad)
        while (cluster < kRowsMaxCluster && (n_vec + cluster - 1) / cluster > kStashVecs) cluster *= 2;
    auto kern = rows_kernel<T, kOp>;
    size_t smem = 0;
    for (;; cluster *= 2) {
        const int per = (n_vec + cluster - 1) / cluster;
        P.stash_vecs = grad ? (per < kStashVecs ? per : kStashVecs) : 0;
        smem = (size_t)P.stash_vecs * 16;
        if (kOp == OP_DISTILL && P.tail == DM_TAIL_BUCKET) smem += ((size_t)per * N + 31) / 32 * 4;
        if (kOp == OP_LOGPROBS && P.n_top > 0)
            smem += (size_t)(kCandCap + kRowsMaxTop + cluster * P.n_top) * sizeof(unsigned long long);
        if (smem <= kRowsSmemLimit) break;
        if (cluster >= kRowsMaxCluster) return DM_EUNSUPPORTED;
    }
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
