// Operators on rows of logits x[N][V] in global memory (fp32 or bf16, any row stride):
//   logprobs       z = x / temperature;  lse = log sum_v exp z_v;  log-probability of a given token
//                  z_tok - lse;  entropy -sum_v p_v log p_v;  the n_top largest entries
//   logprobs_grad  gradient of g_lp * logprob + g_H * entropy with respect to x:
//                  (1/T) [ g_lp (1[v = tok] - p_v) - g_H p_v (log p_v + H) ]
//   distill        KL(teacher || student) for a teacher known by its top tokens, and its gradient
//                  (the teacher's rules stand in dm_rows_dev.cuh)
//
// A row belongs to one thread-block cluster; its CTAs take contiguous shares of the row, cut at
// 16-byte boundaries.  One pass over the share keeps, per warp, the exact maximum m so far (one
// reduction of the warp per 512 fp32 or 1024 bf16 entries) and, per lane, the sum of
// e = 2^((x - m) log2(e) / T) and of e times its exponent (entropy) over the entries below m; entries equal
// to m are counted.  A batch whose maximum stays below m takes the short path.  Warps meet in the
// block, CTAs through distributed shared memory.  Sums never contain the row's largest entry, so that
// log(1 + rest) keeps its precision next to a near-certain token.
//
// Bound: memory, one read of x.  Measured on 622 MB of bf16 logits (2047 rows of 151936): 106 us for the
// sums (5.9 TB/s, 0.90 of a measured copy's rate), 117-119 us with the 5 largest entries, 139 us with 20, 181 us
// with 100 (under sustained load, at the clock the power cap leaves, 121, 132 and 149); two thirds of the
// issue slots are taken.  Loss of a distillation alone, bucket, 64 tokens: 60 us for 1024 rows of 128256 bf16,
// 62 us for 512 rows of fp32 (133 and 160 if the tail of every row is summed anew).  Batches of six vectors per
// thread with three CTAs per SM were slower (146 against 136 us).  Few rows are bound by latency: some 12 us for
// one row of 128256.
#include <cooperative_groups.h>

#include <atomic>

#include "dm_rows_dev.cuh"

namespace dm {

namespace {

namespace cg = cooperative_groups;
using namespace rows;

constexpr int kRing = 2;               // batches in flight per CTA, eight per SM: three made no difference
constexpr int kCandCap = 1024;         // candidates for the top entries of a CTA's share
constexpr int kHitCap = 1024;          // batches that hold them
constexpr int kMaxSlots = 16, kWalkSlots = 8;   // maxima a thread keeps of its batches (for finding the top entries again)

struct RowsShared {
    uint4 answer;                // to the request for another row
    uint64_t answer_bar;
    int next_row;
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
    float t_q[kRowsMaxTop], t_v[kRowsMaxTop], t_x[kRowsMaxTop];
    float t_max[kRowsMaxTop / 32];
    double t_sum[kRowsMaxTop / 32];
    int t_distinct, t_repeated, t_any;
    float raised[kRowsMaxCluster * kWarps];   // parts of a tail that is summed anew, from every CTA
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
    for (int r = 1; r < n_cta; ++r) a = join(a, ss.part[r], c);
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

// ------------------------------------------------------------------------------------ the kernel
// Gradients are written by a second pass that reads the row again (rows whose shares fit in shared
// memory take the kernel of dm_rows_grad.cu instead).
// kWalk (logprobs, rows of one CTA): there is a CTA per row in the grid; a running one takes over rows of
// CTAs that have not started, so that the first batches of its next row are on their way while the
// present one's entries are selected (2047 rows of 151936, 5 alternatives: 147 -> 138 us when it was
// introduced).  Only where more rows than CTAs fit: with fewer there is nothing to take over.
// Four CTAs of 256 threads per SM; five, or CTAs of 128 or 512 threads, were no faster.
// kGrad: with a gradient (distillation has a kernel without, which needs fewer registers).
template <typename T, int kOp, bool kWalk, bool kGrad>
__global__ void __launch_bounds__(kThreads, 4)
rows_kernel(const RowsParams P) {
    static_assert(!kWalk || kOp == OP_LOGPROBS, "only rows without a gradient are walked over");
    constexpr int N = RowVec<T>::N;
    constexpr bool kEntropy = kOp != OP_DISTILL, kTail = kOp == OP_DISTILL;
    constexpr int kBatch = kUnroll * kThreads;
    // (16-byte copies of a warp land in whole 128-byte lines: off that boundary they took up to a tenth longer)
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ RowsShared ss;
    cg::cluster_group cluster = cg::this_cluster();
    const int n_cta = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    if (n_cta > 1) cluster_arrive();   // (waited for before anything is written to another CTA's shared memory)
    uint4* stash = reinterpret_cast<uint4*>(smem);                                      // the ring
    unsigned char* bitmap = reinterpret_cast<unsigned char*>(stash + P.stash_vecs);     // distill: teacher tokens of the share, a byte per vector
    // logprobs: behind the ring what is kept while the row streams, in the ring's place what comes after
    // (behind it, too, where the ring is busy with the next row by then)
    unsigned long long* merged = reinterpret_cast<unsigned long long*>(stash + kRing * kBatch);   // rank 0: every CTA's sorted list
    uint32_t* slots = reinterpret_cast<uint32_t*>(merged + (n_cta > 1 ? n_cta * P.n_top : 0));    // maxima of the threads' batches
    unsigned long long* cand = kWalk ? reinterpret_cast<unsigned long long*>(slots + P.n_slots * kThreads)
                                     : reinterpret_cast<unsigned long long*>(smem);     // candidates
    unsigned long long* sorted = cand + kCandCap;                                       // the largest of the share, sorted
    int* hits = reinterpret_cast<int*>(sorted + kRowsMaxTop);                           // [kHitCap]

    int row = (int)(blockIdx.x / (unsigned)n_cta);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float c = P.c;

    Share<T> sh = share_of<T>(P, row, n_cta, rank);
    T* grad_row = kGrad ? static_cast<T*>(P.out_grad) + (long long)row * P.ld_grad : nullptr;

    const int n_share = sh.last - sh.first, n_batches = kWalk ? P.n_batches : (n_share + kBatch - 1) / kBatch;
    uint4* ring = stash + tid;
    const uint32_t answer = ptx::smem_u32(&ss.answer), answer_bar = ptx::smem_u32(&ss.answer_bar);
    if (kWalk && tid == 0) {
        ptx::mbar_init(answer_bar, 1);
        ptx::fence_mbar_init();
        ptx::fence_proxy_async_smem();
    }
    // on its way before anything else is looked at: the first batches
    for (int b = 0; b < kRing; ++b) sh.fetch_batch(sh.first + b * kBatch, stash + b * kBatch + tid);

    for (uint32_t parity = 0;; parity ^= 1u) {
        if (kWalk && tid == 0) {
            ptx::mbar_arrive_expect_tx(answer_bar, 16);
            ptx::request_next_cluster(answer, answer_bar);
        }
        int next_row = -1;
        float w = P.inv_temp;   // factor of the gradient
        int tok = -1;
        float tok_x = neg_inf();
        if (kOp != OP_DISTILL && P.tokens != nullptr) {
            tok = P.tokens[row];
            if (tok < 0 || tok >= P.V) tok = -1;
            if (tok >= 0) tok_x = RowVec<T>::get_early(sh.row + tok);
        }
        float g_lp = 0.0f, g_h = 0.0f;
        bool zero_grad = false;
        if (kOp == OP_GRAD) {
            g_lp = P.g_logprob != nullptr && tok >= 0 ? P.g_logprob[row] : 0.0f;
            g_h = P.g_entropy != nullptr ? P.g_entropy[row] : 0.0f;
            zero_grad = g_lp == 0.0f && g_h == 0.0f;
        }
        const bool use_bits = kOp == OP_DISTILL && (kGrad || P.tail == DM_TAIL_BUCKET);
        TeacherEntry te{-1, neg_inf(), neg_inf(), false, 0.0};
        if (kOp == OP_DISTILL) {
            if (P.weight != nullptr) { const float wt = P.weight[row]; zero_grad = wt == 0.0f; w *= wt; }
            if (tid < P.k) {
                te.id = P.t_ids[(long long)row * P.k + tid];
                te.v = P.t_logprob[(long long)row * P.k + tid];
                if (te.id < 0 || te.id >= P.V) te.id = -1;
                if (te.id >= 0) te.x = RowVec<T>::get_early(sh.row + te.id);
                ss.t_id[tid] = te.id;
            }
            if (tid == 0) ss.t_distinct = ss.t_repeated = ss.t_any = 0;
            if (use_bits)
                for (int i = tid; i < n_batches * kBatch / 4; i += kThreads) reinterpret_cast<uint32_t*>(bitmap)[i] = 0u;
            if (warp < kRowsMaxTop / 32) {
                float vm = te.id >= 0 ? te.v : neg_inf();
#pragma unroll
                for (int off = 16; off > 0; off >>= 1) vm = fmaxf(vm, __shfl_xor_sync(0xFFFFFFFFu, vm, off));
                if (lane == 0) ss.t_max[warp] = vm;
            }
            __syncthreads();
            if (te.id >= 0) ss.t_any = 1;     // read behind the barriers below
            if (use_bits && te.id >= 0) {
                const int at = (te.id + sh.phase) / N - sh.first;   // vector within the share
                if (at >= 0 && at < sh.last - sh.first) {
                    const uint32_t bit = mark_bit(at, (te.id + sh.phase) % N);
                    te.first = (atomicOr(mark_word(bitmap, at), bit) & bit) == 0u;
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
            uint32_t* slot = slots + tid;
            uint32_t slot_key = 0u;
            int in_slot = 0;
            Share<T> from = sh;                        // what is fetched: this row, at its end the next one
            int ahead = kRing;
            for (int b = 0; b < n_batches; ++b) {   // the same for the whole block; kRing batches in flight
                uint4 v[kUnroll];
                copy_wait(kRing - 1);
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) v[u] = ring[u * kThreads];
                const uint32_t marks = bucket ? reinterpret_cast<const uint32_t*>(bitmap)[b * kThreads + tid] : 0u;
                if (kWalk && b == n_batches - kRing) {
                    if (tid == 0) ss.next_row = granted_row(P, answer, answer_bar, parity);
                    __syncthreads();
                    next_row = ss.next_row;
                    if (next_row >= 0) { from = share_of<T>(P, next_row, 1, 0); ahead = kRing - n_batches; }
                }
                from.fetch_batch(from.first + (b + ahead) * kBatch, ring);   // (past the end of a share: masked entries)
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
                st.add<T, kEntropy, kTail>(v, lane_max, c, P.gap, marks);
            }
            if (!kWalk) copy_wait(0);   // (what is still in flight are empty batches)
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
            if (n_cta > 1) {
                // the same meeting as over a row that is summed: another kernel may change a weight meanwhile, and no
                // CTA may leave while another writes to it or waits for it
                cluster_wait();
                const float nan = __uint_as_float(0x7FC00000u);
                if (tid < n_cta) cluster.map_shared_rank(&ss, tid)->part[rank] = Merged{nan, nan, nan, nan};
                __syncwarp();
                cluster_arrive();
                cluster_wait();
            }
            if (tid == 0) {
                ss.all = Merged{0.0f, 0.0f, 0.0f, 0.0f};
                ss.log_total = ss.inv_total = 0.0f;
            }
        }
        __syncthreads();
        Merged a = ss.all;
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
        float raised = -1.0f;             // the tail where it was summed anew
        if (kOp == OP_DISTILL) {
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < kRowsMaxTop / 32; ++i) sum += ss.t_sum[i];
            const double scale = P.tail == DM_TAIL_RENORM ? (sum != 0.0 ? 1.0 / sum : 0.0) : 1.0;
            mass = (float)(sum * scale);
            // tokens outside the teacher's exist unless k reaches V (such a row is one CTA's)
            if (P.tail == DM_TAIL_BUCKET && ss.t_any != 0 && (P.k < P.V || ss.t_distinct < P.V)) rest = 1.0 - sum > 0.0 || sum != sum ? (float)(1.0 - sum) : 0.0f;
            if (tid < P.k) { ss.t_q[tid] = (float)(te.q * scale); ss.t_v[tid] = te.v; ss.t_x[tid] = te.x; }
            __syncthreads();
            if (P.tail == DM_TAIL_BUCKET && need_stats && small_tail(a, P.V)) {   // the row is read again
                raised = 0.0f;
#pragma unroll 1
                for (int at = tid; at < n_share; at += kThreads)
                    raised += raised_sum<T>(sh.load(sh.first + at), *mark_word(bitmap, at) >> (at / kThreads % kUnroll * 8), a.m, c);
                raised = warp_sum(raised);
                if (lane < n_cta) (n_cta == 1 ? &ss : cluster.map_shared_rank(&ss, lane))->raised[rank * kWarps + warp] = raised;
                if (n_cta == 1) {
                    __syncthreads();
                } else {
                    __syncwarp();
                    cluster_arrive();
                    cluster_wait();
                }
                raised = (lane < n_cta * kWarps ? ss.raised[lane] : 0.0f) + (lane + 32 < n_cta * kWarps ? ss.raised[lane + 32] : 0.0f);
                raised = counted_tail(warp_sum(raised), inv_total);
                a.tail = raised * kTailInv;
            }
            if (rank == 0 && warp == kWarps - 1 && P.out_loss != nullptr) {
                const float loss = teacher_loss(P, a, ss.t_id, ss.t_v, ss.t_x, ss.t_q, sum, sum * scale, rest != 0.0f ? 1.0 - sum : 0.0);
                if (lane == 0) P.out_loss[row] = loss;
            }
        }

        if (kGrad) {
            const bool none = zero_grad || dead || (kOp == OP_DISTILL && ss.t_any == 0);   // (a row without a teacher counts for nothing)
            GradFactors f = kOp == OP_GRAD ? logprob_factors(w, g_lp, g_h, entropy, log_total, inv_total)
                                           : distill_factors(w, mass, rest, a.tail, inv_total);
            if (kOp == OP_DISTILL && (raised >= 0.0f || f.A == neg_inf()))
                f = raised_factors(w, mass, rest, raised >= 0.0f ? raised : a.tail / kTailInv, inv_total);
            const bool same_phase = phase_of(grad_row, sh.phase);
#pragma unroll 4
            for (int j = sh.first + tid; j < sh.last; j += kThreads)
                store_vector(grad_row, sh, j, same_phase, none ? make_uint4(0u, 0u, 0u, 0u) : grad_vector<T, kOp, true>(sh.load(j), a.m, c, GradShift{}, f));
            __syncthreads();   // the entries that differ are written over by one thread each
            if (!none) {
                const int lo = sh.entry0(sh.first), hi = sh.entry0(sh.last);   // this share's entries
                if (kOp == OP_GRAD) {
                    if (tid == 0 && tok >= 0 && tok >= lo && tok < hi)   // (entries below 0 are the padding of the first vector)
                        RowVec<T>::put(grad_row + tok, token_grad(tok_x, a, c, w, g_lp, g_h, entropy, log_total, inv_total));
                } else if (te.first) {                       // (set only for tokens of this share)
                    float q = ss.t_q[tid];
                    if (ss.t_repeated) {
                        q = 0.0f;
                        for (int o = 0; o < P.k; ++o) q += ss.t_id[o] == te.id ? ss.t_q[o] : 0.0f;
                    }
                    const float e = ex2((te.x - a.m) * c);
                    RowVec<T>::put(grad_row + te.id, fmaf(f.top, e, -w * q));
                }
            }
        }
        if (!kWalk || next_row < 0) break;
        row = next_row;
        sh = share_of<T>(P, row, n_cta, rank);
    }
}

template <typename T, int kOp>
int launch_rows(RowsParams P, cudaStream_t stream) {
    constexpr int N = RowVec<T>::N, kBatch = kUnroll * kThreads;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return DM_ECUDA;
    }
    const int n_vec = (P.V + 2 * N - 2) / N;          // at most, whatever the row's alignment
    // CTAs per row: as many as run at once where rows are few, not less than one batch each
    int cluster = 1;
    while (cluster < kRowsMaxCluster && 2ll * P.rows * cluster <= 4ll * sms && n_vec > cluster * kBatch) cluster *= 2;
    size_t smem = 0;
    bool walk = false;
    for (;; cluster *= 2) {
        const int per = (n_vec + cluster - 1) / cluster, batches = (per + kBatch - 1) / kBatch;
        P.stash_vecs = kRing * kBatch;
        P.n_batches = batches;
        walk = kOp == OP_LOGPROBS && cluster == 1 && batches >= kRing && P.rows > 4 * sms;
        smem = (size_t)P.stash_vecs * 16;
        if (kOp == OP_DISTILL && (P.tail == DM_TAIL_BUCKET || P.out_grad != nullptr)) smem += (size_t)batches * kBatch;
        if (kOp == OP_LOGPROBS && P.n_top > 0) {
            const int most = walk ? kWalkSlots : kMaxSlots;
            P.slot_batches = (batches + most - 1) / most;
            P.n_slots = (batches + P.slot_batches - 1) / P.slot_batches;
            smem += (size_t)P.n_slots * kThreads * sizeof(uint32_t);
            if (cluster > 1) smem += (size_t)cluster * P.n_top * sizeof(unsigned long long);
            constexpr size_t lists = (kCandCap + kRowsMaxTop) * sizeof(unsigned long long) + kHitCap * sizeof(int);
            static_assert(lists <= (size_t)kRing * kBatch * 16, "the lists fit the ring");
            if (walk) smem += lists;
        }
        if (smem <= kRowsSmemLimit) break;
        if (cluster >= kRowsMaxCluster) return DM_EUNSUPPORTED;
    }
    if (P.wait_limit <= 0) P.wait_limit = kRowsWaitCycles;
    static std::atomic<unsigned long long> prepared{0}, prepared_walk{0}, prepared_loss{0};
    if (walk)
        return launch_clusters(rows_kernel<T, kOp, kOp == OP_LOGPROBS, kOp != OP_LOGPROBS>, prepared_walk, dev, P, (long long)P.rows, 1, smem, stream);
    if (kOp == OP_DISTILL && P.out_grad == nullptr)
        return launch_clusters(rows_kernel<T, kOp, false, kOp == OP_GRAD>, prepared_loss, dev, P, (long long)P.rows * cluster, cluster, smem, stream);
    return launch_clusters(rows_kernel<T, kOp, false, kOp != OP_LOGPROBS>, prepared, dev, P, (long long)P.rows * cluster, cluster, smem, stream);
}

}  // namespace

int launch_rows_logprobs(const RowsParams& P, int dtype, cudaStream_t stream) {
    return dtype == DM_F32 ? launch_rows<float, OP_LOGPROBS>(P, stream) : launch_rows<__nv_bfloat16, OP_LOGPROBS>(P, stream);
}
int launch_rows_grad(const RowsParams& P, int dtype, cudaStream_t stream) {
    int st;
    if (launch_rows_resident(P, dtype, false, stream, &st)) return st;
    return dtype == DM_F32 ? launch_rows<float, OP_GRAD>(P, stream) : launch_rows<__nv_bfloat16, OP_GRAD>(P, stream);
}
int launch_rows_distill(const RowsParams& P, int dtype, cudaStream_t stream) {
    int st;
    if (P.out_grad != nullptr && launch_rows_resident(P, dtype, true, stream, &st)) return st;
    return dtype == DM_F32 ? launch_rows<float, OP_DISTILL>(P, stream) : launch_rows<__nv_bfloat16, OP_DISTILL>(P, stream);
}

}  // namespace dm
