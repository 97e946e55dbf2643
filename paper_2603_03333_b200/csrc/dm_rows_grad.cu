// Gradients on rows of logits whose shares fit in shared memory: the gradient of log-probability and
// entropy, and distillation with its gradient (dm_rows.cu states the mathematics).
//
// A cluster of CTAs takes row after row (there is one cluster per row in the grid; a running one takes
// over rows of clusters that have not started, so that fast and slow SMs share the rows out between
// them: 175 -> 139 us for the step below).  Each CTA keeps its share, up to 64 KB as a rule and three CTAs
// per SM, in shared memory: one pass over it finds the maximum, one sums, one writes the gradient.  As
// soon as a thread has converted a batch, the copies of the next row's batch into the same slots are on
// their way, so that loading overlaps the tail of the row, its barriers and the beginning of the next
// one.  The CTAs of a cluster meet once per row: every warp writes its sums into every CTA's shared
// memory ahead of one cluster barrier.
//
// Bound: memory, one read and one write of the row.  Measured: distillation with its gradient, 1024
// rows of 128256 bf16 (525 MB in all), 119-120 us = 4.4 TB/s (167 us if the tail of every row is summed anew);
// gradient of log-probability and entropy, 513 rows of 128256 fp32 (526 MB), 100-103 us = 5.1 to 5.3 TB/s;
// 1021 rows of 32003 bf16 (131 MB), 37-38 us = 3.5 TB/s.
// What keeps it there is the chain of a row: of some 21 thousand cycles that a CTA spends on 64 KB, the
// two passes with exponentials (16 per cycle and SM) take 8, waiting for the cluster 3 to 4, barriers,
// sums, merge and the teacher the rest; three CTAs per SM hide half of it.  Tried, on the step: shares of
// 32 KB with five CTAs per SM (the fixed part doubles), shares held in registers with the next row always
// in flight (two CTAs per SM: 181 against 134 us at the time), a maximum per warp in place of the block's
// (142 against 138), sums sent with asynchronous stores that count on a barrier instead of the cluster
// barrier (136 against 127), CTAs of 128 and 512 threads.
#include <cooperative_groups.h>

#include "dm_rows_dev.cuh"

namespace dm {

namespace {

namespace cg = cooperative_groups;
using namespace rows;

constexpr int kBatch = kUnroll * kThreads;
constexpr int kShareVecs = 4096;        // share up to which a row is cut: 64 KB, three CTAs per SM
constexpr int kTeacherWarps = kRowsMaxTop / 32;

// A warp's part of a row: its CTA's maximum, and relative to it the sum of exponentials over the entries
// below it, the same weighted with the exponents (gradient of the entropy) or over the tail (distillation,
// maximum included), and how many entries equal the maximum.
struct __align__(16) WarpSums { float m, s, x, cnt; };
struct PendingLoss { Merged a; double q_sum, mass, rest; int row; };   // row -1: none

struct ResidentShared {
    // written by every CTA of the cluster, twice over: a CTA may be one row ahead of another
    WarpSums part[2][kRowsMaxCluster * kWarps];
    uint4 answer;                  // to the request for another row (rank 0)
    uint64_t answer_bar;
    int next_row[2];               // written by rank 0 into every CTA, twice over
    float w_max[kWarps];
    // teacher (distill), twice over: the loss of a row is finished while the next one is under way
    int t_id[2][kRowsMaxTop];
    float t_v[2][kRowsMaxTop], t_x[2][kRowsMaxTop], t_q[2][kRowsMaxTop];
    int t_distinct[2], t_repeated[2], t_any[2];   // tokens of the share, named twice; whether the row has a token at all
    float t_max[kTeacherWarps];
    double t_sum[kTeacherWarps];
    float raised[kRowsMaxCluster * kWarps];   // parts of a tail that is summed anew, from every CTA
    PendingLoss loss;              // of the row before, until its warp finds the time (rank 0)
};

// The row's statistics from its warps' parts: every warp does the same for itself (some 100 instructions)
// instead of one that keeps the others waiting behind another barrier (2000 cycles of a row's 16 to 27 thousand).
template <bool kEntropy, bool kTail>
__device__ __forceinline__ Merged merge_parts(const WarpSums* part, int n, float c) {
    const int lane = threadIdx.x & 31;
    const WarpSums none{neg_inf(), 0.0f, 0.0f, 0.0f};
    const WarpSums r0 = lane < n ? part[lane] : none;
    const WarpSums r1 = lane + 32 < n ? part[lane + 32] : none;
    Merged a{warp_max_nan(max_nan(r0.m, r1.m)), 0.0f, 0.0f, 0.0f};
    float cnt = 0.0f;
    const auto take = [&](const WarpSums& r) {
        if (r.m == a.m) {
            a.rest += r.s; cnt += r.cnt;
            if (kEntropy) a.t += r.x;
            if (kTail) a.tail += r.x;
        } else if (r.m != neg_inf()) {
            const float d = fmaxf((r.m - a.m) * c, kFloorExp), f = ex2(d), all = r.s + r.cnt;
            a.rest = fmaf(f, all, a.rest);
            if (kEntropy) a.t = fmaf(f, fmaf(d, all, r.x), a.t);
            if (kTail) a.tail = fmaf(f, r.x, a.tail);
        }
    };
    take(r0);
    if (n > 32) take(r1);
    __syncwarp();
    a.rest = warp_sum(a.rest);
    if (kEntropy) a.t = warp_sum(a.t);
    if (kTail) a.tail = warp_sum(a.tail);
    a.rest += fmaxf(warp_sum(cnt) - 1.0f, 0.0f);
    if (!(a.m < __uint_as_float(0x7F800000u))) a.rest = a.t = a.tail = __uint_as_float(0x7FC00000u);   // NaN or +inf: no distribution
    return a;
}

// The tail of a row that is summed anew, 2^64 times as large, or 0 if it counts as nothing.  By all threads of
// the cluster, while the shares without the teacher's tokens still lie in shared memory.
template <typename T>
__device__ __noinline__ float resident_tail(const uint4* stash, int n_batches, float m, float c, float inv_total, ResidentShared& ss) {
    cg::cluster_group cluster = cg::this_cluster();
    const int n_cta = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float raised = 0.0f;
#pragma unroll 4
    for (int i = 0; i < n_batches * kUnroll; ++i) raised += raised_sum<T>(stash[i * kThreads + threadIdx.x], 0u, m, c);
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
    return counted_tail(warp_sum(raised), inv_total);
}

template <typename T, int kOp>
__global__ void __launch_bounds__(kThreads, 3)
rows_resident_kernel(const RowsParams P) {
    constexpr int N = RowVec<T>::N;
    constexpr bool kEntropy = kOp == OP_GRAD, kTail = kOp == OP_DISTILL;
    // (16-byte copies of a warp land in whole 128-byte lines: off that boundary they took up to a tenth longer)
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ ResidentShared ss;
    uint4* stash = reinterpret_cast<uint4*>(smem);                                    // [stash_vecs]
    unsigned char* bitmap = reinterpret_cast<unsigned char*>(stash + P.stash_vecs);   // distill: teacher tokens of the share, a byte per vector: tells repeated ones apart
    cg::cluster_group cluster = cg::this_cluster();
    const int n_cta = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    if (n_cta > 1) cluster_arrive();   // (waited for before anything is written to another CTA's shared memory)
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n_batches = P.stash_vecs / kBatch;   // of the longest share; what a row does not fill is masked
    const float c = P.c;
    const bool bucket = kTail && P.tail == DM_TAIL_BUCKET;

    int row = (int)blockIdx.x / n_cta;
    Share<T> sh = share_of<T>(P, row, n_cta, rank);
    for (int b = 0; b < n_batches; ++b) sh.fetch_batch(sh.first + b * kBatch, stash + b * kBatch + tid);
    if (kTail) {
        for (int i = tid; i < P.stash_vecs / 4; i += kThreads) reinterpret_cast<uint32_t*>(bitmap)[i] = 0u;
        if (tid < 2) ss.t_distinct[tid] = ss.t_repeated[tid] = ss.t_any[tid] = 0;
        __syncthreads();
    }
    // the row's small inputs, one row ahead
    int next_id = -1;              // token, or this thread's teacher token
    float next_a = 0.0f, next_b = 0.0f;   // gradients of log-probability and entropy, or the teacher's value and the weight
    const auto load_small = [&](int r) {
        if (kOp == OP_GRAD) {
            next_id = P.tokens != nullptr ? P.tokens[r] : -1;
            next_a = P.g_logprob != nullptr ? P.g_logprob[r] : 0.0f;
            next_b = P.g_entropy != nullptr ? P.g_entropy[r] : 0.0f;
        } else {
            if (tid < P.k) {
                next_id = P.t_ids[(long long)r * P.k + tid];
                next_a = P.t_logprob[(long long)r * P.k + tid];
            }
            next_b = P.weight != nullptr ? P.weight[r] : 1.0f;
        }
    };
    load_small(row);
    const uint32_t answer = ptx::smem_u32(&ss.answer), answer_bar = ptx::smem_u32(&ss.answer_bar);
    if (tid == 0) {
        ptx::mbar_init(answer_bar, 1);
        ptx::fence_mbar_init();
        ptx::fence_proxy_async_smem();
    }
    bool started = n_cta == 1;

    // The loss of a distillation row is left to one warp, which finishes it where the cluster meets over
    // the row after it: its logarithms take some 3000 cycles that the others would wait for.
    const auto finish_loss = [&](int p) {
        if (kOp != OP_DISTILL || rank != 0 || warp != kWarps - 1) return;
        __syncwarp();
        const PendingLoss of = ss.loss;
        if (of.row >= 0) {
            const float loss = teacher_loss(P, of.a, ss.t_id[p], ss.t_v[p], ss.t_x[p], ss.t_q[p], of.q_sum, of.mass, of.rest);
            if (lane == 0) P.out_loss[of.row] = loss;
        }
        __syncwarp();
    };
    if (tid == kThreads - 32) ss.loss.row = -1;

    int last_par = 0;
    for (int par = 0; row >= 0; par ^= 1) {
        last_par = par;
        const int n_share = sh.last - sh.first;
        if (rank == 0 && tid == 0) {   // the answer is waited for when the row's sums are known
            ptx::mbar_arrive_expect_tx(answer_bar, 16);
            ptx::request_next_cluster(answer, answer_bar);
        }
        T* grad_row = static_cast<T*>(P.out_grad) + (long long)row * P.ld_grad;
        float w = P.inv_temp, g_lp = 0.0f, g_h = 0.0f;
        int tok = -1;
        float tok_x = neg_inf();
        bool zero_grad;
        TeacherEntry te{-1, neg_inf(), neg_inf(), false, 0.0};
        uint32_t* my_word = nullptr;   // word of the bitmap in which this thread's token is marked
        if (kOp == OP_GRAD) {
            if (next_id >= 0 && next_id < P.V) { tok = next_id; tok_x = RowVec<T>::get_early(sh.row + tok); g_lp = next_a; }
            g_h = next_b;
            zero_grad = g_lp == 0.0f && g_h == 0.0f;
        } else {
            zero_grad = next_b == 0.0f;
            w *= next_b;
            if (tid < P.k && next_id >= 0 && next_id < P.V) {
                te.id = next_id;
                te.v = next_a;
                te.x = RowVec<T>::get_early(sh.row + te.id);
            }
            if (te.id >= 0) {
                ss.t_any[par] = 1;
                const int at = (te.id + sh.phase) / N - sh.first;   // vector within the share
                if (at >= 0 && at < n_share) {
                    const uint32_t bit = mark_bit(at, (te.id + sh.phase) % N);
                    my_word = mark_word(bitmap, at);
                    te.first = (atomicOr(my_word, bit) & bit) == 0u;
                    if (te.first) atomicAdd(&ss.t_distinct[par], 1); else ss.t_repeated[par] = 1;
                }
            }
            if (tid < P.k) { ss.t_id[par][tid] = te.id; ss.t_v[par][tid] = te.v; }
            if (warp < kTeacherWarps) {
                const float vm = warp_max(te.v);
                if (lane == 0) ss.t_max[warp] = vm;
            }
        }

        // A row whose gradient is zero whatever it holds is not looked at (unless its loss is wanted).
        const bool need_stats = !(zero_grad && (kOp == OP_GRAD || P.out_loss == nullptr));
        // which row comes next, told to every CTA ahead of the row's cluster barrier
        const auto tell_next = [&]() {
            if (rank == 0 && warp == 0) {
                int next = -1;
                if (lane == 0) {
                    next = granted_row(P, answer, answer_bar, (uint32_t)par);
                    if (next >= 0) next /= n_cta;
                }
                next = __shfl_sync(0xFFFFFFFFu, next, 0);
                if (lane < n_cta) (n_cta == 1 ? &ss : cluster.map_shared_rank(&ss, lane))->next_row[par] = next;
                __syncwarp();
            }
        };
        const auto meet = [&]() {
            if (n_cta == 1) {
                __syncthreads();
                finish_loss(par ^ 1);
            } else {
                __syncwarp();
                cluster_arrive();
                finish_loss(par ^ 1);
                cluster_wait();
            }
        };
        if (!started) { cluster_wait(); started = true; }
        if (need_stats) {
            float thread_max = neg_inf();
            for (int b = 0; b < n_batches; ++b) {
                copy_wait(n_batches - 1 - b);
                uint4 v[kUnroll];
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) v[u] = stash[b * kBatch + u * kThreads + tid];
                thread_max = max_nan(thread_max, RowVec<T>::vmax(v));
            }
            const float warp_top = warp_max_nan(thread_max);
            if (lane == 0) ss.w_max[warp] = warp_top;
            __syncthreads();
            float m = ss.w_max[0];
#pragma unroll
            for (int i = 1; i < kWarps; ++i) m = max_nan(m, ss.w_max[i]);
            if (kTail) {
                // the teacher's tokens leave the share by their threads' hands: what is left is the tail
                if (bucket) {
                    if (ss.t_repeated[par] != 0 && te.id >= 0) {   // of those that name one token the first counts, whichever was faster
                        te.first = my_word != nullptr;
                        for (int o = 0; o < tid; ++o) te.first = te.first && ss.t_id[par][o] != te.id;
                    }
                    if (te.first) RowVec<T>::put(reinterpret_cast<T*>(stash) + (te.id + sh.phase - sh.first * N), neg_inf());
                    __syncthreads();
                }
                if (warp < kTeacherWarps) {   // q in fp64, relative to the largest value (renorm)
                    float vm = ss.t_max[0];
#pragma unroll
                    for (int i = 1; i < kTeacherWarps; ++i) vm = fmaxf(vm, ss.t_max[i]);
                    const double shift = P.tail == DM_TAIL_RENORM && vm > neg_inf() ? (double)vm : 0.0;
                    if (te.id >= 0) te.q = exp((double)te.v - shift);
                    double sum = te.q;
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
                    if (lane == 0) ss.t_sum[warp] = sum;
                }
            }
            Stats st;
            st.init();
            st.set_maximum<T>(m, c, P.gap);
            const bool holder = warp_top == m && m != neg_inf();
            for (int b = 0; b < n_batches && (holder || st.ce != 0.0f); ++b) {
                uint4 v[kUnroll];
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) v[u] = stash[b * kBatch + u * kThreads + tid];
                if (holder) st.take<T, false>(v, 0u);
                if (st.ce != 0.0f) st.sum<T, kEntropy, false>(v, 0u);
            }
            if (kTail) {
                st.tail = fmaf((float)st.cnt, st.of_maximum(), st.s);
                if (bucket && te.first) {   // the teacher's tokens, by their threads
                    if (te.x == m) st.cnt += m != neg_inf() ? 1 : 0;
                    else if (st.ce != 0.0f) st.s += ex2(fmaf(te.x, st.ce, -st.rc));
                }
            }
            st.finish();
            const WarpSums r{m, warp_sum(st.s), warp_sum(kTail ? st.tail : st.t), (float)__reduce_add_sync(0xFFFFFFFFu, st.cnt)};
            if (lane < n_cta) (n_cta == 1 ? &ss : cluster.map_shared_rank(&ss, lane))->part[par][rank * kWarps + warp] = r;
        } else {
            copy_wait(0);
            // whether the cluster meets again over this row hangs on what is exchanged here, in every CTA alike,
            // even where another kernel changes a weight meanwhile
            if (kTail && lane < n_cta)
                (n_cta == 1 ? &ss : cluster.map_shared_rank(&ss, lane))->part[par][rank * kWarps + warp] =
                    WarpSums{__uint_as_float(0x7FC00000u), 0.0f, 0.0f, 0.0f};
        }
        tell_next();
        meet();
        const int next_row = ss.next_row[par];
        const bool more = next_row >= 0;
        if (more) load_small(next_row);
        Merged a = need_stats ? merge_parts<kEntropy, kTail>(ss.part[par], n_cta * kWarps, c) : Merged{0.0f, 0.0f, 0.0f, 0.0f};
        const float log_total = log1pf(a.rest), inv_total = 1.0f / (1.0f + a.rest);
        // (the marks have served; so have the counters of the row before)
        if (kOp == OP_DISTILL && my_word != nullptr) *my_word = 0u;
        if (kOp == OP_DISTILL && tid == 0) ss.t_distinct[par ^ 1] = ss.t_repeated[par ^ 1] = ss.t_any[par ^ 1] = 0;
        float mass = 0.0f, rest = 0.0f, q = 0.0f;   // sum of the teacher's q, mass of its bucket, this thread's q
        double q_sum = 0.0;
        if (kOp == OP_DISTILL) {
#pragma unroll
            for (int i = 0; i < kTeacherWarps; ++i) q_sum += ss.t_sum[i];
            const double scale = P.tail == DM_TAIL_RENORM ? (q_sum != 0.0 ? 1.0 / q_sum : 0.0) : 1.0;
            mass = (float)(q_sum * scale);
            // tokens outside the teacher's exist unless k reaches V (such a row is one CTA's)
            if (bucket && ss.t_any[par] != 0 && (P.k < P.V || ss.t_distinct[par] < P.V)) rest = 1.0 - q_sum > 0.0 || q_sum != q_sum ? (float)(1.0 - q_sum) : 0.0f;
            q = (float)(te.q * scale);
            if (tid < P.k) { ss.t_q[par][tid] = q; ss.t_x[par][tid] = te.x; }
        }
        const bool repeated = kOp == OP_DISTILL && ss.t_repeated[par] != 0;
        const bool dead = a.m == neg_inf();                 // every entry masked: no distribution
        const float entropy = dead ? 0.0f : fmaf(-kLn2 * inv_total, a.t, log_total);
        const bool taught = kOp != OP_DISTILL || ss.t_any[par] != 0;   // (a row without a teacher counts for nothing)
        const bool none = zero_grad || dead || !taught;
        const float rc = a.m * c;
        bool plain = !(fabsf(rc) < kSmallShift);   // exponents of differences
        GradFactors f = kOp == OP_GRAD ? logprob_factors(w, g_lp, g_h, entropy, log_total, inv_total)
                                       : distill_factors(w, mass, rest, a.tail, inv_total);
        if (kOp == OP_DISTILL && bucket && need_stats && (small_tail(a, P.V) || f.A == neg_inf())) {
            float raised = a.tail / kTailInv;
            if (small_tail(a, P.V)) {   // (the teacher's tokens have left the share)
                raised = resident_tail<T>(stash, n_batches, a.m, c, inv_total, ss);
                a.tail = raised * kTailInv;
            }
            f = raised_factors(w, mass, rest, raised, inv_total);
            plain = plain || f.up != 0.0f;
        }

        // the gradient; each batch's slots are handed to the next row at once (a thread reads its slots in
        // program order before its copies into them are issued, and only ever touches its own)
        const bool same_phase = phase_of(grad_row, sh.phase);
        const Share<T> next = more ? share_of<T>(P, next_row, n_cta, rank) : sh;
        const GradShift shift{rc, RowVec<T>::floor_word(a.m - P.gap)};
        const GradFactors g = factors_against(f, fmaf(a.m, c, -rc));
        if (same_phase && !none && !plain) {
            uint4* dst = reinterpret_cast<uint4*>(grad_row - sh.phase) + sh.first + tid;
            for (int b = 0; b < n_batches; ++b) {
                uint4 v[kUnroll];
                uint4* slot = stash + b * kBatch + tid;
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) v[u] = slot[u * kThreads];
                if (more) next.fetch_batch(next.first + b * kBatch, slot);
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) v[u] = grad_vector<T, kOp>(v[u], a.m, c, shift, g);
                if (sh.whole_batch(sh.first + b * kBatch)) {
#pragma unroll
                    for (int u = 0; u < kUnroll; ++u) __stcs(dst + b * kBatch + u * kThreads, v[u]);
                } else {
                    const int j = sh.first + b * kBatch + tid, n = sh.whole_end - j, lo = sh.whole_lo - j;
#pragma unroll
                    for (int u = 0; u < kUnroll; ++u) {
                        if (u * kThreads < n && u * kThreads >= lo) __stcs(dst + b * kBatch + u * kThreads, v[u]);
                        else if (j + u * kThreads < sh.last) store_vector(grad_row, sh, j + u * kThreads, true, v[u]);   // the row's first and last
                    }
                }
            }
        } else {
            for (int b = 0; b < n_batches; ++b) {
                uint4* slot = stash + b * kBatch + tid;
#pragma unroll 1
                for (int u = 0; u < kUnroll; ++u) {
                    const int j = sh.first + b * kBatch + u * kThreads + tid;
                    if (j < sh.last)
                        store_vector(grad_row, sh, j, same_phase,
                                     none    ? make_uint4(0u, 0u, 0u, 0u)
                                     : plain ? grad_vector<T, kOp, true>(slot[u * kThreads], a.m, c, shift, f)
                                             : grad_vector<T, kOp>(slot[u * kThreads], a.m, c, shift, g));
                }
                if (more) next.fetch_batch(next.first + b * kBatch, slot);
            }
        }
        if (kOp == OP_GRAD) {
            // the token's entry, by the thread that has just written its vector
            const int at = tok >= 0 && !none ? (tok + sh.phase) / N - sh.first : -1;
            if (at >= 0 && at < n_share && at % kThreads == tid)
                RowVec<T>::put(grad_row + tok, token_grad(tok_x, a, c, w, g_lp, g_h, entropy, log_total, inv_total));
        } else {
            __syncthreads();   // the teacher's entries are written over by one thread each
            if (te.first && !none) {                         // (set only for tokens of this share)
                if (repeated) {
                    q = 0.0f;
                    for (int o = 0; o < P.k; ++o) q += ss.t_id[par][o] == te.id ? ss.t_q[par][o] : 0.0f;
                }
                RowVec<T>::put(grad_row + te.id, fmaf(f.top, ex2((te.x - a.m) * c), -w * q));
            }
            if (rank == 0 && tid == kThreads - 32) {
                const double scale = P.tail == DM_TAIL_RENORM ? (q_sum != 0.0 ? 1.0 / q_sum : 0.0) : 1.0;
                ss.loss = PendingLoss{a, q_sum, q_sum * scale, rest != 0.0f ? 1.0 - q_sum : 0.0, P.out_loss != nullptr ? row : -1};
            }
        }
        sh = next;
        row = next_row;
    }
    finish_loss(last_par);
}

template <typename T, int kOp>
bool launch(RowsParams P, cudaStream_t stream, int* status) {
    constexpr int N = RowVec<T>::N;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        *status = DM_ECUDA;
        return true;
    }
    const int n_vec = (P.V + 2 * N - 2) / N;          // at most, whatever the row's alignment
    // CTAs per row: as many as run at once where rows are few, not less than one batch each; and until
    // three shares fit an SM's shared memory
    int cluster = 1;
    while (cluster < kRowsMaxCluster && 2ll * P.rows * cluster <= 3ll * sms && n_vec > cluster * kBatch) cluster *= 2;
    while (cluster < kRowsMaxCluster && (n_vec + cluster - 1) / cluster > kShareVecs) cluster *= 2;
    const int per = (n_vec + cluster - 1) / cluster;
    P.stash_vecs = (per + kBatch - 1) / kBatch * kBatch;
    const size_t smem = (size_t)P.stash_vecs * 16 + (kOp == OP_DISTILL ? (size_t)P.stash_vecs : 0);
    if (smem > kRowsSmemLimit) return false;
    if (P.wait_limit <= 0) P.wait_limit = kRowsWaitCycles;
    static std::atomic<unsigned long long> prepared{0};
    *status = launch_clusters(rows_resident_kernel<T, kOp>, prepared, dev, P, (long long)P.rows * cluster, cluster, smem, stream);
    return true;
}

}  // namespace

bool launch_rows_resident(const RowsParams& P, int dtype, bool distill, cudaStream_t stream, int* status) {
    if (dtype == DM_F32) return distill ? launch<float, OP_DISTILL>(P, stream, status) : launch<float, OP_GRAD>(P, stream, status);
    return distill ? launch<__nv_bfloat16, OP_DISTILL>(P, stream, status) : launch<__nv_bfloat16, OP_GRAD>(P, stream, status);
}

}  // namespace dm
