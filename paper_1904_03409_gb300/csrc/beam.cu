// beam.cu -- beam search over StackLSTM hypotheses: the rows' normalisers, the selection over
// beams and classes, the reordering of the stacks and the push of a new state, and their C ABI
// (include/stacklstm.h, stacklstm_beam_*).
//
// Hypothesis k of sentence b has the score s[b][k] and the logits z[b][k][0 .. V); candidate
// (k, v) scores s[b][k] + (z[b][k][v] - lse[b][k]), each operation rounded to fp32, so that the
// order is a matter of the inputs alone. The K best of the K V candidates of a sentence go on,
// best first, of equal ones the lowest k V + v first. A candidate becomes one 64-bit key: the
// score's order in the upper half, the complement of its place in the lower one. Keys are
// distinct, and the K best are the same whatever order they are looked at in. Key 0 is no
// candidate (-inf or NaN).
#include "rowvec.cuh"

namespace sl {
namespace {

typedef unsigned long long u64;

// A CTA of NT threads looks at NI candidates a thread: 256 x 32, or 512 x 64 where there are many.
constexpr int kMergeItems = 16;                        // keys a thread and pass of the merge
constexpr int kWideRow = 1024;                         // classes from which a CTA keeps to one row
constexpr int kMaxBeams = 64;

// ------------------------------------------------------------------ normalisers
// Read once where a row fits its threads' registers: 512 x 32003 bf16, one wave of CTAs, 8.1 us a call.
template <typename T, int TPR, int NP>
__global__ void __launch_bounds__(row_cta(TPR), row_ctas_per_sm(TPR))
lse_rows(int rows, int V, const T *__restrict__ z, float *__restrict__ lse)
{
    constexpr int E = RowVec<T>::E;
    __shared__ float sm[32];
    after_previous();
    const int r = blockIdx.x * rows_per_cta(TPR) + (TPR <= 32 ? threadIdx.x / TPR : 0), t = threadIdx.x % TPR;
    const RowVec<T> row(r, V);
    const int n = r < rows ? row.pieces() : 0;  // (a row past the end has no pieces: its lanes stay for the joins)
    uint4 q[NP > 0 ? NP : 1];
    if constexpr (NP > 0) {
#pragma unroll
        for (int j = 0; j < NP; ++j)
            if (j * TPR + t < n) q[j] = row.load(z, j * TPR + t);
    }
    auto each = [&](auto f) {
        if constexpr (NP > 0) {
#pragma unroll
            for (int j = 0; j < NP; ++j)
                if (j * TPR + t < n) {
                    float v[E];
                    unpack<T>(q[j], v);
                    f(v);
                }
        } else {
            for (int p = t; p < n; p += TPR) {
                float v[E];
                unpack<T>(row.load(z, p), v);
                f(v);
            }
        }
    };
    float m[1] = {-INFINITY}, s[1] = {0.0f};
    if constexpr (NP > 0) {
#pragma unroll
        for (int j = 0; j < NP; ++j)
            if (j * TPR + t < n) m[0] = max_nan(m[0], piece_max<T, true>(q[j]));
    } else {
        for (int p = t; p < n; p += TPR) m[0] = max_nan(m[0], piece_max<T, true>(row.load(z, p)));
    }
    row_join<true, TPR>(m, sm);
    const float base = m[0] == -INFINITY ? 0.0f : m[0];  // a row of -inf sums to 0: its lse is -inf
    each([&](const float (&v)[E]) {
#pragma unroll
        for (int i = 0; i < E; ++i) s[0] += exp2_hw((v[i] - base) * kLog2e);
    });
    row_join<false, TPR>(s, sm);
    if (t == 0 && r < rows) lse[r] = base == INFINITY ? base : base + logf(s[0]);  // (+inf: its differences are NaN)
}

template <typename T>
cudaError_t launch_lse(int rows, int V, const void *z, float *lse, cudaStream_t st)
{
    int tpr, np;
    row_plan<T>(V, &tpr, &np);
    const unsigned grid = ceil_div(rows, rows_per_cta(tpr));
#define SL_LSE(t, n) \
    if (tpr == t && np == n) return launch_after(lse_rows<T, t, n>, grid, row_cta(t), 0, st, rows, V, (const T *)z, lse);
    SL_ROW_PLANS(SL_LSE)
#undef SL_LSE
    return cudaErrorInvalidValue;  // not reached
}

// ------------------------------------------------------------------ selection
__device__ __forceinline__ u64 make_key(float score, uint32_t place)
{
    if (!(score > -INFINITY)) return 0;  // -inf and NaN
    const uint32_t b = __float_as_uint(score + 0.0f);  // -0 counts as 0
    const uint32_t o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return (u64)o << 32 | (0xFFFFFFFFu - place);
}
__device__ __forceinline__ float key_score(u64 key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float((o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o);
}

constexpr int kList = 1024;  // keys that are ranked together, most times

struct SelShared {
    u64 top[512];          // the threads' best keys
    float group[64];       // the groups' best scores
    u64 best[kMaxBeams];   // the K best, sorted
    u64 list[kList];
    u64 kth;
    int count, last;
    float score[kMaxBeams], lse[kMaxBeams];
    uint8_t done[kMaxBeams];
};

// The K best of the CTA's keys into s.best, sorted. `top` is the best score of the thread's keys
// (-inf: none), push(least, f) calls f with each of the thread's keys of a score >= least, and
// best_key() is its best key. Of any disjoint groups of keys, the K-th best of the groups' best
// scores is no better than the K-th best of all: first the threads' best are grouped (32 groups, 64
// for more than 32 hypotheses) and the keys from that score on are listed and ranked against one
// another. Where they are more than the list holds (most of a row alike, or all of it in few threads),
// the bound is the K-th of the threads' own best keys, from which on there are at most K times a
// thread's keys, in `spill`.
template <int NT, typename Push, typename Best>
__device__ __forceinline__ void block_topk(float top, const Push &push, const Best &best_key, int K, SelShared &s, u64 *spill)
{
    const int tid = threadIdx.x, lane = tid & 31;
    const int width = K <= 32 ? NT / 32 : NT / 64, groups = NT / width;
    float g = top;
    for (int o = 1; o < width; o <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, o));
    __syncthreads();  // (what an earlier call left in s is read)
    if (lane % width == 0) s.group[tid / width] = g;
    if (tid == 0) s.count = 0;
    if (tid < K) s.best[tid] = 0;
    __syncthreads();
    // every warp finds the K-th best group for itself: lane i ranks groups i and i + 32
    float least = -INFINITY;  // fewer than K groups: every candidate counts
    for (int half = 0; half < groups; half += 32) {
        const int me = half + lane;
        const float mine = s.group[me];
        int above = 0;
#pragma unroll 8
        for (int i = 0; i < groups; ++i) above += s.group[i] > mine || (s.group[i] == mine && i < me);
        const unsigned hit = __ballot_sync(0xffffffffu, above == K - 1);
        if (hit) least = __shfl_sync(0xffffffffu, mine, __ffs(hit) - 1);
    }
    if (top > -INFINITY && top >= least)
        push(least, [&](u64 k) {
            const int at = atomicAdd(&s.count, 1);  // any order: they are ranked below
            if (at < kList) s.list[at] = k;
        });
    __syncthreads();
    int n = s.count;
    u64 *list = s.list;
    if (n > kList) {
        list = spill;
        const u64 mine = best_key();
        __syncthreads();
        s.top[tid] = mine;
        if (tid == 0) {
            s.count = 0;
            s.kth = 1;
        }
        __syncthreads();
        int above = 0;
        if (mine)
            for (int i = 0; i < NT; ++i) above += s.top[i] > mine;
        if (mine && above == K - 1) s.kth = mine;
        __syncthreads();
        const u64 kth = s.kth;  // (1: fewer than K threads have a key, and every key counts)
        if (mine >= kth)
            push(kth > 1 ? key_score(kth) : -INFINITY, [&](u64 k) {
                if (k >= kth) list[atomicAdd(&s.count, 1)] = k;
            });
        __syncthreads();
        n = s.count;
    }
    for (int e = tid; e < n; e += NT) {
        const u64 k = list[e];
        int above = 0;
        for (int i = 0; i < n; ++i) above += list[i] > k;
        if (above < K) s.best[above] = k;
    }
    __syncthreads();
}

// Keys that a thread has at hand.
template <int NT, int PT>
__device__ __forceinline__ void keys_topk(const u64 (&key)[PT], int K, SelShared &s, u64 *spill)
{
    u64 mine = 0;
#pragma unroll
    for (int i = 0; i < PT; ++i) mine = key[i] > mine ? key[i] : mine;
    block_topk<NT>(mine ? key_score(mine) : -INFINITY, [&](float least, auto f) {
#pragma unroll
        for (int i = 0; i < PT; ++i)
            if (key[i] && key_score(key[i]) >= least) f(key[i]);
    }, [&] { return mine; }, K, s, spill);
}

// Sentence blockIdx.y; the candidates of segment blockIdx.x: NT NI of the sentence's K V
// (ROWS = false), or NT NI of the V of hypothesis blockIdx.x / per_row. The K best of each
// segment go to `part`, and the sentence's last CTA joins them.
template <typename T, bool ROWS, int NT, int NI>
__global__ void __launch_bounds__(NT, ROWS ? 2048 / NT : 2)
beam_select(int K, int V, int nseg, int per_row, const T *__restrict__ z, const float *__restrict__ lse,
            const float *__restrict__ score, const uint8_t *__restrict__ done, u64 *__restrict__ part,
            int *__restrict__ arrived, float *__restrict__ out_score, int32_t *__restrict__ parent,
            int32_t *__restrict__ token)
{
    __shared__ SelShared s;
    extern __shared__ u64 spill[];
    after_previous();
    const int tid = threadIdx.x, b = blockIdx.y, seg = blockIdx.x;
    if (tid < K) {
        s.score[tid] = score[(size_t)b * K + tid];
        s.lse[tid] = lse ? lse[(size_t)b * K + tid] : 0.0f;
        s.done[tid] = done ? done[(size_t)b * K + tid] : 0;
    }
    if constexpr (ROWS) {
        // The segment is read for the threads' largest logits alone; the few threads whose best makes
        // the bound read their pieces again: at 64 x 8 x 32003 bf16 15.7 us, all CTAs at once (6.5 for
        // the reading alone); 18 to 20 with the pieces held in registers, two CTAs of 512 an SM.
        constexpr int E = RowVec<T>::E, NP = NI / E;
        const int k = seg / per_row, piece0 = seg % per_row * (NT * NI / E) + tid;
        const RowVec<T> row((size_t)b * K + k, V);
        const int n = row.pieces();
        float zmax = -INFINITY;
#pragma unroll
        for (int j0 = 0; j0 < NP; j0 += 4) {
            uint4 q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (piece0 + (j0 + j) * NT < n) q[j] = row.load(z, piece0 + (j0 + j) * NT);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (piece0 + (j0 + j) * NT < n) zmax = fmaxf(zmax, piece_max<T, false>(q[j]));
        }
        __syncthreads();
        const float add = s.score[k], sub = s.lse[k];
        const bool is_done = s.done[k];
        const uint32_t place0 = (uint32_t)k * (uint32_t)V;
        // (rounded operations keep the order: the best score is that of the largest logit)
        const auto cand = [&](float v) { return __fadd_rn(add, __fsub_rn(v, sub)); };
        float top = cand(zmax);
        if (is_done) top = seg % per_row == 0 && tid == 0 ? add : -INFINITY;
        if (!(top > -INFINITY)) top = -INFINITY;
        auto push = [&](float least, auto f) {
            if (is_done) {
                f(make_key(add, place0));
                return;
            }
#pragma unroll 1
            for (int p0 = piece0; p0 < n && p0 < piece0 + NP * NT; p0 += 4 * NT) {
                uint4 q[4];
                unsigned hit = 0;  // the pieces with a candidate
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (p0 + j * NT < n) q[j] = row.load(z, p0 + j * NT);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (p0 + j * NT < n && cand(piece_max<T, false>(q[j])) >= least) hit |= 1u << j;
#pragma unroll 1
                for (; hit; hit &= hit - 1) {  // (its elements one by one: a copy of the code for each cost more)
                    const int c0 = row.column(p0 + (__ffs(hit) - 1) * NT);
#pragma unroll 1
                    for (int c = max(c0, 0); c < min(c0 + E, V); ++c) {
                        const float x = cand(to_f32(z[row.first() + c]));
                        if (x >= least && x > -INFINITY) f(make_key(x, place0 + (uint32_t)c));
                    }
                }
            }
        };
        auto best_key = [&] {
            u64 mine = 0;
            if (top > -INFINITY) push(top, [&](u64 k) { mine = k > mine ? k : mine; });
            return mine;
        };
        block_topk<NT>(top, push, best_key, K, s, spill);
    } else {
        const uint32_t n = (uint32_t)K * (uint32_t)V;
        const T *zb = z + (size_t)b * n;
        float v[NI];
        const uint32_t first = (uint32_t)seg * (NT * NI), e0 = first + tid;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const uint32_t e = e0 + i * NT;
            v[i] = e < n ? to_f32(zb[e]) : -INFINITY;
        }
        __syncthreads();
        u64 key[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const uint32_t e = e0 + i * NT;
            key[i] = 0;
            if (first + i * NT < n && e < n) {  // (the first for the whole CTA: a short segment ends early)
                const uint32_t k = e / (uint32_t)V;
                if (!s.done[k])
                    key[i] = make_key(__fadd_rn(s.score[k], __fsub_rn(v[i], s.lse[k])), e);
                else if (e == k * (uint32_t)V)
                    key[i] = make_key(s.score[k], e);
            }
        }
        keys_topk<NT, NI>(key, K, s, spill);
    }
    if (nseg > 1) {  // the sentence's last CTA joins the segments
        if (tid < K) part[((size_t)b * nseg + seg) * K + tid] = s.best[tid];
        __threadfence();
        __syncthreads();
        if (tid == 0) s.last = atomicAdd(&arrived[b], 1) == nseg - 1;
        __syncthreads();
        if (!s.last) return;
        __threadfence();
        if (tid == 0) arrived[b] = 0;  // for the next call
        const u64 *mine = part + (size_t)b * nseg * K;
        const int total = nseg * K, step = NT * (kMergeItems - 1);
        __syncthreads();  // (every thread has read its best of the segment)
        if (tid < K) s.best[tid] = 0;
        if (total <= NT) {  // few: all of them against one another
            const u64 key = tid < total ? __ldcg(mine + tid) : 0;
            s.top[tid] = key;
            __syncthreads();
            int above = 0;
            if (key)
                for (int i = 0; i < total; ++i) above += s.top[i] > key;
            if (key && above < K) s.best[above] = key;
            __syncthreads();
        }
        for (int at = 0; total > NT && at < total; at += step) {
            u64 key[kMergeItems];
#pragma unroll
            for (int i = 0; i < kMergeItems - 1; ++i) {
                const int e = at + i * NT + tid;
                key[i] = e < total ? __ldcg(mine + e) : 0;
            }
            key[kMergeItems - 1] = tid < K ? s.best[tid] : 0;  // the best so far
            keys_topk<NT, kMergeItems>(key, K, s, spill);
        }
    }
    if (tid < K) {
        const u64 key = s.best[tid];
        const size_t o = (size_t)b * K + tid;
        if (!key) {
            out_score[o] = -INFINITY;
            parent[o] = token[o] = -1;
        } else {
            const uint32_t e = 0xFFFFFFFFu - (uint32_t)key, k = e / (uint32_t)V;
            out_score[o] = key_score(key);
            parent[o] = (int)k;
            token[o] = s.done[k] ? -1 : (int)(e - k * (uint32_t)V);
        }
    }
}

// Segments of a sentence: by rows where a row fills most of a CTA's threads, else across the rows
// (8 x 83 candidates are one CTA's; by rows they would be eight, and their join). Larger CTAs where
// the small ones would be more than run at once four to an SM: 64 x 8 x 32003 bf16 23 us in 2048
// CTAs, 16 in 512.
struct SelPlan {
    bool rows, large;
    int per_row, nseg;
};
template <typename T>
SelPlan select_plan(int B, int K, int V, int sms)
{
    SelPlan p;
    p.rows = V >= kWideRow;
    constexpr size_t E = RowVec<T>::E;
    const size_t pieces = ((size_t)V + E - 1) / E + 1;
    p.per_row = (int)ceil_div(pieces, 256 * 32 / E);
    p.large = p.rows && (size_t)B * K * p.per_row > 4 * (size_t)sms && p.per_row > 1;
    if (p.large) p.per_row = (int)ceil_div(pieces, 512 * 64 / E);
    p.nseg = p.rows ? K * p.per_row : (int)ceil_div((size_t)K * V, 256 * 32);
    return p;
}
template <typename T>
cudaError_t launch_select(const stacklstm_op *op, const void *z, const float *lse, const float *score, const uint8_t *done,
                          float *new_score, int32_t *parent, int32_t *token)
{
    const int K = op->beams, V = op->V;
    const SelPlan p = select_plan<T>(op->B, K, V, op->num_sms);
    auto launch = [&](auto kernel, int nt, int ni) {
        return launch_after(kernel, dim3(p.nseg, op->B), nt, (size_t)K * ni * 8, op->stream,  // (at most 32 KB)
                            K, V, p.nseg, p.per_row, (const T *)z, lse, score, done, (u64 *)op->ws[0], (int *)op->ws[1], new_score,
                            parent, token);
    };
    if (p.large) return launch(beam_select<T, true, 512, 64>, 512, 64);
    if (p.rows) return launch(beam_select<T, true, 256, 32>, 256, 32);
    return launch(beam_select<T, false, 256, 32>, 256, 32);
}

// ------------------------------------------------------------------ stacks
// The row of the old stacks that row n of the new ones comes from, and its pointer. A row whose
// candidate ran out (parent -1) keeps its own stack.
__device__ __forceinline__ int source_row(int n, int K, int S, const int32_t *parent, const int32_t *p, int *top, int32_t *err)
{
    const int b = n / K;
    int par = parent[n];
    if (par < -1 || par >= K) {
        atomicCAS(err, 0, (int)SL_ERR_ARG);
        par = -1;
    }
    const int src = par < 0 ? n : b * K + par;
    int at = p[src];
    if (at < 0 || at >= S) {
        atomicCAS(err, 0, (int)SL_ERR_ARG);
        at = min(max(at, 0), S - 1);
    }
    *top = at;
    return src;
}

// `slots` slots from s0 on of row src to row n, `per` pieces each; slot top also to top_out. The
// CTA's threads take the pieces in order, four copies in flight each.
template <typename Q>
__device__ __forceinline__ void copy_slots(const Q *__restrict__ from, Q *__restrict__ to, Q *__restrict__ top_out, int N,
                                           int src, int n, int s0, int slots, int per, int top)
{
    const int total = slots * per;
    for (int i0 = threadIdx.x; i0 < total; i0 += 4 * blockDim.x) {
        Q v[4];
        size_t at[4];
        bool last[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + u * blockDim.x, slot = i / per, c = i - slot * per;
            at[u] = ((size_t)(s0 + slot) * N) * per + c;
            last[u] = s0 + slot == top;
            if (i < total) v[u] = from[at[u] + (size_t)src * per];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i0 + u * (int)blockDim.x < total) {
                to[at[u] + (size_t)n * per] = v[u];
                if (last[u] && top_out) top_out[(size_t)n * per + (at[u] % per)] = v[u];
            }
    }
}

// Row n (blockIdx.x) of the new stacks: kSlots of the slots 0 .. p of its source row, and its top.
// PH and PC pieces (types QH, QC) of h and c a slot. Bound by HBM: the live slots of 64 x 8 stacks of
// 186 x 200 (bf16 h, fp32 c) are read and written in 22 us (5.2 TB/s). (A CTA a slot kept 75 of 256 threads busy
// at H = 200.)
constexpr int kSlots = 16;
template <typename QH, typename QC>
__global__ void __launch_bounds__(256, 4)
reorder_rows(int N, int K, int S, int PH, int PC, const int32_t *__restrict__ parent, const int32_t *__restrict__ p,
             const QH *__restrict__ h, const QC *__restrict__ c, int32_t *__restrict__ p_out, QH *__restrict__ h_out,
             QC *__restrict__ c_out, QH *__restrict__ top_h, QC *__restrict__ top_c, int32_t *err)
{
    after_previous();
    const int n = blockIdx.x, s0 = blockIdx.y * kSlots;
    int top;
    const int src = source_row(n, K, S, parent, p, &top, err);
    if (blockIdx.y == 0 && threadIdx.x == 0) p_out[n] = top;
    const int slots = min(kSlots, top + 1 - s0);
    if (slots <= 0) return;
    copy_slots(c, c_out, top_c, N, src, n, s0, slots, PC, top);
    copy_slots(h, h_out, top_h, N, src, n, s0, slots, PH, top);
}

// Row n: the new state into slot p + 1 of a push, p moved by the op, the new top out.
template <typename QH, typename QC>
__global__ void __launch_bounds__(128)
push_rows(int N, int S, int PH, int PC, const int8_t *__restrict__ ops, const QH *__restrict__ h_new,
          const QC *__restrict__ c_new, int32_t *__restrict__ p, QH *__restrict__ h, QC *__restrict__ c,
          QH *__restrict__ top_h, QC *__restrict__ top_c, int32_t *err)
{
    after_previous();
    const int n = blockIdx.x;
    int at = p[n], op = ops[n];
    if (threadIdx.x == 0) {
        if (at < 0 || at >= S) atomicCAS(err, 0, (int)SL_ERR_ARG);
        if (op < -1 || op > 1) atomicCAS(err, 0, (int)SL_ERR_OP);
        else if (op == -1 && at <= 0) atomicCAS(err, 0, (int)SL_ERR_UNDERFLOW);
        else if (op == 1 && at >= S - 1) atomicCAS(err, 0, (int)SL_ERR_ARG);
    }
    at = min(max(at, 0), S - 1);
    if (op < -1 || op > 1 || at + op < 0 || at + op >= S) op = 0;  // as a hold
    const int to = at + op;
    for (int i = threadIdx.x; i < PH + PC; i += blockDim.x) {
        const size_t slot = (size_t)to * N + n;
        if (i < PH) {
            QH v;
            if (op == 1) {
                v = h_new[(size_t)n * PH + i];
                h[slot * PH + i] = v;
            } else {
                v = h[slot * PH + i];
            }
            if (top_h) top_h[(size_t)n * PH + i] = v;
        } else {
            const int j = i - PH;
            QC v;
            if (op == 1) {
                v = c_new[(size_t)n * PC + j];
                c[slot * PC + j] = v;
            } else {
                v = c[slot * PC + j];
            }
            if (top_c) top_c[(size_t)n * PC + j] = v;
        }
    }
    __syncthreads();  // every thread has read p
    if (threadIdx.x == 0) p[n] = to;
}

}  // namespace
}  // namespace sl

using namespace sl;

extern "C" {

sl_status stacklstm_beam_create(stacklstm_op_t *out, int B, int K, int V, int S, int H, sl_dtype dtype, int device,
                                void *stream)
{
    if (!out) return SL_ERR_ARG;
    *out = nullptr;
    if (B < 1 || K < 1 || V < 1 || S < 1 || H < 1 || (dtype != SL_FP32 && dtype != SL_BF16)) return SL_ERR_ARG;
    if (K > kMaxBeams || B > 65535 || (long long)K * V > (1LL << 30) || H > (1 << 24) || S > kSlots * 65535) return SL_ERR_UNSUPPORTED;
    sl_status st;
    stacklstm_op *op = op_new(SL_OP_BEAM, dtype, device, stream, &st);
    if (!op) return st;
    op->R = B * K; op->B = B; op->beams = K; op->V = V; op->S = S; op->H = H;
    OpDevice guard(device);
    const size_t nseg = dtype == SL_BF16 ? select_plan<__nv_bfloat16>(B, K, V, op->num_sms).nseg : select_plan<float>(B, K, V, op->num_sms).nseg;
    cudaError_t e = op_workspace(op, 0, (size_t)B * nseg * K * 8);
    if (!e) e = op_workspace(op, 1, (size_t)B * 4);
    if (!e) e = cudaMemsetAsync(op->ws[1], 0, (size_t)B * 4, op->stream);
    if (e) {
        stacklstm_op_destroy(op);
        return SL_ERR_OOM;
    }
    *out = op;
    return SL_OK;
}

sl_status stacklstm_beam_lse(stacklstm_op_t op, const void *logits, float *lse)
{
    if (!op || op->kind != SL_OP_BEAM) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (const char *m = check_pointers({logits, lse}, {})) return op_fail(op, SL_ERR_ARG, m);
    OpDevice guard(op->device);
    const cudaError_t e = op->dt == SL_BF16 ? launch_lse<__nv_bfloat16>(op->R, op->V, logits, lse, op->stream)
                                            : launch_lse<float>(op->R, op->V, logits, lse, op->stream);
    return e ? op_cuda(op, e, "stacklstm_beam_lse") : SL_OK;
}

sl_status stacklstm_beam_select(stacklstm_op_t op, const void *logits, const float *lse, const float *score,
                                const uint8_t *done, float *new_score, int32_t *parent, int32_t *token)
{
    if (!op || op->kind != SL_OP_BEAM) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (const char *m = check_pointers({logits, score, new_score, parent, token}, {lse, done}))
        return op_fail(op, SL_ERR_ARG, m);
    if (new_score == score) return op_fail(op, SL_ERR_ARG, "new_score must not be score: it is read by the whole sentence");
    OpDevice guard(op->device);
    const cudaError_t e = op->dt == SL_BF16
                              ? launch_select<__nv_bfloat16>(op, logits, lse, score, done, new_score, parent, token)
                              : launch_select<float>(op, logits, lse, score, done, new_score, parent, token);
    return e ? op_cuda(op, e, "stacklstm_beam_select") : SL_OK;
}

sl_status stacklstm_beam_reorder(stacklstm_op_t op, const int32_t *parent, const int32_t *p, const void *h_stack,
                                 const float *c_stack, int32_t *p_out, void *h_out, float *c_out, void *top_h, float *top_c)
{
    if (!op || op->kind != SL_OP_BEAM) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (const char *m = check_pointers({parent, p, h_stack, c_stack, p_out, h_out, c_out}, {top_h, top_c}))
        return op_fail(op, SL_ERR_ARG, m);
    if (p_out == p || h_out == h_stack || c_out == c_stack)
        return op_fail(op, SL_ERR_ARG, "the new stacks must not be the old ones: rows are read after others are written");
    OpDevice guard(op->device);
    const int N = op->R, K = op->beams, S = op->S, H = op->H;
    const bool bf = op->dt == SL_BF16;
    const dim3 grid(N, ceil_div(S, kSlots));
    auto copy = [&](auto qh, auto qc, int ph, int pc) {  // in pieces of these types
        using QH = decltype(qh);
        using QC = decltype(qc);
        return launch_after(reorder_rows<QH, QC>, grid, 256, 0, op->stream, N, K, S, ph, pc, parent, p, (const QH *)h_stack,
                            (const QC *)c_stack, p_out, (QH *)h_out, (QC *)c_out, (QH *)top_h, (QC *)top_c, op->err);
    };
    const cudaError_t e = H % 8 == 0 ? copy(uint4(), uint4(), H / (bf ? 8 : 4), H / 4)
                          : bf       ? copy(uint16_t(), uint32_t(), H, H)
                                     : copy(uint32_t(), uint32_t(), H, H);
    return e ? op_cuda(op, e, "stacklstm_beam_reorder") : SL_OK;
}

sl_status stacklstm_beam_push(stacklstm_op_t op, const int8_t *ops, const void *h_new, const float *c_new, int32_t *p,
                              void *h_stack, float *c_stack, void *top_h, float *top_c)
{
    if (!op || op->kind != SL_OP_BEAM) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (const char *m = check_pointers({ops, h_new, c_new, p, h_stack, c_stack}, {top_h, top_c}))
        return op_fail(op, SL_ERR_ARG, m);
    OpDevice guard(op->device);
    const int N = op->R, S = op->S, H = op->H;
    const bool bf = op->dt == SL_BF16;
    auto step = [&](auto qh, auto qc, int ph, int pc) {
        using QH = decltype(qh);
        using QC = decltype(qc);
        return launch_after(push_rows<QH, QC>, N, 128, 0, op->stream, N, S, ph, pc, ops, (const QH *)h_new, (const QC *)c_new, p,
                            (QH *)h_stack, (QC *)c_stack, (QH *)top_h, (QC *)top_c, op->err);
    };
    const cudaError_t e = H % 8 == 0 ? step(uint4(), uint4(), H / (bf ? 8 : 4), H / 4)
                          : bf       ? step(uint16_t(), uint32_t(), H, H)
                                     : step(uint32_t(), uint32_t(), H, H);
    return e ? op_cuda(op, e, "stacklstm_beam_push") : SL_OK;
}

}  // extern "C"
