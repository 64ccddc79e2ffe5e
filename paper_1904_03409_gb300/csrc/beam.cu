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

constexpr int kSelThreads = 256;
constexpr int kSelItems = 32;                          // candidates a thread
constexpr int kSegment = kSelThreads * kSelItems;      // candidates a CTA
constexpr int kMergeItems = 16;                        // keys a thread and pass of the merge
constexpr int kWideRow = 1024;                         // classes from which a CTA keeps to one row
constexpr int kMaxBeams = 64;

// ------------------------------------------------------------------ normalisers
template <typename T, int TPR, int NP>
__global__ void __launch_bounds__(row_cta(TPR), row_ctas_per_sm(TPR))
lse_rows(int rows, int V, const T *__restrict__ z, float *__restrict__ lse)
{
    constexpr int E = RowVec<T>::E, RPC = TPR == 32 ? 8 : 1;
    __shared__ float sm[32];
    const int r = blockIdx.x * RPC + (TPR == 32 ? threadIdx.x / 32 : 0), t = threadIdx.x % TPR;
    if (r >= rows) return;
    const RowVec<T> row(r, V);
    const int n = row.pieces();
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
    each([&](const float (&v)[E]) {
#pragma unroll
        for (int i = 0; i < E; ++i) m[0] = max_nan(m[0], v[i]);
    });
    row_join<true, TPR>(m, sm);
    const float base = m[0] == -INFINITY ? 0.0f : m[0];  // a row of -inf sums to 0: its lse is -inf
    each([&](const float (&v)[E]) {
#pragma unroll
        for (int i = 0; i < E; ++i) s[0] += exp2_hw((v[i] - base) * kLog2e);
    });
    row_join<false, TPR>(s, sm);
    if (t == 0) lse[r] = base + logf(s[0]);
}

template <typename T>
cudaError_t launch_lse(int rows, int V, const void *z, float *lse, cudaStream_t st)
{
    int tpr, np;
    row_plan<T>(V, &tpr, &np);
    const unsigned grid = ceil_div(rows, tpr == 32 ? 8 : 1);
#define SL_LSE(t, n) \
    if (tpr == t && np == n) lse_rows<T, t, n><<<grid, row_cta(t), 0, st>>>(rows, V, (const T *)z, lse);
    SL_ROW_PLANS(SL_LSE)
#undef SL_LSE
    return cudaGetLastError();
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
    u64 top[kSelThreads];  // the groups' (threads') best keys
    u64 best[kMaxBeams];   // the K best, sorted
    u64 list[kList];
    u64 kth;
    int count, last;
    float score[kMaxBeams], lse[kMaxBeams];
    uint8_t done[kMaxBeams];
};

// The K best of the CTA's keys into s.best, sorted. `mine` is the thread's best key and
// push(bound, f) calls f with each of the thread's keys that are >= bound. Of any disjoint groups
// of keys, the K-th best of the groups' best is no better than the K-th best of all: first the
// threads' best are grouped (8 lanes a group, 4 for more than 32 hypotheses) and the keys from
// that bound on are listed and ranked against one another. Where they are more than the list
// holds (most of a row alike), the bound is the K-th of the threads' own best, from which on there
// are at most K times a thread's keys, in `spill`.
template <typename Push>
__device__ __forceinline__ void block_topk(u64 mine, const Push &push, int K, SelShared &s, u64 *spill)
{
    const int tid = threadIdx.x, lane = tid & 31;
    const int width = K <= 32 ? 8 : 4, groups = kSelThreads / width;
    u64 g = mine;
    for (int o = 1; o < width; o <<= 1) {
        const u64 w = __shfl_xor_sync(0xffffffffu, g, o);
        g = w > g ? w : g;
    }
    __syncthreads();
    if (lane % width == 0) s.top[tid / width] = g;
    if (tid == 0) {
        s.count = 0;
        s.kth = 1;  // fewer than K groups with a candidate: every one counts
    }
    if (tid < K) s.best[tid] = 0;
    __syncthreads();
    if (tid < groups) {
        const u64 k = s.top[tid];
        int above = 0;
#pragma unroll 8
        for (int i = 0; i < groups; ++i) above += s.top[i] > k;
        if (k && above == K - 1) s.kth = k;
    }
    __syncthreads();
    const u64 bound = s.kth;
    if (mine >= bound)
        push(bound, [&](u64 k) {
            const int at = atomicAdd(&s.count, 1);  // any order: they are ranked below
            if (at < kList) s.list[at] = k;
        });
    __syncthreads();
    int n = s.count;
    u64 *list = s.list;
    if (n > kList) {
        list = spill;
        __syncthreads();
        s.top[tid] = mine;
        if (tid == 0) {
            s.count = 0;
            s.kth = 1;
        }
        __syncthreads();
        int above = 0;
        if (mine)
            for (int i = 0; i < kSelThreads; ++i) above += s.top[i] > mine;
        if (mine && above == K - 1) s.kth = mine;
        __syncthreads();
        const u64 tight = s.kth;
        if (mine >= tight) push(tight, [&](u64 k) { list[atomicAdd(&s.count, 1)] = k; });
        __syncthreads();
        n = s.count;
    }
    for (int e = tid; e < n; e += kSelThreads) {
        const u64 k = list[e];
        int above = 0;
        for (int i = 0; i < n; ++i) above += list[i] > k;
        if (above < K) s.best[above] = k;
    }
    __syncthreads();
}

// Keys that a thread has at hand.
template <int PT>
__device__ __forceinline__ void keys_topk(const u64 (&key)[PT], int K, SelShared &s, u64 *spill)
{
    u64 mine = 0;
#pragma unroll
    for (int i = 0; i < PT; ++i) mine = key[i] > mine ? key[i] : mine;
    block_topk(mine, [&](u64 bound, auto f) {
#pragma unroll
        for (int i = 0; i < PT; ++i)
            if (key[i] >= bound) f(key[i]);
    }, K, s, spill);
}

// Sentence blockIdx.y; the candidates of segment blockIdx.x: kSegment of the sentence's K V
// (ROWS = false), or kSegment of the V of hypothesis blockIdx.x / per_row. The K best of each
// segment go to `part`, and the sentence's last CTA joins them.
template <typename T, bool ROWS>
__global__ void __launch_bounds__(kSelThreads)
beam_select(int K, int V, int nseg, int per_row, const T *__restrict__ z, const float *__restrict__ lse,
            const float *__restrict__ score, const uint8_t *__restrict__ done, u64 *__restrict__ part,
            int *__restrict__ arrived, float *__restrict__ out_score, int32_t *__restrict__ parent,
            int32_t *__restrict__ token)
{
    __shared__ SelShared s;
    extern __shared__ u64 spill[];
    const int tid = threadIdx.x, b = blockIdx.y, seg = blockIdx.x;
    if (tid < K) {
        s.score[tid] = score[(size_t)b * K + tid];
        s.lse[tid] = lse ? lse[(size_t)b * K + tid] : 0.0f;
        s.done[tid] = done ? done[(size_t)b * K + tid] : 0;
    }
    if constexpr (ROWS) {
        constexpr int E = RowVec<T>::E, NP = kSelItems / E;
        const int k = seg / per_row, piece0 = seg % per_row * (kSegment / E) + tid;
        const RowVec<T> row((size_t)b * K + k, V);
        const int n = row.pieces();
        uint4 q[NP];
#pragma unroll
        for (int j = 0; j < NP; ++j)
            if (piece0 + j * kSelThreads < n) q[j] = row.load(z, piece0 + j * kSelThreads);
        __syncthreads();
        const float add = s.score[k], sub = s.lse[k];
        const bool is_done = s.done[k];
        const uint32_t place0 = (uint32_t)k * (uint32_t)V;
        u64 mine = 0;
        if (is_done) {
            if (seg % per_row == 0 && tid == 0) mine = make_key(add, place0);
        } else {
            float top = -INFINITY;
            uint32_t at = 0;
#pragma unroll
            for (int j = 0; j < NP; ++j)
                if (piece0 + j * kSelThreads < n) {
                    float v[E];
                    unpack<T>(q[j], v);
#pragma unroll
                    for (int i = 0; i < E; ++i) {  // places go up: of equal scores the first stays
                        const float c = __fadd_rn(add, __fsub_rn(v[i], sub));
                        if (c > top) {
                            top = c;
                            at = (uint32_t)(row.column(piece0 + j * kSelThreads) + i);
                        }
                    }
                }
            if (top > -INFINITY) mine = make_key(top, place0 + at);
        }
        block_topk(mine, [&](u64 bound, auto f) {
            if (is_done) {
                f(mine);
                return;
            }
            const float least = bound > 1 ? key_score(bound) : -INFINITY;
#pragma unroll
            for (int j = 0; j < NP; ++j)
                if (piece0 + j * kSelThreads < n) {
                    float v[E];
                    unpack<T>(q[j], v);
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        const float c = __fadd_rn(add, __fsub_rn(v[i], sub));
                        if (c >= least) {
                            const u64 key = make_key(c, place0 + (uint32_t)(row.column(piece0 + j * kSelThreads) + i));
                            if (key >= bound) f(key);
                        }
                    }
                }
        }, K, s, spill);
    } else {
        const uint32_t n = (uint32_t)K * (uint32_t)V;
        const T *zb = z + (size_t)b * n;
        float v[kSelItems];
        const uint32_t e0 = (uint32_t)seg * kSegment + tid;
#pragma unroll
        for (int i = 0; i < kSelItems; ++i) {
            const uint32_t e = e0 + i * kSelThreads;
            v[i] = e < n ? to_f32(zb[e]) : -INFINITY;
        }
        __syncthreads();
        u64 key[kSelItems];
#pragma unroll
        for (int i = 0; i < kSelItems; ++i) {
            const uint32_t e = e0 + i * kSelThreads;
            key[i] = 0;
            if (e < n) {
                const uint32_t k = e / (uint32_t)V;
                if (!s.done[k])
                    key[i] = make_key(__fadd_rn(s.score[k], __fsub_rn(v[i], s.lse[k])), e);
                else if (e == k * (uint32_t)V)
                    key[i] = make_key(s.score[k], e);
            }
        }
        keys_topk<kSelItems>(key, K, s, spill);
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
        const int total = nseg * K, step = kSelThreads * (kMergeItems - 1);
        if (tid < K) s.best[tid] = 0;
        __syncthreads();
        for (int at = 0; at < total; at += step) {
            u64 key[kMergeItems];
#pragma unroll
            for (int i = 0; i < kMergeItems - 1; ++i) {
                const int e = at + i * kSelThreads + tid;
                key[i] = e < total ? __ldcg(mine + e) : 0;
            }
            key[kMergeItems - 1] = tid < K ? s.best[tid] : 0;  // the best so far
            keys_topk<kMergeItems>(key, K, s, spill);
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
// (8 x 83 candidates are one CTA's; by rows they would be eight, and their join).
struct SelPlan {
    bool rows;
    int per_row, nseg;
};
template <typename T>
SelPlan select_plan(int K, int V)
{
    SelPlan p;
    p.rows = V >= kWideRow;
    constexpr size_t E = RowVec<T>::E;
    p.per_row = (int)ceil_div(((size_t)V + E - 1) / E + 1, kSegment / E);
    p.nseg = p.rows ? K * p.per_row : (int)ceil_div((size_t)K * V, kSegment);
    return p;
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

// Row n (blockIdx.x) of the new stacks: the slots 0 .. p of its source row, and its top. PH and
// PC pieces (types QH, QC) of h and c a slot. A CTA takes kSlots slots, its threads their pieces in
// order, four copies in flight each (a CTA a slot kept 75 of 256 threads busy at H = 200).
constexpr int kSlots = 16;
template <typename QH, typename QC>
__global__ void __launch_bounds__(256)
reorder_rows(int N, int K, int S, int PH, int PC, const int32_t *__restrict__ parent, const int32_t *__restrict__ p,
             const QH *__restrict__ h, const QC *__restrict__ c, int32_t *__restrict__ p_out, QH *__restrict__ h_out,
             QC *__restrict__ c_out, QH *__restrict__ top_h, QC *__restrict__ top_c, int32_t *err)
{
    const int n = blockIdx.x, s0 = blockIdx.y * kSlots;
    int top;
    const int src = source_row(n, K, S, parent, p, &top, err);
    if (blockIdx.y == 0 && threadIdx.x == 0) p_out[n] = top;
    const int slots = min(kSlots, top + 1 - s0);
    if (slots <= 0) return;
    const int per = PH + PC, total = slots * per;
    for (int i0 = threadIdx.x; i0 < total; i0 += 4 * 256) {
        QH vh[4];
        QC vc[4];
        int slot[4], at[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + u * 256;
            slot[u] = i / per;
            at[u] = i - slot[u] * per;
            if (i < total) {
                const size_t from = (size_t)(s0 + slot[u]) * N + src;
                if (at[u] < PH)
                    vh[u] = h[from * PH + at[u]];
                else
                    vc[u] = c[from * PC + (at[u] - PH)];
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i0 + u * 256 >= total) break;
            const int s = s0 + slot[u];
            const size_t to = (size_t)s * N + n;
            if (at[u] < PH) {
                h_out[to * PH + at[u]] = vh[u];
                if (s == top && top_h) top_h[(size_t)n * PH + at[u]] = vh[u];
            } else {
                c_out[to * PC + (at[u] - PH)] = vc[u];
                if (s == top && top_c) top_c[(size_t)n * PC + (at[u] - PH)] = vc[u];
            }
        }
    }
}

// Row n: the new state into slot p + 1 of a push, p moved by the op, the new top out.
template <typename QH, typename QC>
__global__ void __launch_bounds__(128)
push_rows(int N, int S, int PH, int PC, const int8_t *__restrict__ ops, const QH *__restrict__ h_new,
          const QC *__restrict__ c_new, int32_t *__restrict__ p, QH *__restrict__ h, QC *__restrict__ c,
          QH *__restrict__ top_h, QC *__restrict__ top_c, int32_t *err)
{
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
    const size_t nseg = dtype == SL_BF16 ? select_plan<__nv_bfloat16>(K, V).nseg : select_plan<float>(K, V).nseg;
    cudaError_t e = op_workspace(op, 0, (size_t)B * nseg * K * 8);
    if (!e) e = op_workspace(op, 1, (size_t)B * 4);
    if (!e) e = cudaMemset(op->ws[1], 0, (size_t)B * 4);
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
    const int K = op->beams, V = op->V;
    const size_t smem = (size_t)K * kSelItems * 8;  // at most 16 KB
    auto launch = [&](auto kernel, const SelPlan &p, auto *z) {
        kernel<<<dim3(p.nseg, op->B), kSelThreads, smem, op->stream>>>(K, V, p.nseg, p.per_row, z, lse, score, done, (u64 *)op->ws[0],
                                                                       (int *)op->ws[1], new_score, parent, token);
    };
    if (op->dt == SL_BF16) {
        const SelPlan p = select_plan<__nv_bfloat16>(K, V);
        launch(p.rows ? beam_select<__nv_bfloat16, true> : beam_select<__nv_bfloat16, false>, p, (const __nv_bfloat16 *)logits);
    } else {
        const SelPlan p = select_plan<float>(K, V);
        launch(p.rows ? beam_select<float, true> : beam_select<float, false>, p, (const float *)logits);
    }
    const cudaError_t e = cudaGetLastError();
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
    if (H % 8 == 0)
        reorder_rows<<<grid, 256, 0, op->stream>>>(N, K, S, H / (bf ? 8 : 4), H / 4, parent, p, (const uint4 *)h_stack,
                                                   (const uint4 *)c_stack, p_out, (uint4 *)h_out, (uint4 *)c_out,
                                                   (uint4 *)top_h, (uint4 *)top_c, op->err);
    else if (bf)
        reorder_rows<<<grid, 256, 0, op->stream>>>(N, K, S, H, H, parent, p, (const uint16_t *)h_stack,
                                                   (const uint32_t *)c_stack, p_out, (uint16_t *)h_out, (uint32_t *)c_out,
                                                   (uint16_t *)top_h, (uint32_t *)top_c, op->err);
    else
        reorder_rows<<<grid, 256, 0, op->stream>>>(N, K, S, H, H, parent, p, (const uint32_t *)h_stack,
                                                   (const uint32_t *)c_stack, p_out, (uint32_t *)h_out, (uint32_t *)c_out,
                                                   (uint32_t *)top_h, (uint32_t *)top_c, op->err);
    const cudaError_t e = cudaGetLastError();
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
    if (H % 8 == 0)
        push_rows<<<N, 128, 0, op->stream>>>(N, S, H / (bf ? 8 : 4), H / 4, ops, (const uint4 *)h_new, (const uint4 *)c_new,
                                             p, (uint4 *)h_stack, (uint4 *)c_stack, (uint4 *)top_h, (uint4 *)top_c, op->err);
    else if (bf)
        push_rows<<<N, 128, 0, op->stream>>>(N, S, H, H, ops, (const uint16_t *)h_new, (const uint32_t *)c_new, p,
                                             (uint16_t *)h_stack, (uint32_t *)c_stack, (uint16_t *)top_h,
                                             (uint32_t *)top_c, op->err);
    else
        push_rows<<<N, 128, 0, op->stream>>>(N, S, H, H, ops, (const uint32_t *)h_new, (const uint32_t *)c_new, p,
                                             (uint32_t *)h_stack, (uint32_t *)c_stack, (uint32_t *)top_h,
                                             (uint32_t *)top_c, op->err);
    const cudaError_t e = cudaGetLastError();
    return e ? op_cuda(op, e, "stacklstm_beam_push") : SL_OK;
}

}  // extern "C"
