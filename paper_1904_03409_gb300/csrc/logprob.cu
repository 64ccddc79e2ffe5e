// logprob.cu -- log probabilities of given classes, the distribution's entropy and its best classes,
// their gradient, and their C ABI (include/stacklstm.h, stacklstm_logprob_*).
//
// A row of V logits z, with x_v = z_v - max z, e_v = exp x_v and s = sum e:
//   lse = max z + ln s,  lp_v = x_v - ln s,  H = -sum p lp = ln s - (sum e x) / s
// (x and e x are exact where a class is the best; z sum-by-sum would cancel). For gradients g of the target's
// lp, g_j of alternative i_j's and h of H, with G = g + sum g_j,
//   dz_v = g [v = target] + sum_j g_j [v = i_j] - p_v (G + h (lp_v + H)).
// lse as a float is off by half a step, 2^-25 of it, and p = exp(z - lse) by a factor that the whole row shares: 1.4e-5 for
// logits shifted by 300, and V for a row of V times -1e9. So the backward takes lse only for a first base and makes
// f = sum_v exp(z_v - lse) itself: p_v = exp(z_v - lse - ln f). (lse is at most 21 off, the logarithm of the most classes.)
// Bound by HBM: a row is read once, and by the backward once more, which writes 4 bytes a class.
#include "select.cuh"

namespace sl {
namespace {

struct LogpArgs {
    int rows, V, k;
    const void *z;
    const int32_t *target;
    float *logp, *entropy, *lse;
    int32_t *top_idx;
    float *top_logp;
    int32_t *err;
    // a row over several CTAs: their statistics and best keys
    int split, per;            // CTAs a row, pieces of each
    float4 *part;              // [rows][split]: max, sum e, sum e x
    u64 *part_key;             // [rows][split][k]
    int *arrived;              // [rows], 0 between calls
};

__device__ __forceinline__ int read_target(const LogpArgs &a, size_t r, bool reports)
{
    const int t = a.target ? a.target[r] : -1;
    if (t >= -1 && t < a.V) return t;
    if (reports) atomicCAS(a.err, 0, (int)SL_ERR_ARG);
    return -1;
}

// A thread's (a row's) largest logit and its sums against it.
struct Stats {
    float m = -INFINITY, s = 0.0f, sx = 0.0f;
    __device__ __forceinline__ void add(float z)  // (z at most m)
    {
        const float x = fmaxf(z - m, -1e30f);  // (-inf: its share of both sums is 0; a NaN is in e)
        const float e = exp2_hw((z - m) * kLog2e);
        s += e;
        sx = fmaf(e, x, sx);
    }
    // the same sums against a larger m
    __device__ __forceinline__ void lift(float to)
    {
        if (m == -INFINITY) {  // nothing yet
            m = to;
            return;
        }
        const float d = m - to, c = exp2_hw(d * kLog2e);
        sx = c * fmaf(d > -1e30f ? d : -1e30f, s, sx);
        s *= c;
        m = to;
    }
};

struct Out {
    float m, ln_s, s, sx;
    __device__ __forceinline__ explicit Out(const Stats &t) : m(t.m), ln_s(logf(t.s)), s(t.s), sx(t.sx) {}
    // a row whose every logit is -inf has no probabilities: lp -inf, entropy 0
    __device__ __forceinline__ bool none() const { return m == -INFINITY; }
    __device__ __forceinline__ float lp(float z) const { return none() ? -INFINITY : (z - m) - ln_s; }
    __device__ __forceinline__ void put(const LogpArgs &a, size_t r, int target, float zt) const
    {
        if (a.logp) a.logp[r] = target < 0 ? 0.0f : lp(zt);
        if (a.entropy) a.entropy[r] = none() ? 0.0f : ln_s - sx / s;
        if (a.lse) a.lse[r] = none() || m == INFINITY ? m : m + ln_s;
    }
};

// Rows of up to 4 pieces a lane: TPR lanes (8 or 32) to a row, NP pieces a lane in registers. The k best are
// found one after the other, the best of the lanes' best. Of 32 lanes each keeps its best, and the one whose best was
// taken looks for its next: 10008 x 432 bf16 with 29 alternatives 54 us, bound by those instructions, 77 with all lanes
// looking for their best below the last one. Of 8 lanes (four rows a warp, whose lanes look at different times) all look: 11840 x
// 83 fp32 with 16 alternatives 16 us, 22 the other way; with 5 forward and backward 13 us, two calls' launches.
template <typename T, int TPR, int NP>
__global__ void __launch_bounds__(256)
logprob_narrow(const __grid_constant__ LogpArgs a)
{
    constexpr int E = RowVec<T>::E, RPC = 256 / TPR;
    after_previous();
    const int sub = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const size_t r = (size_t)blockIdx.x * RPC + sub;
    const bool here = r < (size_t)a.rows;  // (lanes of a row past the end stay for the joins)
    const T *z = (const T *)a.z;
    const RowVec<T> row(r, a.V);
    const int n = here ? row.pieces() : 0;
    float v[NP * E];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        float w[E];
        uint4 q;
        if (j * TPR + t < n) q = row.load(z, j * TPR + t);
        unpack<T>(q, w);
#pragma unroll
        for (int i = 0; i < E; ++i) v[j * E + i] = j * TPR + t < n ? w[i] : -INFINITY;
    }
    const int target = here ? read_target(a, r, t == 0) : -1;
    const float zt = t == 0 && target >= 0 ? to_f32(z[row.first() + target]) : 0.0f;
    float top[1] = {-INFINITY};
#pragma unroll
    for (int i = 0; i < NP * E; ++i) top[0] = max_nan(top[0], v[i]);
    lanes_join<true, TPR>(top);
    Stats st;
    st.m = top[0];
    if (st.m > -INFINITY || isnan(st.m))
#pragma unroll
        for (int i = 0; i < NP * E; ++i) st.add(v[i]);
    float s[2] = {st.s, st.sx};
    lanes_join<false, TPR>(s);
    st.s = s[0];
    st.sx = s[1];
    const Out out(st);
    if (t == 0 && here) out.put(a, r, target, zt);
    if (a.k == 0) return;
    auto put = [&](int j, u64 best) {
        if (t == 0 && here) {
            if (a.top_idx) a.top_idx[r * a.k + j] = best ? (int)(0xFFFFFFFFu - (uint32_t)best) : -1;
            if (a.top_logp) a.top_logp[r * a.k + j] = best ? out.lp(key_score(best)) : -INFINITY;
        }
    };
    if constexpr (TPR == 32) {
        float most;  // the lane's best that is left (of equal ones the first), in its place
        int at;
        auto look = [&]() {
            most = -INFINITY;
            at = 0;
#pragma unroll
            for (int i = 0; i < NP * E; ++i)
                if (v[i] > most) {  // (never a NaN)
                    most = v[i];
                    at = i;
                }
        };
        look();
        for (int j = 0; j < a.k; ++j) {
            const u64 mine = make_key(most, (uint32_t)(row.column(at / E * TPR + t) + at % E));
            const uint32_t score = __reduce_max_sync(0xffffffffu, (uint32_t)(mine >> 32));
            const bool may = (uint32_t)(mine >> 32) == score;
            const uint32_t place = __reduce_max_sync(0xffffffffu, may ? (uint32_t)mine : 0u);
            put(j, (u64)score << 32 | place);
            if (may && score && (uint32_t)mine == place) {
#pragma unroll
                for (int i = 0; i < NP * E; ++i)
                    if (i == at) v[i] = -INFINITY;
                look();
            }
        }
    } else {
        u64 last = ~0ull;
        for (int j = 0; j < a.k; ++j) {
            u64 best = 0;
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const u64 key = make_key(v[p * E + i], (uint32_t)(row.column(p * TPR + t) + i));
                    if (key < last && key > best) best = key;
                }
#pragma unroll
            for (int o = TPR / 2; o > 0; o >>= 1) {
                const u64 w = __shfl_xor_sync(0xffffffffu, best, o);
                best = w > best ? w : best;
            }
            put(j, best);
            last = best ? best : 1;  // (1: below every key)
        }
    }
}

// Wider rows: a CTA of NT threads takes per pieces of one, in segments of NP pieces a thread, four in flight. A
// segment is read for the threads' sums and largest logits alone; the few threads whose best makes the bound read
// their pieces again, from the caches. Where a row is over several CTAs, the last of them to end joins their
// statistics and best keys.
// 4096 x 32003 bf16: 53 us without alternatives (4.9 TB/s), 84 with 8 of them (3.1 TB/s: the search, issue 54 %).
template <typename T, int NT, int NP>
__global__ void __launch_bounds__(NT, 1024 / NT)
logprob_wide(const __grid_constant__ LogpArgs a)
{
    constexpr int E = RowVec<T>::E;
    __shared__ SelShared sel;
    __shared__ float sm[2 * NT / 32];
    extern __shared__ u64 spill[];
    after_previous();
    const int tid = threadIdx.x, k = a.k;
    const size_t r = blockIdx.x / a.split;
    const int part = (int)(blockIdx.x % a.split);
    const T *z = (const T *)a.z;
    const RowVec<T> row(r, a.V);
    const int p_lo = part * a.per, n = min(row.pieces(), p_lo + a.per);
    Stats st;
    if (tid < k) sel.best[tid] = 0;
    const uint4 *whole = (const uint4 *)(z + row.at);  // the row's pieces but the first and the last, which may hold neighbours'
    const int last = row.pieces() - 1;
    for (int p0 = p_lo; p0 < n; p0 += NT * NP) {
        const int end = min(n, p0 + NT * NP);
        float top = -INFINITY;
        auto add = [&](const uint4 *q, int count) {  // count pieces
            float most = -INFINITY;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (u < count) most = max_nan(most, piece_max<T, true>(q[u]));
            if (isnan(most)) {
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (u < count) top = fmaxf(top, piece_max<T, false>(q[u]));
            }
            top = fmaxf(top, most);
            if (!(most <= st.m)) st.lift(max_nan(st.m, most));
            if (st.m == -INFINITY) return;
            // two neighbours at a time
            float2 s2 = {0.0f, 0.0f}, x2 = {0.0f, 0.0f};
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (u < count) {
                    float v[E];
                    unpack<T>(q[u], v);
#pragma unroll
                    for (int i = 0; i < E; i += 2) {
                        const float2 d = __fadd2_rn(make_float2(v[i], v[i + 1]), make_float2(-st.m, -st.m));
                        const float2 w = __fmul2_rn(d, make_float2(kLog2e, kLog2e));
                        const float2 e = make_float2(exp2_hw(w.x), exp2_hw(w.y));
                        s2 = __fadd2_rn(s2, e);
                        x2 = __ffma2_rn(e, make_float2(fmaxf(d.x, -1e30f), fmaxf(d.y, -1e30f)), x2);
                    }
                }
            st.s += s2.x + s2.y;
            st.sx += x2.x + x2.y;
        };
#pragma unroll 1
        for (int p = p0 + tid; p < end; p += 4 * NT) {
            uint4 q[4];
            if (p > 0 && p + 3 * NT < min(end, last)) {
#pragma unroll
                for (int u = 0; u < 4; ++u) q[u] = whole[p + u * NT];
                add(q, 4);
            } else {
#pragma unroll 1
                for (int u = 0; u < 4 && p + u * NT < end; ++u) {
                    q[0] = row.load(z, p + u * NT);
                    add(q, 1);
                }
            }
        }
        if (k) {
            const u64 kept = tid < k && p0 > p_lo ? sel.best[tid] : 0;  // the best so far are candidates too
            if (kept) top = fmaxf(top, key_score(kept));
            auto push = [&](float least, auto f) {
                if (kept && key_score(kept) >= least) f(kept);
#pragma unroll 1
                for (int p = p0 + tid; p < end; p += 4 * NT) {
                    unsigned hit = 0;  // the pieces that may have a candidate
                    if (p > 0 && p + 3 * NT < min(end, last)) {
                        uint4 q[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) q[u] = whole[p + u * NT];
#pragma unroll
                        for (int u = 0; u < 4; ++u) hit |= (unsigned)(piece_max<T, false>(q[u]) >= least) << u;
                    } else {
                        for (int u = 0; u < 4; ++u) hit |= (unsigned)(p + u * NT < end) << u;
                    }
#pragma unroll 1
                    for (; hit; hit &= hit - 1) {
                        const int at = p + (__ffs(hit) - 1) * NT, c0 = row.column(at);
                        const uint4 w = row.load(z, at);  // (from the first cache; the four are not indexed by number)
                        float v[E];
                        unpack<T>(w, v);
#pragma unroll
                        for (int i = 0; i < E; ++i)
                            if (v[i] >= least && v[i] > -INFINITY) f(make_key(v[i], (uint32_t)(c0 + i)));
                    }
                }
            };
            auto best_key = [&] {
                u64 mine = 0;
                if (top > -INFINITY) push(top, [&](u64 x) { mine = x > mine ? x : mine; });
                return mine;
            };
            block_topk<NT>(top, push, best_key, k, sel, spill);
        }
    }
    auto joined = [&]() {  // the threads' statistics, to all of them
        float m[1] = {st.m};
        row_join<true, NT>(m, sm);
        float s[2] = {0.0f, 0.0f};
        if (st.m > -INFINITY || isnan(st.m)) {
            st.lift(m[0]);
            s[0] = st.s;
            s[1] = st.sx;
        }
        row_join<false, NT>(s, sm);
        st.m = m[0];
        st.s = s[0];
        st.sx = s[1];
    };
    joined();
    if (a.split > 1) {
        if (tid == 0) a.part[r * a.split + part] = make_float4(st.m, st.s, st.sx, 0.0f);
        if (tid < k) a.part_key[(r * a.split + part) * k + tid] = sel.best[tid];
        __threadfence();
        __syncthreads();
        if (tid == 0) sel.last = atomicAdd(&a.arrived[r], 1) == a.split - 1;
        __syncthreads();
        if (!sel.last) return;
        __threadfence();
        if (tid == 0) a.arrived[r] = 0;  // for the next call
        st = Stats();
        if (tid < a.split) {
            const float4 w = __ldcg(&a.part[r * a.split + tid]);
            st.m = w.x;
            st.s = w.y;
            st.sx = w.z;
        }
        joined();
        if (k) {
            const u64 *mine = a.part_key + r * a.split * k;
            const int total = a.split * k, step = NT * (kMergeItems - 1);
            __syncthreads();
            if (tid < k) sel.best[tid] = 0;
            __syncthreads();
            for (int at = 0; at < total; at += step) {
                u64 key[kMergeItems];
#pragma unroll
                for (int i = 0; i < kMergeItems - 1; ++i) {
                    const int e = at + i * NT + tid;
                    key[i] = e < total ? __ldcg(mine + e) : 0;
                }
                key[kMergeItems - 1] = tid < k ? sel.best[tid] : 0;  // the best so far
                keys_topk<NT, kMergeItems>(key, k, sel, spill);
            }
        }
    }
    const Out out(st);
    if (tid == 0) {
        const int target = read_target(a, r, true);
        out.put(a, r, target, target >= 0 ? to_f32(z[row.first() + target]) : 0.0f);
    }
    if (tid < k) {
        const u64 key = sel.best[tid];
        if (a.top_idx) a.top_idx[r * k + tid] = key ? (int)(0xFFFFFFFFu - (uint32_t)key) : -1;
        if (a.top_logp) a.top_logp[r * k + tid] = key ? out.lp(key_score(key)) : -INFINITY;
    }
}

// ------------------------------------------------------------------ backward
struct GradArgs {
    int rows, V, k;
    const void *z;
    const int32_t *target, *top_idx;
    const float *entropy, *lse, *dlogp, *dentropy, *dtop;
    float *dz;
    int32_t *err;
    // rows over several CTAs:
    int split;                 // CTAs a row
    int sums;                  // parts of a row whose sums of exponentials are in
    float *part;               //  [rows][sums]
};

// The row's classes that have a gradient of their own: the target and the alternatives (c: class or -1).
__device__ __forceinline__ void read_entry(const GradArgs &a, size_t r, int j, int *c, float *w)
{
    int v = -1;
    float g = 0.0f;
    if (j < a.k) {  // (k is 0 without dtop)
        v = a.top_idx[r * a.k + j];
        g = a.dtop[r * a.k + j];
    } else if (a.target && a.dlogp) {
        v = a.target[r];
        g = a.dlogp[r];
    }
    if (v < -1 || v >= a.V) {
        atomicCAS(a.err, 0, (int)SL_ERR_ARG);  // skipped
        v = -1;
    }
    if (v < 0) g = 0.0f;
    c[j] = v;
    w[j] = g;
}

struct Grad {
    float lse, h, entropy;
    float rest, all;          // lp = z - lse - rest; all = G + h H
    bool none;
    __device__ __forceinline__ Grad(const GradArgs &a, size_t r)
    {
        lse = a.lse[r];
        h = a.dentropy ? a.dentropy[r] : 0.0f;
        entropy = a.dentropy ? a.entropy[r] : 0.0f;
        none = lse == -INFINITY;
    }
    __device__ __forceinline__ void join(int k, const float *w, float f)  // the entries' weights, f of the row
    {
        rest = logf(f);
        all = 0.0f;
        for (int j = 0; j <= k; ++j) all += w[j];
        all = fmaf(h, entropy, all);
    }
    __device__ __forceinline__ float operator()(float z) const
    {
        const float lp = (z - lse) - rest, p = exp2_hw(lp * kLog2e);
        return none ? 0.0f : -p * fmaf(h, fmaxf(lp, -1e4f), all);  // (p is 0 below -104: no inf x 0)
    }
};
// A piece's share of f (what is outside the row is -inf, and counts 0).
template <typename T>
__device__ __forceinline__ float piece_sum(const uint4 &q, float lse)
{
    float v[RowVec<T>::E], s = 0.0f;
    unpack<T>(q, v);
#pragma unroll
    for (int i = 0; i < RowVec<T>::E; ++i) s += exp2_hw((v[i] - lse) * kLog2e);
    return s;
}
// Pieces p_lo .. n of a row are written: the few classes of the entries among them are once more. The first entry of each
// class takes the sum of the class's weights in entry order, so repeated classes need no atomics. (mine: entry t's logit,
// where each thread has one at most)
template <typename T>
__device__ __forceinline__ float entry_logit(const GradArgs &a, const RowVec<T> &row, const int *c, int t)
{
    return t <= a.k && c[t] >= 0 ? to_f32(((const T *)a.z)[row.first() + c[t]]) : 0.0f;
}
template <typename T, int TPR>
__device__ __forceinline__ void put_entries(const GradArgs &a, const Grad &g, const RowVec<T> &row, int p_lo, int n, const int *c, const float *w, int t,
                                            float mine)
{
    const int c_lo = row.column(p_lo), c_hi = row.column(n);
    for (int j = t; j <= a.k; j += TPR) {
        const int v = c[j];
        if (v < c_lo || v >= c_hi || v < 0 || g.none) continue;
        bool first = true;
        float sum = w[j];
        for (int i = 0; i <= a.k; ++i)
            if (c[i] == v) {
                if (i < j) first = false;
                if (i > j) sum += w[i];
            }
        if (first) a.dz[row.first() + v] = g(TPR > 64 ? mine : entry_logit<T>(a, row, c, j)) + sum;
    }
}

// A row's pieces read once for f and for the gradient, NP a thread in registers: TPR lanes (8, 32) to a row, several rows a CTA,
// or a CTA of TPR threads; what 1024 threads do not hold they read again, in part from L2.
// Bound by HBM: 4096 x 32003 bf16 with 8 alternatives 138 us, 5.7 TB/s (6 bytes a class), 121 without; 148 and 128 where what a
// row needs of entropy, weights and entries' logits was read after its sum. (A row over a cluster of CTAs, 2000 x 70001: 222 us, 169 so.)
template <typename T, int TPR, int NP>
__global__ void __launch_bounds__(row_cta(TPR), TPR <= 32 ? 1 : row_ctas_per_sm(TPR))
logprob_grad(const __grid_constant__ GradArgs a)
{
    constexpr int RPC = rows_per_cta(TPR);
    __shared__ float sm[TPR <= 32 ? 1 : TPR / 32];
    extern __shared__ __align__(16) uint8_t dyn[];
    after_previous();
    const int k1 = a.k + 1, sub = TPR <= 32 ? threadIdx.x / TPR : 0, t = threadIdx.x % TPR;
    int *c = (int *)dyn + sub * k1;
    float *w = (float *)(dyn + (size_t)RPC * k1 * 4) + sub * k1;
    const size_t r = (size_t)blockIdx.x * RPC + sub;
    const bool here = r < (size_t)a.rows;  // (lanes of a row past the end stay for the joins)
    const T *z = (const T *)a.z;
    const RowVec<T> row(r, a.V);
    const int n = here ? row.pieces() : 0;
    // the pieces are on their way while the entries are read
    uint4 q[NP];
#pragma unroll
    for (int u = 0; u < NP; ++u)
        if (u * TPR + t < n) q[u] = row.load(z, u * TPR + t);
    if (here)
        for (int j = t; j < k1; j += TPR) read_entry(a, r, j, c, w);
    Grad g(a, here ? r : 0);
    float f[1] = {0.0f};
#pragma unroll
    for (int u = 0; u < NP; ++u)
        if (u * TPR + t < n) f[0] += piece_sum<T>(q[u], g.lse);
    constexpr int U = 4;  // of a longer row's pieces at a time
    if constexpr (TPR == 1024)
        for (int p = NP * TPR + t; p < n; p += U * TPR) {
            uint4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * TPR < n) x[u] = row.load(z, p + u * TPR);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * TPR < n) f[0] += piece_sum<T>(x[u], g.lse);
        }
    row_join<false, TPR>(f, sm);  // (and the entries are written, of a row over a CTA)
    if constexpr (TPR <= 32) __syncwarp();
    if (!here) return;
    g.join(a.k, w, f[0]);
    const float mine = TPR > 64 ? entry_logit<T>(a, row, c, t) : 0.0f;
    const bool aligned = on_32(a.dz);
    auto put = [&](const uint4 &x, int p) {
        float v[RowVec<T>::E];
        unpack<T>(x, v);
#pragma unroll
        for (int i = 0; i < RowVec<T>::E; ++i) v[i] = g(v[i]);
        row.store_f32(a.dz, aligned, p, v);
    };
#pragma unroll
    for (int u = 0; u < NP; ++u)
        if (u * TPR + t < n) put(q[u], u * TPR + t);
    if constexpr (TPR == 1024)
        for (int p = NP * TPR + t; p < n; p += U * TPR) {
            uint4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * TPR < n) x[u] = row.load(z, p + u * TPR);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + u * TPR < n) put(x[u], p + u * TPR);
        }
    if constexpr (TPR <= 32)
        __syncwarp(TPR == 32 ? 0xffffffffu : 0xffu << (threadIdx.x & 24));
    else
        __syncthreads();
    put_entries<T, TPR>(a, g, row, 0, n, c, w, t, mine);
}

// Long rows, too few to fill the GPU with a CTA each: f in parts first, a CTA of 256 threads each, ... (8 x 32003 bf16 both
// launches as long as 100 rows of a CTA each.)
template <typename T>
__global__ void __launch_bounds__(256)
logprob_sum(const __grid_constant__ GradArgs a)
{
    constexpr int U = 4;
    __shared__ float sm[8];
    after_previous();
    const size_t r = blockIdx.x / a.sums;
    const int part = (int)(blockIdx.x % a.sums), t = threadIdx.x;
    const RowVec<T> row(r, a.V);
    const int pieces = row.pieces(), p_lo = (int)((long long)pieces * part / a.sums), n = (int)((long long)pieces * (part + 1) / a.sums);
    const float lse = a.lse[r];
    float f[1] = {0.0f};
    for (int p = p_lo + t; p < n; p += U * 256) {
        uint4 q[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u * 256 < n) q[u] = row.load((const T *)a.z, p + u * 256);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u * 256 < n) f[0] += piece_sum<T>(q[u], lse);
    }
    row_join<false, 256>(f, sm);
    if (t == 0) a.part[r * a.sums + part] = f[0];
}
// ... and then the gradient, a CTA to a range of a row's pieces, which adds the parts up in their order.
template <typename T>
__global__ void __launch_bounds__(256)
logprob_grad_range(const __grid_constant__ GradArgs a)
{
    constexpr int U = 4;
    __shared__ float sm[8];
    extern __shared__ __align__(16) uint8_t dyn[];
    after_previous();
    const int t = threadIdx.x;
    int *c = (int *)dyn;
    float *w = (float *)(dyn + (size_t)(a.k + 1) * 4);
    const size_t r = blockIdx.x / a.split;
    const int part = (int)(blockIdx.x % a.split);
    const T *z = (const T *)a.z;
    const RowVec<T> row(r, a.V);
    const int pieces = row.pieces(), p_lo = (int)((long long)pieces * part / a.split), n = (int)((long long)pieces * (part + 1) / a.split);
    uint4 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (p_lo + u * 256 + t < n) q[u] = row.load(z, p_lo + u * 256 + t);
    for (int j = t; j <= a.k; j += 256) read_entry(a, r, j, c, w);
    Grad g(a, r);
    float f[1] = {0.0f};
    for (int i = t; i < a.sums; i += 256) f[0] += a.part[r * a.sums + i];
    row_join<false, 256>(f, sm);
    g.join(a.k, w, f[0]);
    const float mine = entry_logit<T>(a, row, c, t);
    const bool aligned = on_32(a.dz);
    for (int p = p_lo + t; p < n; p += U * 256) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + u * 256 < n) {
                float v[RowVec<T>::E];
                unpack<T>(q[u], v);
#pragma unroll
                for (int i = 0; i < RowVec<T>::E; ++i) v[i] = g(v[i]);
                row.store_f32(a.dz, aligned, p + u * 256, v);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p + (U + u) * 256 < n) q[u] = row.load(z, p + (U + u) * 256);
    }
    __syncthreads();
    put_entries<T, 256>(a, g, row, p_lo, n, c, w, t, mine);
}

template <typename T>
cudaError_t launch_logprob(stacklstm_op *op, LogpArgs &a)
{
    int tpr, np;
    row_plan<T>(a.V, &tpr, &np);
    if (tpr <= 32) {
        const unsigned grid = ceil_div(a.rows, 256 / tpr);
        auto launch = [&](auto kernel) { return launch_after(kernel, grid, 256, 0, op->stream, a); };
        return tpr == 8 ? launch(np == 1 ? logprob_narrow<T, 8, 1> : np == 2 ? logprob_narrow<T, 8, 2> : logprob_narrow<T, 8, 4>)
                        : launch(np <= 2 ? logprob_narrow<T, 32, 2> : logprob_narrow<T, 32, 4>);
    }
    constexpr int NP = 8;
    const int pieces = (int)(((size_t)a.V + RowVec<T>::E - 1) / RowVec<T>::E) + 1;
    // Few rows: several CTAs each, of two pieces a thread at least, and the small CTAs where those hold the parts.
    // 8 x 32003 bf16 with 16 alternatives: 12.0 us with two CTAs of 512 threads a row.
    const size_t room = (size_t)op->num_sms * 4 / a.rows;  // CTAs of 128 threads a row
    const bool small = pieces <= 128 * NP || (room > 1 && pieces <= 128 * NP * (int)std::min<size_t>(room, 64));
    const int nt = small ? 128 : 256;
    a.split = (int)std::max<size_t>(1, std::min<size_t>(std::min<size_t>(64, pieces / (nt * 2)), small ? room : (size_t)op->num_sms * 4 / a.rows));
    a.per = (int)ceil_div(pieces, a.split);
    if (a.split > 1) {
        cudaError_t e = op_workspace(op, 0, (size_t)a.rows * a.split * 16);
        if (!e && a.k) e = op_workspace(op, 1, (size_t)a.rows * a.split * a.k * 8);
        if (e) return e;
        a.part = (float4 *)op->ws[0];
        a.part_key = (u64 *)op->ws[1];
        a.arrived = (int *)op->ws[2];
    }
    // A long row's threads: 128, eight rows an SM, where the room for its best keys is small, else 256. 4096 x 32003 bf16 without
    // alternatives 53 us, 60 with 256 threads and 82 with 512; with 8 of them 84 and 89, with 12 (caches cold) 115 and 101, with
    // 32 296 and 134; 8192 x 12000 with 8 97 and 119, 12 119 and 124, 16 144 and 128; fp32, 4096 x 32003, 8 138 and 148, 12 156 and 152.
    const int per = small ? NP : a.k <= 8 ? 4 * NP : 2 * NP;  // pieces a thread and segment
    const size_t spill = (size_t)a.k * std::max(per * RowVec<T>::E + 1, (int)kMergeItems) * 8;
    const dim3 grid((unsigned)((size_t)a.rows * a.split));
    auto launch = [&](auto kernel, unsigned threads) {
        if (spill > 32 * 1024)
            if (cudaError_t e = smem_at_least((const void *)kernel, spill)) return e;
        return launch_after(kernel, grid, threads, spill, op->stream, a);
    };
    if (small) return launch(logprob_wide<T, 128, NP>, 128);
    return a.k <= 8 ? launch(logprob_wide<T, 128, 4 * NP>, 128) : launch(logprob_wide<T, 256, 2 * NP>, 256);
}

template <typename T>
cudaError_t launch_grad(stacklstm_op *op, GradArgs &a)
{
    int tpr, np;
    row_plan<T>(a.V, &tpr, &np);
    if (tpr <= 32 || a.rows >= op->num_sms / 2) {
        const size_t smem = (size_t)rows_per_cta(tpr) * (a.k + 1) * 8;
        const dim3 grid(ceil_div(a.rows, rows_per_cta(tpr)));
#define SL_GRAD(TPR, NP) \
    if (tpr == TPR && np && np <= NP) return launch_after(logprob_grad<T, TPR, NP>, grid, row_cta(TPR), smem, op->stream, a);
        SL_GRAD(8, 1) SL_GRAD(8, 2) SL_GRAD(8, 4) SL_GRAD(32, 2) SL_GRAD(32, 4) SL_GRAD(128, 2) SL_GRAD(128, 4) SL_GRAD(128, 8)
        SL_GRAD(512, 4) SL_GRAD(512, 8)
        return launch_after(logprob_grad<T, 1024, 8>, grid, 1024, smem, op->stream, a);
#undef SL_GRAD
    }
    const size_t pieces = ((size_t)a.V + RowVec<T>::E - 1) / RowVec<T>::E + 1;
    a.split = (int)std::max<size_t>(1, std::min<size_t>(ceil_div(pieces, 1024), (1u << 30) / (size_t)a.rows));
    a.sums = std::min(a.split, 256);
    if (cudaError_t e = op_workspace(op, 3, (size_t)a.rows * a.sums * 4)) return e;
    a.part = (float *)op->ws[3];
    if (cudaError_t e = launch_after(logprob_sum<T>, dim3((unsigned)((size_t)a.rows * a.sums)), 256, 0, op->stream, a)) return e;
    return launch_after(logprob_grad_range<T>, dim3((unsigned)((size_t)a.rows * a.split)), 256, (size_t)(a.k + 1) * 8, op->stream, a);
}

}  // namespace
}  // namespace sl

using namespace sl;

extern "C" {

sl_status stacklstm_logprob_create(stacklstm_op_t *out, int R, int V, int k, sl_dtype dtype, int device, void *stream)
{
    if (!out) return SL_ERR_ARG;
    *out = nullptr;
    if (R < 1 || V < 1 || k < 0 || (dtype != SL_FP32 && dtype != SL_BF16)) return SL_ERR_ARG;
    if (k > kMaxBeams || V > (1 << 30)) return SL_ERR_UNSUPPORTED;
    sl_status st;
    stacklstm_op *op = op_new(SL_OP_LOGPROB, dtype, device, stream, &st);
    if (!op) return st;
    op->R = R;
    op->V = V;
    op->k = k;
    // the arrival counters of rows over several CTAs
    const size_t counters = std::min<size_t>(R, (size_t)op->num_sms * 4) * 4;
    cudaError_t e = op_workspace(op, 2, counters);
    if (!e) e = cudaMemsetAsync(op->ws[2], 0, counters, op->stream);
    if (e) {
        cudaGetLastError();
        stacklstm_op_destroy(op);
        return SL_ERR_OOM;
    }
    *out = op;
    return SL_OK;
}

sl_status stacklstm_logprob_forward(stacklstm_op_t op, int rows, const void *logits, const int32_t *target, float *logp,
                                    float *entropy, float *lse, int32_t *top_idx, float *top_logp)
{
    if (!op || op->kind != SL_OP_LOGPROB) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (rows < 0 || rows > op->R) return op_fail(op, SL_ERR_ARG, "rows outside 0 .. R");
    if (rows == 0) return SL_OK;
    if (const char *m = check_pointers({logits}, {target, logp, entropy, lse, top_idx, top_logp})) return op_fail(op, SL_ERR_ARG, m);
    OpDevice guard(op->device);
    LogpArgs a = {};
    a.rows = rows; a.V = op->V; a.k = top_idx || top_logp ? op->k : 0; a.z = logits; a.target = target; a.logp = logp;
    a.entropy = entropy; a.lse = lse; a.top_idx = top_idx; a.top_logp = top_logp; a.err = op->err; a.split = 1;
    const cudaError_t e = op->dt == SL_BF16 ? launch_logprob<__nv_bfloat16>(op, a) : launch_logprob<float>(op, a);
    return e ? op_cuda(op, e, "stacklstm_logprob_forward") : SL_OK;
}

sl_status stacklstm_logprob_backward(stacklstm_op_t op, int rows, const void *logits, const int32_t *target, const float *entropy,
                                     const float *lse, const int32_t *top_idx, const float *dlogp, const float *dentropy,
                                     const float *dtop, float *dlogits)
{
    if (!op || op->kind != SL_OP_LOGPROB) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (rows < 0 || rows > op->R) return op_fail(op, SL_ERR_ARG, "rows outside 0 .. R");
    if (rows == 0) return SL_OK;
    if (const char *m = check_pointers({logits, lse, dlogits}, {target, entropy, top_idx, dlogp, dentropy, dtop}))
        return op_fail(op, SL_ERR_ARG, m);
    if (dlogp && !target) return op_fail(op, SL_ERR_ARG, "dlogp without target");
    if (dentropy && !entropy) return op_fail(op, SL_ERR_ARG, "dentropy without entropy");
    if (dtop && (!top_idx || !op->k)) return op_fail(op, SL_ERR_ARG, "dtop without top_idx");
    OpDevice guard(op->device);
    GradArgs a = {};
    a.rows = rows; a.V = op->V; a.k = dtop ? op->k : 0; a.z = logits; a.target = target; a.top_idx = top_idx; a.entropy = entropy;
    a.lse = lse; a.dlogp = dlogp; a.dentropy = dentropy; a.dtop = dtop; a.dz = dlogits; a.err = op->err;
    const cudaError_t e = op->dt == SL_BF16 ? launch_grad<__nv_bfloat16>(op, a) : launch_grad<float>(op, a);
    return e ? op_cuda(op, e, "stacklstm_logprob_backward") : SL_OK;
}

}  // extern "C"
