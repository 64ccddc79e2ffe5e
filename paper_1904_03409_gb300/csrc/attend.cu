// attend.cu -- attention of a StackLSTM's outputs over an encoder's states of another length, its
// backward, and their C ABI (include/stacklstm.h, stacklstm_attend_*).
//
// For a sentence with n states, query t and state s of one head, with c > 0 the scale,
//   z_ts = c q_t . k_s,   w_ts = exp(z_ts - lse_t),  lse_t = ln sum_{s < n} exp z_ts,   y_t = sum_s w_ts v_s
// and for the gradient dy of y
//   dv_s = sum_t w_ts dy_t,   dz_ts = w_ts (dy_t . v_s - dy_t . y_t),   dq_t = c sum_s dz_ts k_s,   dk_s = c sum_t dz_ts q_t.
// Neither z nor w is ever in memory: the forward goes over the states in tiles of 64 and keeps, for
// each query, the largest z so far, the sum of exponentials and the weighted sum of v against it; the
// backward makes w again from lse, and from f_t = sum_s exp(z_ts - lse_t), 1 but for what lse's rounding lost.
//
// All products run on the tensor cores (tcgen05, bf16 operands, fp32 accumulators in tensor memory).
// A bf16 tensor is one operand; an fp32 number is the sum of three bf16 parts (8 + 8 + 8 significant
// bits) and the product of two of them six partial products, of one with a bf16 number three (what is
// left out is below 2^-23 of it). So gradients, which are fp32, have fp32's accuracy whatever the
// inputs' type: dy, w and dz enter as three parts. The tensor cores' additions cut, so that an accumulator's error
// grows with what it takes: one tile's products (threads add the tiles up in registers, in fp32), or for a bf16
// result those of kRun tiles.
//
// Queries of the heads that share a state's head lie side by side: row r of a tile is query
// t0 + r / G of head r % G of the G, so that a tile reads the states once for all of them, and their
// gradients' sums come from the products themselves.
#include <limits.h>

#include <type_traits>

#include "op.cuh"
#include "tc.cuh"

namespace sl {
namespace {

using tc::elect_one;
using tc::smem_u32;
using tc::warp_wait;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr long long kDrain = 4000000000LL;  // clock cycles: waits for a CTA's own copies and MMAs before it ends
constexpr int kMostGroup = 32;              // heads that share a state's head
constexpr int kMostD = 128;

__device__ __forceinline__ float exp2_hw(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The partial products of PA parts of A and PB of B: those of order i + j <= 2, small ones first.
template <int PA, int PB>
struct Products {
    int n = 0, a[6] = {}, b[6] = {};
    constexpr Products()
    {
        for (int order = 2; order >= 0; --order)
            for (int i = 0; i < PA; ++i)
                if (order - i >= 0 && order - i < PB) {
                    a[n] = i;
                    b[n++] = order - i;
                }
    }
};

// A sentence's length, checked (a length outside 0 .. n is the nearest one).
__device__ __forceinline__ int checked_len(int v, int n, int32_t *err, bool reports)
{
    if (v >= 0 && v <= n) return v;
    if (reports) atomicCAS(err, 0, (int)SL_ERR_ARG);
    return v < 0 ? 0 : n;
}
__device__ __forceinline__ int seq_len(const int32_t *len, int b, int n, int32_t *err, bool reports)
{
    return len ? checked_len(len[b], n, err, reports) : n;
}

// What a CTA works on at a time: tile `tile` of a sentence's queries (states) for one of the states' heads, in split
// `sp` of several.
struct Item {
    int tile, sp, kvh, b, q_len, len;
};
// CTAs take items as they come to them (sentences' lengths differ; with a fixed share of the items a CTA could have
// twice another's work): the loading warp fetches the numbers from a counter and tells the other warps through shared
// memory. Items go over the tiles first, then the heads, the sentences and the splits: a sentence's last split, often a
// short one or empty, is begun late.
constexpr int kItems = 4;  // told ahead at most
constexpr int kSorted = 192;  // sentences at most (256 would not fit beside attend_grad_states<3, 64>'s tiles)
struct ItemRing {
    uint64_t full[kItems], empty[kItems];
    Item item[kItems];     // the last has tile -1
    unsigned char order[kSorted];
};
__device__ __forceinline__ void init_items(ItemRing &r, int readers)
{
    for (int i = 0; i < kItems; ++i) {
        tc::mbar_init(&r.full[i], 1);
        tc::mbar_init(&r.empty[i], readers);
    }
}
// Where the items are few to a CTA (g.sorted), sentences of more states (queries) come first, so that no long item is
// begun when the others end: 4 x 2048 x 4096, heads of 128, 105 us, 115 in the sentences' order.
template <typename A>
__device__ __forceinline__ void sort_sentences(const A &g, ItemRing &ring, const int32_t *len, int *lens)  // (lens: room in shared memory)
{
    for (int b = threadIdx.x; b < g.B; b += blockDim.x) lens[b] = len[b];
    __syncthreads();
    for (int b = threadIdx.x; b < g.B; b += blockDim.x) {
        const int mine = lens[b];
        int before = 0;
        for (int i = 0; i < g.B; ++i) before += lens[i] > mine || (lens[i] == mine && i < b);
        ring.order[before] = (unsigned char)b;
    }
    __syncthreads();
}
// The loading warp's side: f(item) for each item until one says no.
template <typename A, typename F>
__device__ __forceinline__ bool fetch_items(const A &g, ItemRing &ring, volatile int *abort, const F &f)
{
    const int lane = threadIdx.x & 31;
    // Item j + 1's number and lengths are on their way while item j's loads are issued, and the number after it.
    struct {
        Item w;
        int q, len;  // as they are in memory
        bool more;
    } now, after;
    auto look = [&](int it, auto &n) {
        n.more = it < g.items;
        if (!n.more) return;
        unsigned u = (unsigned)it;
        n.w.tile = (int)(u % (unsigned)g.tiles);
        u /= (unsigned)g.tiles;
        n.w.kvh = (int)(u % (unsigned)g.nk);
        u /= (unsigned)g.nk;
        n.w.b = (int)(u % (unsigned)g.B);
        n.w.sp = (int)(u / (unsigned)g.B);
        if (g.sorted) n.w.b = ring.order[n.w.b];
        n.q = g.q_len ? g.q_len[n.w.b] : g.T;
        n.len = g.kv_len ? g.kv_len[n.w.b] : g.S;
    };
    auto take_next = [&] { return lane == 0 ? atomicAdd(g.next, 1) : 0; };
    look(blockIdx.x, now);
    int next = take_next();
    for (int j = 0;; ++j) {
        const int s = j % kItems;
        if (!warp_wait(&ring.empty[s], (uint32_t)(j / kItems + 1) & 1, g.limit, abort)) return false;
        if (now.more) {
            now.w.q_len = checked_len(now.q, g.T, g.err, lane == 0);
            now.w.len = checked_len(now.len, g.S, g.err, lane == 0);
        } else {
            now.w.tile = -1;
        }
        if (lane == 0) {
            ring.item[s] = now.w;
            tc::mbar_arrive(&ring.full[s]);
        }
        if (!now.more) return true;
        look((int)gridDim.x + __shfl_sync(0xffffffffu, next, 0), after);
        next = take_next();
        if (!f(now.w)) return false;
        now = after;
    }
}
// The other warps' side. idle() is called where the next item is not known yet, before the wait for it: the MMA warp
// holds a tile's last products back until it knows what comes next, but no longer (the items in between may have no
// tiles, and other warps may need those products before they make room for more of them).
template <typename A, typename F, typename I>
__device__ __forceinline__ bool each_item(const A &g, ItemRing &ring, volatile int *abort, const F &f, const I &idle)
{
    for (int j = 0;; ++j) {
        const int s = j % kItems;
        if (!__all_sync(0xffffffffu, tc::mbar_test_wait(&ring.full[s], (uint32_t)(j / kItems) & 1)) && !idle()) return false;
        if (!warp_wait(&ring.full[s], (uint32_t)(j / kItems) & 1, g.limit, abort)) return false;
        const Item w = ring.item[s];
        __syncwarp();
        if ((threadIdx.x & 31) == 0) tc::mbar_arrive(&ring.empty[s]);
        if (w.tile < 0) return true;
        if (!f(w)) return false;
    }
}
template <typename A, typename F>
__device__ __forceinline__ bool each_item(const A &g, ItemRing &ring, volatile int *abort, const F &f)
{
    return each_item(g, ring, abort, f, [] { return true; });
}
// The counter for the next launch, by the last CTA to end (next[1] counts those).
__device__ __forceinline__ void items_done(int *next)
{
    __threadfence();
    if (atomicAdd(next + 1, 1) == (int)gridDim.x - 1) {
        next[0] = 0;
        next[1] = 0;
    }
}

// Rows that lie one to a lane to memory through 2 KB of shared memory a warp, so that the lanes of an access lie
// side by side: four 16-byte pieces of each lane's row, to `row` (null: nowhere), the first n elements of them;
// whole: rows and n are whole pieces. (Straight from the lanes an access is 32 lines: stores of a tile's outputs
// took four times the cycles.)
constexpr uint32_t kStageBytes = 2048;
// Element by element, where pieces of a row are not on 16 bytes. (A function of its own: inlined, its code at every
// output slowed the kernels whose heads never need it by a tenth.)
template <typename T>
__device__ __noinline__ void put_elements(uint32_t stage, T *row, int n)
{
    constexpr int E = 16 / (int)sizeof(T), RE = 4 * E;  // elements of a piece, of a row here
    const int lane = threadIdx.x & 31, e = lane % RE;
#pragma unroll 4
    for (int k = 0; k < RE; ++k) {
        const int r = k * (32 / RE) + lane / RE;
        T *to = (T *)__shfl_sync(0xffffffffu, (unsigned long long)row, r);
        const uint32_t from = stage + r * 64 + ((e / E ^ (r >> 1 & 3)) << 4) + e % E * (uint32_t)sizeof(T);
        if (to && e < n) {
            if constexpr (sizeof(T) == 4) {
                float x;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(from));
                to[e] = x;
            } else {
                unsigned short x;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(from));
                to[e] = __ushort_as_bfloat16(x);
            }
        }
    }
}
// A warp's rows: D numbers v of each lane times `by` (or 0 where `none`), as type T, to row (null: nowhere) of memory.
template <typename T, int DP>
__device__ __forceinline__ void put_rows(uint32_t stage, T *row, const float2 (&v)[DP / 2], int D, float by, bool none, bool whole)
{
    constexpr int E = 16 / (int)sizeof(T);
    const int lane = threadIdx.x & 31, piece = lane & 3;
    T *to[4];  // what this lane writes of: rows k 8 + lane / 4
#pragma unroll
    for (int k = 0; k < 4; ++k) to[k] = (T *)__shfl_sync(0xffffffffu, (unsigned long long)row, k * 8 + (lane >> 2));
#pragma unroll
    for (int i = 0; i < DP; i += 4 * E)
        if (i < D) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (sizeof(T) == 4) {
                        const float2 f = v[(i + 4 * j + k) / 2];
                        w[k] = none ? 0u : __float_as_uint((k & 1 ? f.y : f.x) * by);
                    } else {
                        const float2 f = v[(i + 8 * j) / 2 + k];
                        const __nv_bfloat162 h = __floats2bfloat162_rn(f.x * by, f.y * by);
                        w[k] = none ? 0u : *(const uint32_t *)&h;
                    }
                }
                tc::st_shared_v4(stage + lane * 64 + ((j ^ (lane >> 1 & 3)) << 4), w);
            }
            __syncwarp();
            if (whole) {
                uint4 q[4];  // (all reads, then all writes: one after the other a piece took 800 cycles)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int r = k * 8 + (lane >> 2);
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(q[k].x), "=r"(q[k].y), "=r"(q[k].z), "=r"(q[k].w)
                                 : "r"(stage + r * 64 + ((piece ^ (r >> 1 & 3)) << 4)));
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (to[k] && i + piece * E < D) *(uint4 *)(to[k] + i + piece * E) = q[k];
            } else {
                put_elements<T>(stage, row ? row + i : nullptr, min(4 * E, D - i));
            }
            __syncwarp();
        }
}

template <int NP>
struct Maps {
    CUtensorMap q[NP], k[NP], v[NP];
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void *tmap, int c0, int c1, int c2, int c3, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(dst), "l"((uint64_t)tmap), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const void *tmap, int c0, int c1, int c2, int c3, int c4, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
        ::"r"(dst), "l"((uint64_t)tmap), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(smem_u32(bar))
        : "memory");
}

// Operands in shared memory by the lower word of their descriptors (address and leading offset in units of
// 16 bytes): the upper one (rows of 128 bytes, 128-byte swizzle) is that of all of them, and operands are at
// constant distances from one another, so that one register and immediate numbers make every descriptor.
// (With a 64-bit descriptor each the issuing warp's registers were spilled.)
constexpr uint32_t kDescUpper = (1024u >> 4) | (1u << 14) | ((uint32_t)tc::kSwizzle128B << 29);
__host__ __device__ constexpr uint32_t desc_lower(uint32_t lbo_bytes) { return (lbo_bytes >> 4) << 16; }
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescUpper)
        : "memory");
}
// f(k) for the contraction's steps of 16: written out where they are four, else two to a loop's body (8 x 1024 x 1024,
// heads of 128, backward 420 us with all of them written out, 330 so: the warps waited for instructions; heads of 64,
// 256 x 256 x 256, 840 and 790 the other way).
template <int NP, int DP, typename F>
__device__ __forceinline__ void each_step(int steps, const F &f)
{
    if constexpr (NP == 1 && DP == 64) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < steps) f(k);
    } else {
#pragma unroll 2
        for (int k = 0; k < steps; ++k) f(k);
    }
}
// A in tensor memory: its rows are the lanes, two bf16 of the contraction a column.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescUpper)
        : "memory");
}
// Each thread of a warp writes 16 (8) consecutive columns of its own lane.
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The largest of three.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}
// The upper halves of two words (a's below): two fp32 numbers cut to bf16.
__device__ __forceinline__ uint32_t upper2(float a, float b) { return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632); }
// What cutting both to bf16 leaves, exactly: two cuts leave 8 significant bits, a third part of their own.
__device__ __forceinline__ float2 less_upper2(float2 v)
{
    return __fadd2_rn(v, make_float2(-__uint_as_float(__float_as_uint(v.x) & 0xffff0000u), -__uint_as_float(__float_as_uint(v.y) & 0xffff0000u)));
}

// acc += D columns of a lane, so many at a time.
template <int DP, int STEP>
__device__ __forceinline__ void add_columns(uint32_t at, int D, float2 (&acc)[DP / 2])
{
#pragma unroll
    for (int i = 0; i < DP; i += STEP)
        if (i < D) {  // (what is past D is not used)
            uint32_t v[STEP / 16][16];
#pragma unroll
            for (int j = 0; j < STEP / 16; ++j) tc::tmem_ld16_async(at + i + 16 * j, v[j]);
            tc::tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < STEP / 2; ++j)
                acc[i / 2 + j] = __fadd2_rn(acc[i / 2 + j], make_float2(__uint_as_float(v[j / 8][2 * j % 16]), __uint_as_float(v[j / 8][2 * j % 16 + 1])));
        }
}

__device__ __forceinline__ void zero_shared(uint32_t at, uint32_t bytes, int thread, int threads)
{
    const uint32_t z[4] = {0, 0, 0, 0};
    for (uint32_t o = thread * 16; o < bytes; o += threads * 16) tc::st_shared_v4(at + o, z);
}

// ------------------------------------------------------------------ operands made of tensors
// What a call makes of its tensors first, in one launch: an fp32 tensor as three bf16 parts, a bf16
// one whose heads do not start on 16 bytes as a copy whose heads do; with dy also dy . y of each row.
// `lanes` lanes take a head's row, eight elements each.
struct Pack {
    const void *src;      // [rows][heads][D], or null
    __nv_bfloat16 *out;   // [parts][rows][heads][Dp]
    const float *ctx;     // dy alone: y in fp32
    float *delta;         // dy alone: [rows][heads]
    const int32_t *len;
    int n, B, heads, D, Dp, batch_major, fp32, lanes;
    unsigned ctas;
};
struct Packs {
    Pack t[4];
    int32_t *err;
};
template <typename T>
__device__ __forceinline__ void read_eight(const T *p, int n, bool whole, float (&v)[8])
{
    if (whole) {
        load_vec<T, 8>(p, v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? to_f32(p[j]) : 0.0f;
    }
}

union Eight {
    __nv_bfloat162 p[4];
    __nv_bfloat16 b[8];
    uint4 q;
};
// split3 of eight, two at a time. Where a value is not finite, or its first part is not, so is what is left at the end,
// and each is split by itself. (One at a time, with those checks for each, 256 x 256 x 256
// training 1063 us where it takes 1049, 20 x 300 x 300 fp32 heads of 37, backward 129 and 107.)
__device__ __forceinline__ void split_eight(const float (&v)[8], Eight (&o)[3])
{
    float odd = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float2 r = make_float2(v[2 * j], v[2 * j + 1]);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            o[k].p[j] = __float22bfloat162_rn(r);
            const float2 part = __bfloat1622float2(o[k].p[j]);
            if (k < 2) r = __fadd2_rn(r, make_float2(-part.x, -part.y));
        }
        odd = fmaf(r.x, 0.0f, fmaf(r.y, 0.0f, odd));
    }
    if (odd == 0.0f) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        __nv_bfloat16 p[3];
        split3(v[j], p);
#pragma unroll
        for (int k = 0; k < 3; ++k) o[k].b[j] = p[k];
    }
}

__device__ __forceinline__ void pack_block(const Pack &a, unsigned cta, int32_t *err)
{
    const int lane = threadIdx.x % a.lanes, sub = threadIdx.x / a.lanes, per = 256 / a.lanes;
    const size_t items = (size_t)a.n * a.B * a.heads, plane = items * a.Dp;
    const int e0 = lane * 8;
    const bool whole = a.D % 8 == 0;
    {
        const size_t it = (size_t)cta * per + sub;
        bool here = it < items;
        if (here) {
            int b, t;
            if (items < (size_t)1 << 32) {  // (64-bit divisions took as many instructions as all the rest)
                const unsigned row = (unsigned)it / (unsigned)a.heads;
                b = (int)(a.batch_major ? row / (unsigned)a.n : row % (unsigned)a.B);
                t = (int)(a.batch_major ? row % (unsigned)a.n : row / (unsigned)a.B);
            } else {
                const size_t row = it / a.heads;
                b = (int)(a.batch_major ? row / a.n : row % a.B);
                t = (int)(a.batch_major ? row % a.n : row / a.B);
            }
            here = t < seq_len(a.len, b, a.n, err, lane == 0);  // (padding is not read)
        }
        float v[8] = {}, w[8] = {};
        const bool mine = here && e0 < a.D;
        if (mine) {
            if (a.fp32)
                read_eight((const float *)a.src + it * a.D + e0, a.D - e0, whole, v);
            else
                read_eight((const __nv_bfloat16 *)a.src + it * a.D + e0, a.D - e0, whole, v);
            if (a.ctx) read_eight(a.ctx + it * a.D + e0, a.D - e0, whole, w);
        }
        if (here && e0 < a.Dp) {
            if (a.fp32) {
                Eight o[3];
                split_eight(v, o);
#pragma unroll
                for (int k = 0; k < 3; ++k) *(uint4 *)(a.out + k * plane + it * a.Dp + e0) = o[k].q;
            } else {
                store_vec<__nv_bfloat16, 8>(a.out + it * a.Dp + e0, v);
            }
        }
        if (a.delta) {
            float d = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) d = fmaf(v[j], w[j], d);
            for (int o = a.lanes / 2; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
            if (lane == 0 && it < items) a.delta[it] = d;  // (0 of padding)
        }
    }
}

// Bound by HBM and, nearly as much, by instructions: 4 bytes read and 6 written an element (dy: 8 and 6); dy of
// 64 x 256 x 1024 in 36 us, 6.5 TB/s.
__global__ void __launch_bounds__(256)
attend_pack(const __grid_constant__ Packs a)
{
    after_previous();
    unsigned cta = blockIdx.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (cta < a.t[i].ctas) return pack_block(a.t[i], cta, a.err);
        cta -= a.t[i].ctas;
    }
}

// ------------------------------------------------------------------ forward
constexpr int kRows = 128, kKeys = 64;  // of a tile
constexpr uint32_t kQBlock = kRows * 128, kKBlock = kKeys * 128;  // bytes of 64 columns of a tile

// NP: parts of q, k and v; PP: of w. Three of them are w; two (the second rounded) leave out at most 2^-15 of it, which a
// bf16 result, rounded by up to 2^-8, does not show: 4 x 2048 x 4096, heads of 128, is 1.66e-3 off 64 bits, the rounding
// alone, in 130 us (of one part 2.3e-3, 107 us; of three 281 us, sums in registers).
template <int NP, int PP, int DP>
struct FwdShape {
    static constexpr int DB = DP / 64;
    using Out = typename std::conditional<NP == 3, float, __nv_bfloat16>::type;
    static constexpr int kCtas = NP == 3 && DP == 128 ? 1 : 2;  // an SM
    static constexpr int kStages = NP == 3 ? 1 : DP == 64 ? 3 : 2;
    static constexpr int kQs = NP == 1 && DP == 64 ? 2 : 1;     // places for queries
    static constexpr uint32_t kQ = NP * DB * kQBlock, kKV = NP * DB * kKBlock;
    static constexpr uint32_t kK0 = kQs * kQ, kV0 = kK0 + kStages * kKV, kStage0 = kV0 + kStages * kKV, kMain = kStage0 + 4 * kStageBytes;
    static constexpr uint32_t kBars = (5 * kStages + 2 * kQs + 7) * 8 + 16;
    static constexpr uint32_t kSmem = 1024 + kMain + kBars;
    // tensor memory: z, w, w v; where that is more than an SM's half, w over z's second half (which is read first). A
    // bf16 result's sum of w v stays there, with two places for w in turn where there is room; an fp32 result's is added
    // up in registers, tile by tile. (w over the tile's own z, two places of both in turn, with heads of 128: 4 x 2048 x 4096
    // 191 us of equal sentences, 173 so.)
    static constexpr bool kSums = PP == 2;
    // Tiles whose w v are summed in tensor memory before the sum goes to memory, where it is added up in fp32: 8 MMAs a
    // tile, each of which loses 2^-23.8 of the sum (2^20 values of one sign in one sum: y 0.9 % too small), 2^-14.8 in all.
    static constexpr int kRun = 64;
    static constexpr bool kOver = kCtas == 2 && kKeys + PP * kKeys / 2 + DP > 256;
    static constexpr uint32_t kWs = kSums && DP == 64 ? 2 : 1;  // places for w
    static constexpr uint32_t kColW = kOver ? kKeys / 2 : kKeys, kColO = kColW + kWs * PP * kKeys / 2;
    static __device__ uint32_t col_w(int tile, int part) { return kColW + ((uint32_t)tile % kWs * PP + part) * (kKeys / 2); }
    static constexpr uint32_t kCols = kColO + DP <= 256 ? 256 : 512;
    static_assert(kSmem + sizeof(ItemRing) <= (kCtas == 2 ? 113 : 227) * 1024 && (kCtas == 1 || kCols == 256), "tensor and shared memory of a CTA");
};

struct FwdArgs {
    int T, S, B, nk, G, D;
    int q_t, q_b;             // rows of (head, D) from one query (sentence) to the next, in heads
    const int32_t *q_len, *kv_len;
    float scale;
    void *y;
    float *lse, *ctx;
    float *part;              // [split][rows][Dp], or null
    float2 *part_stats;       // [split][rows]: the largest z, the sum of exponentials against it (0: no states)
    float *sums;              // [split][rows][Dp], part or a buffer by itself: a bf16 result's sums of the runs before
    int split, per;           // splits of the key tiles, key tiles of a split
    int tq, tiles, items;     // queries of a tile, tiles; all items
    size_t rows;              // B T heads
    int Dp;
    int *next;                // the items' counter, 0 between launches
    int sorted;               // longer sentences first
    long long limit;
    int32_t *err;
};

// The key tiles lo .. lo + n of an item.
__device__ __forceinline__ void key_tiles(const FwdArgs &g, const Item &w, int &lo, int &n)
{
    lo = w.sp * g.per;
    const int hi = w.tile * g.tq < w.q_len ? min(lo + g.per, (w.len + kKeys - 1) / kKeys) : lo;
    n = max(0, hi - lo);
}

// CTAs take items one after the other: 128 query rows of one sentence and state's head, and a range of its key tiles. Warp 0
// loads (TMA), also the next item's queries and states while this one's outputs are made, warp 1 issues the MMAs, warp 2
// clears what lies behind a sentence's last state, and a thread of warps 4 to 7 has a query: 32 z of a tile at a time
// in registers, and an fp32 result's sum of w v.
// Bound by a tile's chain of MMA, reading z, exponentials and writing w, which two CTAs an SM and z one tile ahead hide
// in part: 64 x 256 x 256, 16 heads of 64, bf16, 52 us (issue 42 %, tensor pipe 23 %), 71 for an fp32 result too; 8 x 1024 x
// 1024, 8 heads of 128, 57 us (tensor pipe 46 %), 112; 4 x 2048 x 4096, 8 heads of 128 over 2, 134 us (455 TFLOP/s).
template <int NP, int PP, int DP>
__global__ void __launch_bounds__(256, FwdShape<NP, PP, DP>::kCtas)
attend_forward(const __grid_constant__ Maps<NP> tm, const __grid_constant__ FwdArgs g)
{
    using Sh = FwdShape<NP, PP, DP>;
    constexpr int DB = Sh::DB, NS = Sh::kStages, QS = Sh::kQs;
    constexpr Products<NP, NP> PS;
    constexpr Products<PP, NP> PO;
    __shared__ ItemRing ring;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t sm = smem_u32(base);
    uint64_t *full_k = (uint64_t *)(base + Sh::kMain), *full_v = full_k + NS, *empty_k = full_v + NS, *empty_v = empty_k + NS,
             *q_full = empty_v + NS, *q_free = q_full + QS, *z_full = q_free + QS, *z_read = z_full + 1, *w_ready = z_read + 1,
             *o_full = w_ready + 2, *fixed = o_full + 2, *done = fixed + NS;
    uint32_t *tmem_slot = (uint32_t *)(done + 1);
    volatile int *abort = (volatile int *)(tmem_slot + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        // (empty_v: the MMAs and warp 2, which has to have seen every tile of a place before the next one's load ends)
        for (uint64_t *bar = full_k; bar <= done; ++bar) tc::mbar_init(bar, bar >= z_read && bar < o_full ? 4 : bar >= empty_v && bar < q_full ? 2 : 1);
        init_items(ring, 6);
        *abort = 0;
        tc::fence_mbar_init();
    }
    if (tid >= 64 && tid < 64 + 3 * NP)
        tc::prefetch_map(tid - 64 < NP ? &tm.q[tid - 64] : tid - 64 < 2 * NP ? &tm.k[tid - 64 - NP] : &tm.v[tid - 64 - 2 * NP]);
    if (warp == 0) tc::tmem_alloc(tmem_slot, Sh::kCols);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    after_previous();
    if (g.sorted) sort_sentences(g, ring, g.kv_len, (int *)(base + Sh::kStage0));

    const long long limit = g.limit;
    auto fail = [&]() {
        *abort = 1;
        atomicCAS(g.err, 0, (int)SL_ERR_TIMEOUT);
    };

    if (warp < 4) {
        if constexpr (Sh::kCtas == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Sh::kSums ? 80 : 48));
        const bool issues = elect_one();
        if (warp == 0) {
            int m = 0, nv = 0, j = 0;  // loads of k, of v, of queries
            const bool ok = fetch_items(g, ring, abort, [&](const Item &w) {
                int lo, n;
                key_tiles(g, w, lo, n);
                if (n == 0) return true;
                if (!warp_wait(&q_free[j % QS], (uint32_t)(j / QS + 1) & 1, limit, abort)) return false;
                if (issues) {
                    tc::mbar_arrive_expect_tx(&q_full[j % QS], NP * DB * (uint32_t)(g.tq * g.G) * 128u);
#pragma unroll
                    for (int p = 0; p < NP; ++p)
                        for (int d = 0; d < DB; ++d)
                            tma_load_5d(sm + j % QS * Sh::kQ + (p * DB + d) * kQBlock, &tm.q[p], d * 64, 0, w.kvh, w.b, w.tile * g.tq, &q_full[j % QS]);
                }
                ++j;
                for (int i = 0; i < n; ++i) {
                    const int s = m % NS, s0 = (lo + i) * kKeys;
                    const uint32_t ph = (uint32_t)(m / NS + 1) & 1;
                    if (!warp_wait(&empty_k[s], ph, limit, abort)) return false;
                    ++m;
                    if (issues) {
                        tc::mbar_arrive_expect_tx(&full_k[s], Sh::kKV);
#pragma unroll
                        for (int p = 0; p < NP; ++p)
                            for (int d = 0; d < DB; ++d)
                                tma_load_4d(sm + Sh::kK0 + s * Sh::kKV + (p * DB + d) * kKBlock, &tm.k[p], d * 64, w.kvh, w.b, s0, &full_k[s]);
                    }
                    if (!warp_wait(&empty_v[s], ph, limit, abort)) return false;
                    ++nv;
                    if (issues) {
                        tc::mbar_arrive_expect_tx(&full_v[s], Sh::kKV);
#pragma unroll
                        for (int p = 0; p < NP; ++p)
                            for (int d = 0; d < DB; ++d)
                                tma_load_4d(sm + Sh::kV0 + s * Sh::kKV + (p * DB + d) * kKBlock, &tm.v[p], d * 64, w.kvh, w.b, s0, &full_v[s]);
                    }
                }
                return true;
            });
            if (!ok && issues) fail();
            // no copy in flight when the CTA ends: the last load of every place has landed
            for (int s = 0; s < QS; ++s)
                if (j > s) tc::mbar_wait(&q_full[s], (uint32_t)((j - 1 - s) / QS) & 1, kDrain, nullptr);
            for (int s = 0; s < NS; ++s) {
                if (m > s) tc::mbar_wait(&full_k[s], (uint32_t)((m - 1 - s) / NS) & 1, kDrain, nullptr);
                if (nv > s) tc::mbar_wait(&full_v[s], (uint32_t)((nv - 1 - s) / NS) & 1, kDrain, nullptr);
            }
        }
        if (warp == 1) {
            const uint32_t at = sm >> 4;  // (shared memory ends below 2^18: no carry into the leading offset)
            const uint32_t id_z = tc::idesc_bf16(kKeys), id_o = tc::idesc_bf16((uint32_t)(g.D + 15) / 16 * 16, 0, 1);
            const int steps = (g.D + 15) / 16;
            int m = -1, j = 0;   // the tile whose w v is next; items begun
            uint32_t cut = 0;    // cleared tiles of each place, modulo 2
            bool starts = false, partial = false;  // of tile m: does it begin a sum, are states of it cleared
            auto scores = [&](int m, bool first, bool last) {  // z of tile m of item j (first, last: of the item)
                const int s = m % NS, qs = j % QS;
                if (first && !warp_wait(&q_full[qs], (uint32_t)(j / QS) & 1, limit, abort)) return false;
                if (!warp_wait(&full_k[s], (uint32_t)(m / NS) & 1, limit, abort)) return false;
                tc::tc_fence_after();
                const uint32_t ak = at + (uint32_t)s * (Sh::kKV >> 4), aq = at + (uint32_t)qs * (Sh::kQ >> 4);
                if (issues) {
#pragma unroll
                    for (int p = 0; p < PS.n; ++p)
                        each_step<NP, DP>(steps, [&](int k) {
                                mma_ss(tmem, aq + desc_lower(16) + (((PS.a[p] * DB + k / 4) * kQBlock) >> 4) + (k % 4) * 2,
                                       ak + desc_lower(16) + ((Sh::kK0 + (PS.b[p] * DB + k / 4) * kKBlock) >> 4) + (k % 4) * 2, id_z, p || k);
                        });
                    tc::mma_commit(&empty_k[s]);
                    if (last) tc::mma_commit(&q_free[qs]);
                    tc::mma_commit(z_full);
                }
                __syncwarp();
                return true;
            };
            // w v of tile m and, where there is one, z of the next tile (first, last: of its item)
            auto sums = [&](bool next, bool first, bool last) {
                const int s = m % NS;
                // the next tile's z while this one's w is made, unless another item's operands are not there yet
                auto scores_next = [&] { return (Sh::kOver || warp_wait(z_read, (uint32_t)m & 1, limit, abort)) && scores(m + 1, first, last); };
                const bool early = !Sh::kOver && next &&
                                   (!first || __all_sync(0xffffffffu, tc::mbar_test_wait(&q_full[j % QS], (uint32_t)(j / QS) & 1) &&
                                                                          tc::mbar_test_wait(&full_k[(m + 1) % NS], (uint32_t)((m + 1) / NS) & 1)));
                if (early && !scores_next()) return false;
                if (!warp_wait(&w_ready[(uint32_t)m % Sh::kWs], (uint32_t)m / Sh::kWs & 1, limit, abort)) return false;
                if (!warp_wait(&full_v[s], (uint32_t)(m / NS) & 1, limit, abort)) return false;
                if (partial) {
                    if (!warp_wait(&fixed[s], cut >> s & 1, limit, abort)) return false;
                    cut ^= 1u << s;
                }
                tc::tc_fence_after();
                const uint32_t av = at + (uint32_t)s * (Sh::kKV >> 4);
                if (issues) {
#pragma unroll
                    for (int p = 0; p < PO.n; ++p)
#pragma unroll
                        for (int k = 0; k < kKeys / 16; ++k)
                            mma_ts(tmem + Sh::kColO, tmem + Sh::col_w(m, PO.a[p]) + k * 8,
                                   av + desc_lower(kKBlock) + ((Sh::kV0 + PO.b[p] * DB * kKBlock) >> 4) + k * 128, id_o, p || k || (Sh::kSums && !starts));
                    tc::mma_commit(&empty_v[s]);
                    tc::mma_commit(&o_full[(uint32_t)m % Sh::kWs]);
                }
                __syncwarp();
                return !next || early || scores_next();
            };
            bool held = false;  // tile m's products are to be issued
            auto release = [&] {
                const bool ok = !held || sums(false, false, false);
                held = false;
                return ok;
            };
            bool ok = each_item(g, ring, abort, [&](const Item &w) {
                int lo, n;
                key_tiles(g, w, lo, n);
                for (int i = 0; i < n; ++i) {
                    if (held ? !sums(true, i == 0, i == n - 1) : !scores(m + 1, true, n == 1)) return false;
                    held = true;
                    ++m;
                    if (i == n - 1) ++j;
                    starts = i % Sh::kRun == 0;
                    partial = (lo + i + 1) * kKeys > w.len;
                }
                return true;
            }, release);
            if (ok) ok = release();
            if (!ok && issues) fail();
            if (issues) tc::mma_commit(done);
            __syncwarp();
            tc::mbar_wait(done, 0, kDrain, nullptr);  // no MMA in flight when tensor memory is freed
        }
        if (warp == 2) {
            // w is 0 behind the last state, but what lies there may be anything: 0 x NaN is NaN
            int m = 0;
            const bool ok = each_item(g, ring, abort, [&](const Item &w) {
                int lo, n;
                key_tiles(g, w, lo, n);
                for (int i = 0; i < n; ++i, ++m) {
                    const int s = m % NS, rows = w.len - (lo + i) * kKeys;
                    if (!warp_wait(&full_v[s], (uint32_t)(m / NS) & 1, limit, abort)) return false;
                    if (lane == 0) tc::mbar_arrive(&empty_v[s]);  // (a wait by parity must not miss a load: this warp may be late)
                    if (rows >= kKeys) continue;
                    for (int k = 0; k < NP * DB; ++k)
                        zero_shared(sm + Sh::kV0 + s * Sh::kKV + k * kKBlock + rows * 128, kKBlock - rows * 128, lane, 32);
                    tc::fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&fixed[s]);
                }
                return true;
            });
            if (!ok && lane == 0) fail();
        }
        __syncwarp();
    } else {
        if constexpr (Sh::kCtas == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Sh::kSums ? 176 : 208));  // (of 256 x 128 in all)
        const int q = warp & 3, r = q * 32 + lane;
        const int t_in = r / g.G, head_in = r % g.G;
        const uint32_t at = tmem + ((uint32_t)(q * 32) << 16), stage = sm + Sh::kStage0 + q * kStageBytes;
        const float c = g.scale * kLog2e;
        const float2 c2 = make_float2(c, c);
        int m0 = 0;  // tiles so far
        // the products of tile m's w are done (a barrier a place of w: a wait is one phase behind at most)
        auto summed = [&](int m) {
            const bool ok = warp_wait(&o_full[(uint32_t)m % Sh::kWs], (uint32_t)m / Sh::kWs & 1, limit, abort);
            tc::tc_fence_after();
            return ok;
        };
        const bool ok = each_item(g, ring, abort, [&](const Item &w) {
            int lo, n;
            key_tiles(g, w, lo, n);
            const int t = w.tile * g.tq + t_in, head = w.kvh * g.G + head_in, len = w.len;
            const bool there = r < g.tq * g.G && t < g.T, here = there && t < w.q_len;
            const bool busy = __any_sync(0xffffffffu, here);  // a warp of no queries only keeps the count
            float2 o[Sh::kSums ? 1 : DP / 2];
            if constexpr (!Sh::kSums)
#pragma unroll
                for (int i = 0; i < DP / 2; ++i) o[i] = make_float2(0.0f, 0.0f);
            // m: what z is taken from before the exponential. For an fp32 result the largest z so far; a bf16
            // result's sum in tensor memory is scaled anew only where that has grown by more than 2^8, a factor
            // that neither w nor the sums mind
            float m = -INFINITY, l = 0.0f, alpha = 1.0f;  // w = 2^(c z - base2), base2 = c m as rounded
            float kept2 = 0.0f;  // base2 of the sums in memory
            float only = 0.0f;   // z of a single state, which is taken from itself
            const size_t row = (size_t)w.b * g.q_b + (size_t)t * g.q_t + head;
            auto kept = [&](int d) { return (float4 *)(g.sums + (w.sp * g.rows + row) * g.Dp + d); };  // four of them
            auto add_o = [&]() {  // o = o alpha + the last tile's w v
                const float2 al = make_float2(alpha, alpha);
#pragma unroll
                for (int i = 0; i < DP; i += 16) {
                    if (i < g.D) {
                        uint32_t v[16];
                        tc::tmem_ld16_async(at + Sh::kColO + i, v);
                        tc::tmem_wait_ld();
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            o[i / 2 + j] = __ffma2_rn(o[i / 2 + j], al, make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])));
                    }
                }
            };
            // the sum in tensor memory, times `by`, to the one in memory (first: it is the first), times `old`
            auto keep_sum = [&](float by, float old, bool first) {
#pragma unroll 1
                for (int i = 0; i < g.Dp; i += 8) {
                    float v[8];
                    tc::tmem_ld8(at + Sh::kColO + i, v);
                    if (here)
#pragma unroll
                        for (int j = 0; j < 8; j += 4) {
                            const float4 x = first ? make_float4(0, 0, 0, 0) : *kept(i + j);
                            *kept(i + j) = make_float4(fmaf(v[j], by, x.x * old), fmaf(v[j + 1], by, x.y * old), fmaf(v[j + 2], by, x.z * old),
                                                       fmaf(v[j + 3], by, x.w * old));
                        }
                }
            };
            auto scale_o = [&](float by) {  // the sum in tensor memory
#pragma unroll
                for (int i = 0; i < DP; i += 16) {
                    if (i < g.D) {
                        uint32_t v[16];
                        tc::tmem_ld16_async(at + Sh::kColO + i, v);
                        tc::tmem_wait_ld();
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * by);
                        tmem_st(at + Sh::kColO + i, v);
                    }
                }
                tmem_wait_st();
            };
#pragma unroll 1
            for (int i = 0; i < n; ++i) {
                const int mi = m0 + i;
                if (!warp_wait(z_full, (uint32_t)mi & 1, limit, abort)) return false;
                tc::tc_fence_after();
                const int left = len - (lo + i) * kKeys;  // states of the tile
                // so many z at a time (128 sums of an output's row leave registers for 16)
                constexpr int CZ = PP == 3 && DP == 128 ? 16 : 32, HZ = kKeys / CZ;
                auto read = [&](int h, float2 (&z)[CZ / 2]) {
                    uint32_t v[CZ / 16][16];
#pragma unroll
                    for (int j = 0; j < CZ / 16; ++j) tc::tmem_ld16_async(at + CZ * h + 16 * j, v[j]);
                    tc::tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < CZ / 2; ++j) z[j] = make_float2(__uint_as_float(v[j / 8][2 * j % 16]), __uint_as_float(v[j / 8][2 * j % 16 + 1]));
                    if (left < kKeys) {
#pragma unroll
                        for (int j = 0; j < CZ / 2; ++j) {
                            if (CZ * h + 2 * j >= left) z[j].x = -INFINITY;
                            if (CZ * h + 2 * j + 1 >= left) z[j].y = -INFINITY;
                        }
                        if (len == 1 && h == 0) {  // its weight is 1, not 2^(what rounding leaves of z's exponent)
                            only = z[0].x;
                            z[0].x -= only;
                        }
                    }
                };
                // all z of the tile stay in registers where the sums do not, and are read twice where they do
                constexpr bool kHold = Sh::kSums;
                float2 held[kHold ? HZ : 1][CZ / 2];
                auto z_done = [&]() {
                    tc::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(z_read);
                };
                float now = 1.0f, base2 = 0.0f;
                if (busy) {
                    float top = m;
                    if constexpr (kHold) {
#pragma unroll
                        for (int h = 0; h < HZ; ++h) read(h, held[h]);
                        z_done();
                    }
#pragma unroll
                    for (int h = 0; h < HZ; ++h) {
                        float2 z[CZ / 2];
                        if constexpr (kHold) {
#pragma unroll
                            for (int j = 0; j < CZ / 2; ++j) z[j] = held[h][j];
                        } else {
                            read(h, z);
                        }
                        float t4[4] = {z[0].x, z[0].y, z[1].x, z[1].y};
#pragma unroll
                        for (int j = 2; j < CZ / 2; ++j) t4[j % 4] = max3(t4[j % 4], z[j].x, z[j].y);
                        top = fmaxf(max3(top, t4[0], t4[1]), fmaxf(t4[2], t4[3]));
                    }
                    const bool keep = Sh::kSums && i > 0 && !(fmaf(top, c, -m * c) > 8.0f);
                    if (keep) top = m;
                    base2 = top == -INFINITY ? 0.0f : __fmul_rn(top, c);
                    now = m == -INFINITY ? 0.0f : keep ? 1.0f : exp2_hw(__fmul_rn(m, c) - base2);
                    m = top;
                }
                // w's place is free, and the sum so far is there, once an earlier tile's products are done
                constexpr int kBack = Sh::kWs;
                if (i >= kBack && !summed(mi - kBack)) return false;
                if (busy) {
                    if constexpr (Sh::kSums) {
                        if (i > 0 && i % Sh::kRun == 0) {
                            if (!summed(mi - 1)) return false;
                            const bool first = i == Sh::kRun;
                            keep_sum(now, first ? 0.0f : exp2_hw(kept2 - base2), first);
                            kept2 = base2;
                        } else if (__any_sync(0xffffffffu, i > 0 && now != 1.0f)) {
                            if (!summed(mi - 1)) return false;
                            scale_o(now);
                        }
                    } else if (i > 0) {
                        add_o();
                    }
                    alpha = now;
                    float2 sum[2] = {};
                    const float2 minus = make_float2(-base2, -base2);
#pragma unroll
                    for (int h = HZ - 1; h >= 0; --h) {
                        float2 z[CZ / 2];
                        if constexpr (kHold) {
#pragma unroll
                            for (int j = 0; j < CZ / 2; ++j) z[j] = held[h][j];
                        } else {
                            read(h, z);
                            if (h == 0 && !Sh::kOver) z_done();
                        }
#pragma unroll
                        for (int j = 0; j < CZ / 2; ++j) {
                            const float2 x = __ffma2_rn(z[j], c2, minus);
                            z[j] = make_float2(exp2_hw(x.x), exp2_hw(x.y));
                            sum[j % 2] = __fadd2_rn(sum[j % 2], z[j]);
                        }
#pragma unroll
                        for (int p = 0; p < PP; ++p) {
                            uint32_t wp[CZ / 2];
#pragma unroll
                            for (int j = 0; j < CZ / 2; ++j) {
                                float2 &a = z[j];
                                if (PP == 2 && p == 1) {  // (rounded, so that sums have no bias)
                                    const __nv_bfloat162 x = __floats2bfloat162_rn(a.x, a.y);
                                    wp[j] = *(const uint32_t *)&x;
                                } else {
                                    wp[j] = upper2(a.x, a.y);
                                    if (p < PP - 1) a = less_upper2(a);
                                }
                            }
                            tmem_st(at + Sh::col_w(mi, p) + CZ / 2 * h, wp);
                        }
                    }
                    sum[0] = __fadd2_rn(sum[0], sum[1]);
                    l = fmaf(l, now, sum[0].x + sum[0].y);
                    tmem_wait_st();
                } else if (!Sh::kOver) {
                    if (lane == 0) tc::mbar_arrive(z_read);
                }
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&w_ready[(uint32_t)mi % Sh::kWs]);  // (a warp may be a tile ahead of another)
            }
            m0 += n;
            if (n > 0 && !summed(m0 - 1)) return false;
            if constexpr (!Sh::kSums)
                if (n > 0 && busy) add_o();
            if (!__any_sync(0xffffffffu, there)) return true;
            const bool some = here && n > 0;
            const float by = some ? 1.0f / l : 0.0f;
            // l is against base2, not c m: an lse that left the difference out was 8e-7 off (2221 states), with it 3e-7
            if (len == 1) m = only;
            const float off = m == -INFINITY || len == 1 ? 0.0f : fmaf(m, c, -__fmul_rn(m, c));
            const bool pieces = g.D % 8 == 0;
            // CD of the outputs' columns, from d0 on
            auto put = [&](auto &v, int d0) __attribute__((always_inline)) {
                constexpr int CD = 2 * (sizeof v / sizeof v[0]);
                if (g.part) {
                    put_rows<float, CD>(stage, some ? g.part + (w.sp * g.rows + row) * g.Dp + d0 : nullptr, v, min(g.Dp - d0, CD), by, false, true);
                } else {
                    using T = typename Sh::Out;
                    put_rows<T, CD>(stage, there ? (T *)g.y + row * g.D + d0 : nullptr, v, min(g.D - d0, CD), by, !some, pieces);
                    if (PP == 3 && g.ctx) put_rows<float, CD>(stage, there ? g.ctx + row * g.D + d0 : nullptr, v, min(g.D - d0, CD), by, !some, pieces);
                }
            };
            if constexpr (Sh::kSums) {  // 64 columns at a time (all 128: 0.7 KB of spills)
#pragma unroll 1
                for (int d0 = 0; d0 < g.D; d0 += 64) {
                    float2 v[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = make_float2(0.0f, 0.0f);
                    if (n > 0 && busy) add_columns<64, 32>(at + Sh::kColO + d0, g.D - d0, v);
                    if (n > Sh::kRun && here) {
                        const float old = exp2_hw(kept2 - (m == -INFINITY ? 0.0f : __fmul_rn(m, c)));
#pragma unroll
                        for (int i = 0; i < 32; i += 2)
                            if (d0 + 2 * i < g.Dp) {
                                const float4 x = *kept(d0 + 2 * i);
                                v[i] = __ffma2_rn(make_float2(x.x, x.y), make_float2(old, old), v[i]);
                                v[i + 1] = __ffma2_rn(make_float2(x.z, x.w), make_float2(old, old), v[i + 1]);
                            }
                    }
                    put(v, d0);
                }
            } else {
                put(o, 0);
            }
            if (there) {
                if (g.part)
                    g.part_stats[w.sp * g.rows + row] = some ? make_float2(m, l * exp2f(-off)) : make_float2(-INFINITY, 0.0f);
                else if (g.lse)
                    g.lse[row] = some ? (l == INFINITY ? l : fmaf(m, g.scale, fmaf(-kLn2, off, logf(l)))) : -INFINITY;
            }
            return true;
        });
        if (!ok && lane == 0) fail();
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 0) tc::tmem_dealloc(tmem, Sh::kCols);
    if (tid == 0) items_done(g.next);
}

// The splits' outputs of each query row joined: a warp a row, a lane a split's weight, then four columns. A weight is made of
// differences of z, as those of states are: of lses, rounded by 2^-25 of them, y was 1.2e-5 off where they are 3200.
constexpr int kMostSplits = 32;
template <typename T>
__global__ void __launch_bounds__(256)
attend_join(const __grid_constant__ FwdArgs g)
{
    after_previous();
    const size_t row = (size_t)blockIdx.x * 8 + threadIdx.x / 32;
    const int lane = threadIdx.x & 31, d = lane * 4;
    if (row >= g.rows) return;
    const float2 e = lane < g.split ? g.part_stats[lane * g.rows + row] : make_float2(-INFINITY, 0.0f);
    float m = e.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const bool there = e.y != 0.0f;  // (else the split had no states, and wrote nothing)
    const float w = there ? e.y * exp2f((e.x - m) * (g.scale * kLog2e)) : 0.0f;
    const float sum = warp_sum(w);
    const unsigned have = __ballot_sync(0xffffffffu, there);
    float v[4] = {};
    constexpr int U = 4;  // reads in flight
    for (int s0 = 0; s0 < g.split; s0 += U) {
        float4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            x[u] = (have >> (s0 + u) & 1) && d < g.Dp ? *(const float4 *)(g.part + ((size_t)(s0 + u) * g.rows + row) * g.Dp + d) : make_float4(0, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float ws = __shfl_sync(0xffffffffu, w, s0 + u);
            v[0] = fmaf(ws, x[u].x, v[0]); v[1] = fmaf(ws, x[u].y, v[1]); v[2] = fmaf(ws, x[u].z, v[2]); v[3] = fmaf(ws, x[u].w, v[3]);
        }
    }
    const float by = have ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (d + j < g.D) {
            ((T *)g.y)[row * g.D + d + j] = from_f32<T>(v[j] * by);
            if (g.ctx) g.ctx[row * g.D + d + j] = v[j] * by;
        }
    if (lane == 0 && g.lse) g.lse[row] = have ? fmaf(m, g.scale, logf(sum)) : -INFINITY;
}

// ------------------------------------------------------------------ backward
// Two kernels, one for the states' gradients and one for the queries', each of which makes z and dw = dy . v again:
// 13 and 7 products of bf16 parts for bf16 inputs where one for all three gradients takes 16, but w and dz then
// go through tensor memory alone. (As one kernel dz had to be in shared memory, read with states along the
// contraction and across it: the MMAs' reads took all of shared memory's bandwidth, and the threads' stores of dq,
// and their reads and writes of w and dz, waited for it: 256 x 256 x 256 of 16 heads of 64 1080 to 1780 us.)
template <int NP>
struct BwdMaps {
    CUtensorMap q[NP], k[NP], v[NP], dy[3];
};

struct BwdArgs {
    int T, S, B, nk, G, D;
    int q_t, q_b, k_t, k_b;   // in heads, as FwdArgs'
    const int32_t *q_len, *kv_len;
    float scale;
    const float *lse, *delta;
    float *norm;              // [B][heads][T] log2 f: made with dq, read for dk and dv
    float *part_norm;         // [split][B][heads][T] f of splits
    size_t rows;              // B T heads
    float *dq, *dk, *dv;
    int tq, tiles;            // queries of a tile, tiles of queries (dq) or of states (dk, dv)
    int split, per;           // splits of the other's tiles, tiles of a split: each has sums of its own
    size_t plane;             // elements from a split's sums to the next one's
    int items;                // sentences x splits x states' heads x tiles
    int *next;                // the items' counter, 0 between launches
    int sorted;               // longer sentences first
    long long limit;
    int32_t *err;
};

// w = exp(scale z - lse) as 2^(c (z - pivot) - rest), c = scale log2 e: where w counts z is near the pivot, so that
// the rounding of the product and of c is that of a small number. (Of c z - lse log2 e it is that of lse, 12 for 2221
// states, for all of a row's w: gradients 1.5e-6 off 64 bits, 6e-7 so.) lse itself is off by half a step, 2^-25 of it, and
// with it all w of a row by one factor, 1.5e-5 where lse is 300: the kernel that makes dq sums a row's w, divides dq by
// that sum f, and leaves log2 f for the kernel that makes dk and dv, whose rest it is added to.
struct RowBase {
    float pivot, rest;
};
__device__ __forceinline__ RowBase row_base(float lse, float scale)
{
    float p = lse / scale;
    if (isinf(p)) {
        if (isinf(lse)) return {p, 0.0f};
        p = 0.0f;
    }
    return {p, fmaf(-p, scale, lse) * kLog2e};
}

// Where a row's f lies: a warp's rows are next to one another (as they lie in lse stores cost 14 us of 256 x 256 x 256).
__device__ __forceinline__ size_t norm_at(const BwdArgs &g, int b, int head, int t) { return ((size_t)b * (g.nk * g.G) + head) * g.T + t; }

// Columns of part p of the 16 fp32 numbers c of a lane (of 64 numbers) as an operand in tensor memory, made in the
// place of the numbers (64 columns and 32 more): the first two parts lie in the 16 numbers' own columns.
__host__ __device__ constexpr uint32_t part_col(int c, int p) { return p < 2 ? c * 16 + p * 8 : 64 + c * 8; }

// 16 fp32 numbers of a lane as three bf16 parts in tensor memory.
__device__ __forceinline__ void put_parts16(uint32_t at, int c, float2 (&v)[8])
{
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w[j] = upper2(v[j].x, v[j].y);
            if (p < 2) v[j] = less_upper2(v[j]);
        }
        tmem_st(at + part_col(c, p), w);
    }
}
__device__ __forceinline__ void read16(uint32_t at, float2 (&z)[8])
{
    uint32_t v[16];
    tc::tmem_ld16_async(at, v);
    tc::tmem_wait_ld();
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
}
__device__ __forceinline__ float2 pair_of(const uint32_t (&v)[2][16], int j)
{
    return make_float2(__uint_as_float(v[j / 8][2 * j % 16]), __uint_as_float(v[j / 8][2 * j % 16 + 1]));
}
// 32 columns of a lane.
__device__ __forceinline__ void read32(uint32_t at, float2 (&z)[16])
{
    uint32_t v[2][16];
    tc::tmem_ld16_async(at, v[0]);
    tc::tmem_ld16_async(at + 16, v[1]);
    tc::tmem_wait_ld();
#pragma unroll
    for (int j = 0; j < 16; ++j) z[j] = pair_of(v, j);
}
// ---- the states' gradients. For a tile of KT states and one of 64 query rows, states in the lanes of tensor memory:
//   z^T = k q^T,  (dw)^T = v dy^T  [KT][64];   dv += w^T dy,  dk += (dz)^T q  [KT][D]
template <int NP, int DP>
struct StatesShape {
    static constexpr int DB = DP / 64, TT = 64;
    static constexpr int KT = NP == 3 && DP == 128 ? 64 : 128;
    static constexpr int kStages = NP == 3 && DP == 128 ? 1 : NP == 1 && DP == 64 ? 3 : 2;  // places for query tiles
    static constexpr uint32_t kKBlock = KT * 128, kQBlock = TT * 128;
    static constexpr uint32_t kK = NP * DB * kKBlock, kQ = NP * DB * kQBlock, kDy = 3 * DB * kQBlock;
    static constexpr int kStates = NP == 1 && DP == 64 ? 2 : 1;  // places for states
    // warps that make w and dz: sixteen hide one another's latencies, where their share of dv and dk leaves registers
    static constexpr int kWarps = DP == 64 ? 16 : 8, kThreads = 128 + 32 * kWarps, kRegs = kWarps == 16 ? 104 : 224, kOther = kWarps == 16 ? 48 : 56;
    static_assert(128 * kOther + 32 * kWarps * kRegs <= kThreads * (kWarps == 16 ? 96 : 168), "registers of a CTA");
    // offsets in shared memory: k and v of each place, q, dy, the output rows' stages
    static constexpr uint32_t kQ0 = 2 * kStates * kK, kY0 = kQ0 + kStages * kQ, kStage0 = kY0 + kStages * kDy, kMain = kStage0 + kWarps * kStageBytes;
    static constexpr uint32_t kBars = (3 * kStages + 2 * kStates + 7) * 8 + 16;
    static constexpr uint32_t kSmem = 1024 + kMain + kStages * 12 * TT + kBars;
    static constexpr uint32_t kColV = 0, kColK = DP, kColZ = 2 * DP, kColW = kColZ + TT, kColD = kColW + TT + TT / 2;  // (dz over dw)
    // a warp's columns of z and dw, of dv or dk
    static constexpr int kParts = kWarps / 4, CW = TT / kParts, CD = 2 * DP / kParts;
    static_assert(kColD + TT + TT / 2 <= 512 && kSmem + sizeof(ItemRing) <= 227 * 1024, "tensor and shared memory of a CTA");
};

// start(item, nt), then tile(item, q, i, nt) for each i of the nt tiles of queries, from q - i on, that the item's
// states meet.
template <int KT, bool FETCH, typename F, typename G, typename I>
__device__ __forceinline__ bool each_tile(const BwdArgs &g, ItemRing &ring, volatile int *abort, const F &start, const G &tile, const I &idle)
{
    auto f = [&](const Item &w) {
        const int lo = w.sp * g.per, hi = w.tile * KT < w.len ? min(lo + g.per, (w.q_len + g.tq - 1) / g.tq) : 0, nt = max(0, hi - lo);
        start(w, nt);
        for (int i = 0; i < nt; ++i)
            if (!tile(w, lo + i, i, nt)) return false;
        return true;
    };
    if constexpr (FETCH)
        return fetch_items(g, ring, abort, f);
    else
        return each_item(g, ring, abort, f, idle);
}
template <int KT, bool FETCH, typename F, typename G>
__device__ __forceinline__ bool each_tile(const BwdArgs &g, ItemRing &ring, volatile int *abort, const F &start, const G &tile)
{
    return each_tile<KT, FETCH>(g, ring, abort, start, tile, [] { return true; });
}

// One CTA an SM takes items one after the other. Warp 0 loads (TMA), warp 1 issues the MMAs, warps 2 and 3 clear what lies
// behind a sentence's last query and fetch the rows' statistics, the others make w and dz of a tile (a thread
// has a state's row and a quarter or half of the queries; heads of 64: eight warps filled 31 % of the issue slots and
// took 480 us where sixteen take 410) and add up dv (the first half of them) and dk of the tile before. Tile n's MMAs are
// issued as dv(n), z(n + 1), dk(n), dw(n + 1): w(n + 1) is made while dk(n) and dw(n + 1) run.
// Bound by the chain z, w, dv, dw, dz, dk of a tile: 64 x 256 x 256, 16 heads of 64, bf16, 146 us, 765 TFLOP/s in 13
// products of parts (tensor pipe 34 %, issue 53 %).
template <int NP, int DP>
__global__ void __launch_bounds__(StatesShape<NP, DP>::kThreads, 1)
attend_grad_states(const __grid_constant__ BwdMaps<NP> tm, const __grid_constant__ BwdArgs g)
{
    using Sh = StatesShape<NP, DP>;
    constexpr int DB = Sh::DB, NS = Sh::kStages, KS = Sh::kStates, TT = Sh::TT, KT = Sh::KT;
    constexpr Products<NP, NP> PZ;   // k q
    constexpr Products<NP, 3> PD;    // v dy
    constexpr Products<3, 3> PV;     // w dy
    constexpr Products<3, NP> PK;    // dz q
    __shared__ ItemRing ring;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t sm = smem_u32(base);
    float *st_pivot = (float *)(base + Sh::kMain), *st_rest = st_pivot + NS * TT, *st_delta = st_rest + NS * TT;
    uint64_t *q_full = (uint64_t *)(st_delta + NS * TT), *q_ready = q_full + NS, *q_free = q_ready + NS, *kv_full = q_free + NS,
             *kv_free = kv_full + KS, *z_full = kv_free + KS, *d_full = z_full + 1, *w_ready = d_full + 1, *z_ready = w_ready + 1,
             *v_full = z_ready + 1, *k_full = v_full + 1, *done = k_full + 1;
    uint32_t *tmem_slot = (uint32_t *)(done + 1);
    volatile int *abort = (volatile int *)(tmem_slot + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (uint64_t *bar = q_full; bar <= done; ++bar)
            tc::mbar_init(bar, bar >= q_ready && bar < q_free ? 2 : bar == w_ready || bar == z_ready ? Sh::kWarps : 1);
        init_items(ring, Sh::kWarps + 3);
        *abort = 0;
        tc::fence_mbar_init();
    }
    // rows that no copy writes (a group of heads that does not divide the tile) stay 0
    if (g.tq * g.G < TT) zero_shared(sm + Sh::kQ0, NS * (Sh::kQ + Sh::kDy), tid, Sh::kThreads);
    tc::fence_proxy_async();
    if (warp == 0) tc::tmem_alloc(tmem_slot, 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    after_previous();
    if (g.sorted) sort_sentences(g, ring, g.q_len, (int *)(base + Sh::kStage0));

    const long long limit = g.limit;
    auto fail = [&]() {
        *abort = 1;
        atomicCAS(g.err, 0, (int)SL_ERR_TIMEOUT);
    };
    auto no_start = [](const Item &, int) {};

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Sh::kOther));
        const bool issues = elect_one();
        if (warp == 0) {
            int n = 0, nj = 0;
            const bool ok = each_tile<KT, true>(g, ring, abort, no_start, [&](const Item &w, int qt, int i, int nt) {
                if (i == 0) {
                    const int s = nj % KS;
                    if (!warp_wait(&kv_free[s], (uint32_t)(nj / KS + 1) & 1, limit, abort)) return false;
                    ++nj;
                    if (issues) {
                        tc::mbar_arrive_expect_tx(&kv_full[s], 2 * Sh::kK);
#pragma unroll
                        for (int p = 0; p < NP; ++p)
                            for (int d = 0; d < DB; ++d) {
                                const uint32_t to = sm + s * 2 * Sh::kK + (p * DB + d) * Sh::kKBlock;
                                tma_load_4d(to, &tm.k[p], d * 64, w.kvh, w.b, w.tile * KT, &kv_full[s]);
                                tma_load_4d(to + Sh::kK, &tm.v[p], d * 64, w.kvh, w.b, w.tile * KT, &kv_full[s]);
                            }
                    }
                }
                const int s = n % NS;
                if (!warp_wait(&q_free[s], (uint32_t)(n / NS + 1) & 1, limit, abort)) return false;
                ++n;
                if (issues) {
                    tc::mbar_arrive_expect_tx(&q_full[s], (NP + 3) * DB * (uint32_t)(g.tq * g.G) * 128u);
#pragma unroll
                    for (int p = 0; p < NP; ++p)
                        for (int d = 0; d < DB; ++d)
                            tma_load_5d(sm + Sh::kQ0 + s * Sh::kQ + (p * DB + d) * Sh::kQBlock, &tm.q[p], d * 64, 0, w.kvh, w.b, qt * g.tq, &q_full[s]);
#pragma unroll
                    for (int p = 0; p < 3; ++p)
                        for (int d = 0; d < DB; ++d)
                            tma_load_5d(sm + Sh::kY0 + s * Sh::kDy + (p * DB + d) * Sh::kQBlock, &tm.dy[p], d * 64, 0, w.kvh, w.b, qt * g.tq, &q_full[s]);
                }
                return true;
            });
            if (!ok && issues) fail();
            // no copy in flight when the CTA ends: the last load of every place has landed
            for (int s = 0; s < KS; ++s)
                if (nj > s) tc::mbar_wait(&kv_full[s], (uint32_t)((nj - 1 - s) / KS) & 1, kDrain, nullptr);
            for (int s = 0; s < NS; ++s)
                if (n > s) tc::mbar_wait(&q_full[s], (uint32_t)((n - 1 - s) / NS) & 1, kDrain, nullptr);
        }
        if (warp == 1) {
            constexpr uint32_t kRowsLo = desc_lower(16), kQueriesLo = desc_lower(Sh::kQBlock);
            const uint32_t at = sm >> 4;  // (everything lies at a constant distance from it)
            const int steps = (g.D + 15) / 16;
            const uint32_t id_z = tc::idesc_bf16(TT), id_g = tc::idesc_bf16((uint32_t)steps * 16, 0, 1);
            int n = -1, nj = 0;  // the tile whose gradients are next; items whose states are in use or were
            auto scores = [&](int m, int kv, bool first) {  // z of tile m, states kv
                const int s = m % NS;
                if (first && !warp_wait(&kv_full[kv % KS], (uint32_t)(kv / KS) & 1, limit, abort)) return false;
                if (!warp_wait(&q_ready[s], (uint32_t)(m / NS) & 1, limit, abort)) return false;
                tc::tc_fence_after();
                if (issues) {
                    const uint32_t aq = at + (uint32_t)s * (Sh::kQ >> 4), ak = at + (uint32_t)(kv % KS) * (2 * Sh::kK >> 4);
#pragma unroll
                    for (int p = 0; p < PZ.n; ++p)
                        each_step<NP, DP>(steps, [&](int k) {
                                mma_ss(tmem + Sh::kColZ, ak + kRowsLo + (((PZ.a[p] * DB + k / 4) * Sh::kKBlock) >> 4) + (k % 4) * 2,
                                       aq + kRowsLo + ((Sh::kQ0 + (PZ.b[p] * DB + k / 4) * Sh::kQBlock) >> 4) + (k % 4) * 2, id_z, p || k);
                        });
                    tc::mma_commit(z_full);
                }
                __syncwarp();
                return true;
            };
            auto scores2 = [&](int m, int kv, bool last) {  // dw of tile m, the last of its item?
                if (issues) {
                    const uint32_t ay = at + (uint32_t)(m % NS) * (Sh::kDy >> 4), ak = at + (uint32_t)(kv % KS) * (2 * Sh::kK >> 4);
#pragma unroll
                    for (int p = 0; p < PD.n; ++p)
                        each_step<NP, DP>(steps, [&](int k) {
                                mma_ss(tmem + Sh::kColD, ak + kRowsLo + ((Sh::kK + (PD.a[p] * DB + k / 4) * Sh::kKBlock) >> 4) + (k % 4) * 2,
                                       ay + kRowsLo + ((Sh::kY0 + (PD.b[p] * DB + k / 4) * Sh::kQBlock) >> 4) + (k % 4) * 2, id_z, p || k);
                        });
                    tc::mma_commit(d_full);
                    if (last) tc::mma_commit(&kv_free[kv % KS]);  // (the gradients' products do not read the states)
                }
                __syncwarp();
                return true;
            };
            // The gradients of tile n and, where there is one, the next tile's scores (first, last: of its item).
            auto gradients = [&](bool next, bool first, bool last) {
                const int s = n % NS;
                const uint32_t aq = at + (uint32_t)s * (Sh::kQ >> 4), ay = at + (uint32_t)s * (Sh::kDy >> 4);
                if (!warp_wait(w_ready, (uint32_t)n & 1, limit, abort)) return false;
                tc::tc_fence_after();
                if (issues) {
#pragma unroll
                    for (int p = 0; p < PV.n; ++p)
#pragma unroll
                        for (int k = 0; k < TT / 16; ++k)
                            mma_ts(tmem + Sh::kColV, tmem + Sh::kColW + part_col(k, PV.a[p]),
                                   ay + kQueriesLo + ((Sh::kY0 + PV.b[p] * DB * Sh::kQBlock) >> 4) + k * 128, id_g, p || k);
                    tc::mma_commit(v_full);
                }
                __syncwarp();
                const int kv = first ? nj : nj - 1;
                if (NS > 1 && next && !scores(n + 1, kv, first)) return false;
                if (!warp_wait(z_ready, (uint32_t)n & 1, limit, abort)) return false;
                tc::tc_fence_after();
                if (issues) {
#pragma unroll
                    for (int p = 0; p < PK.n; ++p)
#pragma unroll
                        for (int k = 0; k < TT / 16; ++k)
                            mma_ts(tmem + Sh::kColK, tmem + Sh::kColD + part_col(k, PK.a[p]),
                                   aq + kQueriesLo + ((Sh::kQ0 + PK.b[p] * DB * Sh::kQBlock) >> 4) + k * 128, id_g, p || k);
                    tc::mma_commit(&q_free[s]);
                    tc::mma_commit(k_full);
                }
                __syncwarp();
                if (!next) return true;
                return (NS > 1 || scores(n + 1, kv, first)) && scores2(n + 1, kv, last);
            };
            bool held = false;  // tile n's products are to be issued
            auto release = [&] {
                const bool ok = !held || gradients(false, false, false);
                held = false;
                return ok;
            };
            bool ok = each_tile<KT, false>(g, ring, abort, no_start, [&](const Item &w, int qt, int i, int nt) {
                const bool last = i == nt - 1;
                if (held ? !gradients(true, i == 0, last) : !(scores(n + 1, nj, true) && scores2(n + 1, nj, last))) return false;
                held = true;
                ++n;
                if (i == 0) ++nj;
                return true;
            }, release);
            if (ok) ok = release();
            if (!ok && issues) fail();
            if (issues) tc::mma_commit(done);
            __syncwarp();
            tc::mbar_wait(done, 0, kDrain, nullptr);  // no MMA in flight when tensor memory is freed
        }
        if (warp >= 2) {
            // what lies behind a sentence's last query may be anything: it is cleared before the products that
            // sum over it; and the rows' statistics
            const int part = warp - 2, r = part * 32 + lane;
            int n = 0;
            const bool ok = each_tile<KT, false>(g, ring, abort, no_start, [&](const Item &w, int qt, int i, int nt) {
                const int s = n % NS, t0 = qt * g.tq, t = t0 + r / g.G;
                RowBase from = {INFINITY, 0.0f};  // (w of no query: exp(-inf))
                float delta = 0.0f;
                if (r < g.tq * g.G && t < w.q_len) {
                    const size_t row = (size_t)w.b * g.q_b + (size_t)t * g.q_t + w.kvh * g.G + r % g.G;
                    from = row_base(g.lse[row], g.scale);
                    from.rest += g.norm[norm_at(g, w.b, w.kvh * g.G + r % g.G, t)];
                    delta = g.delta[row];
                }
                // (the place's statistics of NS tiles ago were read before its gradients were made)
                if (!warp_wait(&q_full[s], (uint32_t)(n / NS) & 1, limit, abort)) return false;
                st_pivot[s * TT + r] = from.pivot;
                st_rest[s * TT + r] = from.rest;
                st_delta[s * TT + r] = delta;
                const int rows = (w.q_len - t0) * g.G;  // with a query
                if (rows < g.tq * g.G) {
                    for (int k = part; k < NP * DB; k += 2)
                        zero_shared(sm + Sh::kQ0 + s * Sh::kQ + k * Sh::kQBlock + rows * 128, Sh::kQBlock - rows * 128, lane, 32);
                    for (int k = part; k < 3 * DB; k += 2)
                        zero_shared(sm + Sh::kY0 + s * Sh::kDy + k * Sh::kQBlock + rows * 128, Sh::kQBlock - rows * 128, lane, 32);
                    tc::fence_proxy_async();
                }
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&q_ready[s]);
                ++n;
                return true;
            });
            if (!ok && lane == 0) fail();
        }
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Sh::kRegs));
        const int q = warp & 3, part = (warp - 4) >> 2, s = q * 32 + lane;  // a state's row; some of the queries' columns
        const bool is_k = part >= Sh::kParts / 2;   // of dk (dv), columns d0 ..
        const int d0 = part % (Sh::kParts / 2) * Sh::CD;
        const uint32_t at = tmem + ((uint32_t)(q * 32) << 16), stage = sm + Sh::kStage0 + (warp - 4) * kStageBytes;
        const float c = g.scale * kLog2e;
        float *const mine = is_k ? g.dk : g.dv;
        const bool puts = mine && d0 < g.D;
        const int width = min(g.D - d0, Sh::CD);
        constexpr int CW = Sh::CW, CD = Sh::CD;
        constexpr bool kLate = Sh::kWarps == 16;  // rows go to memory while the next tile's products run (128 sums a thread: registers spill so)
        float2 acc[CD / 2];
#pragma unroll
        for (int i = 0; i < CD / 2; ++i) acc[i] = make_float2(0.0f, 0.0f);
        int n = 0;
        struct {
            float *out;   // the row's columns in memory (null: nowhere)
            bool dead, last;
        } past = {};  // the tile before: its gradients are still in tensor memory
        // (inlined at each call: a function would have the sums in local memory)
        auto take = [&]() __attribute__((always_inline)) { add_columns<CD, (DP == 64 ? 32 : 16)>(at + (is_k ? Sh::kColK : Sh::kColV) + d0, width, acc); };
        auto put = [&]() __attribute__((always_inline)) {  // an item's rows to memory
            if (puts) put_rows<float, CD>(stage, past.out, acc, width, is_k ? g.scale : 1.0f, past.dead, g.D % 8 == 0);
#pragma unroll
            for (int i = 0; i < CD / 2; ++i) acc[i] = make_float2(0.0f, 0.0f);
        };
        auto row_out = [&](const Item &w) -> float * {
            const int row = w.tile * KT + s;
            return s < KT && row < g.S ? mine + w.sp * g.plane + ((size_t)w.b * g.k_b + (size_t)row * g.k_t + w.kvh) * g.D + d0 : nullptr;
        };
        auto clear = [&](const Item &w, int nt) {  // states without queries, and behind the sentence's end: 0
            // (of several splits the sum knows which have none)
            if (nt == 0 && g.split == 1 && puts) put_rows<float, CD>(stage, row_out(w), acc, width, 0.0f, true, g.D % 8 == 0);
        };
        auto arrive = [&](uint64_t *bar) {
            tmem_wait_st();
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(bar);
        };
        bool ok;
        if (q * 32 >= KT) {  // a warp of no states (tiles of 64) only keeps the count
            ok = each_tile<KT, false>(g, ring, abort, clear, [&](const Item &, int, int, int) {
                for (int i = 0; i < 2; ++i) {
                    if (!warp_wait(i ? d_full : z_full, (uint32_t)n & 1, limit, abort)) return false;
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(i ? z_ready : w_ready);
                }
                ++n;
                return true;
            });
            n = 0;  // (nothing to take)
        } else {
            ok = each_tile<KT, false>(g, ring, abort, clear, [&](const Item &w, int qt, int i, int nt) {
                const bool live = w.tile * KT + s < w.len;
                const bool some_dead = __any_sync(0xffffffffu, !live);
                const float *pivot = st_pivot + n % NS * TT + part * CW, *rest = st_rest + n % NS * TT + part * CW, *delta = st_delta + n % NS * TT + part * CW;
                float2 wv[CW / 16][8];
                if (!warp_wait(z_full, (uint32_t)n & 1, limit, abort)) return false;
                tc::tc_fence_after();
                if (!warp_wait(&q_ready[n % NS], (uint32_t)(n / NS) & 1, limit, abort)) return false;  // (the statistics)
#pragma unroll
                for (int h = 0; h < CW / 16; ++h) {
                    read16(at + Sh::kColZ + part * CW + 16 * h, wv[h]);
#pragma unroll
                    for (int k = 0; k < 8; k += 2) {
                        const float4 pv = *(const float4 *)(pivot + 16 * h + 2 * k), re = *(const float4 *)(rest + 16 * h + 2 * k);
                        const float2 x = __ffma2_rn(__fadd2_rn(wv[h][k], make_float2(-pv.x, -pv.y)), make_float2(c, c), make_float2(-re.x, -re.y));
                        const float2 y = __ffma2_rn(__fadd2_rn(wv[h][k + 1], make_float2(-pv.z, -pv.w)), make_float2(c, c), make_float2(-re.z, -re.w));
                        wv[h][k] = make_float2(exp2_hw(x.x), exp2_hw(x.y));
                        wv[h][k + 1] = make_float2(exp2_hw(y.x), exp2_hw(y.y));
                    }
                    if (some_dead)
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (!live) wv[h][k] = make_float2(0.0f, 0.0f);
                    // (one state has weight 1, whatever z is: not what rounding leaves of it. 0 stays 0, a NaN one)
                    if (w.len == 1)
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            if (wv[h][k].x > 0.0f) wv[h][k].x = 1.0f;
                            if (wv[h][k].y > 0.0f) wv[h][k].y = 1.0f;
                        }
                }
                if (n > 0) {  // w's place is free; the last tile's dv (dk) is there, which the next one's takes the place of
                    if (!warp_wait(v_full, (uint32_t)(n - 1) & 1, limit, abort)) return false;
                    if (is_k && !warp_wait(k_full, (uint32_t)(n - 1) & 1, limit, abort)) return false;
                    tc::tc_fence_after();
                    take();
                    if (!kLate && past.last) put();
                }
#pragma unroll
                for (int h = 0; h < CW / 16; ++h) {
                    float2 w[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) w[k] = wv[h][k];
                    put_parts16(at + Sh::kColW, part * (CW / 16) + h, w);
                }
                arrive(w_ready);
                if (!warp_wait(d_full, (uint32_t)n & 1, limit, abort)) return false;
                tc::tc_fence_after();
#pragma unroll
                for (int h = 0; h < CW / 16; ++h) {
                    float2 dz[8];
                    read16(at + Sh::kColD + part * CW + 16 * h, dz);
#pragma unroll
                    for (int k = 0; k < 8; k += 2) {
                        const float4 de = *(const float4 *)(delta + 16 * h + 2 * k);
                        dz[k] = __fmul2_rn(wv[h][k], __fadd2_rn(dz[k], make_float2(-de.x, -de.y)));
                        dz[k + 1] = __fmul2_rn(wv[h][k + 1], __fadd2_rn(dz[k + 1], make_float2(-de.z, -de.w)));
                    }
                    // (one state has weight 1 whatever z is: dz is 0, not what rounding leaves of it)
                    if (some_dead || w.len == 1)
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (!live || w.len == 1) dz[k] = make_float2(0.0f, 0.0f);
                    put_parts16(at + Sh::kColD, part * (CW / 16) + h, dz);
                }
                arrive(z_ready);
                if (kLate && past.last) put();
                past.last = i == nt - 1;
                if (past.last) {
                    past.out = mine ? row_out(w) : nullptr;
                    past.dead = !live;  // (no state: w and dz are 0, but 0 x NaN is NaN)
                }
                ++n;
                return true;
            });
        }
        if (ok && n > 0) {
            ok = warp_wait(is_k ? k_full : v_full, (uint32_t)(n - 1) & 1, limit, abort);
            tc::tc_fence_after();
            if (ok) {
                take();
                put();
            }
        }
        if (!ok && lane == 0) fail();
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 0) tc::tmem_dealloc(tmem, 512);
    if (tid == 0) items_done(g.next);
}

// ---- the queries' gradients. For a tile of RT query rows and one of 64 states, queries in the lanes:
//   z = q k^T,  dw = dy v^T  [RT][64];   dq += dz k  [RT][D]
template <int NP, int DP>
struct QueriesShape {
    static constexpr int DB = DP / 64;
    static constexpr int RT = NP == 3 && DP == 128 ? 64 : 128;
    static constexpr int kCtas = NP == 1 && DP == 64 ? 2 : 1;  // an SM
    static constexpr int kStages = NP == 3 && DP == 128 ? 1 : 2;
    static constexpr uint32_t kQBlock = RT * 128;
    static constexpr uint32_t kQ = NP * DB * kQBlock, kDy = 3 * DB * kQBlock, kK = NP * DB * kKBlock;
    static constexpr uint32_t kY0 = kQ, kK0 = kY0 + kDy, kV0 = kK0 + kStages * kK, kStage0 = kV0 + kStages * kK, kMain = kStage0 + 4 * kStageBytes;
    static constexpr uint32_t kBars = (5 * kStages + 8) * 8 + 16;
    static constexpr uint32_t kSmem = 1024 + kMain + kBars;
    static constexpr uint32_t kColZ = 0, kColD = kKeys, kColQ = kColD + kKeys + kKeys / 2;  // (dz over dw)
    static constexpr uint32_t kCols = kColQ + DP <= 256 ? 256 : 512;
    static_assert(kSmem + sizeof(ItemRing) <= (kCtas == 2 ? 113 : 227) * 1024 && (kCtas == 1 || kCols == 256), "tensor and shared memory of a CTA");
};

// CTAs take items one after the other: a tile of query rows of one sentence and state's head. Warp 0 loads (TMA), warp 1 issues
// the MMAs, warp 2 clears what lies behind a sentence's last state, and a thread of warps 4 to 7 has a query. Tile
// m's MMAs are issued as z(m + 1), dq(m), dw(m + 1).
// Bound by the chain z, w, dw, dz of a tile, as above: 64 x 256 x 256, 16 heads of 64, bf16, 89 us, 680 TFLOP/s in 7
// products of parts (tensor pipe 31 %, issue 36 %; two CTAs an SM).
template <int NP, int DP>
__global__ void __launch_bounds__(256, QueriesShape<NP, DP>::kCtas)
attend_grad_queries(const __grid_constant__ BwdMaps<NP> tm, const __grid_constant__ BwdArgs g)
{
    using Sh = QueriesShape<NP, DP>;
    constexpr int DB = Sh::DB, NS = Sh::kStages;
    constexpr Products<NP, NP> PZ;   // q k
    constexpr Products<3, NP> PD;    // dy v, dz k
    __shared__ ItemRing ring;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t sm = smem_u32(base);
    uint64_t *full_k = (uint64_t *)(base + Sh::kMain), *full_v = full_k + NS, *empty_k = full_v + NS, *empty_v = empty_k + NS,
             *fixed = empty_v + NS, *q_full = fixed + NS, *q_free = q_full + 1, *z_full = q_free + 1, *d_full = z_full + 1,
             *g_full = d_full + 1, *z_read = g_full + 1, *z_ready = z_read + 1, *done = z_ready + 1;
    uint32_t *tmem_slot = (uint32_t *)(done + 1);
    volatile int *abort = (volatile int *)(tmem_slot + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        // (empty_k: the MMAs and warp 2, as empty_v of the forward)
        for (uint64_t *bar = full_k; bar <= done; ++bar) tc::mbar_init(bar, bar == z_read || bar == z_ready ? 4 : bar >= empty_k && bar < empty_v ? 2 : 1);
        init_items(ring, 6);
        *abort = 0;
        tc::fence_mbar_init();
    }
    if (warp == 0) tc::tmem_alloc(tmem_slot, Sh::kCols);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    after_previous();
    if (g.sorted) sort_sentences(g, ring, g.kv_len, (int *)(base + Sh::kStage0));

    const long long limit = g.limit;
    auto fail = [&]() {
        *abort = 1;
        atomicCAS(g.err, 0, (int)SL_ERR_TIMEOUT);
    };
    // tiles of states: from lo on
    auto tiles = [&](const Item &w, int &lo) {
        lo = w.sp * g.per;
        return w.tile * g.tq < w.q_len ? max(0, min(g.per, (w.len + kKeys - 1) / kKeys - lo)) : 0;
    };

    if (warp < 4) {
        if constexpr (Sh::kCtas == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        const bool issues = elect_one();
        if (warp == 0) {
            int m = 0, nv = 0, j = 0;  // loads of k, of v, of queries
            const bool ok = fetch_items(g, ring, abort, [&](const Item &w) {
                int lo;
                const int n = tiles(w, lo);
                if (n == 0) return true;
                if (!warp_wait(q_free, (uint32_t)(j + 1) & 1, limit, abort)) return false;
                if (issues) {
                    tc::mbar_arrive_expect_tx(q_full, (NP + 3) * DB * (uint32_t)(g.tq * g.G) * 128u);
#pragma unroll
                    for (int p = 0; p < NP; ++p)
                        for (int d = 0; d < DB; ++d) tma_load_5d(sm + (p * DB + d) * Sh::kQBlock, &tm.q[p], d * 64, 0, w.kvh, w.b, w.tile * g.tq, q_full);
#pragma unroll
                    for (int p = 0; p < 3; ++p)
                        for (int d = 0; d < DB; ++d)
                            tma_load_5d(sm + Sh::kY0 + (p * DB + d) * Sh::kQBlock, &tm.dy[p], d * 64, 0, w.kvh, w.b, w.tile * g.tq, q_full);
                }
                ++j;
                for (int i = 0; i < n; ++i) {
                    const int s = m % NS;
                    const uint32_t ph = (uint32_t)(m / NS + 1) & 1;
                    if (!warp_wait(&empty_k[s], ph, limit, abort)) return false;
                    ++m;
                    if (issues) {
                        tc::mbar_arrive_expect_tx(&full_k[s], Sh::kK);
#pragma unroll
                        for (int p = 0; p < NP; ++p)
                            for (int d = 0; d < DB; ++d)
                                tma_load_4d(sm + Sh::kK0 + s * Sh::kK + (p * DB + d) * kKBlock, &tm.k[p], d * 64, w.kvh, w.b, (lo + i) * kKeys, &full_k[s]);
                    }
                    if (!warp_wait(&empty_v[s], ph, limit, abort)) return false;
                    ++nv;
                    if (issues) {
                        tc::mbar_arrive_expect_tx(&full_v[s], Sh::kK);
#pragma unroll
                        for (int p = 0; p < NP; ++p)
                            for (int d = 0; d < DB; ++d)
                                tma_load_4d(sm + Sh::kV0 + s * Sh::kK + (p * DB + d) * kKBlock, &tm.v[p], d * 64, w.kvh, w.b, (lo + i) * kKeys, &full_v[s]);
                    }
                }
                return true;
            });
            if (!ok && issues) fail();
            // no copy in flight when the CTA ends: the last load of every place has landed
            if (j) tc::mbar_wait(q_full, (uint32_t)(j - 1) & 1, kDrain, nullptr);
            for (int s = 0; s < NS; ++s) {
                if (m > s) tc::mbar_wait(&full_k[s], (uint32_t)((m - 1 - s) / NS) & 1, kDrain, nullptr);
                if (nv > s) tc::mbar_wait(&full_v[s], (uint32_t)((nv - 1 - s) / NS) & 1, kDrain, nullptr);
            }
        }
        if (warp == 1) {
            constexpr uint32_t kRowsLo = desc_lower(16), kStatesLo = desc_lower(kKBlock);
            const uint32_t at = sm >> 4;
            const int steps = (g.D + 15) / 16;
            const uint32_t id_z = tc::idesc_bf16(kKeys), id_q = tc::idesc_bf16((uint32_t)steps * 16, 0, 1);
            int m = -1, j = 0;     // the tile whose dq is next; items begun
            uint32_t cut = 0;      // cleared tiles of each place, modulo 2
            bool partial = false;  // of tile m: are states of it cleared
            auto scores = [&](int m, bool first) {  // z of tile m
                const int s = m % NS;
                if (first && !warp_wait(q_full, (uint32_t)j & 1, limit, abort)) return false;
                if (!warp_wait(&full_k[s], (uint32_t)(m / NS) & 1, limit, abort)) return false;
                tc::tc_fence_after();
                if (issues) {
                    const uint32_t ak = at + (uint32_t)s * (Sh::kK >> 4);
#pragma unroll
                    for (int p = 0; p < PZ.n; ++p)
                        each_step<NP, DP>(steps, [&](int k) {
                                mma_ss(tmem + Sh::kColZ, at + kRowsLo + (((PZ.a[p] * DB + k / 4) * Sh::kQBlock) >> 4) + (k % 4) * 2,
                                       ak + kRowsLo + ((Sh::kK0 + (PZ.b[p] * DB + k / 4) * kKBlock) >> 4) + (k % 4) * 2, id_z, p || k);
                        });
                    tc::mma_commit(z_full);
                }
                __syncwarp();
                return true;
            };
            auto scores2 = [&](int m, bool last) {  // dw of tile m, the last of its item?
                const int s = m % NS;
                if (!warp_wait(&full_v[s], (uint32_t)(m / NS) & 1, limit, abort)) return false;
                tc::tc_fence_after();
                if (issues) {
                    const uint32_t av = at + (uint32_t)s * (Sh::kK >> 4);
#pragma unroll
                    for (int p = 0; p < PD.n; ++p)
                        each_step<NP, DP>(steps, [&](int k) {
                                mma_ss(tmem + Sh::kColD, at + kRowsLo + ((Sh::kY0 + (PD.a[p] * DB + k / 4) * Sh::kQBlock) >> 4) + (k % 4) * 2,
                                       av + kRowsLo + ((Sh::kV0 + (PD.b[p] * DB + k / 4) * kKBlock) >> 4) + (k % 4) * 2, id_z, p || k);
                        });
                    tc::mma_commit(&empty_v[s]);
                    if (last) tc::mma_commit(q_free);  // (dq's products read neither q nor dy)
                    tc::mma_commit(d_full);
                }
                __syncwarp();
                return true;
            };
            // dq of tile m and, where there is one, the next tile's scores (first, last: of its item); those of the
            // same item's z while this tile's dz is made
            auto sums = [&](bool next, bool first, bool last) {
                const int s = m % NS;
                const bool early = NS > 1 && next && !first;
                if (early && !(warp_wait(z_read, (uint32_t)m & 1, limit, abort) && scores(m + 1, false))) return false;
                if (!warp_wait(z_ready, (uint32_t)m & 1, limit, abort)) return false;
                if (partial) {
                    if (!warp_wait(&fixed[s], cut >> s & 1, limit, abort)) return false;
                    cut ^= 1u << s;
                }
                tc::tc_fence_after();
                if (issues) {
                    const uint32_t ak = at + (uint32_t)s * (Sh::kK >> 4);
#pragma unroll
                    for (int p = 0; p < PD.n; ++p)
#pragma unroll
                        for (int k = 0; k < kKeys / 16; ++k)
                            mma_ts(tmem + Sh::kColQ, tmem + Sh::kColD + part_col(k, PD.a[p]),
                                   ak + kStatesLo + ((Sh::kK0 + PD.b[p] * DB * kKBlock) >> 4) + k * 128, id_q, p || k);
                    tc::mma_commit(&empty_k[s]);
                    tc::mma_commit(g_full);
                }
                __syncwarp();
                return !next || ((early || scores(m + 1, first)) && scores2(m + 1, last));
            };
            bool held = false;  // tile m's products are to be issued
            auto release = [&] {
                const bool ok = !held || sums(false, false, false);
                held = false;
                return ok;
            };
            bool ok = each_item(g, ring, abort, [&](const Item &w) {
                int lo;
                const int n = tiles(w, lo);
                for (int i = 0; i < n; ++i) {
                    if (held ? !sums(true, i == 0, i == n - 1) : !(scores(m + 1, true) && scores2(m + 1, n == 1))) return false;
                    held = true;
                    ++m;
                    if (i == 0) ++j;
                    partial = (lo + i + 1) * kKeys > w.len;
                }
                return true;
            }, release);
            if (ok) ok = release();
            if (!ok && issues) fail();
            if (issues) tc::mma_commit(done);
            __syncwarp();
            tc::mbar_wait(done, 0, kDrain, nullptr);  // no MMA in flight when tensor memory is freed
        }
        if (warp == 2) {
            // dz is 0 behind the last state, but what lies there may be anything: 0 x NaN is NaN. (z of the tile may
            // be made of what is there or of zeros: those columns are not used.)
            int m = 0;
            const bool ok = each_item(g, ring, abort, [&](const Item &w) {
                int lo;
                const int n = tiles(w, lo);
                for (int i = 0; i < n; ++i, ++m) {
                    const int s = m % NS, rows = w.len - (lo + i) * kKeys;
                    if (!warp_wait(&full_k[s], (uint32_t)(m / NS) & 1, limit, abort)) return false;
                    if (lane == 0) tc::mbar_arrive(&empty_k[s]);
                    if (rows >= kKeys) continue;
                    for (int k = 0; k < NP * DB; ++k)
                        zero_shared(sm + Sh::kK0 + s * Sh::kK + k * kKBlock + rows * 128, kKBlock - rows * 128, lane, 32);
                    tc::fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&fixed[s]);
                }
                return true;
            });
            if (!ok && lane == 0) fail();
        }
        __syncwarp();
    } else {
        if constexpr (Sh::kCtas == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
        const int q = warp & 3, r = q * 32 + lane;
        const int t_in = r / g.G, head_in = r % g.G;
        const uint32_t at = tmem + ((uint32_t)(q * 32) << 16), stage = sm + Sh::kStage0 + q * kStageBytes;
        const float c = g.scale * kLog2e;
        int m0 = 0;  // tiles so far
        auto arrive = [&](uint64_t *bar) {
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(bar);
        };
        const bool ok = each_item(g, ring, abort, [&](const Item &w) {
            int lo;
            const int n = tiles(w, lo), len = w.len;
            const int t = w.tile * g.tq + t_in, head = w.kvh * g.G + head_in;
            const bool there = r < g.tq * g.G && t < g.T, here = there && t < w.q_len;
            const bool busy = __any_sync(0xffffffffu, here);  // a warp of no queries only keeps the count
            const size_t row = (size_t)w.b * g.q_b + (size_t)t * g.q_t + head;
            const RowBase from = here ? row_base(g.lse[row], g.scale) : RowBase{0.0f, 0.0f};
            const float2 pivot = make_float2(-from.pivot, -from.pivot), rest = make_float2(-from.rest, -from.rest);
            const float delta = here ? g.delta[row] : 0.0f;
            float2 acc[DP / 2], f2 = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < DP / 2; ++i) acc[i] = make_float2(0.0f, 0.0f);
#pragma unroll 1
            for (int i = 0; i < n; ++i) {
                const int m = m0 + i, left = len - (lo + i) * kKeys;  // states of the tile
                float2 wv[2][16];
                if (!warp_wait(z_full, (uint32_t)m & 1, limit, abort)) return false;
                tc::tc_fence_after();
                if (busy) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        read32(at + Sh::kColZ + 32 * h, wv[h]);
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const float2 x = __ffma2_rn(__fadd2_rn(wv[h][j], pivot), make_float2(c, c), rest);
                            wv[h][j] = make_float2(exp2_hw(x.x), exp2_hw(x.y));
                        }
                    }
                }
                arrive(z_read);
                if (!warp_wait(d_full, (uint32_t)m & 1, limit, abort)) return false;
                tc::tc_fence_after();
                if (busy) {
                    if (i > 0) {  // (dq of the tile before was made ahead of this tile's dw)
                        if (!warp_wait(g_full, (uint32_t)(m - 1) & 1, limit, abort)) return false;
                        add_columns<DP, (DP == 64 ? 32 : 16)>(at + Sh::kColQ, g.D, acc);
                    }
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        float2 dz[8];
                        read16(at + Sh::kColD + 16 * h, dz);
#pragma unroll
                        for (int j = 0; j < 8; ++j) dz[j] = __fmul2_rn(wv[h / 2][h % 2 * 8 + j], __fadd2_rn(dz[j], make_float2(-delta, -delta)));
                        float2 *const w = &wv[h / 2][h % 2 * 8];
                        if (left < kKeys) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                if (16 * h + 2 * j >= left) dz[j].x = w[j].x = 0.0f;
                                if (16 * h + 2 * j + 1 >= left) dz[j].y = w[j].y = 0.0f;
                            }
                            // (one state has weight 1 whatever z is: dz is 0, not what rounding leaves of it)
                            if (h == 0 && len == 1) dz[0].x = 0.0f;
                        }
                        float2 s2 = __fadd2_rn(w[0], w[1]), u2 = __fadd2_rn(w[2], w[3]);
#pragma unroll
                        for (int j = 4; j < 8; j += 2) {
                            s2 = __fadd2_rn(s2, w[j]);
                            u2 = __fadd2_rn(u2, w[j + 1]);
                        }
                        f2 = __fadd2_rn(f2, __fadd2_rn(s2, u2));
                        put_parts16(at + Sh::kColD, h, dz);
                    }
                    tmem_wait_st();
                }
                arrive(z_ready);
            }
            m0 += n;
            if (n > 0) {
                if (!warp_wait(g_full, (uint32_t)(m0 - 1) & 1, limit, abort)) return false;
                tc::tc_fence_after();
                if (busy) add_columns<DP, (DP == 64 ? 32 : 16)>(at + Sh::kColQ, g.D, acc);
            }
            if (n == 0 && g.split > 1) return true;  // (the sum knows which splits have none)
            const float f = f2.x + f2.y;
            if (here && n > 0) {
                if (g.split > 1)
                    g.part_norm[w.sp * g.rows + norm_at(g, w.b, head, t)] = f;
                else
                    g.norm[norm_at(g, w.b, head, t)] = log2f(f);
            }
            if (g.dq && __any_sync(0xffffffffu, there))
                put_rows<float, DP>(stage, there ? g.dq + w.sp * g.plane + row * g.D : nullptr, acc, g.D, g.split > 1 ? g.scale : g.scale / f, !here || n == 0, g.D % 8 == 0);
            return true;
        });
        if (!ok && lane == 0) fail();
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 0) tc::tmem_dealloc(tmem, Sh::kCols);
    if (tid == 0) items_done(g.next);
}

// The splits' sums of each row added in their order: dk and dv, or dq. A warp a row; what lies behind the end of the
// row's sentence, or meets nothing, is 0.
struct SumArgs {
    const float *part[2];
    float *out[2];           // (each may be null)
    const float *part_norm;  // of dq's rows f of each split, or null
    float *norm;             //  and log2 f
    size_t plane, rows;
    int n, B, heads, D, r_t, r_b;        // the rows' tensor
    const int32_t *len, *other_len;      // of the rows, and of what they were split over
    int other, tile, per, split;         // its length, its tiles' and a split's tiles
};
__global__ void __launch_bounds__(256)
attend_sum(const __grid_constant__ SumArgs a)
{
    after_previous();
    const size_t row = (size_t)blockIdx.x * 8 + threadIdx.x / 32;
    const int lane = threadIdx.x & 31;
    if (row >= a.rows) return;
    const size_t line = row / a.heads;
    const bool by_time = a.r_t > a.r_b;  // (equal: one sentence, or one row of each)
    const int b = a.B == 1 ? 0 : by_time || a.n == 1 ? (int)(line % a.B) : (int)(line / a.n);
    const int t = a.n == 1 ? 0 : by_time || a.B == 1 ? (int)(line / a.B) : (int)(line % a.n);
    const int len = a.len ? min(max(a.len[b], 0), a.n) : a.n, other = a.other_len ? min(max(a.other_len[b], 0), a.other) : a.other;
    const int tiles = (other + a.tile - 1) / a.tile, n = t < len ? min(a.split, (tiles + a.per - 1) / a.per) : 0;
    float by = 1.0f;
    if (a.part_norm && n > 0) {
        const size_t at = ((size_t)b * a.heads + row % a.heads) * a.n + t;
        float f = 0.0f;
        for (int i = 0; i < n; ++i) f += a.part_norm[i * a.rows + at];
        by = 1.0f / f;
        if (lane == 0) a.norm[at] = log2f(f);
    }
#pragma unroll
    for (int o = 0; o < 2; ++o) {
        if (!a.out[o]) continue;
        for (int d = lane; d < a.D; d += 32) {
            const float *p = a.part[o] + row * a.D + d;
            float v = 0.0f;
#pragma unroll 4
            for (int i = 0; i < n; ++i) v += p[i * a.plane];
            a.out[o][row * a.D + d] = v * by;
        }
    }
}

// ------------------------------------------------------------------ host side
enum { kWsQ = 0, kWsK, kWsV, kWsDy, kWsDelta, kWsPart, kWsPartStats, kWsNorm };  // workspace buffers

// q, k, v, y or dy: B sentences of n rows of `heads` heads; D elements a head, or in the workspace Dp.
struct Rows {
    int n, B, heads, D, batch_major;
    int t() const { return batch_major ? heads : B * heads; }  // from one row to the next, in heads
    int b() const { return batch_major ? n * heads : heads; }
};

// The map of a part, read in boxes of 64 columns x G heads x `box` rows of a sentence (of a state's head
// G = 1, and the group's dimension is left out); what is outside reads as zero.
cudaError_t make_map(CUtensorMap *tm, const void *p, const Rows &r, int width, int G, bool grouped, int box)
{
    cudaError_t e;
    auto encode = tensor_map_encoder(&e);
    if (e) return e;
    cuuint64_t dims[5], strides[4];
    cuuint32_t boxes[5], es[5] = {1, 1, 1, 1, 1};
    const cuuint64_t head = (cuuint64_t)width * 2;
    int k = 0;
    dims[k] = width; boxes[k] = 64; ++k;
    if (grouped) { dims[k] = G; strides[k - 1] = head; boxes[k] = G; ++k; }
    dims[k] = r.heads / G; strides[k - 1] = head * G; boxes[k] = 1; ++k;
    dims[k] = r.B; strides[k - 1] = head * r.b(); boxes[k] = 1; ++k;
    dims[k] = r.n; strides[k - 1] = head * r.t(); boxes[k] = box; ++k;
    const CUresult c = encode(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, k, const_cast<void *>(p), dims, strides, boxes, es,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return c == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// What the products read of a tensor: itself, or its parts in the workspace.
struct Operand {
    const void *p = nullptr;
    int width = 0;
    size_t plane = 0;  // elements from one part to the next
    const void *part(int i) const { return (const __nv_bfloat16 *)p + i * plane; }
};
cudaError_t as_operand(stacklstm_op *op, const void *src, bool fp32, const Rows &r, const int32_t *len, int ws, Pack *pack, Operand *o)
{
    const int Dp = (r.D + 7) / 8 * 8;
    const size_t rows = (size_t)r.n * r.B * r.heads;
    *o = {src, r.D, 0};
    if (!fp32 && Dp == r.D) return cudaSuccess;
    if (cudaError_t e = op_workspace(op, ws, rows * Dp * 2 * (fp32 ? 3 : 1))) return e;
    *o = {op->ws[ws], Dp, rows * Dp};
    int lanes = 1;
    while (lanes * 8 < Dp) lanes *= 2;
    *pack = {src, (__nv_bfloat16 *)op->ws[ws], nullptr, nullptr, len, r.n, r.B, r.heads, r.D, Dp, r.batch_major, fp32, lanes,
             ceil_div(rows, (size_t)(256 / lanes))};
    return cudaSuccess;
}
cudaError_t launch_pack(const stacklstm_op *op, const Packs &p)
{
    const unsigned ctas = p.t[0].ctas + p.t[1].ctas + p.t[2].ctas + p.t[3].ctas;
    return ctas ? launch_after(attend_pack, ctas, 256, 0, op->stream, p) : cudaSuccess;
}

struct Call {
    int T, S;
    const void *q, *k, *v;
    const int32_t *q_len, *kv_len;
    float scale;
};
Rows query_rows(const stacklstm_op *op, int T) { return {T, op->B, op->heads, op->D, op->q_layout == SL_BATCH_MAJOR}; }
Rows state_rows(const stacklstm_op *op, int S) { return {S, op->B, op->kv_heads, op->D, op->kv_layout == SL_BATCH_MAJOR}; }

cudaError_t operands(stacklstm_op *op, const Call &c, Packs &packs, Operand (&o)[3])
{
    const bool fp32 = op->dt == SL_FP32;
    const Rows qr = query_rows(op, c.T), kr = state_rows(op, c.S);
    packs.err = op->err;
    cudaError_t e = as_operand(op, c.q, fp32, qr, c.q_len, kWsQ, &packs.t[0], &o[0]);
    if (!e) e = as_operand(op, c.k, fp32, kr, c.kv_len, kWsK, &packs.t[1], &o[1]);
    if (!e) e = as_operand(op, c.v, fp32, kr, c.kv_len, kWsV, &packs.t[2], &o[2]);
    return e;
}
template <int NP, typename M>
cudaError_t make_maps(const stacklstm_op *op, const Call &c, const Operand (&o)[3], int tq, int keys, M &m)
{
    const int G = op->heads / op->kv_heads;
    const Rows qr = query_rows(op, c.T), kr = state_rows(op, c.S);
    cudaError_t e = cudaSuccess;
    for (int p = 0; p < NP && !e; ++p) {
        e = make_map(&m.q[p], o[0].part(p), qr, o[0].width, G, true, tq);
        if (!e) e = make_map(&m.k[p], o[1].part(p), kr, o[1].width, 1, false, keys);
        if (!e) e = make_map(&m.v[p], o[2].part(p), kr, o[2].width, 1, false, keys);
    }
    return e;
}

// Whether items of sentences of different lengths are so few to a CTA that their order matters.
bool few_each(long long items, long long ctas, int B, const int32_t *len)
{
    return len && B > 1 && B <= kSorted && items > ctas && items <= 8 * ctas;
}

// In how many splits (`most` at most) items of `tiles` tiles each go over the `room` CTAs there are. An item's begin and
// end cost `ends` tiles, the join of the splits `join`. Where the sentences differ (uneven) CTAs take what there is, `few`
// items each, so that their work evens out; else the splits are those that end first: 64 x 8 over 4096 states, 16 heads
// of 64 over 4, 256 items for 304 CTAs, in one go 51 us and in three splits each 65. Of lengths from a third of it on, with
// 2, 3, 4, 6 items a CTA: 57, 53, 54, 61 us; 32 x 1 over 8192, 8 heads of 128 over 2: 54, 56, 57, 60; 40 x 8 over 3000, 8 of 128
// over 4: 54, 51, 52, 55; 8 x 16 over 4096, 16 of 64 over 8: 27, 29, 31, 30. Backward, 1 x 1194 x 3442 fp32, 2 heads of 31, 91
// us with two items a CTA, 76 so.
int few_splits(long long items, long long room, int tiles, int most, bool uneven, int few, int ends, int join)
{
    if (items >= room || most < 2) return 1;
    if (uneven) return (int)std::max<long long>(1, std::min<long long>(most, few * room / items));
    int best = 1;
    long long least = LLONG_MAX;
    for (int s = 1; s <= most; ++s) {
        const long long per = ceil_div(tiles, s), n = ceil_div(tiles, per), rounds = ceil_div(items * n, room);
        const long long cost = rounds * (per + ends) + (n > 1 ? join : 0);
        if (cost < least) least = cost, best = (int)n;
    }
    return best;
}

template <int NP, int PP, int DP>
cudaError_t launch_forward(stacklstm_op *op, const Call &c, const Operand (&o)[3], FwdArgs &g)
{
    using Sh = FwdShape<NP, PP, DP>;
    constexpr auto kernel = attend_forward<NP, PP, DP>;
    Maps<NP> m;
    cudaError_t e = make_maps<NP>(op, c, o, g.tq, kKeys, m);
    if (!e) e = smem_at_least((const void *)kernel, Sh::kSmem);
    if (e) return e;
    // few query tiles: the states are split too, where each split still reads more states than it
    // writes sums
    const long long ctas = (long long)g.tiles * g.nk * g.B, room = (long long)op->num_sms * Sh::kCtas;
    const int tiles = (int)ceil_div(c.S, kKeys), rows = std::min(c.T * g.G, kRows);
    const int least = std::max(4, 8 * rows / kKeys);
    g.split = few_splits(ctas, room, tiles, std::min(tiles / least, kMostSplits), c.kv_len && g.B > 1, 3, 3, 4);
    g.per = (int)ceil_div(tiles, g.split);
    g.split = (int)ceil_div(tiles, g.per);
    if (g.split > 1) {
        e = op_workspace(op, kWsPart, (size_t)g.split * g.rows * g.Dp * 4);
        if (!e) e = op_workspace(op, kWsPartStats, (size_t)g.split * g.rows * 8);
        if (e) return e;
        g.part = g.sums = (float *)op->ws[kWsPart];
        g.part_stats = (float2 *)op->ws[kWsPartStats];
    }
    if (Sh::kSums && g.split == 1 && g.per > Sh::kRun) {
        if ((e = op_workspace(op, kWsPart, g.rows * g.Dp * 4))) return e;
        g.sums = (float *)op->ws[kWsPart];
    }
    g.items = (int)(ctas * g.split);
    g.sorted = few_each(g.items, room, g.B, g.kv_len);
    e = launch_after(kernel, dim3((unsigned)std::min<long long>(g.items, room)), 256, Sh::kSmem, op->stream, m, g);
    if (!e && g.split > 1)
        e = op->dt == SL_BF16 ? launch_after(attend_join<__nv_bfloat16>, dim3(ceil_div(g.rows, 8)), 256, 0, op->stream, g)
                       : launch_after(attend_join<float>, dim3(ceil_div(g.rows, 8)), 256, 0, op->stream, g);
    return e;
}

template <int NP, int DP>
cudaError_t launch_backward(stacklstm_op *op, const Call &c, const Operand (&o)[3], const Operand &dy, BwdArgs &g)
{
    const Rows qr = query_rows(op, c.T);
    BwdMaps<NP> m;
    cudaError_t e = cudaSuccess;
    auto maps = [&](int keys) {
        cudaError_t e = make_maps<NP>(op, c, o, g.tq, keys, m);
        for (int p = 0; p < 3 && !e; ++p) e = make_map(&m.dy[p], dy.part(p), qr, dy.width, g.G, true, g.tq);
        return e;
    };
    const long long pairs = (long long)g.B * g.nk;
    // Few items: each of them in several splits of what it goes over, two tiles of it at least, with sums of their own.
    auto split = [&](long long items, int tiles, long long ctas, bool uneven) {
        g.split = few_splits(items, ctas, tiles, std::min(tiles / 2, kMostSplits), uneven, 2, 2, 3);
        g.per = (int)ceil_div(tiles, g.split);
        g.split = (int)ceil_div(tiles, g.per);
        g.items = (int)(items * g.split);
    };
    auto sum = [&](const Rows &r, const int32_t *len, const int32_t *other_len, int other, int tile, const float *p0, const float *p1, float *o0, float *o1,
                   const float *part_norm) {
        const size_t rows = (size_t)r.n * r.B * r.heads;
        const SumArgs a = {{p0, p1}, {o0, o1}, part_norm, g.norm, g.plane, rows, r.n, r.B, r.heads, r.D, r.t(), r.b(), len, other_len, other, tile, g.per, g.split};
        return launch_after(attend_sum, dim3(ceil_div(rows, 8)), 256, 0, op->stream, a);
    };
    float *const dq = g.dq, *const dk = g.dk, *const dv = g.dv;
    g.rows = (size_t)qr.n * qr.B * qr.heads;
    {  // dq, and each row's f (wanted for dk and dv too)
        using Sh = QueriesShape<NP, DP>;
        constexpr auto kernel = attend_grad_queries<NP, DP>;
        g.tq = Sh::RT / g.G;
        g.tiles = (int)ceil_div(c.T, g.tq);
        split(pairs * g.tiles, (int)ceil_div(c.S, kKeys), op->num_sms * Sh::kCtas, (c.q_len || c.kv_len) && g.B > 1);
        g.sorted = few_each(g.items, op->num_sms * Sh::kCtas, g.B, g.kv_len);
        g.plane = (size_t)qr.n * qr.B * qr.heads * qr.D;
        e = maps(kKeys);
        if (!e) e = op_workspace(op, kWsNorm, g.rows * 4);
        g.norm = (float *)op->ws[kWsNorm];
        if (!e && g.split > 1 && dq && !(e = op_workspace(op, kWsPart, g.split * g.plane * 4))) g.dq = (float *)op->ws[kWsPart];
        if (!e && g.split > 1 && !(e = op_workspace(op, kWsPartStats, g.split * g.rows * 4))) g.part_norm = (float *)op->ws[kWsPartStats];
        if (!e) e = smem_at_least((const void *)kernel, Sh::kSmem);
        if (!e) e = launch_after(kernel, dim3((unsigned)std::min(g.items, op->num_sms * Sh::kCtas)), 256, Sh::kSmem, op->stream, m, g);
        if (!e && g.split > 1) e = sum(qr, g.q_len, g.kv_len, c.S, kKeys, g.dq, nullptr, dq, nullptr, g.part_norm);
    }
    if (!e && (dk || dv)) {
        using Sh = StatesShape<NP, DP>;
        constexpr auto kernel = attend_grad_states<NP, DP>;
        const Rows kr = state_rows(op, c.S);
        g.tq = Sh::TT / g.G;
        g.tiles = (int)ceil_div(c.S, Sh::KT);
        split(pairs * g.tiles, (int)ceil_div(c.T, g.tq), op->num_sms, (c.q_len || c.kv_len) && g.B > 1);
        g.sorted = few_each(g.items, op->num_sms, g.B, g.q_len);
        g.plane = (size_t)kr.n * kr.B * kr.heads * kr.D;
        e = maps(Sh::KT);
        if (!e && g.split > 1 && !(e = op_workspace(op, kWsPart, 2 * g.split * g.plane * 4))) {
            if (dk) g.dk = (float *)op->ws[kWsPart];
            if (dv) g.dv = (float *)op->ws[kWsPart] + g.split * g.plane;
        }
        if (!e) e = smem_at_least((const void *)kernel, Sh::kSmem);
        if (!e) e = launch_after(kernel, dim3((unsigned)std::min(g.items, op->num_sms)), Sh::kThreads, Sh::kSmem, op->stream, m, g);
        if (!e && g.split > 1) e = sum(kr, g.kv_len, g.q_len, c.T, g.tq, g.dk, g.dv, dk, dv, nullptr);
    }
    return e;
}

const char *check_call(const stacklstm_op *op, int T, int S, float scale)
{
    if (T < 0 || T > op->T) return "T outside 0 .. T";
    if (S < 1 || S > op->S) return "S outside 1 .. S";
    if (!(scale > 0.0f) || !(scale < INFINITY)) return "scale must be positive and finite";
    return nullptr;
}

}  // namespace
}  // namespace sl

using namespace sl;

extern "C" {

sl_status stacklstm_attend_create(stacklstm_op_t *out, int T, int S, int B, int heads, int kv_heads, int D, sl_dtype dtype,
                                  sl_layout q_layout, sl_layout kv_layout, int device, void *stream)
{
    if (!out) return SL_ERR_ARG;
    *out = nullptr;
    if (T < 1 || S < 1 || B < 1 || heads < 1 || kv_heads < 1 || D < 1 || heads % kv_heads || (dtype != SL_FP32 && dtype != SL_BF16) ||
        (q_layout != SL_TIME_MAJOR && q_layout != SL_BATCH_MAJOR) || (kv_layout != SL_TIME_MAJOR && kv_layout != SL_BATCH_MAJOR))
        return SL_ERR_ARG;
    const int G = heads / kv_heads;
    if (D > kMostD || G > kMostGroup || T > 1 << 20 || S > 1 << 20 || (long long)B * heads * D > 1 << 30 ||
        (long long)std::max(T, S) * heads > 1 << 30 || (long long)B * T * heads > 1LL << 34 || (long long)B * S * kv_heads > 1LL << 34 ||
        ((long long)T * G / 32 + 1) * kv_heads * B > 1LL << 30 || ((long long)S / 64 + 1) * kv_heads * B > 1LL << 30)
        return SL_ERR_UNSUPPORTED;
    sl_status st;
    stacklstm_op *op = op_new(SL_OP_ATTEND, dtype, device, stream, &st);
    if (!op) return st;
    op->T = T;
    op->S = S;
    op->B = B;
    op->heads = heads;
    op->kv_heads = kv_heads;
    op->D = D;
    op->q_layout = q_layout;
    op->kv_layout = kv_layout;
    *out = op;
    return SL_OK;
}

sl_status stacklstm_attend_forward(stacklstm_op_t op, int T, int S, const void *q, const void *k, const void *v, const int32_t *q_len,
                                   const int32_t *kv_len, float scale, void *y, float *lse, float *ctx)
{
    if (!op || op->kind != SL_OP_ATTEND) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (const char *m = check_call(op, T, S, scale)) return op_fail(op, SL_ERR_ARG, m);
    if (T == 0) return SL_OK;
    if (const char *m = check_pointers({q, k, v, y}, {q_len, kv_len, lse, ctx})) return op_fail(op, SL_ERR_ARG, m);
    OpDevice guard(op->device);
    const Call c = {T, S, q, k, v, q_len, kv_len, scale};
    Packs packs = {};
    Operand o[3];
    cudaError_t e = operands(op, c, packs, o);
    if (!e) e = launch_pack(op, packs);
    const Rows qr = query_rows(op, T);
    FwdArgs g = {};
    g.T = T; g.S = S; g.B = op->B; g.nk = op->kv_heads; g.G = op->heads / op->kv_heads; g.D = op->D;
    g.q_t = qr.t(); g.q_b = qr.b(); g.q_len = q_len; g.kv_len = kv_len; g.scale = scale;
    g.y = y; g.lse = lse; g.ctx = ctx;
    g.tq = kRows / g.G; g.tiles = (int)ceil_div(T, g.tq);
    g.rows = (size_t)op->B * T * op->heads; g.Dp = (op->D + 7) / 8 * 8;
    g.limit = op->wait_limit; g.err = op->err; g.next = op->err + 2;
    const bool wide = op->D > 64;
    if (!e) {
        if (op->dt == SL_FP32)
            e = wide ? launch_forward<3, 3, 128>(op, c, o, g) : launch_forward<3, 3, 64>(op, c, o, g);
        else if (ctx)
            e = wide ? launch_forward<1, 3, 128>(op, c, o, g) : launch_forward<1, 3, 64>(op, c, o, g);
        else
            e = wide ? launch_forward<1, 2, 128>(op, c, o, g) : launch_forward<1, 2, 64>(op, c, o, g);
    }
    return e ? op_cuda(op, e, "stacklstm_attend_forward") : SL_OK;
}

sl_status stacklstm_attend_backward(stacklstm_op_t op, int T, int S, const float *dy, const void *q, const void *k, const void *v,
                                    const int32_t *q_len, const int32_t *kv_len, float scale, const float *lse, const float *ctx,
                                    float *dq, float *dk, float *dv)
{
    if (!op || op->kind != SL_OP_ATTEND) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (const char *m = check_call(op, T, S, scale)) return op_fail(op, SL_ERR_ARG, m);
    if (T > 0) {
        if (const char *m = check_pointers({dy, q, k, v, lse, ctx}, {q_len, kv_len, dq, dk, dv})) return op_fail(op, SL_ERR_ARG, m);
    } else if (const char *m = check_pointers({}, {dk, dv})) {
        return op_fail(op, SL_ERR_ARG, m);
    }
    if (!dq && !dk && !dv) return SL_OK;
    OpDevice guard(op->device);
    cudaError_t e = cudaSuccess;
    if (T == 0) {  // no queries: the states' gradients are sums of nothing
        const size_t bytes = (size_t)S * op->B * op->kv_heads * op->D * 4;
        if (dk) e = cudaMemsetAsync(dk, 0, bytes, op->stream);
        if (!e && dv) e = cudaMemsetAsync(dv, 0, bytes, op->stream);
        return e ? op_cuda(op, e, "stacklstm_attend_backward") : SL_OK;
    }
    const Call c = {T, S, q, k, v, q_len, kv_len, scale};
    const Rows qr = query_rows(op, T), kr = state_rows(op, S);
    Packs packs = {};
    Operand o[3], d;
    e = operands(op, c, packs, o);
    if (!e) e = as_operand(op, dy, true, qr, q_len, kWsDy, &packs.t[3], &d);
    if (!e) e = op_workspace(op, kWsDelta, (size_t)op->B * T * op->heads * 4);
    packs.t[3].ctx = ctx;
    packs.t[3].delta = (float *)op->ws[kWsDelta];
    if (!e) e = launch_pack(op, packs);
    BwdArgs g = {};
    g.T = T; g.S = S; g.B = op->B; g.nk = op->kv_heads; g.G = op->heads / op->kv_heads; g.D = op->D;
    g.q_t = qr.t(); g.q_b = qr.b(); g.k_t = kr.t(); g.k_b = kr.b(); g.q_len = q_len; g.kv_len = kv_len; g.scale = scale;
    g.lse = lse; g.delta = packs.t[3].delta; g.dq = dq; g.dk = dk; g.dv = dv;
    g.limit = op->wait_limit; g.err = op->err; g.next = op->err + 2;
    const bool wide = op->D > 64;
    if (!e) {
        if (op->dt == SL_FP32)
            e = wide ? launch_backward<3, 128>(op, c, o, d, g) : launch_backward<3, 64>(op, c, o, d, g);
        else
            e = wide ? launch_backward<1, 128>(op, c, o, d, g) : launch_backward<1, 64>(op, c, o, d, g);
    }
    return e ? op_cuda(op, e, "stacklstm_attend_backward") : SL_OK;
}

}  // extern "C"
