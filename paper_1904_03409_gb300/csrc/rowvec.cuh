// rowvec.cuh -- rows of any width read in whole 16-byte pieces. Row r of a [R][V] tensor covers
// the flat elements r V .. r V + V - 1; a piece is the 16 bytes of flat elements P E .. P E + E - 1
// (E elements of type T), so every piece is aligned whatever V is, and a row's first and last
// piece may hold neighbours' elements, which are masked. An fp32 tensor of the same shape has the
// same flat elements, so a piece of it is aligned too.
#pragma once

#include "op.cuh"

namespace sl {

// The elements of a piece as fp32.
template <typename T>
__device__ __forceinline__ void unpack(const uint4 &q, float (&v)[16 / sizeof(T)])
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) {
            v[j] = __uint_as_float(w[j]);
        } else {
            v[2 * j] = __uint_as_float(w[j] << 16);
            v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
}

template <typename T>
struct RowVec {
    static constexpr int E = 16 / (int)sizeof(T);
    size_t at;   // the row's first piece's first flat element
    int lead;    // elements of that piece that come before the row
    int V;
    __device__ __forceinline__ RowVec(size_t r, int V_) : V(V_)
    {
        const size_t first = r * V_;
        lead = (int)(first % E);
        at = first - lead;
    }
    // pieces the row touches, and the column of a piece's element 0 (negative before the row)
    __device__ __forceinline__ int pieces() const { return (lead + V + E - 1) / E; }
    __device__ __forceinline__ int column(int p) const { return p * E - lead; }
    __device__ __forceinline__ bool whole(int p) const
    {
        const int c = column(p);
        return c >= 0 && c + E <= V;
    }
    __device__ __forceinline__ size_t first() const { return at + lead; }
    // piece p as it lies in memory, with -inf in the place of what is outside the row (which is
    // not read)
    __device__ __forceinline__ uint4 load(const T *base, int p) const
    {
        const size_t o = at + (size_t)p * E;
        if (whole(p)) return *(const uint4 *)(base + o);
        union {
            T e[E];
            uint4 q;
        } u;
        const int c = column(p);
#pragma unroll
        for (int i = 0; i < E; ++i) u.e[i] = c + i >= 0 && c + i < V ? base[o + i] : from_f32<T>(-INFINITY);
        return u.q;
    }
    // (aligned: base is on 32 bytes, so pieces of eight are)
    __device__ __forceinline__ void store_f32(float *base, bool aligned, int p, const float (&v)[E]) const
    {
        const size_t o = at + (size_t)p * E;
        if (whole(p)) {
            if constexpr (E == 8)
                store8(base + o, aligned, v);
            else
                store_vec<float, E>(base + o, v);
        } else {
            const int c = column(p);
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (c + i >= 0 && c + i < V) base[o + i] = v[i];
        }
    }
};

// The larger of two values, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}

// The largest element of a piece: NaN if any is (NANS), or of those that are not.
template <typename T, bool NANS>
__device__ __forceinline__ float piece_max(const uint4 &q)
{
    if constexpr (sizeof(T) == 4) {
        float v[4];
        unpack<T>(q, v);
        return NANS ? max_nan(max_nan(v[0], v[1]), max_nan(v[2], v[3])) : fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
    } else {  // two at a time
        const __nv_bfloat162 *h = (const __nv_bfloat162 *)&q;
        const __nv_bfloat162 m = NANS ? __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]))
                                      : __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        const float a = __low2float(m), b = __high2float(m);
        return NANS ? max_nan(a, b) : fmaxf(a, b);
    }
}

// The sums (maxima) of NV values at once over groups of G lanes (of a warp), their shuffles in
// flight together.
template <bool MAX, int G, int NV>
__device__ __forceinline__ void lanes_join(float (&v)[NV])
{
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) {
        float w[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) w[i] = __shfl_xor_sync(0xffffffffu, v[i], o);
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = MAX ? max_nan(v[i], w[i]) : v[i] + w[i];
    }
}
// The same over the TPR threads of a row: some lanes of a warp, or the whole CTA through `sm`
// (NV TPR / 32 floats; free again after the call, or with KEEP after the CTA's next barrier).
template <bool MAX, int TPR, bool KEEP = false, int NV>
__device__ __forceinline__ void row_join(float (&v)[NV], float *sm)
{
    lanes_join<MAX, (TPR < 32 ? TPR : 32)>(v);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        const int lane = threadIdx.x & 31;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < NV; ++i) sm[i * W + (threadIdx.x >> 5)] = v[i];
        __syncthreads();
        // every warp joins the warps' values, lane by lane and then in a butterfly
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = lane < W ? sm[i * W + lane] : MAX ? -INFINITY : 0.0f;
        lanes_join<MAX, 32>(v);
        if constexpr (!KEEP) __syncthreads();
    }
}

__device__ __forceinline__ float exp2_hw(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;

// How a row of V elements is spread: over 8 lanes or a warp where four pieces a lane hold it, else
// over the least of 128, 512 and 1024 threads with up to eight pieces in the registers of each; the
// widest rows are read again in each pass (NP = 0). (Eight lanes: four rows share a warp's
// instructions; 11840 rows of 83 fp32 classes a warp each were bound by them.)
template <typename T>
inline void row_plan(int V, int *tpr, int *np)
{
    const int n = (int)(((size_t)V + RowVec<T>::E - 1) / RowVec<T>::E) + 1;  // most pieces of a row
    auto up = [](unsigned v) { return v <= 1 ? 1 : v <= 2 ? 2 : v <= 4 ? 4 : v <= 8 ? 8 : 0; };
    for (int t : {8, 32, 128, 512, 1024}) {
        *tpr = t;
        *np = up(ceil_div(n, t));
        if (*np && *np <= (t <= 32 ? 4 : 8)) return;
    }
    *np = 0;
}
// the kernels that row_plan can ask for: X(threads, pieces)
#define SL_ROW_PLANS(X) \
    X(8, 1) X(8, 2) X(8, 4) X(32, 2) X(32, 4) X(128, 2) X(128, 4) X(128, 8) X(512, 4) X(512, 8) X(1024, 8) X(1024, 0)
__host__ __device__ constexpr int row_cta(int tpr) { return tpr <= 32 ? 256 : tpr; }
__host__ __device__ constexpr int row_ctas_per_sm(int tpr) { return tpr <= 32 ? 5 : tpr == 128 ? 8 : tpr == 512 ? 2 : 1; }
__host__ __device__ constexpr int rows_per_cta(int tpr) { return tpr <= 32 ? 256 / tpr : 1; }

}  // namespace sl
