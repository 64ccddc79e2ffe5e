// rowvec.cuh -- rows of any width read in whole 16-byte pieces. Row r of a [R][V] tensor covers
// the flat elements r V .. r V + V - 1; a piece is the 16 bytes of flat elements P E .. P E + E - 1
// (E elements of type T), so every piece is aligned whatever V is, and a row's first and last
// piece may hold neighbours' elements, which are masked. An fp32 tensor of the same shape has the
// same flat elements, so a piece of it is aligned too.
#pragma once

#include "op.cuh"

namespace sl {

template <typename T>
struct RowVec {
    static constexpr int E = 16 / (int)sizeof(T);
    size_t first;  // the row's first flat element
    size_t total;  // elements of the whole tensor: nothing is read beyond them
    int V;
    __device__ __forceinline__ RowVec(int r, int V_, size_t rows) : first((size_t)r * V_), total(rows * V_), V(V_) {}
    // pieces the row touches, and the column of a piece's element 0 (negative before the row)
    __device__ __forceinline__ int pieces() const { return (int)((first + V - 1) / E - first / E) + 1; }
    __device__ __forceinline__ int column(int p) const { return p * E - (int)(first % E); }
    // piece p in v, what is outside the row as -inf
    __device__ __forceinline__ void load(const T *base, int p, float (&v)[E]) const
    {
        const size_t at = (first / E + p) * E;
        const int c = column(p);
        if (c >= 0 && c + E <= V) {
            load_vec<T, E>(base + at, v);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = c + i >= 0 && c + i < V ? to_f32(base[at + i]) : -INFINITY;
        }
    }
    __device__ __forceinline__ void store_f32(float *base, int p, const float (&v)[E]) const
    {
        const size_t at = (first / E + p) * E;
        const int c = column(p);
        if (c >= 0 && c + E <= V) {
            store_vec<float, E>(base + at, v);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (c + i >= 0 && c + i < V) base[at + i] = v[i];
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
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
template <int TPR>
__device__ __forceinline__ float row_max(float v, float *sm)
{
    v = warp_max(v);
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
        __syncthreads();
        v = sm[0];
#pragma unroll
        for (int i = 1; i < TPR / 32; ++i) v = max_nan(v, sm[i]);
        __syncthreads();
    }
    return v;
}

__device__ __forceinline__ float exp2_hw(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;

// How a row of V elements is spread: a warp or a CTA of kRowThreads, its pieces in the threads'
// registers (NP a thread) or, for the widest rows, read again in each pass (NP = 0).
constexpr int kRowThreads = 512;
template <typename T>
inline void row_plan(int V, int *tpr, int *np)
{
    const int n = (int)(((size_t)V + RowVec<T>::E - 1) / RowVec<T>::E) + 1;  // most pieces of a row
    auto up = [](int v) { return v <= 1 ? 1 : v <= 2 ? 2 : v <= 4 ? 4 : v <= 8 ? 8 : v <= 16 ? 16 : 0; };
    *tpr = 32;
    *np = up((int)ceil_div(n, 32));
    if (*np == 0 || *np > 4) {
        *tpr = kRowThreads;
        *np = up((int)ceil_div(n, kRowThreads));
    }
}

}  // namespace sl
