// op.cuh -- the handle of the output-layer and search operators (layer norm, linear layer,
// distillation, beam search) and what their translation units share: argument checks, the
// device guard, element access by type and the reductions over a warp or a CTA.
#pragma once

#include <stdio.h>

#include <algorithm>
#include <new>

#include <utility>

#include "common.cuh"
#include "tc.cuh"

enum sl_op_kind { SL_OP_NORM = 1, SL_OP_LINEAR, SL_OP_DISTILL, SL_OP_BEAM };

// One operator: its sizes, stream and workspace. Plain data (its calls throw nothing).
struct stacklstm_op {
    int kind = 0;
    int device = 0, num_sms = 0;
    cudaStream_t stream = nullptr;
    sl_dtype dt = SL_FP32;
    int R = 0;                         // most rows of a call (beam: B * K)
    int N = 0, K = 0, act = 0;         // norm: N; linear: x [R][K], W [N][K]
    int pairs = 0;                     // linear: pairs of CTAs that run at once
    int V = 0, k = 0;                  // distill: classes, teacher entries a row; beam: V
    int B = 0, beams = 0, S = 0, H = 0;  // beam
    int32_t *err = nullptr;            // device-detected status (first error wins)
    long long wait_limit = 0;          // clock cycles one bounded device-side wait may spin
    void *ws[8] = {};                  // workspace buffers, by kind
    size_t ws_bytes[8] = {};
    char last_error[192] = {};
};

namespace sl {

sl_status op_fail(stacklstm_op *op, sl_status st, const char *msg);
sl_status op_cuda(stacklstm_op *op, cudaError_t e, const char *where);
// a handle with its device checked and its status word allocated (nullptr: *st says why)
stacklstm_op *op_new(int kind, sl_dtype dt, int device, void *stream, sl_status *st);
// workspace buffer i, at least `bytes` (grown only: a kernel of an earlier call may read the old
// one, which is freed after the stream has run dry)
cudaError_t op_workspace(stacklstm_op *op, int i, size_t bytes);

// the operator's device current for the time of a call, the caller's put back after it
struct OpDevice {
    int prev = -1;
    explicit OpDevice(int device)
    {
        int cur = -1;
        if (cudaGetDevice(&cur) == cudaSuccess && cur != device) {
            prev = cur;
            cudaSetDevice(device);
        }
    }
    ~OpDevice()
    {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

// 0 if every pointer is set and 16-byte aligned (those of `may` may be null), else the message
inline const char *check_pointers(std::initializer_list<const void *> need, std::initializer_list<const void *> may)
{
    for (const void *p : need)
        if (!p) return "null pointer";
    for (const void *p : need)
        if (!aligned16(p)) return "tensors must be 16-byte aligned";
    for (const void *p : may)
        if (!aligned16(p)) return "tensors must be 16-byte aligned";
    return nullptr;
}

#ifdef __CUDACC__
// A launch that may begin while the kernel before it on the stream ends. Every kernel launched so
// lets the next one begin and waits for all the work before it (after_previous) before it touches
// memory, so the order on the stream is that of plain launches; what is saved is
// the start of a kernel, one to two microseconds of the short calls.
template <typename... P, typename... A>
inline cudaError_t launch_cluster(void (*kernel)(P...), unsigned cluster, dim3 grid, unsigned threads, size_t smem, cudaStream_t st,
                                  A &&...args)
{
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
}
template <typename... P, typename... A>
inline cudaError_t launch_after(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, A &&...args)
{
    return launch_cluster(kernel, 1, grid, threads, smem, st, std::forward<A>(args)...);
}
__device__ __forceinline__ void after_previous()
{
    tc::grid_dep_launch();
    tc::grid_dep_wait();
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16(v); }

// VEC consecutive elements (one access of VEC * sizeof(T) bytes, so aligned, or VEC = 1)
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T *p, float *v)
{
    if constexpr (VEC == 1) {
        v[0] = to_f32(*p);
    } else if constexpr (sizeof(T) == 4) {
        static_assert(VEC % 4 == 0, "16-byte pieces");
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i) {
            const float4 q = *(const float4 *)(p + 4 * i);
            v[4 * i] = q.x; v[4 * i + 1] = q.y; v[4 * i + 2] = q.z; v[4 * i + 3] = q.w;
        }
    } else {
        static_assert(VEC % 8 == 0, "16-byte pieces");
#pragma unroll
        for (int i = 0; i < VEC / 8; ++i) {
            const uint4 q = *(const uint4 *)(p + 8 * i);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
                v[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
            }
        }
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T *p, const float *v)
{
    if constexpr (VEC == 1) {
        *p = from_f32<T>(v[0]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i)
            *(float4 *)(p + 4 * i) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 8; ++i) {
            union {
                __nv_bfloat162 b[4];
                uint4 q;
            } o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o.b[j] = __floats2bfloat162_rn(v[8 * i + 2 * j], v[8 * i + 2 * j + 1]);
            *(uint4 *)(p + 8 * i) = o.q;
        }
    }
}

// 8 fp32 values as one 32-byte access where `whole` (the address is on 32 bytes), else as two of 16:
// neighbouring lanes' 32 bytes in two accesses move every sector twice between L1 and L2.
__device__ __forceinline__ void load8(const float *p, bool whole, float *v)
{
    if (whole)
        asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                     : "l"(p));
    else
        load_vec<float, 8>(p, v);
}
__device__ __forceinline__ void store8(float *p, bool whole, const float *v)
{
    if (whole)
        asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                     "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                     : "memory");
    else
        store_vec<float, 8>(p, v);
}
__device__ __forceinline__ bool on_32(const void *p) { return ((uintptr_t)p & 31u) == 0; }

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// The sum over the TPR threads of a row, to all of them: a warp (TPR = 32), or the whole CTA
// through `sm` (TPR / 32 floats, free again after the call).
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *sm)
{
    v = warp_sum(v);
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / 32; ++i) v += sm[i];
        __syncthreads();
    }
    return v;
}
#endif

}  // namespace sl
