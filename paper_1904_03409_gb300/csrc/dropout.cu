// dropout.cu -- dropout whose mask is never stored, forward and backward, and its C ABI
// (include/stacklstm.h, stacklstm_dropout_*).
//
//   y = residual + keep x / (1 - p)
// Element e of the mask (of mask_rows rows of N; row r of x uses its row r mod mask_rows) is kept where
// word e mod 4 of block e / 4 is at least p 2^32. A block's four words are those of Philox4x32-7 (Salmon,
// Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011: seven rounds are the
// fewest that pass all of their tests), counter (block, step), key seed: the backward makes the mask
// again. Bound by HBM; a block is 14 wide products for four elements.
#include <cmath>

#include "rowvec.cuh"

namespace sl {
namespace {

struct DropArgs {
    size_t total, period;      // elements of x and of the mask
    const void *x, *residual;
    void *y;
    uint32_t k0, k1, last;     // the key; kept: word > last, or all
    int all;
    float by;
    const long long *step;
    unsigned copies;           // uses of each mask element (2^31 - 1 at most), of which a thread takes
    unsigned per;              //  so many
};

__device__ __forceinline__ void philox7(uint32_t (&c)[4], uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const unsigned long long a = (unsigned long long)c[0] * 0xD2511F53u, b = (unsigned long long)c[2] * 0xCD9E8D57u;
        const uint32_t n0 = (uint32_t)(b >> 32) ^ c[1] ^ k0, n2 = (uint32_t)(a >> 32) ^ c[3] ^ k1;
        c[1] = (uint32_t)b;
        c[3] = (uint32_t)a;
        c[0] = n0;
        c[2] = n2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

constexpr int kE = 8;      // mask elements of a piece: two blocks
constexpr int kInFlight = 4;

// The factors of mask elements kE piece ..: 1 / (1 - p) or 0, as bits.
__device__ __forceinline__ uint32_t kept(const DropArgs &a, size_t piece, uint32_t s0, uint32_t s1)
{
    uint32_t bits = 0;
#pragma unroll
    for (int h = 0; h < kE / 4; ++h) {
        const unsigned long long block = piece * (kE / 4) + h;
        uint32_t c[4] = {(uint32_t)block, (uint32_t)(block >> 32), s0, s1};
        philox7(c, a.k0, a.k1);
#pragma unroll
        for (int i = 0; i < 4; ++i) bits |= (uint32_t)(c[i] > a.last) << (4 * h + i);
    }
    return a.all ? 0xffffffffu : bits;
}

// A piece of x as it lies in memory.
template <typename T>
struct Eight {
    uint4 q[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = ((const uint4 *)p)[i];
    }
    __device__ __forceinline__ void get(float (&v)[kE]) const
    {
        if constexpr (sizeof(T) == 2) {
            unpack<T>(q[0], v);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float w[4];
                unpack<T>(q[i], w);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[4 * i + j] = w[j];
            }
        }
    }
};

// WHOLE: the mask's rows end on a piece, so every piece of x is whole and on 16 bytes. MANY: a mask
// element serves several rows, and a thread keeps a piece of the mask for a.per of them; else it takes
// kInFlight pieces of the mask. 65536 x 1024: bf16 with residual and float gradient in 146 us together, 6.4 TB/s.
template <typename T, bool WHOLE, bool MANY>
__global__ void __launch_bounds__(256)
dropout(const __grid_constant__ DropArgs a)
{
    after_previous();
    const long long step = a.step ? *a.step : 0;
    const uint32_t s0 = (uint32_t)step, s1 = (uint32_t)((unsigned long long)step >> 32);
    const size_t pieces = (a.period + kE - 1) / kE;
    const size_t first = MANY ? (size_t)blockIdx.x * 256 + threadIdx.x : (size_t)blockIdx.x * (256 * kInFlight) + threadIdx.x;
    const T *x = (const T *)a.x, *res = (const T *)a.residual;
    T *y = (T *)a.y;
    if (MANY && first >= pieces) return;
    const uint32_t mine = MANY ? kept(a, first, s0, s1) : 0;
    const unsigned c_lo = MANY ? blockIdx.y * a.per : 0, c_hi = MANY ? min(c_lo + a.per, a.copies) : kInFlight;
    for (unsigned c0 = c_lo; c0 < c_hi; c0 += kInFlight) {
        size_t at[kInFlight];
        Eight<T> q[kInFlight], w[kInFlight];
        bool here[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const size_t piece = MANY ? first : first + (size_t)u * 256;
            at[u] = MANY ? (size_t)(c0 + u) * a.period + piece * kE : piece * kE;
            here[u] = (MANY ? c0 + u < c_hi : piece < pieces) && at[u] < a.total;
            if (WHOLE && here[u]) {
                q[u].load(x + at[u]);
                if (res) w[u].load(res + at[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            if (!here[u]) continue;
            const size_t piece = MANY ? first : first + (size_t)u * 256;
            const uint32_t bits = MANY ? mine : kept(a, piece, s0, s1);
            float v[kE], r[kE];
            if (WHOLE) {
                q[u].get(v);
                if (res) w[u].get(r);
#pragma unroll
                for (int i = 0; i < kE; ++i) {
                    v[i] = bits >> i & 1 ? v[i] * a.by : 0.0f;
                    if (res) v[i] += r[i];
                }
                store_vec<T, kE>(y + at[u], v);
            } else {
                const size_t left = min(a.period - piece * kE, a.total - at[u]);
#pragma unroll
                for (int i = 0; i < kE; ++i)
                    if ((size_t)i < left) {
                        float z = bits >> i & 1 ? to_f32(x[at[u] + i]) * a.by : 0.0f;
                        if (res) z += to_f32(res[at[u] + i]);
                        y[at[u] + i] = from_f32<T>(z);
                    }
            }
        }
    }
}

template <typename T>
cudaError_t launch_dropout(const stacklstm_op *op, DropArgs &a)
{
    const size_t pieces = (a.period + kE - 1) / kE;
    const bool whole = a.period % kE == 0 && a.total % kE == 0;
    if (a.copies == 1) {
        const dim3 grid(ceil_div(pieces, 256 * kInFlight));
        return whole ? launch_after(dropout<T, true, false>, grid, 256, 0, op->stream, a)
                     : launch_after(dropout<T, false, false>, grid, 256, 0, op->stream, a);
    }
    // as few uses a thread as fill the GPU with threads, kInFlight at least
    const size_t ctas = ceil_div(pieces, 256);
    const size_t groups = std::max<size_t>(1, (size_t)op->num_sms * 8 / ctas);
    a.per = (unsigned)std::max<size_t>(kInFlight, std::max(ceil_div(a.copies, groups), ceil_div(a.copies, 65535)));
    a.per = (a.per + kInFlight - 1) / kInFlight * kInFlight;
    const dim3 grid((unsigned)ctas, ceil_div(a.copies, a.per));
    return whole ? launch_after(dropout<T, true, true>, grid, 256, 0, op->stream, a)
                 : launch_after(dropout<T, false, true>, grid, 256, 0, op->stream, a);
}

sl_status run(stacklstm_op *op, int rows, const void *x, const void *residual, double p, uint64_t seed, const int64_t *step,
              int mask_rows, void *y, bool fp32, const char *where)
{
    if (!op || op->kind != SL_OP_DROPOUT) return SL_ERR_ARG;
    op->last_error[0] = 0;
    if (rows < 0 || rows > op->R) return op_fail(op, SL_ERR_ARG, "rows outside 0 .. R");
    if (!(p >= 0.0 && p <= 1.0)) return op_fail(op, SL_ERR_ARG, "p outside 0 .. 1");
    if (mask_rows < 0) return op_fail(op, SL_ERR_ARG, "mask_rows must not be negative");
    if (rows == 0) return SL_OK;
    if (const char *m = check_pointers({x, y}, {residual})) return op_fail(op, SL_ERR_ARG, m);
    if ((uintptr_t)step & 7u) return op_fail(op, SL_ERR_ARG, "step must be 8-byte aligned");
    OpDevice guard(op->device);
    DropArgs a = {};
    const int period = mask_rows == 0 || mask_rows > rows ? rows : mask_rows;
    a.total = (size_t)rows * op->N;
    a.period = (size_t)period * op->N;
    a.copies = ((unsigned)rows + (unsigned)period - 1) / (unsigned)period;
    a.x = x; a.residual = residual; a.y = y; a.step = (const long long *)step;
    a.k0 = (uint32_t)seed; a.k1 = (uint32_t)(seed >> 32);
    const unsigned long long least = (unsigned long long)nearbyint(p * 4294967296.0);  // kept from this word on
    a.all = least == 0;
    a.last = (uint32_t)(least - 1);
    a.by = p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.0f;
    const cudaError_t e = fp32 || op->dt == SL_FP32 ? launch_dropout<float>(op, a) : launch_dropout<__nv_bfloat16>(op, a);
    return e ? op_cuda(op, e, where) : SL_OK;
}

}  // namespace
}  // namespace sl

using namespace sl;

extern "C" {

sl_status stacklstm_dropout_create(stacklstm_op_t *out, int R, int N, sl_dtype dtype, int device, void *stream)
{
    if (!out) return SL_ERR_ARG;
    *out = nullptr;
    if (R < 1 || N < 1 || (dtype != SL_FP32 && dtype != SL_BF16)) return SL_ERR_ARG;
    if ((long long)R * N > 1LL << 38) return SL_ERR_UNSUPPORTED;  // (CTAs of a launch)
    sl_status st;
    stacklstm_op *op = op_new(SL_OP_DROPOUT, dtype, device, stream, &st);
    if (!op) return st;
    op->R = R;
    op->N = N;
    *out = op;
    return SL_OK;
}

sl_status stacklstm_dropout_forward(stacklstm_op_t op, int rows, const void *x, const void *residual, double p, uint64_t seed,
                                    const int64_t *step, int mask_rows, void *y)
{
    return run(op, rows, x, residual, p, seed, step, mask_rows, y, false, "stacklstm_dropout_forward");
}

sl_status stacklstm_dropout_backward(stacklstm_op_t op, int rows, const float *dy, const float *add, double p, uint64_t seed,
                                     const int64_t *step, int mask_rows, float *dx)
{
    return run(op, rows, dy, add, p, seed, step, mask_rows, dx, true, "stacklstm_dropout_backward");
}

}  // extern "C"
