// op.cu -- what the output-layer and search operators have in common: the handle's life, its
// stream, its status word and workspace, and their C ABI (include/stacklstm.h, stacklstm_op_*).
#include <stdlib.h>

#include "op.cuh"

namespace sl {

sl_status op_fail(stacklstm_op *op, sl_status st, const char *msg)
{
    if (op) snprintf(op->last_error, sizeof op->last_error, "%s", msg);
    return st;
}

sl_status op_cuda(stacklstm_op *op, cudaError_t e, const char *where)
{
    if (op) snprintf(op->last_error, sizeof op->last_error, "%s: %s", where, cudaGetErrorString(e));
    return e == cudaErrorMemoryAllocation ? SL_ERR_OOM : SL_ERR_CUDA;
}

stacklstm_op *op_new(int kind, sl_dtype dt, int device, void *stream, sl_status *st)
{
    *st = SL_ERR_OOM;
    stacklstm_op *op = new (std::nothrow) stacklstm_op;
    if (!op) return nullptr;
    op->kind = kind;
    op->dt = dt;
    op->device = device;
    op->stream = (cudaStream_t)stream;
    const char *limit = getenv("STACKLSTM_WAIT_LIMIT_CYCLES");  // test hook (include/stacklstm.h)
    op->wait_limit = limit ? atoll(limit) : 4000000000LL;
    int devices = 0;
    if (cudaGetDeviceCount(&devices) != cudaSuccess || device < 0 || device >= devices) {
        cudaGetLastError();
        delete op;
        *st = SL_ERR_ARG;  // no such device
        return nullptr;
    }
    OpDevice guard(device);
    bool ok = cudaDeviceGetAttribute(&op->num_sms, cudaDevAttrMultiProcessorCount, device) == cudaSuccess;
    if (ok) ok = cudaMalloc((void **)&op->err, 16) == cudaSuccess;
    // (on the handle's stream, as every clearing: cudaMemset is ordered with the default stream's work
    // alone, and a stream that does not wait for that one could have a call's work before it)
    if (ok) ok = cudaMemsetAsync(op->err, 0, 16, op->stream) == cudaSuccess;
    if (!ok) {
        cudaGetLastError();
        stacklstm_op_destroy(op);
        return nullptr;
    }
    *st = SL_OK;
    return op;
}

cudaError_t op_workspace(stacklstm_op *op, int i, size_t bytes)
{
    if (bytes <= op->ws_bytes[i]) return cudaSuccess;
    cudaError_t e = cudaSuccess;
    if (op->ws[i]) {
        if ((e = cudaStreamSynchronize(op->stream))) return e;
        if ((e = cudaFree(op->ws[i]))) return e;
        op->ws[i] = nullptr;
        op->ws_bytes[i] = 0;
    }
    if ((e = cudaMalloc(&op->ws[i], bytes))) {
        op->ws[i] = nullptr;
        cudaGetLastError();  // reported by this call's status alone
        return e;
    }
    op->ws_bytes[i] = bytes;
    return cudaSuccess;
}

}  // namespace sl

using namespace sl;

extern "C" {

sl_status stacklstm_op_set_stream(stacklstm_op_t op, void *stream)
{
    if (!op) return SL_ERR_ARG;
    OpDevice guard(op->device);
    // work queued on the old stream still uses the workspace
    const cudaError_t e = op->stream == (cudaStream_t)stream ? cudaSuccess : cudaStreamSynchronize(op->stream);
    if (e) return op_cuda(op, e, "stacklstm_op_set_stream");
    op->stream = (cudaStream_t)stream;
    return SL_OK;
}

sl_status stacklstm_op_status(stacklstm_op_t op)
{
    if (!op) return SL_ERR_ARG;
    OpDevice guard(op->device);
    int32_t v = 0;
    cudaError_t e = cudaStreamSynchronize(op->stream);
    if (!e) e = cudaMemcpy(&v, op->err, 4, cudaMemcpyDeviceToHost);
    if (!e && v) e = cudaMemsetAsync(op->err, 0, 4, op->stream);
    if (e) return op_cuda(op, e, "stacklstm_op_status");
    if (v == SL_ERR_TIMEOUT) return op_fail(op, SL_ERR_TIMEOUT, "a device-side wait of a contraction ran out");
    if (v == SL_ERR_OP) return op_fail(op, SL_ERR_OP, "an op outside {-1, 0, +1} ran as a hold");
    if (v == SL_ERR_UNDERFLOW) return op_fail(op, SL_ERR_UNDERFLOW, "a pop at depth 0 ran as a hold");
    if (v == SL_ERR_ARG) return op_fail(op, SL_ERR_ARG, "an index outside its range was skipped");
    if (v) return op_fail(op, (sl_status)v, "a device-detected error");
    return SL_OK;
}

sl_status stacklstm_op_destroy(stacklstm_op_t op)
{
    if (!op) return SL_OK;
    {
        OpDevice guard(op->device);
        cudaStreamSynchronize(op->stream);
        if (op->err) cudaFree(op->err);
        for (void *p : op->ws)
            if (p) cudaFree(p);
    }
    delete op;
    return SL_OK;
}

const char *stacklstm_op_last_error(stacklstm_op_t op) { return op ? op->last_error : "null handle"; }

}  // extern "C"
