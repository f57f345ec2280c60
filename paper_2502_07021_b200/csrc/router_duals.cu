// fs_router_duals: entry point, and the kernel (router_duals.cuh) on fp32 scores.
#include "router_duals.cuh"

cudaError_t fsr::run_duals_f32(const DualsArgs &A, bool vec, cudaStream_t st) { return run_duals<float>(A, vec, st); }

extern "C" int fs_router_duals(const void *logits_dev, int dtype, int64_t ld, int64_t tokens, int32_t experts,
                               const uint8_t *mask_dev, const float *target_dev, double eps, int32_t iters,
                               const float *g_start_dev, float *f_out_dev, float *g_out_dev, float *err_out_dev, void *work_dev,
                               int64_t work_bytes, void *stream) {
    using namespace fsr;
    if ((tokens > 0 && !logits_dev) || !g_out_dev || !work_dev) return FS_ERR_NULL;
    if ((dtype != FS_F32 && dtype != FS_BF16 && dtype != FS_F16) || tokens < 0 || experts < 1 || (tokens > 1 && ld < experts) || iters < 1)
        return FS_ERR_BAD_N;
    // eps and log2(e) / eps are used as fp32
    if (!(eps > 0) || !isfinite((float)eps) || !((float)eps > 0) || !isfinite((float)(1.4426950408889634 / eps))) return FS_ERR_BAD_EPS;
    if (experts > FS_ROUTER_MAX_EXPERTS || tokens > INT32_MAX || work_bytes < workspace_bytes(tokens, experts, 1))
        return FS_ERR_TOO_LARGE;
    if ((reinterpret_cast<uintptr_t>(work_dev) & 15) || reinterpret_cast<uintptr_t>(logits_dev) % type_size(dtype))
        return FS_ERR_UNSUPPORTED;
    DualsArgs A;
    A.logits = logits_dev, A.ld = ld, A.tokens = tokens, A.E = experts, A.iters = iters, A.mask = mask_dev;
    A.target = target_dev, A.g_start = g_start_dev, A.eps = (float)eps, A.scale = (float)(1.4426950408889634 / eps);
    A.f = f_out_dev, A.g = g_out_dev, A.err = err_out_dev;
    A.counter = static_cast<unsigned *>(work_dev);
    A.total = reinterpret_cast<unsigned long long *>(static_cast<char *>(work_dev) + 256);
    A.part_log = nullptr, A.fix = 0, A.cached = A.log_parts = 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool vec = rows_aligned(logits_dev, ld, dtype);
    const cudaError_t e = dtype == FS_F32 ? run_duals_f32(A, vec, st) : dtype == FS_BF16 ? run_duals_bf16(A, vec, st) : run_duals_f16(A, vec, st);
    return e == cudaSuccess ? FS_OK : fsk_cuda_failed(e, "fs_router_duals");
}
