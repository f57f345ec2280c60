// The balance's kernel (router_duals.cuh) on fp16 scores.
#include "router_duals.cuh"

cudaError_t fsr::run_duals_f16(const DualsArgs &A, bool vec, cudaStream_t st) { return run_duals<__half>(A, vec, st); }
