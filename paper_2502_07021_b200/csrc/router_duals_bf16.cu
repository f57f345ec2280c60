// The balance's kernel (router_duals.cuh) on bf16 scores.
#include "router_duals.cuh"

cudaError_t fsr::run_duals_bf16(const DualsArgs &A, bool vec, cudaStream_t st) { return run_duals<__nv_bfloat16>(A, vec, st); }
