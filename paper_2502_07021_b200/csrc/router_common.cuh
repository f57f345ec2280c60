// Shared by the router kernels (router.cu, router_duals.cu): a row of E logits is held in the registers of a group of G
// lanes, NE entries each; loads in the caller's type, arithmetic in fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <atomic>

#include "fs_internal.cuh"

namespace fsr {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f32<__half>(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ float rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float lg2(float x) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// two 16-bit numbers of a word, and back (rounded to nearest even)
template <typename T> __device__ __forceinline__ void both(uint32_t w, float &a, float &b);
template <> __device__ __forceinline__ void both<__nv_bfloat16>(uint32_t w, float &a, float &b) {
    a = __uint_as_float(w << 16), b = __uint_as_float(w & 0xffff0000u);
}
template <> __device__ __forceinline__ void both<__half>(uint32_t w, float &a, float &b) {
    const float2 f = __half22float2(*reinterpret_cast<__half2 *>(&w));
    a = f.x, b = f.y;
}
template <typename T> __device__ __forceinline__ uint32_t joined(float a, float b);
template <> __device__ __forceinline__ uint32_t joined<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <> __device__ __forceinline__ uint32_t joined<__half>(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
// two fp32 operations per instruction
struct Pair {
    unsigned long long v;
};
__device__ __forceinline__ Pair pair(float a, float b) {
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(a), "f"(b));
    return p;
}
__device__ __forceinline__ void split(Pair p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.v)); }
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
template <int BYTES> struct Word;
template <> struct Word<2> { typedef uint16_t type; };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<8> { typedef uint2 type; };
template <> struct Word<16> { typedef uint4 type; };

// Entry i of lane `sub` (0 .. G-1) is column (i / VW * G + sub) * VW + i % VW: chunks of VW consecutive columns, one
// load of VW * sizeof(T) <= 16 bytes each, dealt round robin to the lanes.  VEC needs rows that start on such a
// boundary; without it VW = 1.
template <typename T, int G, int NE, bool VEC> struct RowMap {
    static constexpr int kMaxVW = 16 / (int)sizeof(T);
    static constexpr int VW = VEC ? (NE < kMaxVW ? NE : kMaxVW) : 1;
    static constexpr int CH = NE / VW;
    typedef typename Word<VW * (int)sizeof(T)>::type W;

    __device__ static __forceinline__ int col(int i, int sub) { return ((i / VW) * G + sub) * VW + i % VW; }

    // A row as loaded, to be taken apart later: the loads can be under way while another row is worked on.
    struct Raw {
        W w[CH];
    };
    __device__ static __forceinline__ void load_raw(const T *row, int E, int sub, Raw &r) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e0 = (c * G + sub) * VW;
            if (e0 + VW <= E) {
                r.w[c] = *reinterpret_cast<const W *>(row + e0);
            } else {
                union {
                    W w;
                    T t[VW];
                } u;
#pragma unroll
                for (int v = 0; v < VW; ++v) u.t[v] = e0 + v < E ? row[e0 + v] : from_f32<T>(-INFINITY);
                r.w[c] = u.w;
            }
        }
    }
    // a row with every column closed
    __device__ static __forceinline__ void empty(Raw &r) {
        union {
            W w;
            T t[VW];
        } u;
#pragma unroll
        for (int v = 0; v < VW; ++v) u.t[v] = from_f32<T>(-INFINITY);
#pragma unroll
        for (int c = 0; c < CH; ++c) r.w[c] = u.w;
    }
    // columns beyond E are -inf
    __device__ static __forceinline__ void unpack(const Raw &r, float (&x)[NE]) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            union {
                W w;
                T t[VW];
                uint32_t u[(VW * (int)sizeof(T) + 3) / 4];
            } u;
            u.w = r.w[c];
            if constexpr (sizeof(T) == 2 && VW >= 2) {
#pragma unroll
                for (int v = 0; v < VW / 2; ++v) both<T>(u.u[v], x[c * VW + 2 * v], x[c * VW + 2 * v + 1]);
            } else {
#pragma unroll
                for (int v = 0; v < VW; ++v) x[c * VW + v] = to_f32<T>(u.t[v]);
            }
        }
    }
    // a row of fp32 numbers in shared memory (16-byte aligned), one entry per column
    __device__ static __forceinline__ void read(const float *row, int sub, float (&x)[NE]) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const float *p = row + (c * G + sub) * VW;
            if constexpr (VW % 4 == 0) {
#pragma unroll
                for (int v = 0; v < VW / 4; ++v) {
                    const float4 q = reinterpret_cast<const float4 *>(p)[v];
                    x[c * VW + 4 * v] = q.x, x[c * VW + 4 * v + 1] = q.y, x[c * VW + 4 * v + 2] = q.z, x[c * VW + 4 * v + 3] = q.w;
                }
            } else {
#pragma unroll
                for (int v = 0; v < VW; ++v) x[c * VW + v] = p[v];
            }
        }
    }
    __device__ static __forceinline__ void load(const T *row, int E, int sub, float (&x)[NE]) {
        Raw r;
        load_raw(row, E, sub, r);
        unpack(r, x);
    }
    __device__ static __forceinline__ void store(T *row, int E, int sub, const float (&x)[NE]) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e0 = (c * G + sub) * VW;
            union {
                W w;
                T t[VW];
                uint32_t u[(VW * (int)sizeof(T) + 3) / 4];
            } u;
            if constexpr (sizeof(T) == 2 && VW >= 2) {
#pragma unroll
                for (int v = 0; v < VW / 2; ++v) u.u[v] = joined<T>(x[c * VW + 2 * v], x[c * VW + 2 * v + 1]);
            } else {
#pragma unroll
                for (int v = 0; v < VW; ++v) u.t[v] = from_f32<T>(x[c * VW + v]);
            }
            if (e0 + VW <= E) {
                *reinterpret_cast<W *>(row + e0) = u.w;
            } else {
#pragma unroll
                for (int v = 0; v < VW; ++v)
                    if (e0 + v < E) row[e0 + v] = u.t[v];
            }
        }
    }
};

// all-reduce over the G lanes of a group; the order of the additions is the same in every lane
template <int G> __device__ __forceinline__ float group_sum(float x) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
template <int G> __device__ __forceinline__ float group_max(float x) {
    if constexpr (G == 32) { // one instruction for a whole warp; like fmaxf it passes over a NaN
        asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(x) : "f"(x));
    } else {
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    }
    return x;
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a float of another block of the cluster, by the address that it has here
__device__ __forceinline__ float remote(const float *p, uint32_t rank) {
    uint32_t a;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

// Calls F.template run<T, G, NE, VEC>() for the instance that serves E experts of type dtype: the fewest lanes that hold
// a row with at most 8 entries each up to 256 experts (so that several rows share a warp), a whole warp beyond.
template <typename F, typename T, bool VEC> cudaError_t by_experts(F &f, int E) {
    if (E <= 16) return f.template run<T, 4, 4, VEC>();
    if (E <= 32) return f.template run<T, 8, 4, VEC>();
    if (E <= 64) return f.template run<T, 8, 8, VEC>();
    if (E <= 128) return f.template run<T, 16, 8, VEC>();
    if (E <= 256) return f.template run<T, 32, 8, VEC>();
    if (E <= 512) return f.template run<T, 32, 16, VEC>();
    return f.template run<T, 32, 32, VEC>();
}
template <typename F> cudaError_t by_type(F &f, int dtype, int E, bool vec) {
    switch (dtype) {
    case FS_F32: return vec ? by_experts<F, float, true>(f, E) : by_experts<F, float, false>(f, E);
    case FS_BF16: return vec ? by_experts<F, __nv_bfloat16, true>(f, E) : by_experts<F, __nv_bfloat16, false>(f, E);
    default: return vec ? by_experts<F, __half, true>(f, E) : by_experts<F, __half, false>(f, E);
    }
}
// The same with 16 entries per lane (fewer lanes per row, so fewer shuffles per entry), for kernels that keep little else.
template <typename F, typename T, bool VEC> cudaError_t by_experts_wide(F &f, int E) {
    if (E <= 16) return f.template run<T, 1, 16, VEC>();
    if (E <= 32) return f.template run<T, 2, 16, VEC>();
    if (E <= 64) return f.template run<T, 4, 16, VEC>();
    if (E <= 128) return f.template run<T, 8, 16, VEC>();
    if (E <= 256) return f.template run<T, 16, 16, VEC>();
    if (E <= 512) return f.template run<T, 32, 16, VEC>();
    return f.template run<T, 32, 32, VEC>();
}
inline int type_size(int dtype) { return dtype == FS_F32 ? 4 : 2; }
// rows that start on 16-byte boundaries (the widest load of any instance)
inline bool rows_aligned(const void *p, int64_t ld, int dtype) {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld * type_size(dtype)) % 16 == 0;
}
inline int current_device() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) {
        cudaGetLastError();
        return 0;
    }
    return dev;
}
inline int sm_count() { // looked up once per device
    static std::atomic<int> known[64];
    const int dev = current_device();
    int sms = dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0;
    if (sms > 0) return sms;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) {
        cudaGetLastError();
        return 148;
    }
    if (dev < 64) known[dev].store(sms, std::memory_order_relaxed);
    return sms;
}
// What has to be done once per device and kernel (attributes of a kernel): run() until it succeeded on this device.
struct OncePerDevice {
    std::atomic<uint64_t> done{0};
    template <typename F> cudaError_t operator()(F &&run) {
        const int dev = current_device();
        const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
        if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
        const cudaError_t e = run();
        if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
        return e;
    }
};

// the layout of fs_router_workspace's bytes
constexpr int kMaxBlocks = 1024;  // blocks that leave partial sums
// Pairs per block of the dispatch: a multiple of 2048 that keeps the blocks, each of which adds up all blocks' counts, at 512 or fewer.
constexpr int kChunkPairs = 2048;
inline int64_t chunk_pairs(int64_t pairs) { return kChunkPairs * ((pairs + 512 * kChunkPairs - 1) / (512 * kChunkPairs) + (pairs == 0)); }
int64_t workspace_bytes(int64_t tokens, int32_t experts, int32_t topk);

} // namespace fsr
