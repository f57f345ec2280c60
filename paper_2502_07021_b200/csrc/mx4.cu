// fs_mx4_quantize / fs_mx4_dequantize: rows of fp32, bf16 or fp16 to the microscaled 4-bit form and back.
//
// Four lanes share a block of 32 columns, eight consecutive columns each: one 16-byte load (two for fp32), a maximum of
// eight, two shuffles for the block's maximum, the scale exponent from the maximum's exponent bits, eight exact products with a
// power of two, four conversions (cvt.rn.satfinite.e2m1x2), one 4-byte store.  Both directions are bound by HBM: what
// they move is the matrix once and its 17/32-byte-per-entry packed form once.
// 16384 x 8192 bf16: 58 - 60 us to 4 bits and as much back, 340 MB each way, 5.7 - 5.9 TB/s (0.88 - 0.91 of the copy rate).  Rows on
// odd addresses go element by element: 109 and 350 us with a pitch of 8193.  One span per warp at a time:
// 116 and 75 us; four spans with fp32 arithmetic throughout: 89 and 82, 66 % of the issue slots busy -- hence the packed 16-bit maxima
// and products, and the decoding by byte permutes.
#include "router_common.cuh"

namespace fsr {
namespace {

constexpr int kThreads = 256;

constexpr int kWarps = kThreads / 32;
constexpr int kSpan = 256; // columns of a warp step: eight per lane

// eight consecutive entries as loaded: 16 bytes (32 for fp32)
template <typename T> struct Raw8 {
    static constexpr int N = 16 / (int)sizeof(T), W = 8 / N;
    union {
        uint4 w[W];
        T t[8];
    };
};
template <typename T> __device__ __forceinline__ void load8(const T *p, bool vec, int valid, Raw8<T> &r) {
    if (vec && valid >= 8) {
#pragma unroll
        for (int h = 0; h < Raw8<T>::W; ++h)
            asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(r.w[h].x), "=r"(r.w[h].y), "=r"(r.w[h].z), "=r"(r.w[h].w)
                         : "l"(reinterpret_cast<const uint4 *>(p) + h));
    } else {
#pragma unroll
        for (int v = 0; v < 8; ++v) r.t[v] = v < valid ? p[v] : from_f32<T>(0.f);
    }
}

// eight values -> eight codes, the first in the lowest nibble
__device__ __forceinline__ uint32_t e2m1x8(const float (&v)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 t0, t1, t2, t3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 t0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 t1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 t2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 t3, %8, %7;\n\t"
        "mov.b32 %0, {t0, t1, t2, t3};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// Largest magnitude of a block as fp32 bits: magnitudes compare like their bits, and a NaN's are above infinity's.  The
// 16-bit types are compared two at a time.
__device__ __forceinline__ uint32_t block_max(const Raw8<float> &r) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(r.t[i]) & 0x7fffffffu);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    return max(top, __shfl_xor_sync(0xffffffffu, top, 2));
}
template <typename T> __device__ __forceinline__ uint32_t block_max(const Raw8<T> &r) {
    constexpr uint32_t M = 0x7fff7fffu;
    uint32_t top = __vmaxu2(__vmaxu2(r.w[0].x & M, r.w[0].y & M), __vmaxu2(r.w[0].z & M, r.w[0].w & M));
    top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 2));
    union {
        uint16_t u;
        T t;
    } o;
    o.u = (uint16_t)max(top & 0xffffu, top >> 16);
    return __float_as_uint(to_f32<T>(o.t));
}
// the entries times a power of two: exact, or so small that they round to zero
template <typename T> __device__ __forceinline__ void scaled(const Raw8<T> &r, float unit, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32<T>(r.t[i]) * unit;
}
template <> __device__ __forceinline__ void scaled<__nv_bfloat16>(const Raw8<__nv_bfloat16> &r, float unit, float (&v)[8]) {
    const __nv_bfloat162 u2 = __float2bfloat162_rn(unit); // bf16 has fp32's exponents
    const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        union {
            __nv_bfloat162 b;
            uint32_t u;
        } m;
        m.u = w[i];
        m.b = __hmul2(m.b, u2);
        v[2 * i] = __uint_as_float(m.u << 16), v[2 * i + 1] = __uint_as_float(m.u & 0xffff0000u);
    }
}

// A warp takes U spans of 256 columns of one row: all its loads are under way before the first is used.  blockIdx.y =
// group of U spans, warps along the rows.
template <typename T, int U>
__global__ void __launch_bounds__(kThreads)
mx4_quantize_kernel(const T *x, int64_t ld, int64_t src_rows, int64_t cols, const int32_t *slot, int copies, int64_t rows,
                    uint8_t *q, int64_t q_pitch, uint8_t *s, int64_t s_pitch, int vec) {
    const int lane = threadIdx.x & 31;
    const int nb = (int)((cols + 31) / 32), nb4 = (nb + 3) & ~3;
    const int b0 = blockIdx.y * (U * kSpan / 32); // first block of 32 columns
    const bool full = vec && (int64_t)b0 * 32 + U * kSpan <= cols;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int64_t r = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); r < src_rows; r += (int64_t)gridDim.x * kWarps) {
        Raw8<T> raw[U];
        if (full) {
            const T *p = x + r * ld + (int64_t)b0 * 32 + lane * 8;
#pragma unroll
            for (int u = 0; u < U; ++u) load8<T>(p + u * kSpan, true, 8, raw[u]);
        } else {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int64_t c0 = ((int64_t)b0 + u * (kSpan / 32)) * 32 + lane * 8, left = cols - c0;
            load8<T>(x + r * ld + c0, vec != 0, left > 8 ? 8 : left < 0 ? 0 : (int)left, raw[u]);
          }
        }
        uint32_t code[U], word[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int ex = (int)(block_max(raw[u]) >> 23); // biased exponent of the maximum; 0 below 2^-126
            const uint32_t sb = ex >= 255 ? 255u : (uint32_t)max(ex - 2, 0);
            // 2^-X = 2^(127 - sb): bits of an exponent 254 - sb, in 2 .. 254
            const float unit = __uint_as_float((254u - (ex >= 255 ? 0u : sb)) << 23);
            float v[8];
            scaled<T>(raw[u], unit, v);
            code[u] = ex >= 255 ? 0u : e2m1x8(v);
            // four neighbouring blocks' scales as one word
            const int b = b0 + u * (kSpan / 32) + (lane >> 2);
            const uint32_t mine = full || b < nb ? sb << (8 * ((lane >> 2) & 3)) : 0u;
            word[u] = mine | __shfl_xor_sync(0xffffffffu, mine, 4);
            word[u] |= __shfl_xor_sync(0xffffffffu, word[u], 8);
        }
        for (int j = 0; j < copies; ++j) {
            const int64_t to = slot ? slot[r * copies + j] : r;
            if (to < 0 || to >= rows) continue;
            uint32_t *qo = reinterpret_cast<uint32_t *>(q + to * q_pitch + (int64_t)b0 * 16) + lane;
            uint32_t *so = reinterpret_cast<uint32_t *>(s + to * s_pitch + b0) + (lane >> 4);
            if (full) {
#pragma unroll
                for (int u = 0; u < U; ++u) qo[u * (kSpan / 8)] = code[u];
                if ((lane & 15) == 0) {
#pragma unroll
                    for (int u = 0; u < U; ++u) so[u * (kSpan / 128)] = word[u];
                }
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int b = b0 + u * (kSpan / 32) + (lane >> 2);
                    if (b < nb) qo[u * (kSpan / 8)] = code[u];
                    if ((lane & 15) == 0 && b < nb4) so[u * (kSpan / 128)] = word[u];
                }
            }
        }
    }
}

// Codes -> bf16: the eight magnitudes' high and low bytes are looked up by byte permutes, four codes at a time, the signs
// moved to bits 15 and 31.  w[i] holds codes 2i and 2i + 1.
__device__ __forceinline__ void e2m1_to_bf16(uint32_t code, uint32_t (&w)[4]) {
    constexpr uint32_t H0 = 0x3f3f3f00u, H1 = 0x40404040u; // 0 .5 1 1.5 | 2 3 4 6
    constexpr uint32_t L0 = 0xc0800000u, L1 = 0xc0804000u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t c = h ? code >> 16 : code, sel = c & 0x7777u;
        const uint32_t hi = __byte_perm(H0, H1, sel), lo = __byte_perm(L0, L1, sel);
        w[2 * h] = __byte_perm(lo, hi, 0x5140) | ((c << 12) & 0x8000u) | ((c << 24) & 0x80000000u);
        w[2 * h + 1] = __byte_perm(lo, hi, 0x7362) | ((c << 4) & 0x8000u) | ((c << 16) & 0x80000000u);
    }
}
template <typename T> __device__ __forceinline__ void decode8(uint32_t code, float unit, Raw8<T> &o) {
    uint32_t w[4];
    e2m1_to_bf16(code, w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        o.t[2 * i] = from_f32<T>(__uint_as_float(w[i] << 16) * unit);
        o.t[2 * i + 1] = from_f32<T>(__uint_as_float(w[i] & 0xffff0000u) * unit);
    }
}
template <> __device__ __forceinline__ void decode8<__nv_bfloat16>(uint32_t code, float unit, Raw8<__nv_bfloat16> &o) {
    uint32_t w[4];
    e2m1_to_bf16(code, w);
    const __nv_bfloat162 u2 = __float2bfloat162_rn(unit); // exact, and so are the products
    union {
        __nv_bfloat162 b;
        uint32_t u;
    } m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i].u = w[i];
        m[i].b = __hmul2(m[i].b, u2);
    }
    o.w[0] = make_uint4(m[0].u, m[1].u, m[2].u, m[3].u);
}
// 2^(s - 127); NaN for 255
__device__ __forceinline__ float unit_of(uint32_t s) {
    return s == 255 ? NAN : s == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23);
}

// The same division of the work.
template <typename T, int U>
__global__ void __launch_bounds__(kThreads)
mx4_dequantize_kernel(const uint8_t *q, int64_t q_pitch, const uint8_t *s, int64_t s_pitch, int64_t rows, int64_t cols, T *out,
                      int64_t ldo, int vec) {
    const int lane = threadIdx.x & 31;
    const int64_t c0 = (int64_t)blockIdx.y * (U * kSpan) + lane * 8;
    const bool full = vec && (int64_t)(blockIdx.y + 1) * (U * kSpan) <= cols;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int64_t r = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); r < rows; r += (int64_t)gridDim.x * kWarps) {
        const uint32_t *qi = reinterpret_cast<const uint32_t *>(q + r * q_pitch + c0 / 2);
        const uint8_t *si = s + r * s_pitch + c0 / 32;
        T *to = out + r * ldo + c0;
        uint32_t code[U], sb[U];
        if (full) {
#pragma unroll
            for (int u = 0; u < U; ++u) code[u] = __ldg(qi + u * (kSpan / 8)), sb[u] = __ldg(si + u * (kSpan / 32));
#pragma unroll
            for (int u = 0; u < U; ++u) {
                Raw8<T> o;
                decode8<T>(code[u], unit_of(sb[u]), o);
#pragma unroll
                for (int h = 0; h < Raw8<T>::W; ++h) reinterpret_cast<uint4 *>(to + u * kSpan)[h] = o.w[h];
            }
            continue;
        }
#pragma unroll 1
        for (int u = 0; u < U; ++u) {
            const int64_t c = c0 + u * kSpan;
            if (c >= cols) break;
            Raw8<T> o;
            decode8<T>(__ldg(qi + u * (kSpan / 8)), unit_of(__ldg(si + u * (kSpan / 32))), o);
            T *p = to + u * kSpan;
            if (vec && c + 8 <= cols) {
#pragma unroll
                for (int h = 0; h < Raw8<T>::W; ++h) reinterpret_cast<uint4 *>(p)[h] = o.w[h];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < cols) p[i] = o.t[i];
            }
        }
    }
}

int check_packed(const void *q, int64_t q_pitch, const void *s, int64_t s_pitch, int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1) return FS_ERR_BAD_N;
    if (cols > FS_MX4_MAX_COLS) return FS_ERR_TOO_LARGE;
    const int64_t nb = (cols + 31) / 32;
    if (q_pitch < 16 * nb || (q_pitch & 15) || s_pitch < nb || (s_pitch & 3)) return FS_ERR_BAD_N;
    if (rows > 0 && (!q || !s)) return FS_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(q) & 15) || (reinterpret_cast<uintptr_t>(s) & 3)) return FS_ERR_UNSUPPORTED;
    return FS_OK;
}
// Spans per warp: four when that still leaves eight warps per SM, so that large matrices have many loads under way and
// small ones many warps.
int spans_per_warp(int64_t rows, int64_t cols) {
    return rows * ((cols + 4 * kSpan - 1) / (4 * kSpan)) >= 8 * (int64_t)sm_count() && cols > kSpan ? 4 : 1;
}
template <typename... Params, typename... Args>
cudaError_t launch_rows(void (*kernel)(Params...), int spans, int64_t rows, int64_t cols, cudaStream_t st, Args... args) {
    const int64_t groups = (cols + (int64_t)spans * kSpan - 1) / ((int64_t)spans * kSpan);
    const int64_t along = (rows + kWarps - 1) / kWarps, limit = 1 << 20;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(along < limit ? along : limit), (unsigned)groups), cfg.blockDim = dim3(kThreads), cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr, cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <typename T>
cudaError_t quantize(const void *x, int64_t ld, int64_t src_rows, int64_t cols, const int32_t *slot, int copies, int64_t rows,
                     void *q, int64_t q_pitch, void *s, int64_t s_pitch, bool vec, cudaStream_t st) {
    const int u = spans_per_warp(src_rows, cols);
    return launch_rows(u == 4 ? mx4_quantize_kernel<T, 4> : mx4_quantize_kernel<T, 1>, u, src_rows, cols, st,
                       static_cast<const T *>(x), ld, src_rows, cols, slot, copies, rows, static_cast<uint8_t *>(q), q_pitch,
                       static_cast<uint8_t *>(s), s_pitch, (int)vec);
}
template <typename T>
cudaError_t dequantize(const void *q, int64_t q_pitch, const void *s, int64_t s_pitch, int64_t rows, int64_t cols, void *out,
                       int64_t ldo, bool vec, cudaStream_t st) {
    const int u = spans_per_warp(rows, cols);
    return launch_rows(u == 4 ? mx4_dequantize_kernel<T, 4> : mx4_dequantize_kernel<T, 1>, u, rows, cols, st,
                       static_cast<const uint8_t *>(q), q_pitch, static_cast<const uint8_t *>(s), s_pitch, rows, cols,
                       static_cast<T *>(out), ldo, (int)vec);
}

} // namespace
} // namespace fsr

extern "C" int fs_mx4_quantize(const void *x_dev, int dtype, int64_t ld, int64_t src_rows, int64_t cols,
                               const int32_t *slot_dev, int32_t copies, int64_t rows, void *q_out, int64_t q_pitch,
                               void *s_out, int64_t s_pitch, void *stream) {
    using namespace fsr;
    if (dtype != FS_F32 && dtype != FS_BF16 && dtype != FS_F16) return FS_ERR_BAD_N;
    if (int rc = check_packed(q_out, q_pitch, s_out, s_pitch, rows, cols)) return rc;
    if ((src_rows > 1 && ld < cols) || src_rows < 0 || copies < 1 || (!slot_dev && src_rows > 0 && (copies != 1 || rows < src_rows))) return FS_ERR_BAD_N;
    if (rows == 0 || src_rows == 0) return FS_OK;
    if (!x_dev) return FS_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(x_dev) % type_size(dtype)) return FS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool vec = rows_aligned(x_dev, ld, dtype);
    cudaError_t e;
    if (dtype == FS_F32) e = quantize<float>(x_dev, ld, src_rows, cols, slot_dev, copies, rows, q_out, q_pitch, s_out, s_pitch, vec, st);
    else if (dtype == FS_BF16) e = quantize<__nv_bfloat16>(x_dev, ld, src_rows, cols, slot_dev, copies, rows, q_out, q_pitch, s_out, s_pitch, vec, st);
    else e = quantize<__half>(x_dev, ld, src_rows, cols, slot_dev, copies, rows, q_out, q_pitch, s_out, s_pitch, vec, st);
    return e == cudaSuccess ? FS_OK : fsk_cuda_failed(e, "fs_mx4_quantize");
}

extern "C" int fs_mx4_dequantize(const void *q_dev, int64_t q_pitch, const void *s_dev, int64_t s_pitch, int64_t rows,
                                 int64_t cols, void *out, int dtype, int64_t ldo, void *stream) {
    using namespace fsr;
    if (dtype != FS_F32 && dtype != FS_BF16 && dtype != FS_F16) return FS_ERR_BAD_N;
    if (int rc = check_packed(q_dev, q_pitch, s_dev, s_pitch, rows, cols)) return rc;
    if (rows > 1 && ldo < cols) return FS_ERR_BAD_N;
    if (rows == 0) return FS_OK;
    if (!out) return FS_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(out) % type_size(dtype)) return FS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool vec = rows_aligned(out, ldo, dtype);
    cudaError_t e;
    if (dtype == FS_F32) e = dequantize<float>(q_dev, q_pitch, s_dev, s_pitch, rows, cols, out, ldo, vec, st);
    else if (dtype == FS_BF16) e = dequantize<__nv_bfloat16>(q_dev, q_pitch, s_dev, s_pitch, rows, cols, out, ldo, vec, st);
    else e = dequantize<__half>(q_dev, q_pitch, s_dev, s_pitch, rows, cols, out, ldo, vec, st);
    return e == cudaSuccess ? FS_OK : fsk_cuda_failed(e, "fs_mx4_dequantize");
}
