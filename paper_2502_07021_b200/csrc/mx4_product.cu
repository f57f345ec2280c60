// fs_mx4_product: rows of microscaled 4-bit values times the transposed 4-bit weights of their group, on the tensor cores.
//
// y_rn = sum_k x_rk w_gnk for the rows r of group g.  Both operands are contiguous along k, which is what
// tcgen05.mma.kind::mxf4.block_scale multiplies: 64 k-values per instruction, each 32 of a row scaled by its own power of
// two taken from tensor memory, exact products, fp32 accumulation in tensor memory.  The weights are the M side (128
// rows of a weight matrix, i.e. outputs), the rows of x the N side, in tiles of NT that the host picks from the mean group
// size: a decode step with one row per group fills a 16-wide tile instead of a 128-wide one.
//
// One persistent CTA per SM; tile list = (row tile of a group) x (128 outputs), laid out from the offsets by every CTA itself,
// so nothing about the groups has to reach the host.
//   warp 0      TMA: per 256 k-values (128 bytes) a 128-row weight box and an NT-row x box, 128-byte swizzle
//   warps 2-9   scale bytes, two teams in turn: 16 per row (512 k-values) in one load, one step ahead, then stored in the order that
//               tcgen05.cp wants -- 512-byte units of 128 rows and 128 k-values, entry (row % 32) * 16 + (row / 32) * 4 --
//               so scales stay row-major in memory and a tile may start at any row
//   warp 1      tcgen05.cp of the stage's scales into tensor memory (each ring stage has columns of its own), four
//               tcgen05.mma, commit to the stage's barrier
//   warps 10-17 tcgen05.ld of a finished accumulator (two of them, so this overlaps the next tile), rounding, stores
// Every wait is bounded; if one runs out the CTA's remaining outputs become NaN and it leaves.
//
// Bound and measured.  32768 rows in 32 groups, 4096 x 4096: 304 - 314 us, 3.5 PFLOP/s (0.53 of four times the bf16 rate); no single
// part bounds it: without the operand loads 247, the scales 254, three of four matrix instructions 238, the stores 276.  A ring stage
// goes round in about 780 cycles, and tensor memory (504 of 512 columns) and shared memory have no room for a sixth.  One row for each
// of 8 groups, 4096 -> 2048, where 16-wide tiles keep 10 stages of weights under way: 10.9 us for 36 MB of weights from HBM (3.3 TB/s,
// eight sets of groups in turn), 8.1 us when the same 36 MB are still in L2.
// 192 rows per tile is the widest with two accumulators beside the scales' columns.
#include <cuda.h>

#include "router_common.cuh"
#include "tcgen05_ptx.cuh"

namespace fsr {
namespace {
using namespace fstc;
using fsr::ex2;

constexpr int BM = 128;              // outputs per tile
constexpr int KB_BYTES = 128;        // 256 k-values per ring stage
constexpr int kScaleTeam = 4, kScaleWarps = 2 * kScaleTeam, kEpilogueWarps = 8;
constexpr int kThreads = 32 * (2 + kScaleWarps + kEpilogueWarps);
constexpr int W_BYTES = BM * KB_BYTES;

template <int NT> struct Shape {
    static constexpr int RA = (NT + 127) / 128;               // 128-row units of x's scales
    static constexpr int X_BYTES = NT * KB_BYTES;
    static constexpr int SF_BYTES = 2 * 512 * (1 + RA);       // two 128-k units each
    static constexpr int STAGE = W_BYTES + X_BYTES + SF_BYTES;
    static constexpr int STAGES = NT == 192 ? 5 : NT == 128 ? 6 : NT == 64 ? 8 : NT == 32 ? 9 : 10;
    static constexpr int SF_COLS = 8 * (1 + RA);              // tensor-memory columns of a stage's scales
    static constexpr int USED_COLS = 2 * NT + STAGES * SF_COLS;
    static constexpr int COLS = USED_COLS <= 256 ? 256 : 512;
    static constexpr int BARS = 2 * STAGES + 4;
    static_assert(USED_COLS <= 512, "tensor memory");
    // A team of scale warps comes back after at most four ring stages; with four stages or more the stage that it then
    // waits for has at most one use outstanding, so a barrier's phase cannot be mistaken for the one before the last.
    static_assert(STAGES >= 4, "phases");
    static constexpr int smem(int groups) { return 1024 + STAGES * STAGE + 8 * BARS + 16 + 8 * (groups + 1); }
};
static_assert(Shape<192>::smem(FS_MX4_MAX_GROUPS) <= 232448, "shared memory");
static_assert(Shape<128>::smem(FS_MX4_MAX_GROUPS) <= 232448, "shared memory");
static_assert(Shape<64>::smem(FS_MX4_MAX_GROUPS) <= 232448, "shared memory");
static_assert(Shape<32>::smem(FS_MX4_MAX_GROUPS) <= 232448, "shared memory");
static_assert(Shape<16>::smem(FS_MX4_MAX_GROUPS) <= 232448, "shared memory");

struct ProductArgs {
    const uint8_t *xs, *ws;
    int64_t xs_pitch, ws_pitch, ldo;
    int rows, outs, groups, nb, nkb, ntiles_n; // nb: 32-column blocks per row; nkb: ring stages per tile
    int wide;                                  // scale rows can be read 16 bytes at a time
    const int32_t *offsets;
    void *out;
};

// Instruction descriptor of kind::mxf4: A, B e2m1 (1), both along k, scales ue8m0 (bit 23), M = 128; the ids of the two
// scale bytes within their 32-bit word go to bits 29-30 (A) and 4-5 (B).
__host__ __device__ constexpr uint32_t idesc_mxf4(int n, uint32_t id) {
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(BM >> 4) << 24) | (id << 29) | (id << 4);
}
// Unswizzled 32-row x 16-byte unit for tcgen05.cp: 8-row groups of 128 consecutive bytes.
__device__ __forceinline__ uint64_t scale_desc(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFF) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
}
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
}
__device__ __forceinline__ void tma_load_3d(const CUtensorMap *map, uint32_t dst, uint32_t bar, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void st_word(uint32_t addr, uint32_t x) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(x) : "memory"); }

__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

struct Tile {
    int group, row0, rows, n0; // rows: valid ones, at most NT
};

// N accumulator columns of this thread's tensor-memory lane
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&r)[32]) {
    tmem_ld32_issue(taddr, r);
    tmem_ld_wait32(r);
}
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr) : "memory");
}

template <int NT, typename OutT>
__global__ void __launch_bounds__(kThreads, 1)
mx4_product_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const ProductArgs A) {
    typedef Shape<NT> S;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bars = base + S::STAGES * S::STAGE;
    const uint32_t full = bars, empty = bars + 8 * S::STAGES, acc_full = empty + 8 * S::STAGES, acc_empty = acc_full + 16;
    const uint32_t tmem_slot = bars + 8 * S::BARS;
    uint8_t *gbase = smem_raw + (base - smem_u32(smem_raw));
    uint32_t *tmem_slot_ptr = reinterpret_cast<uint32_t *>(gbase + (tmem_slot - base));
    int *tile_start = reinterpret_cast<int *>(gbase + (tmem_slot + 16 - base)); // [groups + 1] row tiles before each group
    int *row_start = tile_start + A.groups + 1;                                 // [groups + 1] offsets, clamped
    __shared__ int scan_w[kThreads / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) {
            mbar_init(full + 8 * s, 1 + kScaleTeam); // TMA thread, one team of scale warps
            mbar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full + 8 * b, 1);
            mbar_init(acc_empty + 8 * b, kEpilogueWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tmem_slot), "r"(S::COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    griddep_launch_dependents();
    griddep_wait(); // everything this kernel reads may come from the one before it

    // offsets, and row tiles per group -> exclusive sums; thread i takes `per` consecutive groups
    for (int g = threadIdx.x; g <= A.groups; g += kThreads)
        row_start[g] = A.offsets ? min(max(__ldg(A.offsets + g), 0), A.rows) : (g == 0 ? 0 : A.rows);
    __syncthreads();
    const int per = (A.groups + kThreads - 1) / kThreads;
    int mine = 0;
    for (int k = 0; k < per; ++k) {
        const int g = threadIdx.x * per + k;
        if (g < A.groups) mine += (max(row_start[g + 1] - row_start[g], 0) + NT - 1) / NT;
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) scan_w[warp] = incl;
    __syncthreads();
    int at = incl - mine;
    for (int w = 0; w < warp; ++w) at += scan_w[w];
    for (int k = 0; k < per; ++k) {
        const int g = threadIdx.x * per + k;
        if (g >= A.groups) break;
        tile_start[g] = at;
        at += (max(row_start[g + 1] - row_start[g], 0) + NT - 1) / NT;
        if (g == A.groups - 1) tile_start[A.groups] = at;
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_slot_ptr;
    const int total = tile_start[A.groups] * A.ntiles_n; // fits: at most rows * outs / 128 and both are 31-bit sized grids

    auto tile_at = [&](int i) {
        Tile t;
        const int rt = i / A.ntiles_n;
        t.n0 = (i % A.ntiles_n) * BM;
        int lo = 0, hi = A.groups - 1; // the last group whose first tile is <= rt
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (tile_start[mid] <= rt) lo = mid;
            else hi = mid - 1;
        }
        t.group = lo;
        t.row0 = row_start[lo] + (rt - tile_start[lo]) * NT;
        t.rows = min(NT, row_start[lo + 1] - t.row0);
        return t;
    };

    // The two issuing warps run their loops with all lanes, so that addresses and descriptors are computed once per warp in
    // uniform registers, and let one elected lane issue.
    bool ok = true;
    if (warp == 0) {
        const bool leader = elect_one();
        int s = 0, issued = 0;
        uint32_t ph = 0;
        for (int i = blockIdx.x; i < total && ok; i += gridDim.x) {
            const Tile t = tile_at(i);
            for (int kb = 0; kb < A.nkb; ++kb) {
                if (!mbar_wait(empty + 8 * s, ph ^ 1u)) { ok = false; break; }
                if (leader) {
                    const uint32_t bar = full + 8 * s, dst = base + s * S::STAGE;
                    mbar_expect_tx(bar, W_BYTES + S::X_BYTES);
                    tma_load_3d(&tm_w, dst, bar, kb * KB_BYTES, t.n0, t.group);
                    tma_load_2d(&tm_x, dst + W_BYTES, bar, kb * KB_BYTES, t.row0);
                }
                ++issued;
                if (++s == S::STAGES) s = 0, ph ^= 1u;
            }
        }
        if (!ok) // copies in flight must land before the shared memory goes away
            for (int j = max(0, issued - S::STAGES); j < issued; ++j)
                (void)mbar_wait(full + 8 * (j % S::STAGES), (uint32_t)(j / S::STAGES) & 1u);
    } else if (warp == 1) {
        const bool leader = elect_one();
        int s = 0, buf = 0;
        uint32_t ph = 0, aph = 0;
        for (int i = blockIdx.x; i < total && ok; i += gridDim.x) {
            if (!mbar_wait(acc_empty + 8 * buf, aph ^ 1u)) { ok = false; break; }
            fence_after();
            const uint32_t acc = tmem + (uint32_t)(buf * NT);
            for (int kb = 0; kb < A.nkb; ++kb) {
                if (!mbar_wait(full + 8 * s, ph)) { ok = false; break; }
                fence_after();
                if (leader) {
                    const uint32_t st = base + s * S::STAGE;
                    const uint64_t sf = scale_desc(st + W_BYTES + S::X_BYTES);
                    const uint32_t tw = tmem + (uint32_t)(2 * NT + s * S::SF_COLS), tx = tw + 8;
#pragma unroll
                    for (int h = 0; h < 2; ++h) { // 128-k units
                        copy_scales(tw + 4 * h, sf + 32 * h);
#pragma unroll
                        for (int r = 0; r < S::RA; ++r) copy_scales(tx + 4 * (h * S::RA + r), sf + 64 + 32 * (h * S::RA + r));
                    }
                    const uint64_t a = make_desc(st), b = make_desc(st + W_BYTES);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_mxf4(acc, a + 2 * kk, b + 2 * kk, idesc_mxf4(NT, (kk & 1) * 2), tw + 4 * (kk >> 1),
                                 tx + 4 * S::RA * (kk >> 1), (kb > 0 || kk > 0) ? 1u : 0u);
                    commit(empty + 8 * s);
                    if (kb == A.nkb - 1) commit(acc_full + 8 * buf);
                }
                if (++s == S::STAGES) s = 0, ph ^= 1u;
            }
            if (++buf == 2) buf = 0, aph ^= 1u;
        }
    } else if (warp < 2 + kScaleWarps) {
        // Scale bytes.  A step is two ring stages, 16 bytes per row; two teams of four warps take the steps in turn, each with
        // its next step's loads under way in registers.  Lane l of a team's warp q has the rows q * 8 + l / 4 + 32 (l % 4) of
        // each 128, so that a warp's stores are 128 consecutive bytes.
        const int team = (warp - 2) / kScaleTeam;
        const int r0 = ((warp - 2) % kScaleTeam) * 8 + (lane >> 2) + 32 * (lane & 3);
        constexpr int RX = (NT + 127) / 128;
        int s = 0;
        uint32_t ph = 0;
        auto fetch_row = [&](const uint8_t *row, int b0, uint4 &v) {
            v = make_uint4(0u, 0u, 0u, 0u);
            const int left = A.nb - b0;
            if (A.wide) {
                v = __ldg(reinterpret_cast<const uint4 *>(row + b0));
            } else {
                const uint32_t *w = reinterpret_cast<const uint32_t *>(row + b0);
                v.x = __ldg(w);
                if (left > 4) v.y = __ldg(w + 1);
                if (left > 8) v.z = __ldg(w + 2);
                if (left > 12) v.w = __ldg(w + 3);
            }
            if (left < 16) { // bytes behind the row's last block are not scales
                auto keep = [&](uint32_t x, int n) { return n >= 4 ? x : n <= 0 ? 0u : x & ((1u << (8 * n)) - 1u); };
                v.x = keep(v.x, left), v.y = keep(v.y, left - 4), v.z = keep(v.z, left - 8), v.w = keep(v.w, left - 12);
            }
        };
        auto fetch = [&](const Tile &t, int kb, uint4 &w, uint4 (&x)[RX]) {
            w = make_uint4(0u, 0u, 0u, 0u);
            if (t.n0 + r0 < A.outs) fetch_row(A.ws + ((int64_t)t.group * A.outs + t.n0 + r0) * A.ws_pitch, kb * 8, w);
#pragma unroll
            for (int m = 0; m < RX; ++m) {
                x[m] = make_uint4(0u, 0u, 0u, 0u);
                const int r = r0 + 128 * m;
                if (r < NT && t.row0 + r < A.rows) fetch_row(A.xs + (int64_t)(t.row0 + r) * A.xs_pitch, kb * 8, x[m]);
            }
        };
        struct Step {
            int i, kb;
            Tile t;
        };
        auto stages_of = [&](const Step &c) { return min(2, A.nkb - c.kb); };
        auto advance = [&](Step &c) {
            c.kb += 2;
            if (c.kb >= A.nkb) {
                c.kb = 0;
                c.i += gridDim.x;
                if (c.i < total) c.t = tile_at(c.i);
            }
        };
        auto skip = [&](int n) {
            s += n;
            if (s >= S::STAGES) s -= S::STAGES, ph ^= 1u;
        };
        uint4 w, x[RX];
        Step cur;
        cur.i = blockIdx.x, cur.kb = 0;
        if (cur.i < total) {
            cur.t = tile_at(cur.i);
            if (team == 1) {
                skip(stages_of(cur));
                advance(cur);
            }
        }
        if (cur.i < total) fetch(cur.t, cur.kb, w, x);
        while (cur.i < total && ok) {
            const uint4 cw = w;
            uint4 cx[RX];
#pragma unroll
            for (int m = 0; m < RX; ++m) cx[m] = x[m];
            const int mine = stages_of(cur);
            int theirs = 0;
            advance(cur);
            if (cur.i < total) {
                theirs = stages_of(cur);
                advance(cur);
                if (cur.i < total) fetch(cur.t, cur.kb, w, x);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (half >= mine) break;
                ok = mbar_wait(empty + 8 * s, ph ^ 1u);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t sf = base + s * S::STAGE + W_BYTES + S::X_BYTES;
                const uint32_t dst = sf + (uint32_t)((r0 & 31) * 16 + (r0 >> 5) * 4);
                st_word(dst, half ? cw.z : cw.x);
                st_word(dst + 512, half ? cw.w : cw.y);
#pragma unroll
                for (int m = 0; m < RX; ++m) {
                    if (r0 + 128 * m < NT) {
                        st_word(dst + 1024 + 512 * m, half ? cx[m].z : cx[m].x);
                        st_word(dst + 1024 + 512 * (S::RA + m), half ? cx[m].w : cx[m].y);
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(full + 8 * s);
                skip(1);
            }
            skip(theirs);
        }
    } else {
        // a warp reads the tensor-memory lanes of its quarter (its rank mod 4): lane = output, columns = rows of x, of which
        // two warps share the quarter's; a store is 32 consecutive outputs of one row
        const int quarter = warp & 3, side = (warp - 2 - kScaleWarps) >> 2;
        constexpr int HALF = NT / 2, CW = HALF < 32 ? HALF : 32;
        int buf = 0;
        uint32_t aph = 0;
        OutT *out = static_cast<OutT *>(A.out);
        for (int i = blockIdx.x; i < total; i += gridDim.x) {
            const Tile t = tile_at(i);
            const int n = t.n0 + quarter * 32 + lane;
            if (ok) {
                ok = mbar_wait(acc_full + 8 * buf, aph);
                ok = __all_sync(0xffffffffu, ok);
                fence_after();
            }
            const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * NT + side * HALF);
            OutT *o = out + (int64_t)(t.row0 + side * HALF) * A.ldo + n;
            const int mine = t.rows - side * HALF; // rows of this warp, may be none
#pragma unroll 1
            for (int c = 0; c < HALF && c < mine; c += CW) {
                uint32_t r[CW];
                if (ok) {
                    tmem_load(taddr + c, r);
                } else {
#pragma unroll
                    for (int j = 0; j < CW; ++j) r[j] = 0x7fc00000u; // a wait ran out: not a result
                }
                if (n < A.outs) {
                    if (mine - c >= CW) {
#pragma unroll
                        for (int j = 0; j < CW; ++j, o += A.ldo) *o = from_f32<OutT>(__uint_as_float(r[j]));
                    } else {
#pragma unroll
                        for (int j = 0; j < CW; ++j, o += A.ldo)
                            if (j < mine - c) *o = from_f32<OutT>(__uint_as_float(r[j]));
                    }
                }
                __syncwarp(); // the next load is the whole warp's
            }
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty + 8 * buf);
            if (++buf == 2) buf = 0, aph ^= 1u;
        }
        // rows that no group has: before the first one's and behind the last one's
        const int first = row_start[0], done = row_start[A.groups], et = threadIdx.x - 32 * (2 + kScaleWarps);
        for (int64_t k = blockIdx.x; k < first + (int64_t)(A.rows - done); k += gridDim.x) {
            const int64_t r = k < first ? k : done + (k - first);
            for (int n = et; n < A.outs; n += 32 * kEpilogueWarps) out[r * A.ldo + n] = from_f32<OutT>(0.f);
        }
    }
    fence_before();
    __syncthreads();
    __syncwarp();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::COLS) : "memory");
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = []() -> EncodeTiledFn {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        return reinterpret_cast<EncodeTiledFn>(p);
    }();
    return fn;
}
// bytes x rows (x groups); boxes of 128 bytes x box_rows; whatever lies outside reads as zero codes
bool make_map(CUtensorMap *map, const void *ptr, int64_t bytes, int64_t rows, int64_t pitch, int64_t groups, int box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const int rank = groups > 0 ? 3 : 2;
    cuuint64_t dims[3] = {(cuuint64_t)bytes, (cuuint64_t)rows, (cuuint64_t)(groups > 0 ? groups : 1)};
    cuuint64_t strides[2] = {(cuuint64_t)pitch, (cuuint64_t)(pitch * rows)};
    cuuint32_t box[3] = {KB_BYTES, (cuuint32_t)box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, rank, const_cast<void *>(ptr), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NT, typename OutT>
cudaError_t launch(const CUtensorMap &tm_w, const void *xq, int64_t xq_pitch, const ProductArgs &A, cudaStream_t st) {
    CUtensorMap tm_x;
    if (!make_map(&tm_x, xq, 16 * (int64_t)A.nb, A.rows, xq_pitch, 0, NT)) return cudaErrorInvalidValue;
    auto kernel = mx4_product_kernel<NT, OutT>;
    const int smem = Shape<NT>::smem(A.groups);
    static OncePerDevice prepared;
    const cudaError_t e = prepared([&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<NT>::smem(FS_MX4_MAX_GROUPS));
    });
    if (e != cudaSuccess) return e;
    // every group adds at most one partly filled row tile
    const int64_t row_tiles = A.rows / NT + (A.groups < A.rows ? A.groups : A.rows);
    const int64_t tiles = row_tiles * A.ntiles_n;
    const int sms = sm_count();
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles < sms ? tiles : sms)), cfg.blockDim = dim3(kThreads), cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr, cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, tm_w, tm_x, A);
}
template <typename OutT>
cudaError_t by_rows(const CUtensorMap &tm_w, const void *xq, int64_t xq_pitch, const ProductArgs &A, cudaStream_t st) {
    const int mean = (A.rows + A.groups - 1) / A.groups;
    if (mean <= 16) return launch<16, OutT>(tm_w, xq, xq_pitch, A, st);
    if (mean <= 32) return launch<32, OutT>(tm_w, xq, xq_pitch, A, st);
    if (mean <= 64) return launch<64, OutT>(tm_w, xq, xq_pitch, A, st);
    if (mean <= 128) return launch<128, OutT>(tm_w, xq, xq_pitch, A, st);
    return launch<192, OutT>(tm_w, xq, xq_pitch, A, st);
}

} // namespace
} // namespace fsr

extern "C" int fs_mx4_product(const void *xq_dev, int64_t xq_pitch, const void *xs_dev, int64_t xs_pitch, int64_t rows,
                              const void *wq_dev, int64_t wq_pitch, const void *ws_dev, int64_t ws_pitch, int32_t groups,
                              const int32_t *offsets_dev, int64_t outs, int64_t cols, void *out, int dtype, int64_t ldo,
                              void *stream) {
    using namespace fsr;
    if (dtype != FS_F32 && dtype != FS_BF16 && dtype != FS_F16) return FS_ERR_BAD_N;
    if (rows < 0 || groups < 1 || outs < 1 || cols < 1 || (rows > 1 && ldo < outs)) return FS_ERR_BAD_N;
    const int64_t nb = (cols + 31) / 32;
    if (xq_pitch < 16 * nb || (xq_pitch & 15) || wq_pitch < 16 * nb || (wq_pitch & 15) || xs_pitch < nb || (xs_pitch & 3) ||
        ws_pitch < nb || (ws_pitch & 3))
        return FS_ERR_BAD_N;
    const int64_t ntiles_n = (outs + BM - 1) / BM;
    if (groups > FS_MX4_MAX_GROUPS || rows > INT32_MAX / 2 || outs > INT32_MAX / 2 || cols > FS_MX4_MAX_COLS ||
        (rows / 16 + groups) * ntiles_n > INT32_MAX / 2)
        return FS_ERR_TOO_LARGE;
    if (!offsets_dev && groups != 1) return FS_ERR_NULL;
    if (rows == 0) return FS_OK;
    if (!xq_dev || !xs_dev || !wq_dev || !ws_dev || !out) return FS_ERR_NULL;
    if (((reinterpret_cast<uintptr_t>(xq_dev) | reinterpret_cast<uintptr_t>(wq_dev)) & 15) ||
        ((reinterpret_cast<uintptr_t>(xs_dev) | reinterpret_cast<uintptr_t>(ws_dev)) & 3) ||
        reinterpret_cast<uintptr_t>(out) % type_size(dtype))
        return FS_ERR_UNSUPPORTED;
    ProductArgs A;
    A.xs = static_cast<const uint8_t *>(xs_dev), A.ws = static_cast<const uint8_t *>(ws_dev);
    A.xs_pitch = xs_pitch, A.ws_pitch = ws_pitch, A.ldo = ldo;
    A.rows = (int)rows, A.outs = (int)outs, A.groups = groups, A.nb = (int)nb, A.nkb = (int)((nb + 7) / 8);
    A.ntiles_n = (int)ntiles_n, A.offsets = offsets_dev, A.out = out;
    A.wide = ((reinterpret_cast<uintptr_t>(xs_dev) | reinterpret_cast<uintptr_t>(ws_dev) | xs_pitch | ws_pitch) & 15) == 0;
    CUtensorMap tm_w;
    if (!make_map(&tm_w, wq_dev, 16 * nb, outs, wq_pitch, groups, BM)) return fsk_cuda_failed(cudaErrorInvalidValue, "fs_mx4_product");
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == FS_F32 ? by_rows<float>(tm_w, xq_dev, xq_pitch, A, st)
                          : dtype == FS_BF16 ? by_rows<__nv_bfloat16>(tm_w, xq_dev, xq_pitch, A, st)
                                             : by_rows<__half>(tm_w, xq_dev, xq_pitch, A, st);
    return e == cudaSuccess ? FS_OK : fsk_cuda_failed(e, "fs_mx4_product");
}
