// fs_router_duals: Sinkhorn in the log domain on a rectangular T x E score matrix, T tokens with one unit each.
//
// One iteration from ONE sweep over the rows.  A group of lanes holds a row in registers; with the current g and a reference
// r_t it forms
//      p_e = 2^((l + g - r) log2(e)/eps),  P_te = p_e / sum p,  r_t <- r_t + eps log sum p
// -- r after the update is -f_t, the row half-step -- and each lane adds P into its NE running column sums.  Any r
// gives the same P; the r of the iteration before keeps sum p near 1 without a maximum over the row, and a sum outside
// 2^-20 .. 2^20 (g moved far) sends the row once more through the maximum.  c_e = sum_t P_te is all that the column
// half-step needs: g_e += eps (log(T' b_e) - log c_e).  A c_e that flushed powers or the sums' resolution could touch by more than
// 2^-20 of itself is redone in the log domain, maximum first, before it is used.
//
// All iterations run in one launch; as many rows as fit stay in shared memory in their own type, the rest is read again
// from L2.  How the blocks' column sums meet goes by the number of rows.  One block: __syncthreads.  One cluster of up to 16
// blocks: each keeps its E sums in its shared memory (two buffers in turn), a cluster barrier, and every block adds all 16 lists in rank
// order.  More rows: a cooperative grid, one block per SM, that meets once per iteration (monotone counter, bounded wait): each block adds its E column sums to a common array as 64-bit fixed point,
// which is exact in any order, so the result does not depend on it, and reads E totals back.  Three such arrays alternate,
// so that one is cleared while the next is in use.
//
// Bound and measured.  Per entry and iteration one exponential (16 per clock and SM: 1.9 us for 32768 x 256) and about six other
// instructions.  32768 x 256 bf16, 10 iterations: 85 us, of an iteration's 8 us the rows take 3.4, the meeting of the grid 2.9 (its bare
// barrier 1.2), sums and column step 1.2; with a list of sums per block, read by every block, and true row maxima it was 191 us.
// 2048 x 64, 10 iterations: 28 us in one cluster, 49 on the grid.  512 x 16 fp32, 20 iterations: 33 us in one block, all latency.
#pragma once

#include "router_common.cuh"

namespace fsr {

struct DualsArgs {
    const void *logits;
    int64_t ld, tokens;
    int E, iters;
    int log_parts;
    int cached;        // sweeps whose rows stay in shared memory (a multiple of rows_for)
    const uint8_t *mask;
    const float *target, *g_start;
    float eps, scale;  // scale = log2(e) / eps
    int fix;           // common column sums: fixed point with `fix` fractional bits at level 0, T 2^fix < 2^62
    float *f, *g, *err;
    unsigned *counter;
    unsigned long long *total; // [3][kLevels E + 2]: column sums by level, NaN marks, active rows
    float *part_log;           // [2][blocks][E]: maxima, sums
};
// One translation unit per type (router_duals.cu, router_duals_bf16.cu, router_duals_f16.cu): 42 instances each, which build side by side.
cudaError_t run_duals_f32(const DualsArgs &A, bool vec, cudaStream_t st);
cudaError_t run_duals_bf16(const DualsArgs &A, bool vec, cudaStream_t st);
cudaError_t run_duals_f16(const DualsArgs &A, bool vec, cudaStream_t st);

namespace {

constexpr uint32_t kPollLimit = 1u << 21;
// A column sum below n kHidden is redone in the log domain.  Powers below 2^-126 are flushed, and in a row whose powers sum to as
// little as kSumLow that hides up to 2^-106 of a column; n rows hide less than 2^-20 of a sum that is n 2^-86 or more.
constexpr float kHidden = 1.2924697e-26f; // 2^-86
constexpr float kSumLow = 9.5367e-7f, kSumHigh = 1048576.f; // 2^-20, 2^20
constexpr int kMaxThreads = 512;
constexpr int kSmemBudget = 220 * 1024;
// A block's column sum c goes to level q of the common sums, the first with c >= 2^(26 - fix - 26 q), as a whole number of
// 2^-(fix + 26 q): exact to 2^-27 of itself at any size down to 2^(26 - fix - 26 (kLevels - 1)), about 1e-30 for 32768 rows, and
// the sum of 1024 blocks stays below 2^62 at every level.
constexpr int kLevels = 4, kLevelBits = 26;
constexpr int kAloneSweeps = 4, kClusterBlocks = 16, kClusterSweeps = 8;

// All blocks meet.  Returns false when the wait ran out here or did so earlier.
__device__ __forceinline__ bool meet(unsigned *counter, unsigned target, int *flag_s) {
    __syncthreads();
    if (threadIdx.x == 0 && *flag_s == 0) {
        asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(counter) : "memory");
        uint32_t it = 0;
        for (; it < kPollLimit; ++it) {
            unsigned seen;
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(counter) : "memory");
            if (seen >= target) break;
            if (it > 64) __nanosleep(32);
        }
        if (it == kPollLimit) *flag_s = 1;
    }
    __syncthreads();
    return *flag_s == 0;
}

// rows that a group works on at a time, so that their chains of loads, sums and shuffles overlap, as registers allow
template <int NE> __host__ __device__ constexpr int rows_for() { return NE <= 16 ? 2 : 1; }
// columns of the working arrays: what the lanes of a group hold, open-ended columns included
template <int G, int NE> __host__ __device__ constexpr int width_for() { return G * NE; }

template <int N> struct Const {
    static constexpr int value = N;
};
enum { kAlone = 0, kCluster = 1, kGrid = 2 };
// shared memory: red[warps][E'] (E' = G NE + 4) | part[4][G NE] (cluster only: sums in two buffers, then maxima and sums) | g_s, c_s, want, log_want, closed [G NE each] | r_s[cached][groups] | cached rows
template <typename T, int G, int NE, bool VEC, int MODE>
__global__ void __launch_bounds__(kMaxThreads, 1) router_duals_kernel(const DualsArgs A) {
    typedef RowMap<T, G, NE, VEC> Map;
    typedef typename Map::W W;
    constexpr int R = rows_for<NE>(), WIDE = width_for<G, NE>(), PITCH = WIDE + 4;
    const int nthreads = blockDim.x, nwarps = nthreads >> 5, groups = nthreads / G;
    extern __shared__ __align__(16) uint8_t sm[];
    const int E = A.E, sub = threadIdx.x % G, grp = threadIdx.x / G, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int blocks = MODE == kAlone ? 1 : gridDim.x;
    float *red = reinterpret_cast<float *>(sm), *part = red + nwarps * PITCH, *g_s = part + (MODE == kCluster ? 4 * WIDE : 0), *c_s = g_s + WIDE, *want = c_s + WIDE;
    float *log_want = want + WIDE;
    int *closed = reinterpret_cast<int *>(log_want + WIDE);
    float *r_s = reinterpret_cast<float *>(closed + WIDE);
    W *cache = reinterpret_cast<W *>(sm + ((4 * ((size_t)nwarps * PITCH + (MODE == kCluster ? 9 : 5) * WIDE + (size_t)A.cached * groups) + 15) & ~(size_t)15));
    __shared__ int flag_s, n_s;
    const T *logits = static_cast<const T *>(A.logits);
    if (threadIdx.x == 0) flag_s = 0, n_s = 0;
    for (int e = threadIdx.x; e < WIDE; e += nthreads) g_s[e] = A.g_start && e < E ? A.g_start[e] : 0.f, closed[e] = 0;
    __syncthreads();
    unsigned meetings = 0;
    bool ok = true;
    int n = 0;
    const int sweeps = (int)((A.tokens + (int64_t)blocks * groups - 1) / ((int64_t)blocks * groups));
    auto row_of = [&](int k) { return ((int64_t)k * blocks + blockIdx.x) * groups + grp; };

    // sweep k's row: from shared memory, or from memory (padding rows and rows beyond the end as empty ones)
    auto from_cache = [&](int k, float (&x)[NE]) {
        typename Map::Raw raw;
#pragma unroll
        for (int c = 0; c < Map::CH; ++c) raw.w[c] = cache[(k * Map::CH + c) * nthreads + threadIdx.x];
        Map::unpack(raw, x);
    };
    auto from_memory = [&](int k, bool keep, float (&x)[NE]) {
        typename Map::Raw raw;
        const int64_t t = row_of(k);
        if (k < sweeps && t < A.tokens && (!A.mask || A.mask[t] != 0)) Map::load_raw(logits + t * A.ld, E, sub, raw);
        else Map::empty(raw);
        if (keep) {
#pragma unroll
            for (int c = 0; c < Map::CH; ++c) cache[(k * Map::CH + c) * nthreads + threadIdx.x] = raw.w[c];
        }
        Map::unpack(raw, x);
    };
    // the row's maximum; +inf where it holds a NaN, so that its p become NaN
    auto top_of = [&](const float (&x)[NE]) {
        float m = -INFINITY;
        bool nan = false;
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            m = fmaxf(m, x[i]);
            nan |= x[i] != x[i];
        }
        return group_max<G>(nan ? INFINITY : m);
    };

    for (int it = 0; it < A.iters && ok; ++it) {
        Pair g2[NE / 2], acc2[NE / 2];
#pragma unroll
        for (int i = 0; i < NE / 2; ++i) {
            g2[i] = pair(g_s[Map::col(2 * i, sub)], g_s[Map::col(2 * i + 1, sub)]);
            acc2[i] = pair(0.f, 0.f);
        }
        int active = 0;
        const bool first = it == 0, last = it == A.iters - 1;
        const Pair scale2 = pair(A.scale, A.scale);
        // l + g -> p, relative to r
        auto powers = [&](float r, Pair (&p)[NE / 2]) {
            const float ro = r != -INFINITY ? -r : 0.f; // an empty row: every p is 0
            const Pair r2 = pair(ro, ro);              // difference first: l log2(e)/eps may overflow
            Pair s2 = pair(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < NE / 2; ++i) {
                float lo, hi;
                split(mul2(add2(p[i], r2), scale2), lo, hi);
                p[i] = pair(ex2(lo), ex2(hi));
                s2 = add2(s2, p[i]);
            }
            float lo, hi;
            split(s2, lo, hi);
            return lo + hi;
        };
        // P into the column sums, and the row's next reference
        auto settle = [&](int k, float r, float sum, const Pair (&p)[NE / 2]) {
            const bool on = r != -INFINITY; // a NaN stays one
            const float inv = on ? rcp(sum) : 0.f;
            const Pair inv2 = pair(inv, inv);
#pragma unroll
            for (int i = 0; i < NE / 2; ++i) acc2[i] = fma2(p[i], inv2, acc2[i]);
            // as a reference any r near the row's logarithm will do; as -f it is taken exactly
            if (sub == 0 && k < A.cached) r_s[k * groups + grp] = fmaf(A.eps * kLn2, lg2(sum), r); // -inf - inf where empty
            if (last && A.f && sub == 0 && k < sweeps) {
                const int64_t t = row_of(k);
                if (t < A.tokens) A.f[t] = on ? -fmaf(A.eps, logf(sum), r) : 0.f;
            }
        };
        // the general form: rows from anywhere, the maximum as reference
        auto careful = [&](int k, auto count) {
            constexpr int N = decltype(count)::value;
            float x[N][NE];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if (!first && k + j < A.cached) from_cache(k + j, x[j]);
                else from_memory(k + j, first && k + j < A.cached, x[j]);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                Pair p[NE / 2];
#pragma unroll
                for (int i = 0; i < NE / 2; ++i) {
                    p[i] = add2(pair(x[j][2 * i], x[j][2 * i + 1]), g2[i]);
                    split(p[i], x[j][2 * i], x[j][2 * i + 1]);
                }
                const float r = top_of(x[j]);
                const float sum = group_sum<G>(powers(r, p));
                if (sub == 0) active += r != -INFINITY;
                settle(k + j, r, sum, p);
            }
        };
        // N kept rows, each with the reference of the iteration before
        auto steady = [&](int k, auto count) {
            constexpr int N = decltype(count)::value;
            Pair p[N][NE / 2];
            float r[N], sum[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float x[NE];
                from_cache(k + j, x);
                r[j] = r_s[(k + j) * groups + grp];
#pragma unroll
                for (int i = 0; i < NE / 2; ++i) p[j][i] = add2(pair(x[2 * i], x[2 * i + 1]), g2[i]);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] = powers(r[j], p[j]);
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] = group_sum<G>(sum[j]);
            bool far = false;
#pragma unroll
            for (int j = 0; j < N; ++j) far |= r[j] != -INFINITY && !(sum[j] > kSumLow && sum[j] < kSumHigh);
            if (__any_sync(0xffffffffu, far)) { // (also: every lane has its r before the next one is stored)
                careful(k, count);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) settle(k + j, r[j], sum[j], p[j]);
            }
            __syncwarp();
        };
        const int kept = first ? 0 : min(A.cached, sweeps);
        int k = 0;
        for (; k + R <= kept; k += R) steady(k, Const<R>());
        for (; k < kept; ++k) steady(k, Const<1>());
        for (; k + R <= sweeps; k += R) careful(k, Const<R>());
        for (; k < sweeps; ++k) careful(k, Const<1>());
        // Column sums.  The groups of a warp: at each distance a lane keeps one half of its columns and gives the other away, so
        // every column's sum ends in one lane; then the warps through shared memory.
        {
            float acc[NE];
#pragma unroll
            for (int i = 0; i < NE / 2; ++i) split(acc2[i], acc[2 * i], acc[2 * i + 1]);
            constexpr int HALVINGS = G >= 32 ? 0 : G == 16 ? 1 : G == 8 ? 2 : G == 4 ? 3 : 4; // NE = 16 below 32 lanes
            int at = 0; // first of the columns that this lane still has
#pragma unroll
            for (int h = 0; h < HALVINGS; ++h) {
                const int o = 16 >> h, half = NE >> (h + 1);
                const bool up = (lane & o) != 0;
#pragma unroll
                for (int i = 0; i < half; ++i) {
                    const float keep = up ? acc[half + i] : acc[i], give = up ? acc[i] : acc[half + i];
                    acc[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                }
                at += up ? half : 0;
            }
            if (G == 1) acc[0] += __shfl_xor_sync(0xffffffffu, acc[0], 1); // one column left and one distance to go
            constexpr int LEFT = NE >> HALVINGS;
            if (G > 1 || (lane & 1) == 0) {
#pragma unroll
                for (int i = 0; i < LEFT; ++i) red[warp * PITCH + Map::col(at + i, sub)] = acc[i];
            }
        }
        if (first) {
            active = __reduce_add_sync(0xffffffffu, active);
            if (lane == 0) atomicAdd(&n_s, active);
        }
        __syncthreads();
        // `parts` neighbouring lanes share a column of the warps' sums
        unsigned long long *total = A.total + (size_t)(it % 3) * (kLevels * E + 2);
        if (first && MODE == kAlone) n = n_s;
        int starved = 0;
        float low = 0.f;
        auto set_low = [&]() { // n is known
            low = (float)max(n, 1) * kHidden;
            if (MODE == kGrid) low = fmaxf(low, (float)blocks * ldexpf(1.f, kLevelBits - A.fix - kLevelBits * (kLevels - 1)));
        };
        if (MODE == kAlone) set_low();
        auto half_step = [&](int e, float c) {
            if (first) {
                want[e] = (float)n * (A.target ? A.target[e] : 1.f / (float)E);
                log_want[e] = logf(want[e]);
            }
            c_s[e] = c;
            if (!closed[e]) {
                if (c < low) starved = 1;
                else g_s[e] += A.eps * kLn2 * lg2(want[e] * rcp(c)); // near its fixed point the ratio is near 1
            }
        };
        for (int i0 = 0; i0 < (E << A.log_parts); i0 += nthreads) { // one round where lanes share columns
            const int i = i0 + (int)threadIdx.x, e = i >> A.log_parts, share = i & ((1 << A.log_parts) - 1);
            float c = 0.f;
            if (e < E) {
                for (int w = share; w < nwarps; w += 8 << A.log_parts) {
                    float v[8];
#pragma unroll
                    for (int h = 0; h < 8; ++h) {
                        const int row = w + (h << A.log_parts);
                        v[h] = row < nwarps ? red[row * PITCH + e] : 0.f;
                    }
                    c += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
                }
            }
            for (int o = 1; o < (1 << A.log_parts); o <<= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
            if (share != 0 || e >= E) continue;
            if (MODE == kAlone) half_step(e, c);
            else if (MODE == kCluster) part[(it & 1) * WIDE + e] = c;
            else if (c != c) atomicAdd(total + kLevels * E, 1ull);
            else if (c != 0.f) {
                const int ex = (int)(__float_as_uint(c) >> 23) - 127; // c >= 2^ex
                const int q = min(max((kLevelBits - A.fix - ex + kLevelBits - 1) / kLevelBits, 0), kLevels - 1);
                const unsigned long long v = (unsigned long long)__float2ll_rn(ldexpf(c, A.fix + kLevelBits * q));
                if (v) atomicAdd(total + q * E + e, v);
            }
        }
        if (MODE == kCluster) {
            __syncwarp();
            cluster_sync(); // a block that is ahead writes the other buffer; it meets this one before it writes this buffer again
            if (first)
                for (int b = 0; b < blocks; ++b) n += __float_as_int(remote(reinterpret_cast<const float *>(&n_s), b));
            set_low();
            for (int e = threadIdx.x; e < E; e += nthreads) {
                float v[kClusterBlocks], c = 0.f;
#pragma unroll
                for (int b = 0; b < kClusterBlocks; ++b) v[b] = b < blocks ? remote(part + (it & 1) * WIDE + e, b) : 0.f;
#pragma unroll
                for (int b = 0; b < kClusterBlocks; ++b) c += v[b];
                half_step(e, c);
            }
        } else if (MODE == kGrid) {
            if (first && threadIdx.x == 0 && n_s) atomicAdd(total + kLevels * E + 1, (unsigned long long)n_s);
            ok = meet(A.counter, ++meetings * blocks, &flag_s);
            if (!ok) break;
            const bool nan = __ldcg(total + kLevels * E) != 0;
            if (first) n = (int)__ldcg(total + kLevels * E + 1);
            set_low();
            for (int e = threadIdx.x; e < E; e += nthreads) {
                unsigned long long v[kLevels];
#pragma unroll
                for (int q = 0; q < kLevels; ++q) v[q] = __ldcg(total + q * E + e);
                float c = 0.f;
#pragma unroll
                for (int q = kLevels - 1; q >= 0; --q) c += ldexpf((float)(long long)v[q], -A.fix - kLevelBits * q);
                half_step(e, nan ? NAN : c);
            }
            // everybody has read the array before this one (it met above): clear it for the iteration after the next
            if (blockIdx.x == 0)
                for (int e = threadIdx.x; e < kLevels * E + 2; e += nthreads)
                    A.total[(size_t)((it + 2) % 3) * (kLevels * E + 2) + e] = 0;
        }
        starved = __syncthreads_or(starved);
        if (blockIdx.x == 0 && A.err && warp == nwarps - 1) { // c_s changes only behind the next barrier
            float miss = 0.f;
            for (int e = lane; e < E; e += 32) miss += fabsf(c_s[e] - want[e]);
            miss = group_sum<32>(miss);
            if (lane == 0) A.err[it] = miss / fmaxf((float)n, 1.f);
        }
        if (starved && n > 0) {
            // the starved columns again: running maximum and sum of 2^(log2 P - maximum).  g2 is the state before this
            // iteration for every row.
            float mx[NE], s[NE];
#pragma unroll
            for (int i = 0; i < NE; ++i) mx[i] = -INFINITY, s[i] = 0.f;
#pragma unroll 1
            for (int q = 0; q < sweeps; ++q) {
                float x[NE];
                if (q < A.cached) from_cache(q, x);
                else from_memory(q, false, x);
#pragma unroll
                for (int i = 0; i < NE / 2; ++i) split(add2(pair(x[2 * i], x[2 * i + 1]), g2[i]), x[2 * i], x[2 * i + 1]);
                const float m = top_of(x), mo = m > -INFINITY ? m : 0.f;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < NE; ++i) {
                    x[i] = (x[i] - mo) * A.scale;
                    sum += ex2(x[i]);
                }
                sum = group_sum<G>(sum);
                if (m > -INFINITY) {
                    const float l2 = log2f(sum);
#pragma unroll
                    for (int i = 0; i < NE; ++i) {
                        const float v = x[i] - l2;
                        if (v > mx[i]) s[i] = fmaf(s[i], ex2(mx[i] - v), 1.f), mx[i] = v;
                        else if (v > -INFINITY) s[i] += ex2(v - mx[i]);
                    }
                }
                __syncwarp();
            }
            // groups of a warp, then warps, then blocks
#pragma unroll
            for (int i = 0; i < NE; ++i) {
#pragma unroll
                for (int o = 16; o >= G; o >>= 1) {
                    const float om = __shfl_xor_sync(0xffffffffu, mx[i], o), os = __shfl_xor_sync(0xffffffffu, s[i], o);
                    const float top = fmaxf(mx[i], om);
                    if (top > -INFINITY) s[i] = s[i] * ex2(mx[i] - top) + os * ex2(om - top);
                    mx[i] = top;
                }
            }
            if (lane < G) {
#pragma unroll
                for (int i = 0; i < NE; ++i) red[warp * PITCH + Map::col(i, sub)] = mx[i];
            }
            __syncthreads();
            constexpr int PER = (FS_ROUTER_MAX_EXPERTS + 127) / 128; // columns of a thread, for blocks of 128 threads and more
            float top[PER], ssum[PER];
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                const int e = q * nthreads + (int)threadIdx.x;
                top[q] = -INFINITY, ssum[q] = 0.f;
                if (e < E)
                    for (int w = 0; w < nwarps; ++w) top[q] = fmaxf(top[q], red[w * PITCH + e]);
            }
            __syncthreads();
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                const int e = q * nthreads + (int)threadIdx.x;
                if (e < E) red[e] = top[q];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NE; ++i) { // every warp's sums relative to the block's maximum
                const int e = Map::col(i, sub);
                const float bm = e < E ? red[e] : -INFINITY;
                s[i] = bm > -INFINITY ? s[i] * ex2(mx[i] - bm) : 0.f;
            }
            __syncthreads();
            if (lane < G) {
#pragma unroll
                for (int i = 0; i < NE; ++i) red[warp * PITCH + Map::col(i, sub)] = s[i];
            }
            __syncthreads();
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                const int e = q * nthreads + (int)threadIdx.x;
                if (e >= E) continue;
                for (int w = 0; w < nwarps; ++w) ssum[q] += red[w * PITCH + e];
                if (MODE == kCluster) {
                    part[2 * WIDE + e] = top[q], part[3 * WIDE + e] = ssum[q];
                } else if (MODE == kGrid) {
                    A.part_log[(int64_t)blockIdx.x * E + e] = top[q];
                    A.part_log[(int64_t)(blocks + blockIdx.x) * E + e] = ssum[q];
                }
            }
            if (MODE == kCluster) {
                __syncwarp();
                cluster_sync();
            } else if (MODE == kGrid) {
                ok = meet(A.counter, ++meetings * blocks, &flag_s);
                if (!ok) break;
            }
#pragma unroll
            for (int q = 0; q < PER; ++q) {
                const int e = q * nthreads + (int)threadIdx.x;
                if (e >= E || closed[e] || !(c_s[e] < low)) continue;
                float tm = top[q], ts = ssum[q];
                if (MODE != kAlone) {
                    auto list = [&](int b, int sums) {
                        return MODE == kCluster ? remote(part + (2 + sums) * WIDE + e, b)
                                                : __ldcg(A.part_log + (int64_t)(b + sums * blocks) * E + e);
                    };
                    tm = -INFINITY, ts = 0.f;
                    for (int b = 0; b < blocks; ++b) tm = fmaxf(tm, list(b, 0));
                    for (int b = 0; b < blocks && tm > -INFINITY; ++b) ts += list(b, 1) * ex2(list(b, 0) - tm);
                }
                if (tm > -INFINITY) {
                    g_s[e] += A.eps * (log_want[e] - kLn2 * (tm + log2f(ts)));
                } else {
                    closed[e] = 1; // no row can use this expert: its dual stays as it is
                }
            }
            // the maxima and sums have one buffer: nobody writes the next ones before everybody has read these
            __syncwarp();
            if (MODE == kCluster) cluster_sync();
            __syncthreads();
        }
    }
    __syncwarp();
    if (MODE == kCluster) cluster_sync(); // no block leaves while another may still read its shared memory
    __syncthreads();
    if (!ok) { // nothing of this is a result
        if (A.f)
            for (int64_t t = (int64_t)blockIdx.x * nthreads + threadIdx.x; t < A.tokens; t += (int64_t)blocks * nthreads) A.f[t] = NAN;
        if (blockIdx.x == 0) {
            for (int e = threadIdx.x; e < E; e += nthreads) A.g[e] = NAN;
            if (A.err)
                for (int k = threadIdx.x; k < A.iters; k += nthreads) A.err[k] = NAN;
        }
        return;
    }
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e < E; e += nthreads) A.g[e] = g_s[e];
}

// the counter and the three arrays of totals behind it start at zero
__global__ void __launch_bounds__(256) clear_kernel(unsigned long long *p, int words) {
    for (int i = threadIdx.x; i < words; i += 256) p[i] = 0;
}

struct DualsLaunch {
    DualsArgs A;
    cudaStream_t st;
    template <typename T, int G, int NE, bool VEC> cudaError_t run() {
        const int sms = sm_count();
        // One block as long as each of its groups has few rows (small batches in smaller blocks, whose fixed cost per warp is
        // less), then one cluster, then the grid.
        int threads = kMaxThreads;
        while (threads > 128 && A.tokens <= (int64_t)(threads / 2 / G) * rows_for<NE>()) threads >>= 1;
        const int64_t all = (A.tokens + threads / G - 1) / (threads / G); // sweeps that one block would make
        if (all <= kAloneSweeps) return start<T, G, NE, VEC, kAlone>(1, threads, all);
        if (all <= kClusterBlocks * kClusterSweeps && cluster_fits<T, G, NE, VEC>()) {
            const int blocks = (int)(all < kClusterBlocks ? all : kClusterBlocks);
            return start<T, G, NE, VEC, kCluster>(blocks, threads, (all + blocks - 1) / blocks);
        }
        const int64_t blocks = all < sms ? all : sms;
        return start<T, G, NE, VEC, kGrid>((int)blocks, threads, (all + blocks - 1) / blocks);
    }
    // whether this device holds a cluster of kClusterBlocks of the largest blocks at all
    template <typename T, int G, int NE, bool VEC> bool cluster_fits() {
        static OncePerDevice asked;
        return asked([&] {
            auto kernel = router_duals_kernel<T, G, NE, VEC, kCluster>;
            cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBudget);
            if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
            cudaLaunchConfig_t cfg{};
            cfg.gridDim = dim3(kClusterBlocks), cfg.blockDim = dim3(kMaxThreads), cfg.dynamicSmemBytes = kSmemBudget;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = kClusterBlocks, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr, cfg.numAttrs = 1;
            int n = 0;
            if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
            if (e != cudaSuccess) cudaGetLastError();
            return e == cudaSuccess && n < 1 ? cudaErrorInvalidConfiguration : e;
        }) == cudaSuccess;
    }
    template <typename T, int G, int NE, bool VEC, int MODE> cudaError_t start(int blocks, int threads, int64_t sweeps) {
        constexpr int R = rows_for<NE>(), WIDE = width_for<G, NE>();
        auto kernel = router_duals_kernel<T, G, NE, VEC, MODE>;
        const int groups = threads / G;
        const size_t fixed = 4 * ((size_t)(threads / 32) * (WIDE + 4) + (MODE == kCluster ? 9 : 5) * (size_t)WIDE) + 16;
        const size_t per = (size_t)groups * 4 + (size_t)NE * sizeof(T) * threads; // a sweep's references and rows
        const int64_t fit = (int64_t)((kSmemBudget - fixed) / per) / R * R, whole = (sweeps + R - 1) / R * R;
        A.cached = (int)(fit < whole ? fit : whole);
        A.log_parts = 0; // lanes that share a column when the warps' sums are added
        while (A.log_parts < 3 && (A.E << (A.log_parts + 1)) <= threads && (1 << (A.log_parts + 1)) <= threads / 32) ++A.log_parts;
        const size_t smem = fixed + A.cached * per;
        static OncePerDevice prepared;
        cudaError_t e = prepared([&] {
            const cudaError_t r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBudget);
            if (r != cudaSuccess || MODE != kCluster) return r;
            return cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        });
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)blocks), cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem, cfg.stream = st;
        cudaLaunchAttribute attr[1];
        cfg.attrs = attr, cfg.numAttrs = 0;
        if (MODE == kAlone) return cudaLaunchKernelEx(&cfg, kernel, A);
        cfg.numAttrs = 1;
        if (MODE == kCluster) {
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = (unsigned)blocks, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
            return cudaLaunchKernelEx(&cfg, kernel, A);
        }
        int k = 62;
        for (int64_t t = A.tokens; t > 0; t >>= 1) --k;
        A.fix = k;
        clear_kernel<<<1, 256, 0, st>>>(reinterpret_cast<unsigned long long *>(A.counter), 32 + 3 * (kLevels * A.E + 2));
        A.part_log = reinterpret_cast<float *>(A.total + 3 * (kLevels * (size_t)A.E + 2));
        attr[0].id = cudaLaunchAttributeCooperative;
        attr[0].val.cooperative = 1;
        return cudaLaunchKernelEx(&cfg, kernel, A);
    }
};

template <typename T> cudaError_t run_duals(const DualsArgs &A, bool vec, cudaStream_t st) {
    DualsLaunch D{A, st};
    return vec ? by_experts_wide<DualsLaunch, T, true>(D, A.E) : by_experts_wide<DualsLaunch, T, false>(D, A.E);
}

} // namespace
} // namespace fsr
