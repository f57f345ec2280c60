// fs_router_forward / fs_router_backward: selection of experts, gates, balance loss and its gradient.
//
// Forward.  A group of G lanes holds the E logits of a token in registers (router_common.cuh), the next token's row is under
// way meanwhile.  One sweep gives the row's maximum m, the sum of e = 2^((l - m) log2 e) and so lse and p = e / sum.  Choice,
// groups of 16 and 32 lanes: the topk-th largest of the lanes' own maxima bounds the topk-th score from below, and little more
// than topk scores reach it; those go to shared memory as 64-bit keys (score, then lower column), one lane takes each and
// counts the keys above its own, which is its rank.  Otherwise, and where more scores tie with the bound than lanes are there:
// each lane sorts its own scores l + bias in descending order (values only, a network of max / min), then topk rounds take the
// largest head of the group's lists; the winner moves its list up.  Which of its columns a value came from is looked up after
// the rounds, once per chosen value of a lane instead of once per round; equal heads in several lanes are settled at once, by
// the lower column.  For training each lane adds p into NE running column sums that live in its registers over all tokens of
// its group, so that the column sums cost one addition per entry and no traffic; the block joins its groups' sums in shared
// memory in a fixed order and leaves E partial sums and E integer counts, which a second small kernel (one cluster, columns
// dealt to its CTAs, started early by programmatic dependent launch) adds in block order and turns into load, prob and the two
// losses.  One block finishes by itself, up to eight form a cluster whose first block reads the others' sums.  Floating sums never meet an atomic; the integer counts do, where
// order does not matter.
//
// Backward.  One sweep per token: p = 2^((l - lse) log2 e), over its sum where lse is large, the gate terms scattered into a per-group
// row in shared memory (topk stores, cleared again after use), F = sum p load by a group reduction, and
//      dl = direct + p (S (load - F) + Z - a)
// with S = d0 E / T', Z = 2 d1 lse / T' and the gate's constants; logits are read once and the gradient written once.
//
// Measured at 32768 x 256 bf16, top 8.  Forward 34 us: bound by instruction issue, about 650 warp instructions per token, 400 of
// them the choice (rounds of an arg max over value and column: 73 us; sorted lists: 51); finishing kernel about 5 of it.  At 64
// registers, two blocks of 512, the instances for 33 to 256 experts spill 84 to 172 bytes a thread.
// Backward 13.3 us for 33.5 MB (2.5 TB/s), issue again, about 250 instructions per token.  Ordering 131072 pairs of 128 experts: 11 us.
#include "router_common.cuh"

namespace fsr {
namespace {

constexpr int kThreads = 256;       // backward
constexpr int kJointBlocks = 8;     // a portable cluster
constexpr int kFinishCtas = 8;
constexpr int kFinishThreads = 1024;

struct ForwardArgs {
    const void *logits;
    int64_t ld, tokens;
    int E, topk, normalize, stats;
    int joint; // the blocks are one cluster, whose first block finishes
    const uint8_t *mask;
    const float *bias;
    int32_t *idx;
    float *gate, *lse;
    int32_t *counts;
    float *load, *prob, *loss;
    // partial results of the blocks: [blocks][E] sums, [blocks][E] counts, [blocks] sums of lse^2, [blocks] active rows
    float *part_p;
    int32_t *part_c;
    float *part_z;
    int32_t *part_n;
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// load, prob and the block's share of the two losses from column totals; called by all threads of a block for its columns
__device__ __forceinline__ void finish_column(const ForwardArgs &A, int e, float p, int c, int n, float &bal) {
    const float nf = (float)max(n, 1);
    const float load = (float)c / ((float)A.topk * nf), prob = p / nf;
    if (A.counts) A.counts[e] = c;
    if (A.load) A.load[e] = load;
    if (A.prob) A.prob[e] = prob;
    bal = fmaf(load, prob, bal);
}

// sum over the block, same order every time; red: one float per warp
__device__ __forceinline__ float block_sum(float x, float *red, int nwarps) {
    x = group_sum<32>(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    float s = 0.f;
    for (int w = 0; w < nwarps; ++w) s += red[w];
    return s;
}

// x in descending order
template <int NE> __device__ __forceinline__ void sort_down(float (&x)[NE]) {
#pragma unroll
    for (int p = 1; p < NE; p *= 2) {
#pragma unroll
        for (int k = p; k >= 1; k /= 2) {
#pragma unroll
            for (int j = k % p; j + k < NE; j += 2 * k) {
#pragma unroll
                for (int i = 0; i < k; ++i) {
                    if (i + j + k < NE && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                        const float hi = fmaxf(x[i + j], x[i + j + k]), lo = fminf(x[i + j], x[i + j + k]);
                        x[i + j] = hi, x[i + j + k] = lo;
                    }
                }
            }
        }
    }
}

// shared memory: sel[groups][topk] | keys[threads], logit_of[threads] (from 16 lanes on) | counts[E] | red[kWarps][E] | sums[E] (with stats)
template <int NE> __host__ __device__ constexpr int forward_threads() { return NE <= 8 ? 512 : 256; }
template <typename T, int G, int NE, bool VEC>
__global__ void __launch_bounds__(forward_threads<NE>(), NE <= 8 ? 2 : 1) router_forward_kernel(const ForwardArgs A) {
    typedef RowMap<T, G, NE, VEC> Map;
    constexpr int kThreads = forward_threads<NE>(), kWarps = kThreads / 32, GROUPS = kThreads / G;
    extern __shared__ __align__(16) uint8_t smem[];
    float2 *sel = reinterpret_cast<float2 *>(smem) + (threadIdx.x / G) * A.topk; // (column bits, score, then logit) per choice
    unsigned long long *keys = reinterpret_cast<unsigned long long *>(smem + (size_t)GROUPS * A.topk * sizeof(float2)) + (threadIdx.x / G) * G; // 16-byte aligned: GROUPS is even
    float *logit_of = reinterpret_cast<float *>(smem + (size_t)GROUPS * A.topk * sizeof(float2) + (G >= 16 ? 8 * kThreads : 0)) + (threadIdx.x / G) * G;
    int *cnt = reinterpret_cast<int *>(smem + (size_t)GROUPS * A.topk * sizeof(float2) + (G >= 16 ? 12 * kThreads : 0));
    float *red = reinterpret_cast<float *>(cnt + A.E);
    __shared__ float red_w[kWarps], lost[kWarps]; // lost: NaN where the bias holds one, else 0; one copy per warp
    const int E = A.E, sub = threadIdx.x % G, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int base = lane & ~(G - 1); // the group's first lane
    const T *logits = static_cast<const T *>(A.logits);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    float bias[NE];
    Pair acc2[NE / 2];
#pragma unroll
    for (int i = 0; i < NE; ++i) {
        const int e = Map::col(i, sub);
        bias[i] = A.bias && e < E ? A.bias[e] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < NE / 2; ++i) acc2[i] = pair(0.f, 0.f);
    if (A.stats) {
        for (int e = threadIdx.x; e < E; e += kThreads) cnt[e] = 0;
        __syncthreads();
    }
    float z2 = 0.f;
    int active = 0;
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t t = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G;
    typename Map::Raw raw;
    bool live = false;
    const T *row = logits + t * A.ld; // of the token to be fetched next
    auto fetch = [&](int64_t at) { // padding rows are read like the others, and not used
        live = false;
        if (at < A.tokens) {
            live = !A.mask || A.mask[at] != 0;
            Map::load_raw(row, E, sub, raw);
        }
        row += step * A.ld;
    };
    fetch(t);
    bool nan = false; // asked with the first row under way
#pragma unroll
    for (int i = 0; i < NE; ++i) nan |= bias[i] != bias[i];
    nan = __any_sync(0xffffffffu, nan); // a group's lanes have all columns
    if (lane == 0) lost[warp] = nan ? NAN : 0.f;
    __syncwarp();
    int32_t *idx_t = A.idx + t * A.topk;
    float *gate_t = A.gate + t * A.topk;
    // every lane of a warp makes the same number of rounds (the shuffles name the whole warp)
    for (int64_t t0 = (int64_t)blockIdx.x * GROUPS; t0 < A.tokens; t0 += step, t += step) {
        const bool in = t < A.tokens;
        float x[NE];
        if (live) {
            Map::unpack(raw, x);
        } else {
#pragma unroll
            for (int i = 0; i < NE; ++i) x[i] = -INFINITY;
        }
        const bool now = live;
        fetch(t + step);
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < NE; ++i) m = fmaxf(m, x[i]);
        m = group_max<G>(m);
        float mm = m > -INFINITY ? m : 0.f;
        Pair p[NE / 2], s2 = pair(0.f, 0.f);
        const Pair log2e2 = pair(kLog2e, kLog2e), mm2 = pair(-mm, -mm); // difference first: l log2 e may overflow
#pragma unroll
        for (int i = 0; i < NE / 2; ++i) {
            float lo, hi;
            split(mul2(add2(pair(x[2 * i], x[2 * i + 1]), mm2), log2e2), lo, hi);
            p[i] = pair(ex2(lo), ex2(hi));
            s2 = add2(s2, p[i]);
        }
        float sum, sum1;
        split(s2, sum, sum1);
        sum = group_sum<G>(sum + sum1); // NaN where the row holds one, +inf included
        const bool on = now && (m > -INFINITY || sum != sum);
        const float inv = on ? rcp(sum) : 0.f;
        const float lse = on ? fmaf(lg2(sum), kLn2, mm) : 0.f;
        if (A.stats) {
#pragma unroll
            for (int i = 0; i < NE / 2; ++i) acc2[i] = fma2(p[i], pair(inv, inv), acc2[i]);
            if (sub == 0 && on) {
                z2 = fmaf(lse, lse, z2);
                ++active;
            }
        }
        if (A.lse && in && sub == 0) A.lse[t] = lse;
        float d[NE];
        auto score = [&](int i) { return fmaxf(x[i] + bias[i], -INFINITY); }; // a NaN becomes -inf and is passed over
#pragma unroll
        for (int i = 0; i < NE; ++i) d[i] = score(i);
        bool chosen = false;
        if constexpr (G >= 16) {
            if (A.topk <= G / 2) {
                float h = d[0];
#pragma unroll
                for (int i = 1; i < NE; ++i) h = fmaxf(h, d[i]);
                float bound = -INFINITY;
                for (int j = 0; j < A.topk; ++j) { // equal maxima go together: the bound only gets lower
                    bound = group_max<G>(h);
                    if (h == bound) h = -INFINITY;
                }
                bool mine[NE];
                int n = 0;
                unsigned before[NE];
#pragma unroll
                for (int i = 0; i < NE; ++i) {
                    mine[i] = d[i] >= bound && d[i] > -INFINITY;
                    unsigned who = __ballot_sync(0xffffffffu, mine[i]) >> base;
                    if (G < 32) who &= (1u << (G & 31)) - 1u;
                    before[i] = n + __popc(who & ((1u << sub) - 1u));
                    n += __popc(who);
                }
                if (!__any_sync(0xffffffffu, n > G)) {
                    chosen = true;
#pragma unroll
                    for (int i = 0; i < NE; ++i) {
                        if (mine[i]) {
                            const uint32_t bits = __float_as_uint(d[i] + 0.f); // -0 is 0
                            const uint32_t up = bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u);
                            keys[before[i]] = (unsigned long long)up << 32 | (uint32_t)~Map::col(i, sub);
                            logit_of[before[i]] = x[i];
                        }
                    }
                    if (sub >= n) keys[sub] = 0ull; // below every key
                    __syncwarp();
                    const unsigned long long key = keys[sub];
                    int rank = 0;
                    const int most = G < 32 ? __reduce_max_sync(0xffffffffu, n) : n;
                    for (int q = 0; q < most; q += 4) { // G is a multiple of four
                        const ulonglong2 a = *reinterpret_cast<const ulonglong2 *>(keys + q);
                        const ulonglong2 b = *reinterpret_cast<const ulonglong2 *>(keys + q + 2);
                        rank += (int)(a.x > key) + (int)(a.y > key) + (int)(b.x > key) + (int)(b.y > key);
                    }
                    const bool take = sub < n && rank < A.topk;
                    float l = take ? logit_of[sub] : -INFINITY, top = mm, scale = inv;
                    const float w0 = ex2((l - mm) * kLog2e);
                    float w = w0;
                    if (A.normalize) {
                        top = group_max<G>(l);
                        if (top == -INFINITY) top = 0.f;
                        w = ex2((l - top) * kLog2e);
                        const float all = group_sum<G>(w);
                        scale = all > 0.f ? rcp(all) : 0.f;
                    }
                    if (on) scale += lost[warp] + (sum - sum); // a NaN in the row or in the bias reaches all its gates
                    if (in) {
                        if (take) {
                            const int e = (int)~(uint32_t)key;
                            idx_t[rank] = e;
                            gate_t[rank] = w * scale;
                            if (A.stats) atomicAdd(&cnt[e], 1);
                        }
                        if (sub >= n && sub < A.topk) idx_t[sub] = -1, gate_t[sub] = 0.f * scale; // fewer than topk open
                    }
                    __syncwarp();
                }
            }
        }
        if (!chosen) {
        // d = the lane's scores in descending order
        sort_down<NE>(d);
        unsigned won = 0, taken = 0; // rounds that this lane won and has not looked up; columns that it has given
        auto look_up = [&]() {
            while (__any_sync(0xffffffffu, won != 0)) {
                if (won != 0) {
                    const int r = __ffs(won) - 1;
                    const float v = sel[r].y;
                    int slot = 0;
                    float l = 0.f;
#pragma unroll
                    for (int i = NE - 1; i >= 0; --i)
                        if (score(i) == v && !((taken >> i) & 1u)) slot = i, l = x[i];
                    taken |= 1u << slot;
                    won &= won - 1;
                    sel[r] = make_float2(__int_as_float(Map::col(slot, sub)), l);
                }
                __syncwarp();
            }
        };
        for (int j = 0; j < A.topk; ++j) {
            const float best = group_max<G>(d[0]);
            const bool head = d[0] == best && best > -INFINITY;
            unsigned heads = __ballot_sync(0xffffffffu, head) >> base;
            if (G < 32) heads &= (1u << (G & 31)) - 1u;
            int winner = __ffs(heads) - 1; // -1: nothing left
            if (__any_sync(0xffffffffu, (heads & (heads - 1)) != 0)) {
                // equal heads: the lane with the lowest column of that score that it has not given yet
                look_up();
                int col = 0x7fffffff;
                if (head) {
#pragma unroll
                    for (int i = NE - 1; i >= 0; --i)
                        if (score(i) == best && !((taken >> i) & 1u)) col = Map::col(i, sub);
                }
                int low = col;
#pragma unroll
                for (int o = G / 2; o > 0; o >>= 1) low = min(low, __shfl_xor_sync(0xffffffffu, low, o));
                const unsigned at = __ballot_sync(0xffffffffu, head && col == low) >> base;
                winner = __ffs(G < 32 ? at & ((1u << (G & 31)) - 1u) : at) - 1;
            }
            if (sub == winner) {
                sel[j].y = best;
                won |= 1u << j;
#pragma unroll
                for (int i = 0; i + 1 < NE; ++i) d[i] = d[i + 1];
                d[NE - 1] = -INFINITY;
            }
            if (winner < 0 && sub == 0) sel[j] = make_float2(__int_as_float(-1), -INFINITY);
        }
        __syncwarp();
        look_up();
        __syncwarp();
        float top = mm, scale = inv;
        if (A.normalize) {
            top = -INFINITY;
            for (int j = 0; j < A.topk; ++j) top = fmaxf(top, sel[j].y);
            if (top == -INFINITY) top = 0.f;
            float w = 0.f;
            for (int j = 0; j < A.topk; ++j) w += ex2((sel[j].y - top) * kLog2e);
            scale = w > 0.f ? rcp(w) : 0.f;
        }
        if (on) scale += lost[warp] + (sum - sum); // as above
        if (in) {
            for (int j = sub; j < A.topk; j += G) {
                const float2 c = sel[j];
                const int e = __float_as_int(c.x);
                idx_t[j] = e;
                gate_t[j] = (e >= 0 ? ex2((c.y - top) * kLog2e) : 0.f) * scale;
                if (A.stats && e >= 0) atomicAdd(&cnt[e], 1);
            }
        }
        __syncwarp();
        }
        idx_t += step * A.topk, gate_t += step * A.topk;
    }
    if (!A.stats) return;

    // the block's column sums: groups of a warp by shuffles, then the warps in order
    float acc[NE];
#pragma unroll
    for (int i = 0; i < NE / 2; ++i) split(acc2[i], acc[2 * i], acc[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < NE; ++i) {
#pragma unroll
        for (int o = 16; o >= G; o >>= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
        const int e = Map::col(i, sub);
        if (lane < G && e < E) red[warp * E + e] = acc[i];
    }
    const float zsum = block_sum(z2, red_w, kWarps);
    const int nsum = (int)block_sum((float)active, red_w, kWarps); // exact: fewer than 2^24 rows per block
    if (A.joint) {
        float *sums = red + kWarps * E;
        __shared__ float z_s;
        __shared__ int n_s;
        for (int e = threadIdx.x; e < E; e += kThreads) {
            float p = 0.f;
            for (int w = 0; w < kWarps; ++w) p += red[w * E + e];
            sums[e] = p;
        }
        if (threadIdx.x == 0) z_s = zsum, n_s = nsum;
        __syncwarp();
        cluster_sync();
        if (cluster_rank() == 0) {
            const int blocks = gridDim.x;
            float z = 0.f, bal = 0.f;
            int n = 0;
            for (int b = 0; b < blocks; ++b) z += remote(&z_s, b), n += __float_as_int(remote(reinterpret_cast<float *>(&n_s), b));
            for (int e = threadIdx.x; e < E; e += kThreads) {
                float p = 0.f;
                int c = 0;
#pragma unroll 4
                for (int b = 0; b < blocks; ++b) {
                    p += remote(sums + e, b);
                    c += __float_as_int(remote(reinterpret_cast<float *>(cnt + e), b));
                }
                finish_column(A, e, p, c, n, bal);
            }
            bal = block_sum(bal, red_w, kWarps);
            if (threadIdx.x == 0) {
                if (A.counts) A.counts[E] = n;
                if (A.loss) A.loss[0] = (float)E * bal, A.loss[1] = z / (float)max(n, 1);
            }
        }
        __syncwarp();
        cluster_sync(); // the others' shared memory stays until it has been read
        return;
    }
    if (gridDim.x > 1) {
        for (int e = threadIdx.x; e < E; e += kThreads) {
            float p = 0.f;
            for (int w = 0; w < kWarps; ++w) p += red[w * E + e];
            A.part_p[(int64_t)blockIdx.x * E + e] = p;
            A.part_c[(int64_t)blockIdx.x * E + e] = cnt[e];
        }
        if (threadIdx.x == 0) A.part_z[blockIdx.x] = zsum, A.part_n[blockIdx.x] = nsum;
        return;
    }
    float bal = 0.f;
    for (int e = threadIdx.x; e < E; e += kThreads) {
        float p = 0.f;
        for (int w = 0; w < kWarps; ++w) p += red[w * E + e];
        finish_column(A, e, p, cnt[e], nsum, bal);
    }
    bal = block_sum(bal, red_w, kWarps);
    if (threadIdx.x == 0) {
        if (A.counts) A.counts[E] = nsum;
        if (A.loss) A.loss[0] = (float)E * bal, A.loss[1] = zsum / (float)max(nsum, 1);
    }
}

// One cluster of kFinishCtas CTAs: strips of 32 columns are dealt to the CTAs, 32 lanes along the blocks per column.
__global__ void __cluster_dims__(kFinishCtas, 1, 1) __launch_bounds__(kFinishThreads)
router_finish_kernel(const ForwardArgs A, int blocks) {
    __shared__ float ps[32][33], red_w[32], share[kFinishCtas];
    __shared__ int cs[32][33];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, E = A.E;
    const uint32_t rank = cluster_rank();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float zb = 0.f;
    int n = 0;
    for (int b = threadIdx.x; b < blocks; b += kFinishThreads) zb += A.part_z[b], n += A.part_n[b];
    n = __reduce_add_sync(0xffffffffu, n);
    if (tx == 0) cs[0][ty] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < 32; ++w) n += cs[0][w];
    const float z = block_sum(zb, red_w, 32);
    float bal = 0.f;
    for (int e0 = (int)rank * 32; e0 < E; e0 += kFinishCtas * 32) {
        const int e = e0 + tx;
        float p = 0.f;
        int c = 0;
        if (e < E) {
#pragma unroll 8
            for (int b = ty; b < blocks; b += 32) {
                p += A.part_p[(int64_t)b * E + e];
                c += A.part_c[(int64_t)b * E + e];
            }
        }
        __syncthreads();
        ps[ty][tx] = p, cs[ty][tx] = c;
        __syncthreads();
        if (ty == 0 && e < E) {
            p = 0.f, c = 0;
            for (int y = 0; y < 32; ++y) p += ps[y][tx], c += cs[y][tx];
            finish_column(A, e, p, c, n, bal);
        }
    }
    if (ty == 0) bal = group_sum<32>(bal);
    if (threadIdx.x == 0) {
        uint32_t addr = (uint32_t)__cvta_generic_to_shared(&share[rank]), dst;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"(addr), "r"(0));
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst), "f"(bal) : "memory");
    }
    cluster_sync();
    if (rank == 0 && threadIdx.x == 0) {
        float s = 0.f;
        for (int r = 0; r < kFinishCtas; ++r) s += share[r];
        if (A.counts) A.counts[E] = n;
        if (A.loss) A.loss[0] = (float)E * s, A.loss[1] = z / (float)max(n, 1);
    }
}

struct ForwardLaunch {
    ForwardArgs A;
    cudaStream_t st;
    template <typename T, int G, int NE, bool VEC> cudaError_t run() {
        constexpr int kThreads = forward_threads<NE>(), kWarps = kThreads / 32, GROUPS = kThreads / G;
        const int64_t want = (A.tokens + GROUPS - 1) / GROUPS;
        const int limit = min(kMaxBlocks, 2 * sm_count()); // what is resident at once for up to 256 experts
        const int blocks = (int)(want < 1 ? 1 : want < limit ? want : limit);
        A.joint = A.stats && blocks > 1 && blocks <= kJointBlocks;
        const size_t smem = (size_t)GROUPS * A.topk * sizeof(float2) + (G >= 16 ? 12 * kThreads : 0) + (A.stats ? (size_t)A.E * 4 * (2 + kWarps) : 0);
        cudaLaunchConfig_t cfg{};
        cudaLaunchAttribute attr[1];
        cfg.gridDim = dim3((unsigned)blocks), cfg.blockDim = dim3(kThreads), cfg.dynamicSmemBytes = smem, cfg.stream = st;
        cfg.attrs = attr, cfg.numAttrs = A.joint;
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)blocks, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
        cudaError_t e = cudaLaunchKernelEx(&cfg, router_forward_kernel<T, G, NE, VEC>, A);
        if (e != cudaSuccess || !A.stats || blocks == 1 || A.joint) return e;
        cfg.gridDim = dim3(kFinishCtas), cfg.blockDim = dim3(kFinishThreads), cfg.dynamicSmemBytes = 0;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr, cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, router_finish_kernel, A, blocks);
    }
};

// ---- backward --------------------------------------------------------------------------------
struct BackwardArgs {
    const void *logits;
    int64_t ld, tokens, ld_out;
    int E, topk, normalize;
    const uint8_t *mask;
    const int32_t *idx;
    const float *gate, *lse;
    const int32_t *counts;
    const float *load, *d_gate, *d_loss;
    void *out;
};

// shared memory: direct[groups][G NE], columns beyond E included
template <typename T, int G, int NE, bool VEC>
__global__ void __launch_bounds__(kThreads) router_backward_kernel(const BackwardArgs A) {
    typedef RowMap<T, G, NE, VEC> Map;
    constexpr int GROUPS = kThreads / G;
    __shared__ __align__(16) float direct_all[GROUPS * G * NE];
    const int E = A.E, sub = threadIdx.x % G;
    float *direct = direct_all + (threadIdx.x / G) * (G * NE);
    const T *logits = static_cast<const T *>(A.logits);
    T *out = static_cast<T *>(A.out);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float S = 0.f, Zc = 0.f;
    if (A.d_loss) {
        const float nf = (float)max(A.counts[E], 1);
        S = A.d_loss[0] * (float)E / nf;
        Zc = 2.f * A.d_loss[1] / nf;
    }
    Pair share[NE / 2]; // S load: what the balance loss adds to dl / p, up to the row's constant
#pragma unroll
    for (int i = 0; i < NE / 2; ++i) {
        const int e = Map::col(2 * i, sub), f = Map::col(2 * i + 1, sub);
        share[i] = pair(A.d_loss && e < E ? S * A.load[e] : 0.f, A.d_loss && f < E ? S * A.load[f] : 0.f);
    }
#pragma unroll
    for (int i = 0; i < NE; ++i) direct[Map::col(i, sub)] = 0.f;
    __syncwarp();
    // the next token's row and gate terms (a lane's first choice) are under way while this one is worked on
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    int64_t t = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G;
    typename Map::Raw raw;
    bool live = false;
    float lse_next = 0.f, w_next = 0.f, dw_next = 0.f;
    int e_next = -1;
    const T *row = logits + t * A.ld; // of the token to be fetched next; the pointers move along
    int64_t pair_at = t * A.topk + sub;
    auto fetch = [&](int64_t at) {
        live = false;
        if (at < A.tokens) {
            live = !A.mask || A.mask[at] != 0;
            Map::load_raw(row, E, sub, raw);
            lse_next = A.lse[at];
            if (A.d_gate && sub < A.topk) {
                e_next = A.idx[pair_at];
                w_next = A.gate[pair_at];
                dw_next = A.d_gate[pair_at];
            }
        }
        row += step * A.ld, pair_at += step * A.topk;
    };
    fetch(t);
    T *to = out + t * A.ld_out;
    const bool more = A.topk > G; // choices beyond a lane's first
    for (int64_t t0 = (int64_t)blockIdx.x * GROUPS; t0 < A.tokens; t0 += step, t += step) {
        const bool in = t < A.tokens;
        float x[NE];
        if (live) {
            Map::unpack(raw, x);
        } else {
#pragma unroll
            for (int i = 0; i < NE; ++i) x[i] = -INFINITY;
        }
        const float lse = lse_next, w0 = w_next, dw0 = dw_next;
        const int e0 = e_next;
        fetch(t + step);
        // gate terms: a = sum w dw over the choices, then each choice's own term
        const bool gates = A.d_gate && in;
        float a = 0.f;
        if (gates) {
            if (e0 >= 0) a = w0 * dw0;
            for (int j = sub + G; more && j < A.topk; j += G)
                if (A.idx[t * A.topk + j] >= 0) a = fmaf(A.gate[t * A.topk + j], A.d_gate[t * A.topk + j], a);
        }
        a = group_sum<G>(a);
        if (gates) {
            if (e0 >= 0 && e0 < E) direct[e0] = A.normalize ? w0 * (dw0 - a) : dw0;
            for (int j = sub + G; more && j < A.topk; j += G) {
                const int e = A.idx[t * A.topk + j];
                if (e < 0 || e >= E) continue;
                const float dw = A.d_gate[t * A.topk + j];
                direct[e] = A.normalize ? A.gate[t * A.topk + j] * (dw - a) : dw;
            }
        }
        Pair p[NE / 2], f2 = pair(0.f, 0.f);
        const Pair log2e2 = pair(kLog2e, kLog2e), lse2 = pair(-lse, -lse);
#pragma unroll
        for (int i = 0; i < NE / 2; ++i) {
            float lo, hi;
            split(mul2(add2(pair(x[2 * i], x[2 * i + 1]), lse2), log2e2), lo, hi);
            p[i] = pair(ex2(lo), ex2(hi));
            f2 = fma2(p[i], share[i], f2);
        }
        float F, F1;
        split(f2, F, F1);
        F = group_sum<G>(F + F1);
        // lse is rounded at its own size: below 16 that costs every p less than 5e-7, in a row of the type's lowest value lse
        // equals the entries and every p is 1.  So rows beyond that have their powers summed again.
        float inv = 1.f;
        if (__any_sync(0xffffffffu, fabsf(lse) > 16.f)) {
            Pair s2 = p[0];
#pragma unroll
            for (int i = 1; i < NE / 2; ++i) s2 = add2(s2, p[i]);
            float sum, sum1;
            split(s2, sum, sum1);
            sum = group_sum<G>(sum + sum1);
            if (fabsf(lse) > 16.f) inv = rcp(sum); // by the row's own lse: what shares the warp changes nothing
        }
        __syncwarp();
        const float base = inv * (fmaf(Zc, lse, -F * inv) - (A.normalize ? 0.f : a));
        const Pair inv2 = pair(inv, inv), base2 = pair(base, base);
        float d[NE], own_v[NE];
        Map::read(direct, sub, own_v);
#pragma unroll
        for (int i = 0; i < NE / 2; ++i) {
            const Pair own = pair(own_v[2 * i], own_v[2 * i + 1]);
            const Pair g = A.normalize ? fma2(p[i], fma2(share[i], inv2, base2), own) : mul2(p[i], fma2(add2(share[i], own), inv2, base2));
            split(g, d[2 * i], d[2 * i + 1]);
        }
        if (in) Map::store(to, E, sub, d);
        to += step * A.ld_out;
        __syncwarp();
        if (gates) {
            if (e0 >= 0 && e0 < E) direct[e0] = 0.f;
            for (int j = sub + G; more && j < A.topk; j += G) {
                const int e = A.idx[t * A.topk + j];
                if (e >= 0 && e < E) direct[e] = 0.f;
            }
        }
        __syncwarp();
    }
}

struct BackwardLaunch {
    BackwardArgs A;
    cudaStream_t st;
    template <typename T, int G, int NE, bool VEC> cudaError_t run() {
        constexpr int GROUPS = kThreads / G;
        const int64_t want = (A.tokens + GROUPS - 1) / GROUPS;
        const int limit = 8 * sm_count();
        const int blocks = (int)(want < limit ? want : limit);
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)blocks), cfg.blockDim = dim3(kThreads), cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr, cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, router_backward_kernel<T, G, NE, VEC>, A);
    }
};

// ---- dispatch --------------------------------------------------------------------------------
// A stable counting sort of the pairs by expert.  Each block owns `chunk` consecutive pairs; each of its warps owns
// consecutive 32-pair rounds of them, so "earlier pair" is (block, warp, round, lane) in order.  Kernel 1 leaves the
// block's counts; kernel 2 adds the counts of all blocks (the total, for the offsets) and of the earlier ones (the
// block's base), counts its warps, and places every pair by its rank among the equal lanes before it.
constexpr int kSortThreads = 256;
constexpr int kSortWarps = kSortThreads / 32;

__device__ __forceinline__ int pair_expert(const int32_t *idx, int64_t i, int64_t pairs, int E) {
    if (i >= pairs) return -1;
    const int e = idx[i];
    return e >= 0 && e < E ? e : -1;
}

__global__ void __launch_bounds__(kSortThreads) dispatch_count_kernel(const int32_t *idx, int64_t pairs, int chunk, int E, int32_t *hist) {
    extern __shared__ int cnt[];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    for (int e = threadIdx.x; e < E; e += kSortThreads) cnt[e] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * chunk;
    for (int k = threadIdx.x; k < chunk; k += kSortThreads) {
        const int e = pair_expert(idx, i0 + k, pairs, E);
        if (e >= 0) atomicAdd(&cnt[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kSortThreads) hist[(int64_t)blockIdx.x * E + e] = cnt[e];
}

// shared memory: warp_base[kSortWarps][E] | start[E]
__global__ void __launch_bounds__(kSortThreads)
dispatch_place_kernel(const int32_t *idx, int64_t pairs, int chunk, int topk, int E, int blocks, const int32_t *hist, int32_t *offsets,
                      int32_t *rows, int32_t *slot) {
    extern __shared__ int sm[];
    int *wbase = sm, *start = sm + kSortWarps * E;
    __shared__ int scan_w[kSortWarps], carry;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per_warp = chunk / kSortWarps; // a multiple of 256
    const int64_t i0 = (int64_t)blockIdx.x * chunk + (int64_t)warp * per_warp;
    for (int k = threadIdx.x; k < kSortWarps * E; k += kSortThreads) wbase[k] = 0;
    if (threadIdx.x == 0) carry = 0;
    __syncthreads();
    for (int k = 0; k < per_warp; k += 32) {
        const int e = pair_expert(idx, i0 + k + lane, pairs, E);
        if (e >= 0) atomicAdd(&wbase[warp * E + e], 1);
    }
    if (blocks > 1) asm volatile("griddepcontrol.wait;" ::: "memory");
    __syncthreads();
    // start[e] = pairs of lower experts + pairs of e in earlier blocks
    for (int e0 = 0; e0 < E; e0 += kSortThreads) {
        const int e = e0 + threadIdx.x;
        int total = 0, before = 0;
        if (e < E) {
            if (blocks > 1) {
#pragma unroll 8
                for (int b = 0; b < blocks; ++b) {
                    const int c = hist[(int64_t)b * E + e];
                    total += c;
                    if (b < (int)blockIdx.x) before += c;
                }
            } else {
                for (int w = 0; w < kSortWarps; ++w) total += wbase[w * E + e];
            }
        }
        int incl = total;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane == 31) scan_w[warp] = incl;
        __syncthreads();
        int below = carry;
        for (int w = 0; w < warp; ++w) below += scan_w[w];
        const int off = below + incl - total;
        if (e < E) {
            start[e] = off + before;
            if (blockIdx.x == 0) offsets[e] = off;
        }
        __syncthreads();
        if (threadIdx.x == kSortThreads - 1) carry = below + incl;
        __syncthreads();
    }
    const int placed = carry;
    if (blockIdx.x == 0 && threadIdx.x == 0) offsets[E] = placed;
    // counts of the warps -> their bases
    for (int e = threadIdx.x; e < E; e += kSortThreads) {
        int at = start[e];
        for (int w = 0; w < kSortWarps; ++w) {
            const int c = wbase[w * E + e];
            wbase[w * E + e] = at;
            at += c;
        }
    }
    __syncthreads();
    for (int k = 0; k < per_warp; k += 32) {
        const int64_t i = i0 + k + lane;
        const int e = pair_expert(idx, i, pairs, E);
        const unsigned same = __match_any_sync(0xffffffffu, e);
        const int rank = __popc(same & ((1u << lane) - 1u));
        int at = 0;
        if (e >= 0) at = wbase[warp * E + e] + rank;
        __syncwarp();
        if (e >= 0 && rank == 0) wbase[warp * E + e] += __popc(same);
        __syncwarp();
        if (e >= 0) rows[at] = (int32_t)(i / topk);
        if (i < pairs) {
            if (slot) slot[i] = e >= 0 ? at : -1;
            if (i >= placed) rows[i] = -1; // behind the last pair; no pair's place lies there
        }
    }
}

bool bad_type(int dtype) { return dtype != FS_F32 && dtype != FS_BF16 && dtype != FS_F16; }

int check_common(const void *logits, int dtype, int64_t ld, int64_t tokens, int32_t experts) {
    if (tokens > 0 && !logits) return FS_ERR_NULL;
    if (bad_type(dtype) || tokens < 0 || experts < 1 || (tokens > 1 && ld < experts)) return FS_ERR_BAD_N; // one row: ld is not used
    if (experts > FS_ROUTER_MAX_EXPERTS) return FS_ERR_TOO_LARGE;
    if (reinterpret_cast<uintptr_t>(logits) % type_size(dtype)) return FS_ERR_UNSUPPORTED;
    return FS_OK;
}
int check_work(const void *work, int64_t work_bytes, int64_t need) {
    if (!work) return FS_ERR_NULL;
    if (work_bytes < need) return FS_ERR_TOO_LARGE;
    if (reinterpret_cast<uintptr_t>(work) & 15) return FS_ERR_UNSUPPORTED;
    return FS_OK;
}

} // namespace

// The calls use the scratch one after another, so it is as large as the largest of them needs:
//   forward   kMaxBlocks x (2 E + 2) words          duals   256 bytes + kMaxBlocks x (3 E + 1) words
//   dispatch  blocks x E words
int64_t workspace_bytes(int64_t tokens, int32_t experts, int32_t topk) {
    const int64_t sums = 256 + (int64_t)kMaxBlocks * (3 * (int64_t)experts + 2) * 4;
    const int64_t chunk = chunk_pairs(tokens * topk), chunks = (tokens * topk + chunk - 1) / chunk;
    const int64_t sort = chunks * experts * 4;
    return ((sums > sort ? sums : sort) + 255) / 256 * 256;
}

} // namespace fsr

extern "C" int64_t fs_router_workspace(int64_t tokens, int32_t experts, int32_t topk) {
    if (tokens < 0 || experts < 1 || experts > FS_ROUTER_MAX_EXPERTS || topk < 1 || topk > FS_ROUTER_MAX_TOPK || topk > experts ||
        tokens > INT32_MAX / topk)
        return 0;
    return fsr::workspace_bytes(tokens, experts, topk);
}

extern "C" int fs_router_forward(const void *logits_dev, int dtype, int64_t ld, int64_t tokens, int32_t experts,
                                 const uint8_t *mask_dev, const float *bias_dev, int32_t topk, int flags, int32_t *idx_out,
                                 float *gate_out, float *lse_out, int32_t *counts_out, float *load_out, float *prob_out,
                                 float *loss_out, void *work_dev, int64_t work_bytes, void *stream) {
    using namespace fsr;
    if (int rc = check_common(logits_dev, dtype, ld, tokens, experts)) return rc;
    if (tokens > 0 && (!idx_out || !gate_out)) return FS_ERR_NULL;
    if (topk < 1 || topk > experts || (flags & ~FS_ROUTE_NORMALIZE)) return FS_ERR_BAD_N;
    if (topk > FS_ROUTER_MAX_TOPK || tokens > INT32_MAX / topk) return FS_ERR_TOO_LARGE;
    if (int rc = check_work(work_dev, work_bytes, workspace_bytes(tokens, experts, topk))) return rc;
    ForwardLaunch F;
    ForwardArgs &A = F.A;
    A.logits = logits_dev, A.ld = ld, A.tokens = tokens, A.E = experts, A.topk = topk;
    A.normalize = flags & FS_ROUTE_NORMALIZE, A.joint = 0;
    A.stats = counts_out || load_out || prob_out || loss_out;
    A.mask = mask_dev, A.bias = bias_dev, A.idx = idx_out, A.gate = gate_out, A.lse = lse_out;
    A.counts = counts_out, A.load = load_out, A.prob = prob_out, A.loss = loss_out;
    A.part_p = static_cast<float *>(work_dev);
    A.part_c = reinterpret_cast<int32_t *>(A.part_p + (int64_t)kMaxBlocks * experts);
    A.part_z = reinterpret_cast<float *>(A.part_c + (int64_t)kMaxBlocks * experts);
    A.part_n = reinterpret_cast<int32_t *>(A.part_z + kMaxBlocks);
    F.st = static_cast<cudaStream_t>(stream);
    if (tokens == 0 && !A.stats) return FS_OK;
    const cudaError_t e = by_type(F, dtype, experts, rows_aligned(logits_dev, ld, dtype));
    return e == cudaSuccess ? FS_OK : fsk_cuda_failed(e, "fs_router_forward");
}

extern "C" int fs_router_backward(const void *logits_dev, int dtype, int64_t ld, int64_t tokens, int32_t experts,
                                  const uint8_t *mask_dev, int32_t topk, int flags, const int32_t *idx_dev,
                                  const float *gate_dev, const float *lse_dev, const int32_t *counts_dev, const float *load_dev,
                                  const float *d_gate_dev, const float *d_loss_dev, void *d_logits_out, int64_t ld_out,
                                  void *stream) {
    using namespace fsr;
    if (int rc = check_common(logits_dev, dtype, ld, tokens, experts)) return rc;
    if (tokens > 0 && (!lse_dev || !d_logits_out)) return FS_ERR_NULL;
    if (tokens > 0 && d_gate_dev && (!idx_dev || !gate_dev)) return FS_ERR_NULL;
    if (d_loss_dev && (!counts_dev || !load_dev)) return FS_ERR_NULL;
    if (topk < 1 || topk > experts || (flags & ~FS_ROUTE_NORMALIZE) || (tokens > 1 && ld_out < experts)) return FS_ERR_BAD_N;
    if (topk > FS_ROUTER_MAX_TOPK || tokens > INT32_MAX / topk) return FS_ERR_TOO_LARGE;
    if (reinterpret_cast<uintptr_t>(d_logits_out) % type_size(dtype)) return FS_ERR_UNSUPPORTED;
    if (tokens == 0) return FS_OK;
    BackwardLaunch B;
    BackwardArgs &A = B.A;
    A.logits = logits_dev, A.ld = ld, A.tokens = tokens, A.ld_out = ld_out, A.E = experts, A.topk = topk;
    A.normalize = flags & FS_ROUTE_NORMALIZE;
    A.mask = mask_dev, A.idx = idx_dev, A.gate = gate_dev, A.lse = lse_dev, A.counts = counts_dev, A.load = load_dev;
    A.d_gate = d_gate_dev, A.d_loss = d_loss_dev, A.out = d_logits_out;
    B.st = static_cast<cudaStream_t>(stream);
    const bool vec = rows_aligned(logits_dev, ld, dtype) && rows_aligned(d_logits_out, ld_out, dtype);
    const cudaError_t e = by_type(B, dtype, experts, vec);
    return e == cudaSuccess ? FS_OK : fsk_cuda_failed(e, "fs_router_backward");
}

extern "C" int fs_router_dispatch(const int32_t *idx_dev, int64_t tokens, int32_t topk, int32_t experts, int32_t *offsets_out,
                                  int32_t *rows_out, int32_t *slot_out, void *work_dev, int64_t work_bytes, void *stream) {
    using namespace fsr;
    if (!offsets_out || (tokens > 0 && (!idx_dev || !rows_out))) return FS_ERR_NULL;
    if (tokens < 0 || experts < 1 || topk < 1 || topk > experts) return FS_ERR_BAD_N;
    if (experts > FS_ROUTER_MAX_EXPERTS || topk > FS_ROUTER_MAX_TOPK || tokens > INT32_MAX / topk) return FS_ERR_TOO_LARGE;
    if (int rc = check_work(work_dev, work_bytes, workspace_bytes(tokens, experts, topk))) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t pairs = tokens * topk;
    const int chunk = (int)chunk_pairs(pairs), blocks = (int)(pairs > chunk ? (pairs + chunk - 1) / chunk : 1);
    int32_t *hist = static_cast<int32_t *>(work_dev);
    const size_t smem = (size_t)(kSortWarps + 1) * experts * sizeof(int);
    if (blocks == 1) {
        dispatch_place_kernel<<<1, kSortThreads, smem, st>>>(idx_dev, pairs, chunk, topk, experts, 1, hist, offsets_out, rows_out, slot_out);
        const cudaError_t e = cudaGetLastError();
        return e == cudaSuccess ? FS_OK : fsk_cuda_failed(e, "fs_router_dispatch");
    }
    dispatch_count_kernel<<<blocks, kSortThreads, (size_t)experts * sizeof(int), st>>>(idx_dev, pairs, chunk, experts, hist);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return fsk_cuda_failed(e, "fs_router_dispatch");
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks), cfg.blockDim = dim3(kSortThreads), cfg.dynamicSmemBytes = smem, cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr, cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, dispatch_place_kernel, idx_dev, pairs, chunk, (int)topk, (int)experts, blocks, (const int32_t *)hist,
                           offsets_out, rows_out, slot_out);
    return e == cudaSuccess ? FS_OK : fsk_cuda_failed(e, "fs_router_dispatch");
}
