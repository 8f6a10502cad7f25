// Group norm with an activation over channels-last grids, x [samples, tokens, channels]: mean and variance over the tokens and the channels of a group,
// n = (x - mean) rstd, y = act(n weight + bias); and its backward, with g = d_y act'(z):
//   d_bias = sum g, d_weight = sum g n, d_x = rstd (g weight - mean(g weight) - n mean(g weight n)), the means over the group.
//
// Both need sums over a sample before the first output, so x (backward: and d_y) is read twice:
//   1. a block takes a chunk of tokens, a thread E channels of it that stay the same, and keeps their sums in registers;
//   2. the blocks' sums are joined, in a fixed order;
//   3. blocks on the same chunks, from their last tokens on, write the outputs: what the first pass read last is still in L2.
//
// A thread's mean and squared deviations from it are updated value by value (Welford 1962), those of several threads or blocks joined by the mean of all and the
// deviations about it, so that nothing cancels however far the mean lies from 0; all in fp32.
//
// What bounds it: HBM in large samples (2 x 2203200 x 128, 32 groups, silu, a call on its own: 575 us, 1.1 GB read twice and written; backward 950), the first pass at 5.2 TB/s, the second at
// 6.1; in small ones launches and latency (2048 x 96: one launch, 7.5 us).  By loads into registers instead of the copy engine's stages the first pass took 200 us of 2203200 x 128 instead of 117.
#include "block_act.cuh"
#include "block_kernels.h"
#include "elem_vec.cuh"
#include "tc_common.cuh"

#ifdef TERRA_ELEM_F16
#define launch_group_norm_fwd launch_group_norm_fwd_f16
#define launch_group_norm_bwd launch_group_norm_bwd_f16
#define read_group_norm_status read_group_norm_status_f16
#define g_group_norm_timeout g_group_norm_timeout_f16
#endif

namespace terra {

__device__ int g_group_norm_timeout = 0;       // set when a bounded wait expired

namespace {

constexpr int kBlock = 256;
// Tokens that a thread has of a stage or, where its vectors are smaller than 16 bytes, reads at a time of each of `tensors`.  us of 100000 x 1001 of
// 7 groups and of 300000 x 131 of one: forward 563 and 234 with 4 of them and 3 blocks of an SM, 440 and 125 with 16 and 4; backward 1371 and 403 with
// 4 and 2, 818 and 221 with 16 and 3, 759 and 206 with 8 and 4 (790 and 214 since rstd is a factor of its own in the second pass).
__host__ __device__ constexpr int deep(int elems, int tensors) { return elems == 8 ? 4 : 16 / tensors; }
// Blocks of an SM, and stages of a block: kBlock x 4 vectors of 16 bytes each, of x and, backward, of d_y.
constexpr int kStage = kBlock * deep(8, 1) * 16;
constexpr int kKeepFwd = 8, kKeepBwd = 4, kMostCluster = 8;        // vectors that a thread of the kernels for small samples holds; their blocks that share a sample's slab
constexpr int kSmallBlocksSm = 2;      // those kernels' blocks on an SM, by their registers
constexpr long long kMostHeld = 176 * 1024, kBlockSmem = 227 * 1024, kSmSmem = 228 * 1024;        // bytes of vectors that a block of theirs holds; of a block; of an SM
constexpr int kMostSamples = 65535;
constexpr int kFewSamples = 8;         // so many samples' sums are added up one after the other
// The most blocks that the kernels for small samples are taken for, forward and backward.  us, they / three launches: forward 16 x 1024 x 320 16.6 / 23.1,
// 256 x 256 x 128 28.3 / 23.4; backward 1000 x 64 x 64 45.6 / 50.9, 64 x 1024 x 640 187 / 136.
constexpr long long kSmallBlocksFwd = 4 * kPlanSms, kSmallBlocksBwd = 16 * kPlanSms;
constexpr int kStagesFwd = 4, kStagesBwd = 3;
__host__ __device__ constexpr int blocks(int elems, int tensors) { return elems == 8 ? 4 - tensors : 4; }
constexpr int kRingFwd = kStage * kStagesFwd, kRingBwd = 2 * kStage * kStagesBwd;

struct Pass {
    const uint16_t *x, *d_y;
    uint16_t* out;                     // y, or d_x
    const float *weight, *bias;
    float *stats, *partial, *sums, *d_weight, *d_bias;
    long long tokens, chunk;           // of a sample; of a block
    int channels, groups, per_group;
    int first, samples;                // of this launch
    int all_samples;
    int activation;
    int across, rows;                  // threads side by side along the channels, and tokens at a time
    int slab, pieces;                  // channels of a block; blocks that share a group (1: none)
    int room, half;                    // cluster kernels: where held vectors begin in shared memory, and d_y's behind x's
    float eps;
    double per_value;                  // 1 / values of a group
};

// Where a block and its thread stand.
struct Place {
    int sample, chunk, c0, sub;        // sample of all; first channel; row among the block's
    int s0, s1;                        // channels of the block
    long long t0, t1;
    bool there;
};
template <int E>
__device__ __forceinline__ Place place_of(const Pass& p) {
    Place a;
    const int v = threadIdx.x % p.across;
    a.sub = threadIdx.x / p.across;
    a.sample = p.first + blockIdx.y;
    a.chunk = blockIdx.x;
    // (a slab that is a piece of a group ends with the group)
    a.s0 = p.pieces == 1 ? blockIdx.z * p.slab : blockIdx.z / p.pieces * p.per_group + blockIdx.z % p.pieces * p.slab;
    a.s1 = min(p.pieces == 1 ? p.channels : (int)(blockIdx.z / p.pieces + 1) * p.per_group, a.s0 + p.slab);
    a.c0 = a.s0 + v * E;
    a.t0 = a.chunk * p.chunk;
    a.t1 = min(p.tokens, a.t0 + p.chunk);
    a.there = a.sub < p.rows && a.c0 < a.s1;
    return a;
}

// f(x's, d_y's vectors of deep(E, STREAMS) tokens, how many of them there are, the first one's offset, the offset from one to the next) for the thread's
// channels of all of the chunk's tokens, in order or from the last ones on.  By every thread of the block.
// Vectors of 16 bytes: the copy engine brings stages of tokens into `ring`, so that what is under way does not depend on the registers.  Others: as many reads
// at a time.
template <int E, int STREAMS, int STAGES, bool BACK, class F>
__device__ __forceinline__ void walk(const Pass& p, const Place& a, uint8_t* ring, F f) {
    constexpr int kDeep = deep(E, STREAMS);
    const long long base = (long long)a.sample * p.tokens * p.channels;
    const int s0 = a.s0, s1 = a.s1;
    if constexpr (E == 8) {
        __shared__ unsigned long long full[STAGES];
        __shared__ int abort_flag;
        const int width = s1 - s0, per = p.rows * kDeep;       // channels and tokens of a stage
        const uint32_t ring_at = smem_u32(ring), half = (uint32_t)per * width * 2;
        const int tiles = (int)((a.t1 - a.t0 + per - 1) / per);
        auto bar = [&](int s) { return smem_u32(&full[s]); };
        auto first_token = [&](int i) { return a.t0 + (long long)(BACK ? tiles - 1 - i : i) * per; };
        auto fetch = [&](int i, int s) {               // by one thread
            const long long t = first_token(i);
            const int n = (int)min((long long)per, a.t1 - t);
            tc::mbar_arrive_expect_tx(bar(s), (uint32_t)(STREAMS * n * width * 2));
#pragma unroll
            for (int k = 0; k < STREAMS; ++k) {
                const uint16_t* from = (k ? p.d_y : p.x) + base + t * p.channels + s0;
                const uint32_t to = ring_at + (s * STREAMS + k) * half;
                if (width == p.channels) tc::bulk_load(to, from, (uint32_t)(n * width * 2), bar(s));
                else
                    for (int j = 0; j < n; ++j) tc::bulk_load(to + j * width * 2, from + (long long)j * p.channels, (uint32_t)(width * 2), bar(s));
            }
        };
        if (threadIdx.x == 0) {
            abort_flag = 0;
            for (int s = 0; s < STAGES; ++s) tc::mbar_init(bar(s), 1);
            tc::fence_barrier_init();
            for (int i = 0; i < STAGES && i < tiles; ++i) fetch(i, i);
        }
        __syncthreads();
        int s = 0, i = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (; i < tiles; ++i) {
            ok = tc::mbar_wait<0>(bar(s), phase, &abort_flag);
            if (ok && a.there) {
                const long long t = first_token(i) + a.sub, left = a.t1 - t;
                const uint4* from = reinterpret_cast<const uint4*>(ring + s * STREAMS * half + ((uint32_t)a.sub * width + (a.c0 - s0)) * 2);
                Raw<8> x[kDeep], g[kDeep];
#pragma unroll
                for (int k = 0; k < kDeep; ++k) {      // (rows that are not there: what is left of earlier ones)
                    x[k].v = from[k * p.rows * width / 8];
                    if (STREAMS == 2) g[k].v = from[half / 16 + k * p.rows * width / 8];
                }
                const int n = left > (long long)(kDeep - 1) * p.rows ? kDeep : left <= 0 ? 0 : (int)((left + p.rows - 1) / p.rows);
                f(x, g, n, base + t * p.channels + a.c0, p.rows * p.channels);
            }
            if (!__syncthreads_and(ok)) break;         // the stage has been read
            if (threadIdx.x == 0 && i + STAGES < tiles) fetch(i + STAGES, s);
            if (++s == STAGES) { s = 0; phase ^= 1; }
        }
        if (i < tiles && threadIdx.x == 0) {           // after an expired wait: what is under way lands before the block ends
            int ignore = 0;
            for (int j = i; j < i + STAGES && j < tiles; ++j) tc::mbar_wait<0>(bar(j % STAGES), (j / STAGES) & 1, &ignore, 200000000LL);
            atomicExch(&g_group_norm_timeout, 1);
        }
        __syncthreads();
    } else if (a.there) {
        const long long step = (long long)p.rows * p.channels, tokens = a.t1 - a.t0;
        const long long batches = (tokens + (long long)kDeep * p.rows - 1) / ((long long)kDeep * p.rows);
        for (long long i = 0; i < batches; ++i) {
            const long long t = a.t0 + a.sub + (BACK ? batches - 1 - i : i) * kDeep * p.rows, at = base + t * p.channels + a.c0, left = a.t1 - t;
            const int n = left > (long long)(kDeep - 1) * p.rows ? kDeep : left <= 0 ? 0 : (int)((left + p.rows - 1) / p.rows);
            Raw<E> x[kDeep], g[kDeep];
#pragma unroll
            for (int k = 0; k < kDeep; ++k) {
                x[k].zero();
                g[k].zero();
                if (k < n) {
                    x[k].load(p.x + at + k * step);
                    if (STREAMS == 2) g[k].load(p.d_y + at + k * step);
                }
            }
            f(x, g, n, at, (int)step);
        }
    }
}

// f(k) for the tokens that are there, without a test for each where all of them are
template <int kDeep, class F>
__device__ __forceinline__ void each_token(int n, F f) {
    if (n == kDeep) {
#pragma unroll
        for (int k = 0; k < kDeep; ++k) f(k);
    } else {
#pragma unroll
        for (int k = 0; k < kDeep; ++k)
            if (k < n) f(k);
    }
}

// Moments of values in parts, each with its count, mean and squared deviations, joined by a warp: the mean of all, then the deviations about it.  part(i): the
// i-th of `parts`.  (Means are added up as differences from the first one, so that they neither cancel nor leave fp32's range.)
struct Moments { float n, mean, m2; };
template <class F>
__device__ __forceinline__ Moments joined(int parts, F part) {
    const int lane = threadIdx.x & 31;
    const float about = parts > 0 ? part(0).mean : 0.f;
    float n = 0.f, sum = 0.f, m2 = 0.f;
    for (int i = lane; i < parts; i += 32) {
        const Moments m = part(i);
        n += m.n;
        sum += m.n > 0.f ? m.n * (m.mean - about) : 0.f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        n += __shfl_xor_sync(0xffffffffu, n, o);
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    const float mean = n > 0.f ? about + sum / n : 0.f;
    for (int i = lane; i < parts; i += 32) {
        const Moments m = part(i);
        const float d = m.mean - mean;
        m2 += m.n > 0.f ? fmaf(m.n * d, d, m.m2) : 0.f;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
    return {n, mean, m2};
}

// The same of one part a lane.
__device__ __forceinline__ Moments joined_lanes(Moments m) {
    const float about = __shfl_sync(0xffffffffu, m.mean, 0);
    float n = m.n, sum = m.n > 0.f ? m.n * (m.mean - about) : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        n += __shfl_xor_sync(0xffffffffu, n, o);
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    const float mean = n > 0.f ? about + sum / n : 0.f, d = m.mean - mean;
    float m2 = m.n > 0.f ? fmaf(m.n * d, d, m.m2) : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
    return {n, mean, m2};
}

// The moments of each group's values in a chunk, to partial[sample of the launch][group][piece][chunk].
template <int E>
__global__ void __launch_bounds__(kBlock, blocks(E, 1)) group_stats_kernel(const __grid_constant__ Pass p) {
    extern __shared__ __align__(128) uint8_t shared[];
    let_dependents_start();
    const Place a = place_of<E>(p);
    constexpr int kPairs = E < 2 ? 1 : E / 2;
    Pair minus_mean[kPairs], m2[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) minus_mean[i] = m2[i] = both(0.f);
    float count = 0.f;
    wait_for_prerequisites();
    walk<E, 1, kStagesFwd, false>(p, a, shared, [&](const Raw<E> (&x)[deep(E, 1)], const Raw<E> (&)[deep(E, 1)], int n, long long, int) {
        if (n == 0) return;
        if (count == 0.f) {                            // the first value is the first mean, exactly
            Pair v[kPairs];
            x[0].pairs(v);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) minus_mean[i] = pmul(v[i], both(-1.f));
        }
#pragma unroll
        for (int q = 0; q < deep(E, 1); q += 4) {
            if (q + 4 <= n) {
                // four tokens' own mean and deviations, joined with the others'
                Pair v[4][kPairs];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[q + k].pairs(v[k]);
                const float all = count + 4.f, share = 4.f * fast_rcp(all);
                const Pair minus_share = both(-share), both_count = both(count * share);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k][i] = padd(v[k][i], minus_mean[i]);
                    const Pair d = pmul(padd(padd(v[0][i], v[1][i]), padd(v[2][i], v[3][i])), both(0.25f)), minus_d = pmul(d, both(-1.f));
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const Pair e = padd(v[k][i], minus_d);
                        m2[i] = pfma(e, e, m2[i]);
                    }
                    minus_mean[i] = pfma(d, minus_share, minus_mean[i]);
                    m2[i] = pfma(pmul(d, d), both_count, m2[i]);
                }
                count = all;
            } else {
#pragma unroll
                for (int k = q; k < q + 4; ++k) {
                    if (k >= n) break;
                    Pair v[kPairs];
                    x[k].pairs(v);
                    count += 1.f;
                    const Pair minus_share = both(-fast_rcp(count));
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        const Pair d = padd(v[i], minus_mean[i]);
                        minus_mean[i] = pfma(d, minus_share, minus_mean[i]);
                        m2[i] = pfma(d, padd(v[i], minus_mean[i]), m2[i]);
                    }
                }
            }
        }
    });
    // A thread's channels, then the rows of the block and the channels of a group.
    float mean[E], dev[E];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        float lo, hi;
        split_pair(minus_mean[i], lo, hi);
        mean[2 * i % E] = -lo;
        if (E > 1) mean[(2 * i + 1) % E] = -hi;
        split_pair(m2[i], lo, hi);
        dev[2 * i % E] = lo;
        if (E > 1) dev[(2 * i + 1) % E] = hi;
    }
    const int tid = threadIdx.x, wide = p.across * E, ch = (tid % p.across) * E;
    float *mean_of = reinterpret_cast<float*>(shared), *m2_of = mean_of + kBlock * E, *count_of = m2_of + kBlock * E;       // (the stages have been read)
    if (a.sub < p.rows) {
        if (ch == 0) count_of[a.sub] = count;          // (a row's threads have the same number of tokens)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            mean_of[a.sub * wide + ch + e] = mean[e];
            m2_of[a.sub * wide + ch + e] = dev[e];
        }
    }
    __syncthreads();
    const int s0 = a.s0, s1 = a.s1, g0 = s0 / p.per_group, g1 = (s1 - 1) / p.per_group + 1, warp = tid >> 5, lane = tid & 31;
    for (int g = g0 + warp; g < g1; g += kBlock / 32) {                // a warp to a group
        const int c0 = max(s0, g * p.per_group) - s0, c1 = min(s1, (g + 1) * p.per_group) - s0;
        const int across = c1 - c0;
        const Moments m = joined(p.rows * across, [&](int i) {
            const int r = (int)((unsigned)i / (unsigned)across), c = c0 + i - r * across;
            return Moments{count_of[r], mean_of[r * wide + c], m2_of[r * wide + c]};
        });
        if (lane == 0) {
            float* to = p.partial + 3 * ((((long long)blockIdx.y * p.groups + g) * p.pieces + (p.pieces == 1 ? 0 : blockIdx.z % p.pieces)) * gridDim.x + a.chunk);
            to[0] = m.n;
            to[1] = m.mean;
            to[2] = m.m2;
        }
    }
}

// stats[sample][group] = (mean, rstd), a block to each (groups x samples of them: their product may be more than a grid's first dimension takes): its warps
// join a part of the entries each, the first one those
__global__ void __launch_bounds__(kBlock) group_stats_join_kernel(const __grid_constant__ Pass p, int entries) {
    __shared__ Moments warps[kBlock / 32];
    let_dependents_start();
    wait_for_prerequisites();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, share = (entries + kBlock / 32 - 1) / (kBlock / 32), first = min(entries, warp * share);
    const long long at = (long long)blockIdx.y * p.groups + blockIdx.x;
    const float* from = p.partial + 3 * (at * entries + first);
    Moments m = joined(min(share, entries - first), [&](int i) { return Moments{from[3 * i], from[3 * i + 1], from[3 * i + 2]}; });
    if (lane == 0) warps[warp] = m;
    __syncthreads();
    if (warp) return;
    m = joined_lanes(lane < kBlock / 32 ? warps[lane] : Moments{0.f, 0.f, 0.f});
    if (lane) return;
    float* out = p.stats + 2 * ((long long)p.first * p.groups + at);
    out[0] = m.mean;
    out[1] = rsqrtf((float)((double)m.m2 * p.per_value) + p.eps);
}

// A thread's channels: z = (x - mean) a + b
template <int E>
struct Channels {
    static constexpr int kPairs = E < 2 ? 1 : E / 2;
    Pair minus_mean[kPairs], a[kPairs], b[kPairs];
    __device__ __forceinline__ void load(const Pass& p, const Place& at, const float* stats) {       // mean and rstd of the sample's groups
        float m[2 * kPairs] = {}, s[2 * kPairs] = {}, t[2 * kPairs] = {};
        if (at.there)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int c = at.c0 + e;
                const float* st = stats + 2 * (c / p.per_group);
                m[e] = -st[0];
                s[e] = st[1] * p.weight[c];
                t[e] = p.bias[c];
            }
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            minus_mean[i] = pair_of(m[2 * i], m[2 * i + 1]);
            a[i] = pair_of(s[2 * i], s[2 * i + 1]);
            b[i] = pair_of(t[2 * i], t[2 * i + 1]);
        }
    }
};

template <int E>
__global__ void __launch_bounds__(kBlock, blocks(E, 1)) group_apply_kernel(const __grid_constant__ Pass p) {
    extern __shared__ __align__(128) uint8_t shared[];
    let_dependents_start();
    const Place a = place_of<E>(p);
    wait_for_prerequisites();
    Channels<E> ch;
    ch.load(p, a, p.stats + 2 * (long long)a.sample * p.groups);
    with_act(p.activation, [&](auto tag) {
        walk<E, 1, kStagesFwd, true>(p, a, shared, [&](const Raw<E> (&x)[deep(E, 1)], const Raw<E> (&)[deep(E, 1)], int n, long long at, int step) {
            each_token<deep(E, 1)>(n, [&](int k) {
                Pair v[Channels<E>::kPairs];
                x[k].pairs(v);
#pragma unroll
                for (int i = 0; i < Channels<E>::kPairs; ++i) v[i] = act2<decltype(tag)::value>(pfma(padd(v[i], ch.minus_mean[i]), ch.a[i], ch.b[i]));
                store_pairs<E>(p.out + at + (long long)k * step, v);
            });
        });
    });
}

// Backward, first pass: for each channel the chunk's sums of g and of g (x - mean), to partial[sample of the launch][chunk][channel].
template <int E>
__global__ void __launch_bounds__(kBlock, blocks(E, 2)) group_bwd_sums_kernel(const __grid_constant__ Pass p) {
    extern __shared__ __align__(128) uint8_t shared[];
    float* rows_sums = reinterpret_cast<float*>(shared);       // [rows][across E][2], once the stages have been read
    let_dependents_start();
    const Place a = place_of<E>(p);
    constexpr int kPairs = Channels<E>::kPairs;
    Pair s1[kPairs], s2[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) s1[i] = s2[i] = both(0.f);
    wait_for_prerequisites();
    Channels<E> ch;
    ch.load(p, a, p.stats + 2 * (long long)a.sample * p.groups);
    with_act(p.activation, [&](auto tag) {
        walk<E, 2, kStagesBwd, false>(p, a, shared, [&](const Raw<E> (&x)[deep(E, 2)], const Raw<E> (&d_y)[deep(E, 2)], int n, long long, int) {
            each_token<deep(E, 2)>(n, [&](int k) {
                Pair v[kPairs], g[kPairs];
                x[k].pairs(v);
                d_y[k].pairs(g);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const Pair d = padd(v[i], ch.minus_mean[i]);
                    const Pair gg = pmul(g[i], finite_slope2<decltype(tag)::value>(pfma(d, ch.a[i], ch.b[i])));
                    s1[i] = padd(s1[i], gg);
                    s2[i] = pfma(gg, d, s2[i]);
                }
            });
        });
    });
    const int wide = p.across * E, c = (threadIdx.x % p.across) * E;
    if (a.sub < p.rows)
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            float v[4];
            split_pair(s1[i], v[0], v[2]);
            split_pair(s2[i], v[1], v[3]);
#pragma unroll
            for (int e = 0; e < 2 && e < E; ++e) {
                rows_sums[2 * (a.sub * wide + c + 2 * i + e)] = v[2 * e];
                rows_sums[2 * (a.sub * wide + c + 2 * i + e) + 1] = v[2 * e + 1];
            }
        }
    __syncthreads();
    float* to = p.partial + 2 * (((long long)blockIdx.y * gridDim.x + a.chunk) * p.channels + a.s0);
    for (int i = threadIdx.x; i < 2 * (a.s1 - a.s0); i += kBlock) {
        float s = 0.f;
        for (int r = 0; r < p.rows; ++r) s += rows_sums[2 * r * wide + i];
        to[i] = s;
    }
}

// sums[sample][channel] = the chunks' sums added up: 32 values to a block, 32 slices of the chunks
__global__ void __launch_bounds__(1024) group_bwd_join_kernel(const __grid_constant__ Pass p, int chunks) {
    __shared__ float slices[32][33];
    let_dependents_start();
    wait_for_prerequisites();
    const int cx = threadIdx.x & 31, slice = threadIdx.x >> 5, i = blockIdx.x * 32 + cx, n = 2 * p.channels;
    const float* from = p.partial + (long long)blockIdx.y * chunks * n;
    float s = 0.f;
    if (i < n)
#pragma unroll 4
        for (int c = slice; c < chunks; c += 32) s += from[(long long)c * n + i];
    slices[slice][cx] = s;
    __syncthreads();
    s = slices[cx][slice];
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int w = blockIdx.x * 32 + slice;
    if (cx == 0 && w < n) p.sums[(long long)(p.first + blockIdx.y) * n + w] = s;
}

// The terms of group g's d_x, -rstd mean(g weight) and -rstd mean(g weight n), of its channels' sums (two of each); by a warp.  (The sum goes through
// g weight (x - mean): rstd comes to it factor by factor, so that nothing leaves fp32's range that is not there in d_x.)
__device__ __forceinline__ void group_means(const Pass& p, const Place& a, int g, const float* sums, float* out, int lane) {
    float l = 0.f, m = 0.f;
    for (int c = g * p.per_group + lane; c < (g + 1) * p.per_group; c += 32) {
        const float w = p.weight[c];
        l = fmaf(w, sums[2 * c], l);
        m = fmaf(w, sums[2 * c + 1], m);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        l += __shfl_xor_sync(0xffffffffu, l, o);
        m += __shfl_xor_sync(0xffffffffu, m, o);
    }
    if (lane) return;
    const float rstd = p.stats[2 * ((long long)a.sample * p.groups + g) + 1], by = (float)p.per_value;
    out[0] = -rstd * (l * by);
    out[1] = -(rstd * (rstd * (m * by)));
}
template <int E>
__device__ __forceinline__ void group_terms(const Pass& p, const Place& a, const float* group_sums, Pair (&c0)[Channels<E>::kPairs], Pair (&c1)[Channels<E>::kPairs],
                                            Pair (&rstd)[Channels<E>::kPairs]) {
    const int g0 = a.s0 / p.per_group;
    const float* stats = p.stats + 2 * ((long long)a.sample * p.groups + g0) + 1;
#pragma unroll
    for (int i = 0; i < Channels<E>::kPairs; ++i) {
        const int lo = 2 * ((a.c0 + 2 * i) / p.per_group - g0), hi = E > 1 ? 2 * ((a.c0 + 2 * i + 1) / p.per_group - g0) : lo;
        c0[i] = pair_of(group_sums[lo], group_sums[hi]);
        c1[i] = pair_of(group_sums[lo + 1], group_sums[hi + 1]);
        rstd[i] = pair_of(stats[lo], stats[hi]);
    }
}

// Second pass: d_x = a g + c0 + (x - mean) rstd c1 with c0 = - rstd mean(g weight), c1 = - rstd mean(g weight n) of the group.
// The last launch's blocks also add up the sums of a few samples: d_weight and d_bias.
template <int E>
__global__ void __launch_bounds__(kBlock, blocks(E, 2)) group_bwd_apply_kernel(const __grid_constant__ Pass p) {
    extern __shared__ __align__(128) uint8_t shared[];
    float* group_sums = reinterpret_cast<float*>(shared + (E == 8 ? kRingBwd : 0));       // [groups of the slab][2]
    let_dependents_start();
    const Place a = place_of<E>(p);
    constexpr int kPairs = Channels<E>::kPairs;
    wait_for_prerequisites();
    Channels<E> ch;
    ch.load(p, a, p.stats + 2 * (long long)a.sample * p.groups);
    const int g0 = a.s0 / p.per_group, g1 = (a.s1 - 1) / p.per_group + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int g = g0 + warp; g < g1; g += kBlock / 32) group_means(p, a, g, p.sums + 2ll * a.sample * p.channels, group_sums + 2 * (g - g0), lane);
    __syncthreads();
    if (p.all_samples <= kFewSamples && p.first + p.samples == p.all_samples) {
        const long long block = ((long long)blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x, blocks = (long long)gridDim.x * gridDim.y * gridDim.z;
        for (long long c = block * kBlock + threadIdx.x; c < p.channels; c += blocks * kBlock) {
            float w = 0.f, b = 0.f;
            for (int s = 0; s < p.all_samples; ++s) {
                b += p.sums[2 * ((long long)s * p.channels + c)];
                w = fmaf(p.sums[2 * ((long long)s * p.channels + c) + 1], p.stats[2 * ((long long)s * p.groups + c / p.per_group) + 1], w);
            }
            p.d_weight[c] = w;
            p.d_bias[c] = b;
        }
    }
    Pair c0[kPairs], c1[kPairs], rstd[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) c0[i] = c1[i] = rstd[i] = both(0.f);
    if (a.there) group_terms<E>(p, a, group_sums, c0, c1, rstd);
    with_act(p.activation, [&](auto tag) {
        walk<E, 2, kStagesBwd, true>(p, a, shared, [&](const Raw<E> (&x)[deep(E, 2)], const Raw<E> (&d_y)[deep(E, 2)], int n, long long at, int step) {
            each_token<deep(E, 2)>(n, [&](int k) {
                Pair v[kPairs], g[kPairs];
                x[k].pairs(v);
                d_y[k].pairs(g);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const Pair d = padd(v[i], ch.minus_mean[i]);
                    const Pair gg = pmul(g[i], finite_slope2<decltype(tag)::value>(pfma(d, ch.a[i], ch.b[i])));
                    v[i] = pfma(gg, ch.a[i], pfma(pmul(d, rstd[i]), c1[i], c0[i]));
                }
                store_pairs<E>(p.out + at + (long long)k * step, v);
            });
        });
    });
}

// ---- samples that a cluster of blocks holds ----------------------------------------------------------------------
// One launch: the blocks of a cluster share the tokens of a sample's slab (whole groups), which are read once, up to `KEEP` vectors of a thread into its registers or
// (KEEP 0) as many as there are into shared memory; the blocks' sums meet in shared memory.

// A thread's vectors of the tokens from `from` on, `step` apart; n of them.
template <int E, int KEEP>
struct Held {
    Raw<E> r[KEEP ? KEEP : 1];
    uint4* mine;                       // in shared memory, kBlock of them apart
    __device__ __forceinline__ void load(const uint16_t* from, long long step, int n, uint8_t* room) {
        if constexpr (KEEP) {
#pragma unroll
            for (int k = 0; k < KEEP; ++k) {
                r[k].zero();
                if (k < n) r[k].load(from + k * step);
            }
        } else {
            mine = reinterpret_cast<uint4*>(room) + threadIdx.x;
            for (int k = 0; k < n; ++k) cp_async16(smem_u32(mine + k * kBlock), from + k * step, 16);
            cp_async_commit();
        }
    }
    __device__ __forceinline__ void wait() {           // (each thread reads what it has copied itself)
        if constexpr (!KEEP) cp_async_wait<0>();
    }
    __device__ __forceinline__ void pairs(int k, Pair (&v)[E < 2 ? 1 : E / 2]) const {
        if constexpr (KEEP) {
            r[k].pairs(v);
        } else {
            Raw<8> x;
            x.v = mine[k * kBlock];
            x.pairs(v);
        }
    }
};
// f(k) for each of the n
template <int KEEP, class F>
__device__ __forceinline__ void each_held(int n, F f) {
    if constexpr (KEEP) {
#pragma unroll
        for (int k = 0; k < KEEP; ++k) {
            if (k >= n) break;
            f(k);
        }
    } else {
#pragma unroll 2
        for (int k = 0; k < n; ++k) f(k);
    }
}

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory"); }
__device__ __forceinline__ float at_rank(const float* mine, int rank) {        // the same place in another block of the cluster
    uint32_t there;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(there) : "r"(smem_u32(mine)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(v) : "r"(there) : "memory");
    return v;
}

template <int E, int KEEP>
__global__ void __launch_bounds__(kBlock, kSmallBlocksSm) group_small_kernel(const __grid_constant__ Pass p) {
    extern __shared__ __align__(128) uint8_t shared[];
    float *mean_of = reinterpret_cast<float*>(shared), *m2_of = mean_of + kBlock * E, *count_of = m2_of + kBlock * E, *moments = count_of + kBlock, *stats = moments + 3 * (p.slab / p.per_group);
    constexpr int kPairs = Channels<E>::kPairs;
    let_dependents_start();
    const Place a = place_of<E>(p);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wide = p.across * E, ch0 = (threadIdx.x % p.across) * E, groups = (a.s1 - a.s0) / p.per_group;
    const long long from = ((long long)a.sample * p.tokens + a.t0 + a.sub) * p.channels + a.c0, step = (long long)p.rows * p.channels;
    const int n = a.there && a.t0 + a.sub < a.t1 ? (int)((a.t1 - a.t0 - a.sub + p.rows - 1) / p.rows) : 0;         // tokens of this thread
    wait_for_prerequisites();
    Held<E, KEEP> held;
    held.load(p.x + from, step, n, shared + p.room);
    held.wait();
    // The mean about the first value, then the deviations about it.
    Pair minus_first[kPairs], minus_mean[kPairs], m2[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) minus_first[i] = minus_mean[i] = m2[i] = both(0.f);
    if (n) {
        Pair v[kPairs];
        held.pairs(0, v);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) minus_first[i] = pmul(v[i], both(-1.f));
    }
    each_held<KEEP>(n, [&](int k) {
        Pair v[kPairs];
        held.pairs(k, v);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) minus_mean[i] = padd(minus_mean[i], padd(v[i], minus_first[i]));
    });
    const Pair by = both(n ? -fast_rcp((float)n) : 0.f);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) minus_mean[i] = pfma(minus_mean[i], by, minus_first[i]);
    each_held<KEEP>(n, [&](int k) {
        Pair v[kPairs];
        held.pairs(k, v);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const Pair d = padd(v[i], minus_mean[i]);
            m2[i] = pfma(d, d, m2[i]);
        }
    });
    if (a.sub < p.rows) {
        if (ch0 == 0) count_of[a.sub] = (float)n;
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            float u[4];
            split_pair(minus_mean[i], u[0], u[1]);
            split_pair(m2[i], u[2], u[3]);
#pragma unroll
            for (int e = 0; e < 2 && e < E; ++e) {
                mean_of[a.sub * wide + ch0 + 2 * i + e] = -u[e];
                m2_of[a.sub * wide + ch0 + 2 * i + e] = u[2 + e];
            }
        }
    }
    __syncthreads();
    for (int g = warp; g < groups; g += kBlock / 32) {
        const Moments m = joined(p.rows * p.per_group, [&](int i) {
            const int row = (int)((unsigned)i / (unsigned)p.per_group), c = i - row * p.per_group + g * p.per_group;
            return Moments{count_of[row], mean_of[row * wide + c], m2_of[row * wide + c]};
        });
        if (lane < 3) moments[3 * g + lane] = lane == 0 ? m.n : lane == 1 ? m.mean : m.m2;
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    for (int g = warp; g < groups; g += kBlock / 32) {
        Moments part = {0.f, 0.f, 0.f};
        if (lane < (int)gridDim.x) part = {at_rank(moments + 3 * g, lane), at_rank(moments + 3 * g + 1, lane), at_rank(moments + 3 * g + 2, lane)};
        const Moments m = joined_lanes(part);
        const float rstd = rsqrtf((float)((double)m.m2 * p.per_value) + p.eps);
        if (lane < 2) {
            stats[2 * g + lane] = lane ? rstd : m.mean;
            if (cluster_rank() == 0) p.stats[2 * ((long long)a.sample * p.groups + a.s0 / p.per_group + g) + lane] = lane ? rstd : m.mean;
        }
    }
    __syncwarp();
    cluster_arrive();                                  // what the others read of this block has been read once they all get here
    __syncthreads();
    if (n) {
        Channels<E> ch;
        ch.load(p, a, stats - 2 * (a.s0 / p.per_group));
        with_act(p.activation, [&](auto tag) {
            each_held<KEEP>(n, [&](int k) {
                Pair v[kPairs];
                held.pairs(k, v);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) v[i] = act2<decltype(tag)::value>(pfma(padd(v[i], ch.minus_mean[i]), ch.a[i], ch.b[i]));
                store_pairs<E>(p.out + from + k * step, v);
            });
        });
    }
    __syncwarp();
    cluster_wait();
}

// d_weight and d_bias of one sample come out at once; of more samples their sums, for group_bwd_params_kernel.
template <int E, int KEEP>
__global__ void __launch_bounds__(kBlock, kSmallBlocksSm) group_small_bwd_kernel(const __grid_constant__ Pass p) {
    extern __shared__ __align__(128) uint8_t shared[];
    float *rows_sums = reinterpret_cast<float*>(shared), *mine = rows_sums + 2 * kBlock * E, *total = mine + 2 * p.slab, *group_sums = total + 2 * p.slab;
    constexpr int kPairs = Channels<E>::kPairs;
    let_dependents_start();
    const Place a = place_of<E>(p);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wide = p.across * E, ch0 = (threadIdx.x % p.across) * E, width = a.s1 - a.s0, groups = width / p.per_group;
    const long long from = ((long long)a.sample * p.tokens + a.t0 + a.sub) * p.channels + a.c0, step = (long long)p.rows * p.channels;
    const int n = a.there && a.t0 + a.sub < a.t1 ? (int)((a.t1 - a.t0 - a.sub + p.rows - 1) / p.rows) : 0;
    wait_for_prerequisites();
    Held<E, KEEP> held_x, held_g;
    held_x.load(p.x + from, step, n, shared + p.room);
    held_g.load(p.d_y + from, step, n, shared + p.room + p.half);
    Channels<E> ch;
    ch.load(p, a, p.stats + 2 * (long long)a.sample * p.groups);
    Pair s1[kPairs], s2[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) s1[i] = s2[i] = both(0.f);
    held_x.wait();
    auto slope = [&](auto tag, int k, auto f) {        // f(i, x - mean, g) of the k-th token
        Pair v[kPairs], g[kPairs];
        held_x.pairs(k, v);
        held_g.pairs(k, g);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const Pair d = padd(v[i], ch.minus_mean[i]);
            f(i, d, pmul(g[i], finite_slope2<decltype(tag)::value>(pfma(d, ch.a[i], ch.b[i]))));
        }
    };
    with_act(p.activation, [&](auto tag) {
        each_held<KEEP>(n, [&](int k) {
            slope(tag, k, [&](int i, Pair d, Pair g) {
                s1[i] = padd(s1[i], g);
                s2[i] = pfma(g, d, s2[i]);
            });
        });
    });
    if (a.sub < p.rows)
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            float u[4];
            split_pair(s1[i], u[0], u[2]);
            split_pair(s2[i], u[1], u[3]);
#pragma unroll
            for (int e = 0; e < 2 && e < E; ++e) {
                rows_sums[2 * (a.sub * wide + ch0 + 2 * i + e)] = u[2 * e];
                rows_sums[2 * (a.sub * wide + ch0 + 2 * i + e) + 1] = u[2 * e + 1];
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * width; i += kBlock) {
        float s = 0.f;
        for (int r = 0; r < p.rows; ++r) s += rows_sums[2 * r * wide + i];
        mine[i] = s;
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    for (int i = threadIdx.x; i < 2 * width; i += kBlock) {
        float s = 0.f;
        for (int r = 0; r < (int)gridDim.x; ++r) s += at_rank(mine + i, r);
        total[i] = s;
        if (cluster_rank()) continue;
        const int c = a.s0 + (i >> 1);
        if (p.all_samples > 1) p.sums[2 * ((long long)a.sample * p.channels + c) + (i & 1)] = s;
        else if (i & 1) p.d_weight[c] = s * p.stats[2 * (c / p.per_group) + 1];
        else p.d_bias[c] = s;
    }
    __syncwarp();
    cluster_arrive();
    __syncthreads();
    for (int g = warp; g < groups; g += kBlock / 32) group_means(p, a, g + a.s0 / p.per_group, total - 2 * a.s0, group_sums + 2 * g, lane);
    __syncthreads();
    if (n) {
        Pair c0[kPairs], c1[kPairs], rstd[kPairs];
        group_terms<E>(p, a, group_sums, c0, c1, rstd);
        with_act(p.activation, [&](auto tag) {
            each_held<KEEP>(n, [&](int k) {
                Pair v[kPairs];
                slope(tag, k, [&](int i, Pair d, Pair g) { v[i] = pfma(g, ch.a[i], pfma(pmul(d, rstd[i]), c1[i], c0[i])); });
                store_pairs<E>(p.out + from + k * step, v);
            });
        });
    }
    __syncwarp();
    cluster_wait();
}

// d_weight and d_bias: the samples' sums, 32 channels to a block, 32 slices of the samples
__global__ void __launch_bounds__(1024) group_bwd_params_kernel(const __grid_constant__ Pass p) {
    __shared__ float w_of[32][33], b_of[32][33];
    let_dependents_start();
    wait_for_prerequisites();
    const int cx = threadIdx.x & 31, slice = threadIdx.x >> 5, c = blockIdx.x * 32 + cx;
    float w = 0.f, b = 0.f;
    if (c < p.channels)
        for (int s = slice; s < p.all_samples; s += 32) {
            const float* sums = p.sums + 2 * ((long long)s * p.channels + c);
            b += sums[0];
            w = fmaf(sums[1], p.stats[2 * ((long long)s * p.groups + c / p.per_group) + 1], w);
        }
    w_of[slice][cx] = w;
    b_of[slice][cx] = b;
    __syncthreads();
    w = w_of[cx][slice];
    b = b_of[cx][slice];
    for (int o = 16; o > 0; o >>= 1) {
        w += __shfl_xor_sync(0xffffffffu, w, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    const int to = blockIdx.x * 32 + slice;
    if (cx || to >= p.channels) return;
    p.d_weight[to] = w;
    p.d_bias[to] = b;
}

Pass pass_of(const GroupNormArgs& a, const GroupNormPlan& plan) {
    Pass p = {};
    p.x = (const uint16_t*)a.x;
    p.d_y = (const uint16_t*)a.d_y;
    p.out = (uint16_t*)a.out;
    p.weight = a.weight;
    p.bias = a.bias;
    p.stats = a.stats;
    p.d_weight = a.d_weight;
    p.d_bias = a.d_bias;
    p.partial = (float*)a.workspace;
    p.sums = (float*)((char*)a.workspace + plan.off_sums);
    p.tokens = a.tokens;
    p.chunk = plan.chunk;
    p.channels = a.channels;
    p.groups = a.groups;
    p.per_group = a.channels / a.groups;
    p.all_samples = a.samples;
    p.activation = a.activation;
    p.across = plan.across;
    p.rows = plan.rows;
    p.slab = plan.slab;
    p.pieces = plan.pieces;
    p.half = plan.held * kBlock * 16;
    p.room = (int)plan.smem - (plan.backward ? 2 : 1) * p.half;
    p.eps = a.eps;
    p.per_value = 1. / ((double)a.tokens * p.per_group);
    return p;
}

// Samples are a grid's second dimension, which ends at kMostSamples.
template <int E, class F>
cudaError_t over_samples(Pass p, const GroupNormPlan& plan, F each) {
    for (p.first = 0; p.first < p.all_samples; p.first += kMostSamples) {
        p.samples = p.all_samples - p.first < kMostSamples ? p.all_samples - p.first : kMostSamples;
        const cudaError_t e = each(p, dim3((unsigned)plan.chunks, (unsigned)p.samples, (unsigned)plan.slabs));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename... P, typename... A>
cudaError_t launch(const char* name, void (*kernel)(P...), dim3 grid, unsigned block, unsigned cluster, size_t smem, cudaStream_t stream, A&&... args) {
    cudaError_t e = smem ? prepare_kernel((const void*)kernel, smem) : cudaSuccess;
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = cluster ? 2 : 1;
    prof_begin(name, stream);
    e = cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
    count_launch(stream);
    return e;
}

template <int E>
cudaError_t forward(const GroupNormArgs& a, const GroupNormPlan& plan, cudaStream_t stream) {
    if (plan.cluster)
        return over_samples<E>(pass_of(a, plan), plan, [&](const Pass& p, dim3 grid) {
            if constexpr (E == 8)
                if (plan.held) return launch("group_small_kernel", group_small_kernel<8, 0>, grid, kBlock, plan.cluster, plan.smem, stream, p);
            return launch("group_small_kernel", group_small_kernel<E, kKeepFwd>, grid, kBlock, plan.cluster, plan.smem, stream, p);
        });
    return over_samples<E>(pass_of(a, plan), plan, [&](const Pass& p, dim3 grid) {
        constexpr size_t kRing = E == 8 ? kRingFwd : 0, kMoments = sizeof(float) * kBlock * (2 * E + 1);
        cudaError_t e = launch("group_stats_kernel", group_stats_kernel<E>, grid, kBlock, 0, kRing > kMoments ? kRing : kMoments, stream, p);
        if (e == cudaSuccess) e = launch("group_stats_join_kernel", group_stats_join_kernel, dim3((unsigned)p.groups, (unsigned)p.samples), kBlock, 0, 0, stream, p, plan.chunks * plan.pieces);
        if (e == cudaSuccess) e = launch("group_apply_kernel", group_apply_kernel<E>, grid, kBlock, 0, kRing, stream, p);
        return e;
    });
}

template <int E>
cudaError_t backward(const GroupNormArgs& a, const GroupNormPlan& plan, cudaStream_t stream) {
    if (plan.cluster) {
        const cudaError_t e = over_samples<E>(pass_of(a, plan), plan, [&](const Pass& p, dim3 grid) {
            if constexpr (E == 8)
                if (plan.held) return launch("group_small_bwd_kernel", group_small_bwd_kernel<8, 0>, grid, kBlock, plan.cluster, plan.smem, stream, p);
            return launch("group_small_bwd_kernel", group_small_bwd_kernel<E, kKeepBwd>, grid, kBlock, plan.cluster, plan.smem, stream, p);
        });
        if (e != cudaSuccess || a.samples == 1) return e;
        return launch("group_bwd_params_kernel", group_bwd_params_kernel, dim3((unsigned)(a.channels + 31) / 32), 1024u, 0, 0, stream, pass_of(a, plan));
    }
    const size_t ring = E == 8 ? kRingBwd : 0, rows = sizeof(float) * 2 * plan.rows * plan.across * E, groups = sizeof(float) * 2 * (plan.slab < a.channels / a.groups ? 1 : plan.slab / (a.channels / a.groups) + 1);
    const cudaError_t e = over_samples<E>(pass_of(a, plan), plan, [&](const Pass& p, dim3 grid) {
        cudaError_t e = launch("group_bwd_sums_kernel", group_bwd_sums_kernel<E>, grid, kBlock, 0, rows > ring ? rows : ring, stream, p);
        if (e == cudaSuccess) e = launch("group_bwd_join_kernel", group_bwd_join_kernel, dim3((unsigned)(2 * p.channels + 31) / 32, (unsigned)p.samples), 1024u, 0, 0, stream, p, plan.chunks);
        if (e == cudaSuccess) e = launch("group_bwd_apply_kernel", group_bwd_apply_kernel<E>, grid, kBlock, 0, ring + groups, stream, p);
        return e;
    });
    if (e != cudaSuccess || a.samples <= kFewSamples) return e;
    return launch("group_bwd_params_kernel", group_bwd_params_kernel, dim3((unsigned)(a.channels + 31) / 32), 1024u, 0, 0, stream, pass_of(a, plan));
}

}  // namespace

#ifndef TERRA_ELEM_F16
// Threads: E channels of a token each, side by side over a slab of channels, whole groups of them, or a piece of one where a group has more than a block's.
// Chunks: so many that the blocks fill the GPU, but a thread has twice as many tokens as it takes at a time.
GroupNormPlan plan_group_norm(int samples, long long tokens, int channels, int groups, bool backward) {
    GroupNormPlan p = {};
    p.backward = backward;
    const int per_group = channels / groups;
    auto fits = [&](int e) { return channels % e == 0 && (per_group % e == 0 || channels <= kBlock * e); };
    p.elems = fits(8) ? 8 : fits(2) ? 2 : 1;
    const int most = kBlock * p.elems;
    p.pieces = 1;
    if (channels <= most) {
        p.slab = channels;
        p.slabs = 1;
    } else if (per_group <= most) {
        p.slab = most / per_group * per_group;
        p.slabs = (channels + p.slab - 1) / p.slab;
    } else {
        p.slab = most;
        p.pieces = (per_group + most - 1) / most;
        p.slabs = p.pieces * groups;
    }
    // Samples whose slabs clusters hold: slabs of as few whole groups as make whole vectors, of 64 bytes a token at least.  Shared memory: a block's sums and its
    // groups' (as the kernels lay them out), then the vectors that it holds there.
    int unit = per_group;
    while (unit % p.elems) unit += per_group;
    while (2 * unit < 64 && channels % (2 * unit) == 0) unit *= 2;
    if (unit <= most) {
        const int rows = kBlock / (unit / p.elems), keep = rows * (backward ? kKeepBwd : kKeepFwd);
        const long long least = (tokens + keep - 1) / keep, slabs = (long long)samples * (channels / unit);       // blocks of a cluster; clusters
        const long long floats = backward ? 2ll * kBlock * p.elems + 4 * unit + 2 * (unit / per_group) : kBlock * (2ll * p.elems + 1) + 5 * (unit / per_group);
        const long long sums = (floats * 4 + 127) / 128 * 128;
        if (least <= kMostCluster && least * slabs <= (backward ? kSmallBlocksBwd : kSmallBlocksFwd)) {
            // more blocks of two tokens a thread while they are all on the GPU at a time
            const long long spread = (tokens + 2 * rows - 1) / (2 * rows), fit = 2 * kPlanSms / slabs;
            p.cluster = (int)(spread < fit ? spread : fit);
            if (p.cluster > kMostCluster) p.cluster = kMostCluster;
            if (p.cluster < least) p.cluster = (int)least;
        } else if (p.elems == 8) {
            // In shared memory, where the blocks of all samples are on the GPU at a time (of the SMs of a cluster of 8 some stay over) or, two to an SM, in two turns.
            // us, so / otherwise: 16 x 280 x 960 backward by clusters of 4, 64 blocks that are there at once, 15.2, by clusters of 6 that are not 22.7; in two turns / three
            // launches 100 x 1720 x 96 30.1 / 34.8, 64 x 371 x 256 backward 23.1 / 36.0, but one block to an SM 16 x 6494 x 80 backward 39.9 / 37.3.
            for (int turns = 1; turns <= 2 && !p.cluster; ++turns)
                for (int c = kMostCluster; c >= 1 && !p.cluster; --c) {
                    const long long held = ((tokens + c - 1) / c + rows - 1) / rows, vectors = held * kBlock * 16 * (backward ? 2 : 1);
                    if (vectors > kMostHeld || vectors + sums > kBlockSmem) break;
                    const long long fit = kSmSmem / (vectors + sums + 1024), per_sm = fit < kSmallBlocksSm ? fit : kSmallBlocksSm;     // (1 KB of a block is the system's)
                    if (turns == 2 && per_sm < kSmallBlocksSm) break;
                    if (c * slabs <= turns * per_sm * (kPlanSms * 7 / 8)) {
                        p.cluster = c;
                        p.held = (int)held;
                    }
                }
        }
        if (p.cluster) {
            p.slab = unit;
            p.slabs = channels / unit;
            p.pieces = 1;
            p.across = unit / p.elems;
            p.rows = rows;
            p.smem = (size_t)(sums + (long long)p.held * kBlock * 16 * (backward ? 2 : 1));
            p.chunks = p.cluster;
            p.chunk = (tokens + p.cluster - 1) / p.cluster;
            p.bytes = backward && samples > 1 ? (sizeof(float) * 2 * samples * (size_t)channels + 255) / 256 * 256 : 0;
            return p;
        }
    }
    p.across = p.slab / p.elems;
    p.rows = kBlock / p.across;
    const int at_once = samples < kMostSamples ? samples : kMostSamples;
    const long long fit = blocks(p.elems, 1 + backward) * (long long)kPlanSms, least = 2ll * deep(p.elems, 1 + backward) * p.rows;
    long long chunks = (fit + (long long)at_once * p.slabs - 1) / ((long long)at_once * p.slabs);
    if (chunks > (tokens + least - 1) / least) chunks = (tokens + least - 1) / least;
    p.chunk = (tokens + chunks - 1) / chunks;
    p.chunks = (int)((tokens + p.chunk - 1) / p.chunk);
    const size_t partial = backward ? sizeof(float) * 2 * at_once * p.chunks * (size_t)channels : sizeof(float) * 3 * at_once * (size_t)groups * p.pieces * p.chunks;
    p.off_sums = (partial + 255) / 256 * 256;
    p.bytes = p.off_sums + (backward ? (sizeof(float) * 2 * samples * (size_t)channels + 255) / 256 * 256 : 0);
    return p;
}
#endif

cudaError_t read_group_norm_status(int* timed_out) {
    int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(timed_out, g_group_norm_timeout, sizeof(int));
    if (e != cudaSuccess) return e;
    if (*timed_out) e = cudaMemcpyToSymbol(g_group_norm_timeout, &zero, sizeof(int));
    return e;
}

cudaError_t launch_group_norm_fwd(const GroupNormArgs& a, const GroupNormPlan& plan, cudaStream_t stream) {
    return plan.elems == 8 ? forward<8>(a, plan, stream) : plan.elems == 2 ? forward<2>(a, plan, stream) : forward<1>(a, plan, stream);
}
cudaError_t launch_group_norm_bwd(const GroupNormArgs& a, const GroupNormPlan& plan, cudaStream_t stream) {
    return plan.elems == 8 ? backward<8>(a, plan, stream) : plan.elems == 2 ? backward<2>(a, plan, stream) : backward<1>(a, plan, stream);
}

}  // namespace terra
