// Root-mean-square norm over a token's channels, with the addition of the residual before it: h = x + r, rstd = (mean h^2 + eps)^-1/2,
// y = h rstd weight, and its backward.  y in the activations' type or in e4m3 with one scale per token, scale = max|y| / 448.
// h is stored rounded to the activations' type; y and rstd are taken of the unrounded sum, which is in registers.
//
// A token's row is held by `lanes` threads (a power of two, 4 to 512), V vectors of E elements each, so that one read of the row
// serves the sum of squares, the maximum and the output.  E is 8, 2 or 1 as the channels allow.  Blocks walk over the rows, the next row's reads
// under way while a row is worked on; the weights stay in registers.  All sums in fp32.
#include <cuda_fp8.h>

#include "block_act.cuh"
#include "block_kernels.h"

#ifdef TERRA_ELEM_F16
#define launch_rms_norm_fwd launch_rms_norm_fwd_f16
#define launch_rms_norm_bwd launch_rms_norm_bwd_f16
#endif

namespace terra {
namespace {

constexpr int kBlock = 256;            // threads of a block where a row takes no more
constexpr int kMaxLanes = 512;         // threads of a row at most
constexpr float kE4m3Max = 448.f;

// E elements of a row as they lie in memory
template <int E> struct Raw;
template <> struct Raw<8> {
    uint4 v;
    __device__ void load(const uint16_t* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ void floats(float (&f)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 t = elem2_to_float2(w[i]); f[2 * i] = t.x; f[2 * i + 1] = t.y; }
    }
    __device__ void add_to(float (&f)[8]) const {
        add_elems(f[0], f[1], v.x);
        add_elems(f[2], f[3], v.y);
        add_elems(f[4], f[5], v.z);
        add_elems(f[6], f[7], v.w);
    }
};
template <> struct Raw<2> {
    uint32_t v;
    __device__ void load(const uint16_t* p) { v = *reinterpret_cast<const uint32_t*>(p); }
    __device__ void zero() { v = 0; }
    __device__ void floats(float (&f)[2]) const { const float2 t = elem2_to_float2(v); f[0] = t.x; f[1] = t.y; }
    __device__ void add_to(float (&f)[2]) const { add_elems(f[0], f[1], v); }
};
template <> struct Raw<1> {
    uint32_t v;
    __device__ void load(const uint16_t* p) { v = *p; }
    __device__ void zero() { v = 0; }
    __device__ void floats(float (&f)[1]) const { f[0] = elem2_to_float2(v).x; }
    __device__ void add_to(float (&f)[1]) const { f[0] += elem2_to_float2(v).x; }
};
__device__ __forceinline__ void store(uint16_t* p, const float (&f)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_elem(f[0], f[1]), pack_elem(f[2], f[3]), pack_elem(f[4], f[5]), pack_elem(f[6], f[7]));
}
__device__ __forceinline__ void store(uint16_t* p, const float (&f)[2]) { *reinterpret_cast<uint32_t*>(p) = pack_elem(f[0], f[1]); }
__device__ __forceinline__ void store(uint16_t* p, const float (&f)[1]) { *p = (uint16_t)pack_elem(f[0], 0.f); }
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b) { return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float (&f)[8]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_e4m3(f[0], f[1]) | pack_e4m3(f[2], f[3]) << 16, pack_e4m3(f[4], f[5]) | pack_e4m3(f[6], f[7]) << 16);
}
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float (&f)[2]) { *reinterpret_cast<uint16_t*>(p) = (uint16_t)pack_e4m3(f[0], f[1]); }
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float (&f)[1]) { *p = (uint8_t)pack_e4m3(f[0], 0.f); }

__device__ __forceinline__ float max_nan(float a, float b) {       // a NaN stays one
    float d;
    asm("max.NaN.f32 %0, %1, %2;\n" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// Sum (or maximum) over the threads of a row, to all of them.  `turn` alternates the two halves of `buf` (32 floats each): one
// barrier a reduction is enough, since a half is written again only after the next reduction's barrier.
template <bool MAX>
__device__ __forceinline__ float over_row(float s, int lanes, float* buf, int& turn) {
    const int within = lanes < 32 ? lanes : 32;
    for (int o = within >> 1; o > 0; o >>= 1) {
        const float t = __shfl_xor_sync(0xffffffffu, s, o);
        s = MAX ? max_nan(s, t) : s + t;
    }
    if (lanes <= 32) return s;
    float* b = buf + 32 * turn;
    turn ^= 1;
    const int warp = threadIdx.x >> 5, per_row = lanes >> 5, first = warp & ~(per_row - 1);
    if ((threadIdx.x & 31) == 0) b[warp] = s;
    __syncthreads();
    s = b[first];
    for (int i = 1; i < per_row; ++i) s = MAX ? max_nan(s, b[first + i]) : s + b[first + i];
    return s;
}

// What bounds it: HBM (156672 x 4096 785 us, 6.5 TB/s; e4m3 759 us, 5.9 TB/s).
template <int E, int V, bool E4M3>
__global__ void __launch_bounds__(kMaxLanes, E == 8 && V <= 2 ? 2 : 1)
rms_norm_fwd_kernel(const NormArgs a, int lanes, int lanes_log2) {
    __shared__ float buf[64];
    int turn = 0;
    const int lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> lanes_log2, per_block = blockDim.x >> lanes_log2;
    const int chunks = a.channels / E;
    const float per_channel = 1.f / (float)a.channels;
    float w[V][E];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = lane + v * lanes;
            w[v][e] = c < chunks ? a.weight[c * E + e] : 0.f;
        }
    const uint16_t *x = (const uint16_t*)a.x, *r = (const uint16_t*)a.r;
    uint16_t* h = (uint16_t*)a.h;
    Raw<E> xr[V], rr[V];
    auto fetch = [&](long long row) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = lane + v * lanes;
            xr[v].zero();
            rr[v].zero();
            if (row < a.rows && c < chunks) {
                xr[v].load(x + row * a.channels + c * E);
                if (r) rr[v].load(r + row * a.channels + c * E);
            }
        }
    };
    const long long step = (long long)gridDim.x * per_block;
    // (With the residual's reads and the sum's writes beside a 16-bit output, reads ahead make it slower: 156672 x 4096 789 -> 878 us.  Without the residual
    // they take it from 535 to 440 us, with the output in 8 bits from 938 to 861.)
    const bool ahead = E4M3 || !r;
    if (ahead) fetch((long long)blockIdx.x * per_block + sub);
    for (long long row0 = (long long)blockIdx.x * per_block; row0 < a.rows; row0 += step) {
        const long long row = row0 + sub;
        const bool live = row < a.rows;
        const long long at = row * a.channels;
        if (!ahead) fetch(row);
        float f[V][E], sum = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            xr[v].floats(f[v]);
            if (r) rr[v].add_to(f[v]);
        }
        if (ahead) fetch(row + step);  // (rows of other blocks are not written, so outputs over inputs stay right)
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int e = 0; e < E; ++e) sum = fmaf(f[v][e], f[v][e], sum);
            const int c = lane + v * lanes;
            if (h && live && c < chunks) store(h + at + c * E, f[v]);
        }
        sum = over_row<false>(sum, lanes, buf, turn);
        const float rstd = rsqrtf(fmaf(sum, per_channel, a.eps));
        if (a.rstd && live && lane == 0) a.rstd[row] = rstd;
        if (E4M3) {
            float top = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    f[v][e] *= w[v][e];
                    top = max_nan(top, fabsf(f[v][e]));
                }
            top = over_row<true>(top, lanes, buf, turn) * rstd;
            const float scale = top / kE4m3Max;
            if (live && lane == 0) a.scale[row] = scale;
            const float by = rstd / scale;             // y / scale = f weight by
            if (scale >= 0x1p-100f && by < 0x1p100f) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int c = lane + v * lanes;
#pragma unroll
                    for (int e = 0; e < E; ++e) f[v][e] *= by;
                    if (live && c < chunks) store_e4m3((uint8_t*)a.y + at + c * E, f[v]);
                }
            } else {                                   // far out, by leaves fp32's range; a row of zeros keeps its zeros; NaN stays NaN
                const float div = scale == 0.f ? 1.f : scale;
#pragma unroll 1
                for (int v = 0; v < V; ++v) {
                    const int c = lane + v * lanes;
#pragma unroll
                    for (int e = 0; e < E; ++e) f[0][e] = f[0][e] * rstd / div;
                    if (live && c < chunks) store_e4m3((uint8_t*)a.y + at + c * E, f[0]);
#pragma unroll
                    for (int u = 0; u + 1 < V; ++u)
#pragma unroll
                        for (int e = 0; e < E; ++e) f[u][e] = f[u + 1][e];
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = lane + v * lanes;
#pragma unroll
                for (int e = 0; e < E; ++e) f[v][e] = f[v][e] * rstd * w[v][e];
                if (live && c < chunks) store((uint16_t*)a.y + at + c * E, f[v]);
            }
        }
    }
}

// n = h rstd, g = d_y weight: dx = rstd (g - n mean(g n)) + d_h, dweight = sum over the rows of d_y n.  A block adds up its rows'
// dweight in registers and writes one row of `partial`; sum_partials_kernel adds those in a fixed order.
// What bounds it: HBM (156672 x 4096 806 us, 131072 x 768 134 us, 6.0 to 6.4 TB/s); where the registers of a row's four vectors, or of its single elements and
// pairs, spill and leave none for the next row, what is spilled and the wait for a row's reads (40000 x 16384 1549 us, 3.4 TB/s; 300000 x 1001 968 us, 2.5 TB/s).
template <int E, int V>
__global__ void __launch_bounds__(kMaxLanes)
rms_norm_bwd_kernel(const NormArgs a, int lanes, int lanes_log2) {
    __shared__ float buf[64];
    extern __shared__ float groups_sum[];
    let_dependents_start();
    int turn = 0;
    const int lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> lanes_log2, per_block = blockDim.x >> lanes_log2;
    const int chunks = a.channels / E;
    const float per_channel = 1.f / (float)a.channels;
    float w[V][E], acc[V][E];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = lane + v * lanes;
            w[v][e] = c < chunks ? a.weight[c * E + e] : 0.f;
            acc[v][e] = 0.f;
        }
    const uint16_t *h = (const uint16_t*)a.x, *dh = (const uint16_t*)a.r, *dy = (const uint16_t*)a.d_y;
    constexpr bool kAhead = V * E <= 16;       // the next row's reads are under way while this one is worked on (else the registers do not hold both)
    Raw<E> hr[V], gr[V], dr[V];
    float rstd = 0.f;
    auto fetch = [&](long long row) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = lane + v * lanes;
            hr[v].zero();
            gr[v].zero();
            dr[v].zero();
            if (row < a.rows && c < chunks) {
                hr[v].load(h + row * a.channels + c * E);
                gr[v].load(dy + row * a.channels + c * E);
                if (dh) dr[v].load(dh + row * a.channels + c * E);
            }
        }
        rstd = row < a.rows ? a.rstd_in[row] : 0.f;
    };
    const long long step = (long long)gridDim.x * per_block;
    if (kAhead) fetch((long long)blockIdx.x * per_block + sub);
    for (long long row0 = (long long)blockIdx.x * per_block; row0 < a.rows; row0 += step) {
        const long long row = row0 + sub;
        const bool live = row < a.rows;
        const long long at = row * a.channels;
        if (!kAhead) fetch(row);
        float n[V][E], g[V][E], along = 0.f;
        Raw<E> dn[V];
        const float rs = rstd;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            hr[v].floats(n[v]);
            gr[v].floats(g[v]);
            dn[v] = dr[v];
        }
        if (kAhead) fetch(row + step);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                n[v][e] *= rs;
                const float t = n[v][e] * g[v][e];
                acc[v][e] += t;
                along = fmaf(t, w[v][e], along);
            }
        along = over_row<false>(along, lanes, buf, turn) * per_channel;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float d[E];
            dn[v].floats(d);
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = fmaf(rs, fmaf(g[v][e], w[v][e], -n[v][e] * along), d[e]);
            const int c = lane + v * lanes;
            if (live && c < chunks) store((uint16_t*)a.y + at + c * E, d);
        }
    }
    // rows of this block: the warp's by shuffles, then the warps' (or the rows' of several warps) in shared memory
    for (int o = lanes; o < 32; o <<= 1)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < E; ++e) acc[v][e] += __shfl_xor_sync(0xffffffffu, acc[v][e], o);
    const int wide = lanes < 32 ? 32 : lanes, groups = blockDim.x / wide, group = threadIdx.x / wide;
    float* out = a.partial + (size_t)blockIdx.x * a.channels;
    float* mine = groups > 1 ? groups_sum + (size_t)group * a.channels : out;
    if ((threadIdx.x & (wide - 1)) < lanes)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = lane + v * lanes;
            if (c < chunks)
#pragma unroll
                for (int e = 0; e < E; ++e) mine[c * E + e] = acc[v][e];
        }
    if (groups == 1) return;
    __syncthreads();
    for (int c = threadIdx.x; c < a.channels; c += blockDim.x) {
        float s = 0.f;
        for (int i = 0; i < groups; ++i) s += groups_sum[(size_t)i * a.channels + c];
        out[c] = s;
    }
}

struct Shape { int E, V, lanes, lanes_log2, threads; };

// Threads to a row: the fewest (but 4 at least) of up to `most` vectors each.  With 16-byte vectors V is the number that the row needs
// then, so that 96, 192, 384 and 768 channels (3 vectors) leave no thread idle.  Up to 4 vectors in a warp; in rows of several warps 2, which leaves
// registers for the next row's (156672 x 4096, with the next row ahead: forward 806 -> 785 us, e4m3 976 -> 759, backward 1661 -> 807).  Odd and even
// numbers of channels by 2 and 4 bytes a thread: 300000 x 1001 forward 773 us, x 1002 549, x 1000 396.
Shape shape_for(int channels, bool backward) {
    Shape s;
    s.E = channels % 8 == 0 ? 8 : channels % 2 == 0 ? 2 : 1;
    const int chunks = channels / s.E;
    int most;
    if (s.E == 8) most = chunks > 128 && chunks <= 1024 ? 2 : 4;
    else if (s.E == 2) most = chunks <= 8 * kMaxLanes ? 8 : 16;
    else if (backward) most = chunks <= 4 * kMaxLanes ? 4 : chunks <= 8 * kMaxLanes ? 8 : chunks <= 16 * kMaxLanes ? 16 : 32;
    else most = chunks <= 64 ? 4 : chunks <= 16 * kMaxLanes ? 16 : 32;
    s.lanes = 4;
    s.lanes_log2 = 2;
    while (s.lanes * most < chunks) { s.lanes *= 2; ++s.lanes_log2; }
    s.V = s.E == 8 ? (chunks + s.lanes - 1) / s.lanes : most;
    if (backward && s.V == 4 && s.E == 8 && s.lanes < kMaxLanes) {        // four vectors leave no registers for the next row (300000 x 200: 151 -> 96 us)
        s.lanes *= 2;
        ++s.lanes_log2;
        s.V = 2;
    }
    s.threads = s.lanes < kBlock ? kBlock : s.lanes;
    return s;
}

template <bool E4M3>
auto fwd_kernel(const Shape& s) {
    if (s.E == 1) return s.V == 4 ? rms_norm_fwd_kernel<1, 4, E4M3> : s.V == 16 ? rms_norm_fwd_kernel<1, 16, E4M3> : rms_norm_fwd_kernel<1, 32, E4M3>;
    if (s.E == 2) return s.V == 8 ? rms_norm_fwd_kernel<2, 8, E4M3> : rms_norm_fwd_kernel<2, 16, E4M3>;
    switch (s.V) {
        case 1: return rms_norm_fwd_kernel<8, 1, E4M3>;
        case 2: return rms_norm_fwd_kernel<8, 2, E4M3>;
        case 3: return rms_norm_fwd_kernel<8, 3, E4M3>;
        default: return rms_norm_fwd_kernel<8, 4, E4M3>;
    }
}
auto bwd_kernel(const Shape& s) {
    if (s.E == 1) return s.V == 4 ? rms_norm_bwd_kernel<1, 4> : s.V == 8 ? rms_norm_bwd_kernel<1, 8> : s.V == 16 ? rms_norm_bwd_kernel<1, 16> : rms_norm_bwd_kernel<1, 32>;
    if (s.E == 2) return s.V == 8 ? rms_norm_bwd_kernel<2, 8> : rms_norm_bwd_kernel<2, 16>;
    switch (s.V) {
        case 1: return rms_norm_bwd_kernel<8, 1>;
        case 2: return rms_norm_bwd_kernel<8, 2>;
        case 3: return rms_norm_bwd_kernel<8, 3>;
        default: return rms_norm_bwd_kernel<8, 4>;
    }
}

constexpr int kBwdBlocks = 640;        // rows of `partial` at most

}  // namespace

#ifndef TERRA_ELEM_F16
int norm_bwd_blocks(long long rows, int channels) {
    const Shape s = shape_for(channels, true);
    const long long per_block = s.threads / s.lanes, need = (rows + per_block - 1) / per_block;
    return (int)(need < kBwdBlocks ? need : kBwdBlocks);
}
#endif

cudaError_t launch_rms_norm_fwd(const NormArgs& a, int sm_count, cudaStream_t stream) {
    const Shape s = shape_for(a.channels, false);
    auto kern = a.scale ? fwd_kernel<true>(s) : fwd_kernel<false>(s);
    int occ = 1;
    cudaError_t e = prepare_kernel((const void*)kern, 0, s.threads, &occ);
    if (e != cudaSuccess) return e;
    const long long per_block = s.threads / s.lanes, need = (a.rows + per_block - 1) / per_block, fit = (long long)sm_count * (occ < 1 ? 1 : occ);
    prof_begin("rms_norm_fwd_kernel", stream);
    kern<<<(unsigned)(need < fit ? need : fit), s.threads, 0, stream>>>(a, s.lanes, s.lanes_log2);
    count_launch(stream);
    return cudaGetLastError();
}

cudaError_t launch_rms_norm_bwd(const NormArgs& a, int sm_count, cudaStream_t stream) {
    const Shape s = shape_for(a.channels, true);
    auto kern = bwd_kernel(s);
    const int wide = s.lanes < 32 ? 32 : s.lanes, groups = s.threads / wide;
    const size_t smem = groups > 1 ? (size_t)groups * a.channels * sizeof(float) : 0;
    int occ = 1;
    cudaError_t e = prepare_kernel((const void*)kern, smem, s.threads, &occ);
    if (e != cudaSuccess) return e;
    const long long fit = (long long)sm_count * (occ < 1 ? 1 : occ);
    const int most = norm_bwd_blocks(a.rows, a.channels), blocks = (int)(most < fit ? most : fit);
    prof_begin("rms_norm_bwd_kernel", stream);
    kern<<<blocks, s.threads, smem, stream>>>(a, s.lanes, s.lanes_log2);
    count_launch(stream);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_sum_partials(a.partial, blocks, a.channels, a.dweight, stream);
}

}  // namespace terra
