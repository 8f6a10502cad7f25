// Root-mean-square norm over a token's channels, with the addition of the residual before it: h = x + r, rstd = (mean h^2 + eps)^-1/2,
// y = h rstd weight, and its backward.  y in the activations' type or in 8 bits with one scale per token: e4m3, scale = max|y| / 448, or whole
// numbers, scale = max|y| / 127.  h is stored rounded to the activations' type; y and rstd are taken of the unrounded sum, which is in registers.
// Rows are quantised without a norm (y = x) by quantize_kernel where their channels are a multiple of 8, by the norm's kernel without the norm where they are not
// (300000 x 130 87 us, 100000 x 1001 207: reads of 4 and 2 bytes), and by quantize_wide_kernel where a block does not hold them.
//
// A token's row is held by `lanes` threads (a power of two, 4 to 512), V vectors of E elements each, so that one read of the row
// serves the sum of squares, the maximum and the output.  E is 8, 2 or 1 as the channels allow.  Blocks walk over the rows, the next row's reads
// under way while a row is worked on; the weights stay in registers.  All sums in fp32.
#include <cuda_fp8.h>

#include "block_act.cuh"
#include "block_kernels.h"
#include "elem_vec.cuh"

#ifdef TERRA_ELEM_F16
#define launch_rms_norm_fwd launch_rms_norm_fwd_f16
#define launch_rms_norm_bwd launch_rms_norm_bwd_f16
#endif

namespace terra {
namespace {

constexpr int kBlock = 256;            // threads of a block where a row takes no more
constexpr int kMaxLanes = 512;         // threads of a row at most
constexpr float kE4m3Max = 448.f, kI8Max = 127.f;

__device__ __forceinline__ uint32_t pack_e4m3(float a, float b) { return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3); }
// to the nearest whole number, ties to the even one; of NaN 0
__device__ __forceinline__ uint32_t pack_i8(float a, float b) { return (uint32_t)(__float2int_rn(a) & 0xff) | (uint32_t)(__float2int_rn(b) & 0xff) << 8; }
template <int OUT> __device__ __forceinline__ uint32_t pack_8(float a, float b) { return OUT == kOpsI8 ? pack_i8(a, b) : pack_e4m3(a, b); }

template <int OUT>
__device__ __forceinline__ void store_8(uint8_t* p, const float (&f)[8]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_8<OUT>(f[0], f[1]) | pack_8<OUT>(f[2], f[3]) << 16, pack_8<OUT>(f[4], f[5]) | pack_8<OUT>(f[6], f[7]) << 16);
}
template <int OUT>
__device__ __forceinline__ void store_8(uint8_t* p, const float (&f)[2]) { *reinterpret_cast<uint16_t*>(p) = (uint16_t)pack_8<OUT>(f[0], f[1]); }
template <int OUT>
__device__ __forceinline__ void store_8(uint8_t* p, const float (&f)[1]) { *p = (uint8_t)pack_8<OUT>(f[0], 0.f); }

__device__ __forceinline__ float max_nan(float a, float b) {       // a NaN stays one
    float d;
    asm("max.NaN.f32 %0, %1, %2;\n" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// y / scale where its reciprocal leaves fp32's range: a row of zeros keeps its zeros, NaN stays NaN, and whole numbers stay in theirs where a scale
// below the normal numbers has lost digits
template <int OUT>
__device__ __forceinline__ float far_out(float y, float scale) {
    const float q = y / (scale == 0.f ? 1.f : scale);
    return OUT == kOpsI8 && fabsf(q) > kI8Max ? copysignf(kI8Max, q) : q;
}

// Rows of the activations' type in whole numbers: 127 x / max to the nearest one, ties to the even one.  Of numbers of 11 bits at most, a quotient that is no
// tie is 2^-19 of itself away from one (254 X and an odd multiple of M differ by 1 at least, and 254 X is below 2^19), and ties are numbers that fp32 holds: the quotient to half a step of fp32
// decides both.  That takes the reciprocal to twice fp32's digits, hi + lo; with hi alone x = max / 2, 63.5, went to 63 or 64 as the row's reciprocal was rounded.
// Far out the row is scaled by a power of two first, so that lo stays among the normal numbers.  A row that is not finite gives zeros.
struct Whole {
    float pre, hi, lo;
    __device__ __forceinline__ explicit Whole(float top) {
        pre = top < 0x1p-60f ? 0x1p100f : top > 0x1p60f ? 0x1p-64f : 1.f;
        const float m = top * pre;
        hi = kI8Max * fast_rcp(m);
        lo = fmaf(-hi, m, kI8Max) * (hi * (1.f / kI8Max));
        if (!(m > 0.f && m < INFINITY)) hi = lo = 0.f;
    }
    __device__ __forceinline__ bool near() const { return pre == 1.f && hi > 0.f; }
    __device__ __forceinline__ float operator()(float x) const { return fmaf(x * pre, hi, x * pre * lo); }       // (not finite: 0 or NaN, of which the whole number is 0)
};

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
template <int E, int V, int OUT, bool NORM>
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
            w[v][e] = !NORM ? 1.f : c < chunks ? a.weight[c * E + e] : 0.f;
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
    const bool ahead = OUT != kOps16 || !r;
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
        if (NORM) sum = over_row<false>(sum, lanes, buf, turn);
        const float rstd = NORM ? rsqrtf(fmaf(sum, per_channel, a.eps)) : 1.f;
        if (a.rstd && live && lane == 0) a.rstd[row] = rstd;
        if (OUT != kOps16) {
            float top = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    f[v][e] *= w[v][e];
                    top = max_nan(top, fabsf(f[v][e]));
                }
            top = over_row<true>(top, lanes, buf, turn) * rstd;
            const float scale = top / (OUT == kOpsI8 ? kI8Max : kE4m3Max);
            if (live && lane == 0) a.scale[row] = scale;
            const float by = rstd / scale;             // y / scale = f weight by
            if (!NORM) {
                const Whole whole(top);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int c = lane + v * lanes;
#pragma unroll
                    for (int e = 0; e < E; ++e) f[v][e] = whole(f[v][e]);
                    if (live && c < chunks) store_8<OUT>((uint8_t*)a.y + at + c * E, f[v]);
                }
            } else if (scale >= 0x1p-100f && by < 0x1p100f) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int c = lane + v * lanes;
#pragma unroll
                    for (int e = 0; e < E; ++e) f[v][e] *= by;
                    if (live && c < chunks) store_8<OUT>((uint8_t*)a.y + at + c * E, f[v]);
                }
            } else {                                   // far out, by leaves fp32's range; a row of zeros keeps its zeros; NaN stays NaN
#pragma unroll 1
                for (int v = 0; v < V; ++v) {
                    const int c = lane + v * lanes;
#pragma unroll
                    for (int e = 0; e < E; ++e) f[0][e] = far_out<OUT>(f[0][e] * rstd, scale);
                    if (live && c < chunks) store_8<OUT>((uint8_t*)a.y + at + c * E, f[0]);
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

// the larger of two elements each, a NaN stays one
__device__ __forceinline__ uint32_t max_elem2(uint32_t a, uint32_t b) {
    uint32_t d;
#ifdef TERRA_ELEM_F16
    asm("max.NaN.f16x2 %0, %1, %2;\n" : "=r"(d) : "r"(a), "r"(b));
#else
    asm("max.NaN.bf16x2 %0, %1, %2;\n" : "=r"(d) : "r"(a), "r"(b));
#endif
    return d;
}

// Rows quantised, up to V vectors of 8 to a thread.  A thread has all of its reads under way at once and keeps them as they are, so that many fit: what
// bounds it is HBM behind that (156672 x 4096 298 us, 6.5 TB/s; 1000000 x 96 54, 5.3).  (156672 x 4096, the norm's kernel without the norm, two vectors a thread and the next row's two ahead: 515 us.)
// A quotient + 1.5 2^23 has the nearest whole number in its last byte.
template <int V>
__global__ void __launch_bounds__(kBlock, V == 8 ? 4 : V == 4 ? 5 : 6) quantize_kernel(const NormArgs a, int lanes, int lanes_log2) {
    __shared__ float buf[64];
    int turn = 0;
    const int lane = threadIdx.x & (lanes - 1), sub = threadIdx.x >> lanes_log2, per_block = kBlock >> lanes_log2, chunks = a.channels / 8;
    const long long step = (long long)gridDim.x * per_block;
    for (long long row0 = (long long)blockIdx.x * per_block; row0 < a.rows; row0 += step) {
        const long long row = row0 + sub;
        const bool live = row < a.rows;
        const uint16_t* x = (const uint16_t*)a.x + row * a.channels;
        uint8_t* y = (uint8_t*)a.y + row * a.channels;
        Raw<8> r[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = lane + v * lanes;
            r[v].zero();
            if (live && c < chunks) r[v].load(x + c * 8);
        }
        uint32_t most = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t m = 0x7fff7fffu;
            most = max_elem2(max_elem2(max_elem2(r[v].v.x & m, r[v].v.y & m), max_elem2(r[v].v.z & m, r[v].v.w & m)), most);
        }
        const float2 two = elem2_to_float2(most);
        const float top = over_row<true>(max_nan(two.x, two.y), lanes, buf, turn);
        if (live && lane == 0) a.scale[row] = top / kI8Max;
        const Whole whole(top);
        const Pair hi = both(whole.hi), lo = both(whole.lo);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = lane + v * lanes;
            if (!live || c >= chunks) continue;
            if (whole.near()) {
                Pair p[4];
                r[v].pairs(p);
                uint32_t q[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float a0, a1;
                    split_pair(padd(pfma(p[i], hi, pmul(p[i], lo)), both(12582912.f)), a0, a1);
                    q[2 * i] = __float_as_uint(a0);
                    q[2 * i + 1] = __float_as_uint(a1);
                }
                *reinterpret_cast<uint2*>(y + c * 8) = make_uint2(__byte_perm(__byte_perm(q[0], q[1], 0x40), __byte_perm(q[2], q[3], 0x40), 0x5410),
                                                                  __byte_perm(__byte_perm(q[4], q[5], 0x40), __byte_perm(q[6], q[7], 0x40), 0x5410));
            } else {
                float f[8];
                r[v].floats(f);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = whole(f[e]);
                store_8<kOpsI8>(y + c * 8, f);
            }
        }
    }
}

// Rows of more channels than a block holds, quantised: a block walks over its row twice, the second time out of the caches.  (20000 x 20000 218 us, 5.5 TB/s of what
// is read and written once, 2000 x 65536 92, 4.3; one at a time, channels that are no multiple of 8, 20000 x 16385 294, 3.3.)
template <int E>
__global__ void __launch_bounds__(kMaxLanes) quantize_wide_kernel(const NormArgs a) {
    __shared__ float buf[64];
    int turn = 0;
    const int chunks = a.channels / E;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const uint16_t* x = (const uint16_t*)a.x + row * a.channels;
        uint8_t* y = (uint8_t*)a.y + row * a.channels;
        float top = 0.f;
        for (int c = threadIdx.x; c < chunks; c += kMaxLanes) {
            Raw<E> r;
            r.load(x + c * E);
            float f[E];
            r.floats(f);
#pragma unroll
            for (int e = 0; e < E; ++e) top = max_nan(top, fabsf(f[e]));
        }
        top = over_row<true>(top, kMaxLanes, buf, turn);
        if (threadIdx.x == 0) a.scale[row] = top / kI8Max;
        const Whole whole(top);
        for (int c = threadIdx.x; c < chunks; c += kMaxLanes) {
            Raw<E> r;
            r.load(x + c * E);
            float f[E];
            r.floats(f);
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = whole(f[e]);
            store_8<kOpsI8>(y + c * E, f);
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

template <int OUT, bool NORM>
auto fwd_kernel(const Shape& s) {
    if (s.E == 1) return s.V == 4 ? rms_norm_fwd_kernel<1, 4, OUT, NORM> : s.V == 16 ? rms_norm_fwd_kernel<1, 16, OUT, NORM> : rms_norm_fwd_kernel<1, 32, OUT, NORM>;
    if (s.E == 2) return s.V == 8 ? rms_norm_fwd_kernel<2, 8, OUT, NORM> : rms_norm_fwd_kernel<2, 16, OUT, NORM>;
    switch (s.V) {
        case 1: return rms_norm_fwd_kernel<8, 1, OUT, NORM>;
        case 2: return rms_norm_fwd_kernel<8, 2, OUT, NORM>;
        case 3: return rms_norm_fwd_kernel<8, 3, OUT, NORM>;
        default: return rms_norm_fwd_kernel<8, 4, OUT, NORM>;
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
    if (a.channels > kNormMaxChannels) {       // (a norm's are refused)
        const long long fit = 4ll * sm_count;
        prof_begin("quantize_kernel", stream);
        auto wide = a.channels % 8 == 0 ? quantize_wide_kernel<8> : quantize_wide_kernel<1>;
        wide<<<(unsigned)(a.rows < fit ? a.rows : fit), kMaxLanes, 0, stream>>>(a);
        count_launch(stream);
        return cudaGetLastError();
    }
    if (!a.weight && a.channels % 8 == 0) {
        const int chunks = a.channels / 8;
        int lanes = 4, log2 = 2;
        while (lanes * 8 < chunks && lanes < kBlock) { lanes *= 2; ++log2; }
        const int v = (chunks + lanes - 1) / lanes;
        auto kern = v <= 1 ? quantize_kernel<1> : v <= 2 ? quantize_kernel<2> : v <= 4 ? quantize_kernel<4> : quantize_kernel<8>;
        int occ = 1;
        cudaError_t e = prepare_kernel((const void*)kern, 0, kBlock, &occ);
        if (e != cudaSuccess) return e;
        const long long per_block = kBlock / lanes, need = (a.rows + per_block - 1) / per_block, fit = (long long)sm_count * (occ < 1 ? 1 : occ);
        prof_begin("quantize_kernel", stream);
        kern<<<(unsigned)(need < fit ? need : fit), kBlock, 0, stream>>>(a, lanes, log2);
        count_launch(stream);
        return cudaGetLastError();
    }
    const Shape s = shape_for(a.channels, false);
    auto kern = a.out == kOps16 ? fwd_kernel<kOps16, true>(s) : a.out == kOpsE4m3 ? fwd_kernel<kOpsE4m3, true>(s)
              : a.weight            ? fwd_kernel<kOpsI8, true>(s) : fwd_kernel<kOpsI8, false>(s);
    int occ = 1;
    cudaError_t e = prepare_kernel((const void*)kern, 0, s.threads, &occ);
    if (e != cudaSuccess) return e;
    const long long per_block = s.threads / s.lanes, need = (a.rows + per_block - 1) / per_block, fit = (long long)sm_count * (occ < 1 ? 1 : occ);
    prof_begin(a.weight ? "rms_norm_fwd_kernel" : "quantize_kernel", stream);
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
