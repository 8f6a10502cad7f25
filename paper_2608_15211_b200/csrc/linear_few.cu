// The forward product for a few rows (a conditioning vector, a single token): y = act(x w' + bias) + residual for up to 8 rows of x, on the
// plain arithmetic units, 16-bit or e4m3 operands.  Every weight is read once, in runs of 512 bytes a warp, and meets all rows of x in fp32.
// A block takes kOut rows of w for each of its groups of warps, the warps of a group share the sum over k; no operand needs padding.
// What bounds it: HBM behind a launch's latency (weights not in L2: 2 x 4096 -> 8192, 67 MB, 17.8 us; 2 x 8192 -> 8192, 134 MB, 30.6 us).  The
// tensor-core kernel spends its tiles of 128 rows on zeros there: it keeps a tenth of the bytes in flight that this one does.
#include <cuda_fp8.h>

#include "block_act.cuh"
#include "block_kernels.h"

#ifdef TERRA_ELEM_F16
#define launch_linear_few launch_linear_few_f16
#endif

namespace terra {
namespace {

constexpr int kWarps = 8;

// V values of an operand's row in memory, as pairs of fp32 (V 1: the second is 0)
template <bool E4M3, int V> struct Run;
template <int V> struct Run<false, V> {
    static constexpr int kPairs = V > 1 ? V / 2 : 1;
    uint32_t w[kPairs];
    __device__ __forceinline__ void load(const void* row, long long k) {
        const uint16_t* p = (const uint16_t*)row + k;
        if (V == 8) *reinterpret_cast<uint4*>(w) = __ldg(reinterpret_cast<const uint4*>(p));
        else if (V == 2) w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
        else w[0] = __ldg(p);
    }
    __device__ __forceinline__ Pair pair(int i) const { const float2 t = elem2_to_float2(w[i]); return pair_of(t.x, t.y); }
};
template <int V> struct Run<true, V> {
    static constexpr int kPairs = V > 1 ? V / 2 : 1;
    uint32_t w[V >= 4 ? V / 4 : 1];
    __device__ __forceinline__ void load(const void* row, long long k) {
        const uint8_t* p = (const uint8_t*)row + k;
        if (V == 16) *reinterpret_cast<uint4*>(w) = __ldg(reinterpret_cast<const uint4*>(p));
        else if (V == 4) w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
        else w[0] = __ldg(p);
    }
    __device__ __forceinline__ Pair pair(int i) const {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
        const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&h));
        return pair_of(t.x, t.y);
    }
};

template <bool E4M3, int R, int V>
__global__ void __launch_bounds__(32 * kWarps) linear_few_kernel(const LinearEpilogue e, const void* __restrict__ x, const void* __restrict__ w, int rows, int n_in, int n_out,
                                                                 int share) {
    constexpr int kOut = R == 8 ? 2 : 4, kValues = kOut * R, kElem = E4M3 ? 1 : 2;
    __shared__ float sums[kWarps][kValues];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % share, group = warp / share;
    const int n0 = (blockIdx.x * (kWarps / share) + group) * kOut;
    const char *xr[R], *wr[kOut];
#pragma unroll
    for (int r = 0; r < R; ++r) xr[r] = (const char*)x + (long long)min(r, rows - 1) * n_in * kElem;
#pragma unroll
    for (int o = 0; o < kOut; ++o) wr[o] = (const char*)w + (long long)min(n0 + o, n_out - 1) * n_in * kElem;
    Pair acc[kOut][R];
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[o][r] = 0;
    let_dependents_start();
    wait_for_prerequisites();
#pragma unroll (R >= 4 ? 2 : 4)
    for (int k = (part * 32 + lane) * V; k < n_in; k += share * 32 * V) {
        Run<E4M3, V> wv[kOut], xv[R];
#pragma unroll
        for (int o = 0; o < kOut; ++o) wv[o].load(wr[o], k);
#pragma unroll
        for (int r = 0; r < R; ++r) xv[r].load(xr[r], k);
#pragma unroll
        for (int i = 0; i < Run<E4M3, V>::kPairs; ++i) {
            Pair xp[R];
#pragma unroll
            for (int r = 0; r < R; ++r) xp[r] = xv[r].pair(i);
#pragma unroll
            for (int o = 0; o < kOut; ++o) {
                const Pair wp = wv[o].pair(i);
#pragma unroll
                for (int r = 0; r < R; ++r) acc[o][r] = pfma(wp, xp[r], acc[o][r]);
            }
        }
    }
#pragma unroll
    for (int o = 0; o < kOut; ++o)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float a, b;
            split_pair(acc[o][r], a, b);
            a += b;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
            if (lane == 0) sums[warp][r * kOut + o] = a;
        }
    __syncthreads();
    // a thread of each group to an output
    const int out_group = threadIdx.x / kValues, v = threadIdx.x % kValues, r = v / kOut, n = (blockIdx.x * (kWarps / share) + out_group) * kOut + v % kOut;
    if (out_group >= kWarps / share || r >= rows || n >= n_out) return;
    float z = 0.f;
    for (int i = 0; i < share; ++i) z += sums[out_group * share + i][v];
    const long long at = (long long)r * n_out + n;
    if (E4M3) z = z * e.x_scale[r] * e.w_scale[n];
    if (e.bias) z += e.bias[n];
    if (e.z) ((uint16_t*)e.z)[at] = (uint16_t)pack_elem(z, 0.f);
    const float res = e.residual ? elem2_to_float2(((const uint16_t*)e.residual)[at]).x : 0.f;
    with_act(e.activation, [&](auto tag) { ((uint16_t*)e.y)[at] = (uint16_t)pack_elem(act<decltype(tag)::value>(z) + res, 0.f); });
}

template <bool E4M3, int R>
auto kernel_for(int n_in) {
    constexpr int kWide = E4M3 ? 16 : 8, kMid = E4M3 ? 4 : 2;
    return n_in % kWide == 0 ? linear_few_kernel<E4M3, R, kWide> : n_in % kMid == 0 ? linear_few_kernel<E4M3, R, kMid> : linear_few_kernel<E4M3, R, 1>;
}

}  // namespace

cudaError_t launch_linear_few(bool e4m3, int rows, int n_in, int n_out, const void* x, const void* w, const LinearEpilogue& epi, cudaStream_t stream) {
    const int R = rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8, out = R == 8 ? 2 : 4;
    const int wide = e4m3 ? 16 : 8, mid = e4m3 ? 4 : 2, v = n_in % wide == 0 ? wide : n_in % mid == 0 ? mid : 1;
    // warps that share a sum: as many as fit the device at a time (24 an SM, for one row 40), so that each has many runs and none waits for a place
    // (4096 -> 8192: 2 rows with one warp to a sum 17.1 us, with two 18.6; 8192 -> 8192: 1 row with one warp 29.5, with two 24.2)
    const int sums = (n_out + out - 1) / out;
    int share = 1;
    while (share < kWarps && share * 32 * v < n_in && 2ll * sums * share <= (R == 1 ? 40ll : 24ll) * kPlanSms) share *= 2;
    const int per_block = kWarps / share * out;
    auto kern = e4m3 ? (R == 1 ? kernel_for<true, 1>(n_in) : R == 2 ? kernel_for<true, 2>(n_in) : R == 4 ? kernel_for<true, 4>(n_in) : kernel_for<true, 8>(n_in))
                     : (R == 1 ? kernel_for<false, 1>(n_in) : R == 2 ? kernel_for<false, 2>(n_in) : R == 4 ? kernel_for<false, 4>(n_in) : kernel_for<false, 8>(n_in));
    prof_begin("linear_few_kernel", stream);
    const cudaError_t e = launch_dependent(kern, (unsigned)((n_out + per_block - 1) / per_block), 32u * kWarps, 0, stream, epi, x, w, rows, n_in, n_out, share);
    count_launch(stream);
    return e;
}

}  // namespace terra
