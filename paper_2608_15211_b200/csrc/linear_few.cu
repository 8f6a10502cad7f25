// The forward product for up to 8 rows of x (a conditioning vector, a single token): y = act(x w' + bias) + residual, 16-bit or e4m3 operands (those
// made fp16, which is exact), on the warps' matrix instructions of 16 rows of w x 8 rows of x, sums in fp32.  Every weight is read once,
// straight into the registers of its product: a lane takes 16 consecutive bytes of a row of w and of x for what the instruction calls columns
// 2t, 2t + 1, 2t + 8, 2t + 9 and so on, which only changes the order of the sum.  The warps of a group share the sum over k; no operand needs padding.
// What bounds it: HBM behind a launch's latency (weights not in L2: 2 x 4096 -> 8192, 67 MB, 15.1 us; 2 x 8192 -> 8192, 134 MB, 25.6 us; 8 rows 15.9 and
// 26.5; e4m3 11.2 and 20.1).  tcgen05 wants 128 rows and its operands in shared memory, one more step between HBM and the product (16 rows 19.0 and 33.1
// us).  On the plain arithmetic units, two conversions for a pair of weights and a multiplication for each row of x, these took 18.1 and 32.4 us with 2
// rows, 23.5 and 33 with 8; one row, 8192 -> 8192, took 24.3 there and 25.5 here.
#include <cuda_fp8.h>

#include "block_act.cuh"
#include "block_kernels.h"

#ifdef TERRA_ELEM_F16
#define launch_linear_few launch_linear_few_f16
#endif

namespace terra {
namespace {

constexpr int kWarps = 16, kRows = 16, kDeep = 4;        // of a block; of w at a time; runs of k under way in a warp

// 16 bytes of an operand's row, the part of them that lies before the row's end; V: bytes that all rows are aligned to
template <int V>
__device__ __forceinline__ void load16(const char* row, int at, int bytes, uint32_t (&v)[4]) {
    if (V == 16) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (at < bytes) u = *reinterpret_cast<const uint4*>(row + at);
        v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = 0;
#pragma unroll
            for (int j = 0; j < 4; j += V) {
                const int a = at + 4 * i + j;
                if (a < bytes) {
                    const uint32_t u = V == 4 ? *reinterpret_cast<const uint32_t*>(row + a)
                                     : V == 2 ? *reinterpret_cast<const uint16_t*>(row + a) : *reinterpret_cast<const uint8_t*>(row + a);
                    v[i] |= u << (8 * j);
                }
            }
        }
    }
}

template <bool E4M3>
__device__ __forceinline__ void multiply(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
#ifdef TERRA_ELEM_F16
    constexpr bool kHalf = true;
#else
    constexpr bool kHalf = E4M3;
#endif
    if (kHalf)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t half2_of_e4m3(uint32_t two) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
    return (uint32_t)h.x | (uint32_t)h.y << 16;
}

// A group of `share` warps has `height` rows of w, from n0 on: 4, 8 or kRows.
template <bool E4M3, int V>
__global__ void __launch_bounds__(32 * kWarps, 2) linear_few_kernel(const LinearEpilogue e, const char* x, const char* w, int rows, int n_in,
                                                                    int n_out, int share, int height) {
    __shared__ float sums[kWarps][8][kRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % share, group = warp / share, groups = kWarps / share;
    const int g = lane >> 2, t = lane & 3, bytes = n_in * (E4M3 ? 1 : 2), n0 = (blockIdx.x * groups + group) * height;
    const char* w0 = w + (long long)min(n0 + g, n_out - 1) * bytes;
    const char* w1 = w + (long long)min(n0 + 8 + g, n_out - 1) * bytes;
    const char* xr = x + (long long)g * bytes;
    const int x_bytes = g < rows ? bytes : 0, w0_bytes = g < height ? bytes : 0, w1_bytes = height > 8 ? bytes : 0;        // rows that are not there are zeros
    float total[4] = {0.f, 0.f, 0.f, 0.f};
    let_dependents_start();
    wait_for_prerequisites();
#pragma unroll 1
    for (int at = part * 64 + t * 16; at - t * 16 < bytes && n0 < n_out; at += kDeep * share * 64) {
        // (The instruction cuts its sum off: no more than 16 steps to one.  65536 features of one sign, fp16: 2.6e-5 -> 5e-7 off, at the same time.  Totals in
        // shared memory, for want of registers, took 11.2 us instead of 9.7 where the weights, 2 x 4096 -> 8192, are in L2.)
        float c[4] = {0.f, 0.f, 0.f, 0.f};
        uint32_t a[kDeep][4], b[kDeep][4];
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            load16<V>(w0, at + i * share * 64, w0_bytes, a[i]);
            load16<V>(w1, at + i * share * 64, w1_bytes, b[i]);
        }
#pragma unroll
        for (int i = 0; i < kDeep; ++i) {
            uint32_t xv[4];
            load16<V>(xr, at + i * share * 64, x_bytes, xv);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint32_t p = a[i][2 * s], q = a[i][2 * s + 1], u = b[i][2 * s], v = b[i][2 * s + 1], m = xv[2 * s], n = xv[2 * s + 1];
                if (E4M3) {
                    multiply<true>(c, half2_of_e4m3(p & 0xffff), half2_of_e4m3(u & 0xffff), half2_of_e4m3(p >> 16), half2_of_e4m3(u >> 16), half2_of_e4m3(m & 0xffff), half2_of_e4m3(m >> 16));
                    multiply<true>(c, half2_of_e4m3(q & 0xffff), half2_of_e4m3(v & 0xffff), half2_of_e4m3(q >> 16), half2_of_e4m3(v >> 16), half2_of_e4m3(n & 0xffff), half2_of_e4m3(n >> 16));
                } else {
                    multiply<false>(c, p, u, q, v, m, n);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) total[i] += c[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[warp][2 * t + (i & 1)][g + 8 * (i >> 1)] = total[i];
    __syncthreads();
    // a thread to an output
    for (int i = threadIdx.x; i < groups * rows * height; i += 32 * kWarps) {
        const int o = i % height, r = i / height % rows, of = i / height / rows, n = (blockIdx.x * groups + of) * height + o;
        if (n >= n_out) continue;
        float z = 0.f;
        for (int s = 0; s < share; ++s) z += sums[of * share + s][r][o];
        const long long at = (long long)r * n_out + n;
        if (E4M3) z = z * e.x_scale[r] * e.w_scale[n];
        if (e.bias) z += e.bias[n];
        if (e.z) ((uint16_t*)e.z)[at] = (uint16_t)pack_elem(z, 0.f);
        const float res = e.residual ? elem2_to_float2(((const uint16_t*)e.residual)[at]).x : 0.f;
        with_act(e.activation, [&](auto tag) { ((uint16_t*)e.y)[at] = (uint16_t)pack_elem(act<decltype(tag)::value>(z) + res, 0.f); });
    }
}

}  // namespace

cudaError_t launch_linear_few(bool e4m3, int rows, int n_in, int n_out, const void* x, const void* w, const LinearEpilogue& epi, cudaStream_t stream) {
    const int bytes = n_in * (e4m3 ? 1 : 2), runs = (bytes + 63) / 64;
    constexpr long long kFit = 2 * kWarps * kPlanSms;        // warps on the GPU at a time
    // Rows of w at a time: fewer where that gives more SMs something to read (3 x 4096 -> 372 5.7 -> 5.2 us, 1 x 16384 -> 64 13.1 -> 12.0).
    int height = kRows, share = 1;
    while (height > 4 && 2ll * ((n_out + height - 1) / height) * (runs < kWarps ? runs : kWarps) <= kFit) height /= 2;
    // Warps that share a sum: as many as have 2 kDeep runs each, and more, down to one run, while all of them are on the GPU at a time.  (With kDeep runs each
    // 1 x 1024 -> 65536 29.7 us, with 2 kDeep 28.0; no more warps than are on the GPU at a time: 2 x 8192 -> 8192 28.7 us against 25.6.)
    const int tiles = (n_out + height - 1) / height;
    while (share < kWarps && (4 * share * kDeep <= runs || (2 * share <= runs && 2ll * tiles * share <= kFit))) share *= 2;
    const int groups = kWarps / share;
    auto kern = e4m3 ? (bytes % 16 == 0 ? linear_few_kernel<true, 16> : bytes % 4 == 0 ? linear_few_kernel<true, 4> : linear_few_kernel<true, 1>)
                     : (bytes % 16 == 0 ? linear_few_kernel<false, 16> : bytes % 4 == 0 ? linear_few_kernel<false, 4> : linear_few_kernel<false, 2>);
    prof_begin("linear_few_kernel", stream);
    const cudaError_t e = launch_dependent(kern, (unsigned)((tiles + groups - 1) / groups), 32u * kWarps, 0, stream, epi, (const char*)x, (const char*)w, rows, n_in, n_out, share, height);
    count_launch(stream);
    return e;
}

}  // namespace terra
