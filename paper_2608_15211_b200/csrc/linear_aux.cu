// What the products need beside the matrix instructions: rows padded to 16 bytes for the copy engine, column sums (the bias's
// gradient) and the gradient through an activation that no product follows.  All of them are bound by HBM.
#include "block_act.cuh"
#include "block_kernels.h"

#ifdef TERRA_ELEM_F16
#define launch_column_sums launch_column_sums_f16
#define launch_activation_bwd launch_activation_bwd_f16
#endif

namespace terra {
namespace {

constexpr int kBlock = 256;

#ifndef TERRA_ELEM_F16
// T: the widest unit that all sources' rows are multiples of
template <typename T>
__global__ void __launch_bounds__(kBlock) pad_rows_kernel(const PadJobs jobs) {
    constexpr int kPer = 16 / sizeof(T);
    let_dependents_start();
    wait_for_prerequisites();
#pragma unroll 1
    for (int k = 0; k < jobs.count; ++k) {
        const PadJob& j = jobs.job[k];
        const int units = j.bytes / (int)sizeof(T), vectors = j.stride / 16;
        const long long total = j.rows * vectors;
        const T* src = (const T*)j.src;
        uint4* dst = (uint4*)j.dst;
        for (long long i = blockIdx.x * (long long)kBlock + threadIdx.x; i < total; i += (long long)gridDim.x * kBlock) {
            long long row;
            int v;
            split_item(i, vectors, row, v);
            union { T t[kPer]; uint4 all; } u;
            const T* p = src + row * units + (long long)v * kPer;
#pragma unroll
            for (int e = 0; e < kPer; ++e) u.t[e] = v * kPer + e < units ? p[e] : T(0);
            dst[i] = u.all;
        }
    }
}

// 32 columns to a block, 32 slices of the rows of `partial`
__global__ void __launch_bounds__(1024) sum_partials_kernel(const float* partial, int blocks, int columns, float* out) {
    __shared__ float slices[32][33];
    let_dependents_start();
    wait_for_prerequisites();
    const int cx = threadIdx.x & 31, slice = threadIdx.x >> 5, c = blockIdx.x * 32 + cx;
    float s = 0.f;
    if (c < columns)
#pragma unroll 4
        for (int b = slice; b < blocks; b += 32) s += partial[(size_t)b * columns + c];
    slices[slice][cx] = s;
    __syncthreads();
    s = slices[cx][slice];
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int cw = blockIdx.x * 32 + slice;
    if (cx == 0 && cw < columns) out[cw] = s;
}
#endif

// 256 columns (32 threads x 8) and 8 rows at a time to a block; the row slice blockIdx.y of the partial sums
__global__ void __launch_bounds__(kBlock) column_sums_kernel(const uint16_t* x, long long rows, int columns, long long stride, float* partial) {
    __shared__ float sums[8][256];
    let_dependents_start();
    wait_for_prerequisites();
    const int cx = threadIdx.x & 31, sub = threadIdx.x >> 5, col = blockIdx.x * 256 + cx * 8;
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = 0.f;
    if (col < columns) {                       // (the rows are padded to 16 bytes)
#pragma unroll 4
        for (long long r = (long long)blockIdx.y * 8 + sub; r < rows; r += (long long)gridDim.y * 8) {
            const uint4 v = *reinterpret_cast<const uint4*>(x + r * stride + col);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { const float2 t = elem2_to_float2(w[i]); s[2 * i] += t.x; s[2 * i + 1] += t.y; }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[sub][cx * 8 + e] = s[e];
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    float all = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) all += sums[i][threadIdx.x];
    if (c < columns) partial[(size_t)blockIdx.y * columns + c] = all;
}

// 8 elements a thread; what is behind the last 8 goes element by element to the first threads
__global__ void __launch_bounds__(kBlock) activation_bwd_kernel(const uint16_t* z, const uint16_t* d_y, uint16_t* d_z, long long n, int activation) {
    const long long first = blockIdx.x * (long long)kBlock + threadIdx.x, step = (long long)gridDim.x * kBlock;
    for (long long i = first; i < n / 8; i += step) {
        const uint4 zv = *reinterpret_cast<const uint4*>(z + 8 * i), gv = *reinterpret_cast<const uint4*>(d_y + 8 * i);
        const uint32_t zw[4] = {zv.x, zv.y, zv.z, zv.w}, gw[4] = {gv.x, gv.y, gv.z, gv.w};
        uint32_t out[4];
        with_act(activation, [&](auto tag) {
            constexpr int A = decltype(tag)::value;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 a = elem2_to_float2(zw[k]), g = elem2_to_float2(gw[k]);
                float lo, hi;
                split_pair(pmul(pair_of(g.x, g.y), act_slope2<A>(pair_of(a.x, a.y))), lo, hi);
                out[k] = pack_elem(lo, hi);
            }
        });
        *reinterpret_cast<uint4*>(d_z + 8 * i) = make_uint4(out[0], out[1], out[2], out[3]);
    }
    if (first < n % 8) {
        const long long i = n / 8 * 8 + first;
        const float a = elem2_to_float2(z[i]).x, g = elem2_to_float2(d_y[i]).x;
        with_act(activation, [&](auto tag) { d_z[i] = (uint16_t)pack_elem(g * act_slope<decltype(tag)::value>(a), 0.f); });
    }
}

}  // namespace

#ifndef TERRA_ELEM_F16
cudaError_t launch_pad_rows(const PadJobs& jobs, int sm_count, cudaStream_t stream) {
    long long most = 0;
    int all = 0;
    for (int k = 0; k < jobs.count; ++k) {
        const long long total = jobs.job[k].rows * (jobs.job[k].stride / 16);
        most = total > most ? total : most;
        all |= jobs.job[k].bytes;
    }
    const long long need = (most + kBlock - 1) / kBlock, fit = 16ll * sm_count;
    auto kern = all % 8 == 0 ? pad_rows_kernel<unsigned long long> : all % 4 == 0 ? pad_rows_kernel<uint32_t> : all % 2 == 0 ? pad_rows_kernel<uint16_t> : pad_rows_kernel<uint8_t>;
    prof_begin("pad_rows_kernel", stream);
    const cudaError_t e = launch_dependent(kern, (unsigned)(need < fit ? need : fit), (unsigned)kBlock, 0, stream, jobs);
    count_launch(stream);
    return e;
}

int column_sum_blocks(long long rows, int columns) {
    const long long across = (columns + 255) / 256, fit = (4ll * kPlanSms + across - 1) / across, need = (rows + 63) / 64;
    return (int)(need < fit ? need : fit);
}

cudaError_t launch_sum_partials(const float* partial, int blocks, int columns, float* out, cudaStream_t stream) {
    prof_begin("sum_partials_kernel", stream);
    const cudaError_t e = launch_dependent(sum_partials_kernel, (unsigned)((columns + 31) / 32), 1024u, 0, stream, partial, blocks, columns, out);
    count_launch(stream);
    return e;
}
#endif

cudaError_t launch_column_sums(const void* x, long long rows, int columns, long long stride, float* partial, float* out, cudaStream_t stream) {
    const int slices = column_sum_blocks(rows, columns);
    prof_begin("column_sums_kernel", stream);
    column_sums_kernel<<<dim3((unsigned)((columns + 255) / 256), (unsigned)slices), kBlock, 0, stream>>>((const uint16_t*)x, rows, columns, stride, partial);
    count_launch(stream);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_sum_partials(partial, slices, columns, out, stream);
}

cudaError_t launch_activation_bwd(const void* z, const void* d_y, void* d_z, long long n, int activation, int sm_count, cudaStream_t stream) {
    const long long need = (n / 8 + kBlock) / kBlock, fit = 16ll * sm_count;        // (one thread at least behind the last 8)
    prof_begin("activation_bwd_kernel", stream);
    activation_bwd_kernel<<<(unsigned)(need < fit ? need : fit), kBlock, 0, stream>>>((const uint16_t*)z, (const uint16_t*)d_y, (uint16_t*)d_z, n, activation);
    count_launch(stream);
    return cudaGetLastError();
}

}  // namespace terra
