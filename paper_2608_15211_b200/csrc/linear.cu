// The products' forward, input gradient and weight gradient (linear_tiles.cuh): their launches, and the joining of sums that are split.
#include "linear_tiles.cuh"

#ifdef TERRA_ELEM_F16
#define launch_linear launch_linear_f16
#define read_linear_status read_linear_status_f16
#endif

namespace terra {
namespace {

// Four columns of a joined sum, through the epilogue, to global memory.
template <int KIND>
__device__ __forceinline__ void join4(const LinearEpilogue& e, float (&v)[4], long long row, int col, int N, float* out) {
    const size_t at = (size_t)row * N + col;
    const bool wide = (N & 3) == 0;
    if (KIND == kLinearWeights) {
        if (wide) *reinterpret_cast<float4*>(out + at) = make_float4(v[0], v[1], v[2], v[3]);
        else
            for (int c = 0; c < 4; ++c)
                if (col + c < N) out[at + c] = v[c];
        return;
    }
    const uint16_t* extra = (const uint16_t*)(KIND == kLinearForward ? e.residual : e.z_in);
    float b[4], w[4], t[4], z[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const bool in = col + c < N;
        b[c] = in && KIND == kLinearForward && e.bias ? e.bias[col + c] : 0.f;
        w[c] = in && KIND == kLinearForward && e.w_scale ? e.w_scale[col + c] : 0.f;
        t[c] = in && extra ? elem2_to_float2(extra[at + c]).x : 0.f;
    }
    const bool scaled = KIND == kLinearForward && e.x_scale;
    const Pair xs = both(scaled ? e.x_scale[row] : 1.f);
    with_act(e.activation, [&](auto tag) {
#pragma unroll
        for (int c = 0; c < 4; c += 2) {
            Pair zz = 0, y;
            const Pair d = pair_of(v[c], v[c + 1]), bb = pair_of(b[c], b[c + 1]), in = pair_of(t[c], t[c + 1]);
            if (scaled) y = finish2<KIND, decltype(tag)::value, true>(d, bb, xs, pair_of(w[c], w[c + 1]), in, zz);
            else y = finish2<KIND, decltype(tag)::value, false>(d, bb, 0, 0, in, zz);
            split_pair(y, v[c], v[c + 1]);
            split_pair(zz, z[c], z[c + 1]);
        }
    });
    if (wide) {
        if (KIND == kLinearForward && e.z) *reinterpret_cast<uint2*>((uint16_t*)e.z + at) = make_uint2(pack_elem(z[0], z[1]), pack_elem(z[2], z[3]));
        *reinterpret_cast<uint2*>((uint16_t*)e.y + at) = make_uint2(pack_elem(v[0], v[1]), pack_elem(v[2], v[3]));
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (col + c < N) {
                if (KIND == kLinearForward && e.z) ((uint16_t*)e.z)[at + c] = (uint16_t)pack_elem(z[c], 0.f);
                ((uint16_t*)e.y)[at + c] = (uint16_t)pack_elem(v[c], 0.f);
            }
    }
}
// Joins the parts of a split product: the sum over the splits, in a fixed order, then the epilogue.  WHOLE: parts in 32-bit integers.
template <int KIND, bool WHOLE>
__global__ void __launch_bounds__(256) linear_join_kernel(const LinearEpilogue e, const float* parts, int splits, long long M, int N, float* out,
                                                          const float* a_parts, int a_splits) {
    let_dependents_start();
    wait_for_prerequisites();
    const int per_row = (N + 3) / 4;
    const long long total = M * per_row;
    const size_t part = (size_t)M * N;
    if (KIND == kLinearWeights && a_parts)
        for (long long i = blockIdx.x * 256ll + threadIdx.x; i < M; i += gridDim.x * 256ll) {
            float v = 0.f;
#pragma unroll 8
            for (int s = 0; s < a_splits; ++s) v += a_parts[s * M + i];
            e.a_sums[i] = v;
        }
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        long long row;
        int c4;
        split_item(i, per_row, row, c4);
        typename SumOf<WHOLE>::Type v[4] = {0, 0, 0, 0};
#pragma unroll 8
        for (int s = 0; s < splits; ++s) part4<WHOLE>(parts + s * part + (size_t)row * N + 4 * c4, 4 * c4, N, v);
        float f[4] = {(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
        join4<KIND>(e, f, row, 4 * c4, N, out);
    }
}
// The same for outputs too small to fill the device so: 8 threads share the parts of four columns.  (A thread that adds 64 parts up alone waits for
// memory eight times.)  Blocks from `quads` on add up a_parts.
template <int KIND, bool WHOLE>
__global__ void __launch_bounds__(256) linear_join_small_kernel(const LinearEpilogue e, const float* parts, int splits, long long M, int N, float* out,
                                                                const float* a_parts, int a_splits, int quads) {
    typedef typename SumOf<WHOLE>::Type Sum;
    __shared__ Sum sums[8][32][4];
    let_dependents_start();
    wait_for_prerequisites();
    const int sub = threadIdx.x >> 5, lane = threadIdx.x & 31, per_row = (N + 3) / 4;
    Sum v[4] = {0, 0, 0, 0};
    const bool is_a = KIND == kLinearWeights && (int)blockIdx.x >= quads;
    const long long i = (is_a ? blockIdx.x - quads : blockIdx.x) * 32ll + lane;
    long long row = 0;
    int c4 = 0;
    if (is_a) {
        if (i < M)
#pragma unroll 4
            for (int s = sub; s < a_splits; s += 8) v[0] += a_parts[s * M + i];
    } else if (i < M * per_row) {
        split_item(i, per_row, row, c4);
#pragma unroll 4
        for (int s = sub; s < splits; s += 8) part4<WHOLE>(parts + s * (size_t)M * N + (size_t)row * N + 4 * c4, 4 * c4, N, v);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) sums[sub][lane][c] = v[c];
    __syncthreads();
    if (sub) return;
#pragma unroll
    for (int k = 1; k < 8; ++k)
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] += sums[k][lane][c];
    if (is_a) {
        if (i < M) e.a_sums[i] = v[0];
    } else if (i < M * per_row) {
        float f[4] = {(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
        join4<KIND>(e, f, row, 4 * c4, N, out);
    }
}

// where a thread for four columns leaves most of the device idle and adds up more than a few parts
bool splits_are_many(int splits, long long quads) { return splits >= 4 && quads <= 256ll * kPlanSms; }

template <int KIND, int OPS, bool LONG>
cudaError_t launch_one_tile(bool pair, bool map, const Maps& maps, Job& job, int sm_count, cudaStream_t stream) {
    if (pair) return map ? launch_one<true, KIND, OPS, true, 1, LONG>(maps, job, sm_count, stream) : launch_one<true, KIND, OPS, false, 1, LONG>(maps, job, sm_count, stream);
    return map ? launch_one<false, KIND, OPS, true, 1, LONG>(maps, job, sm_count, stream) : launch_one<false, KIND, OPS, false, 1, LONG>(maps, job, sm_count, stream);
}
template <int KIND, int OPS>
cudaError_t launch_kind(bool pair, bool map, int tiles, const Maps& maps, Job& job, int sm_count, cudaStream_t stream) {
    if constexpr (OPS == kOps16)
        if (pair && tiles == 2) return launch_one<true, KIND, OPS, true, 2, false>(maps, job, sm_count, stream);
    if constexpr (OPS == kOpsI8)
        if (tiles == 3) {
            if (pair) return map ? launch_one<true, KIND, OPS, true, 3, false>(maps, job, sm_count, stream) : launch_one<true, KIND, OPS, false, 3, false>(maps, job, sm_count, stream);
            return map ? launch_one<false, KIND, OPS, true, 3, false>(maps, job, sm_count, stream) : launch_one<false, KIND, OPS, false, 3, false>(maps, job, sm_count, stream);
        }
    if constexpr (OPS != kOpsI8)
        if (job.kb_per_split > kLinearLongChunk) return launch_one_tile<KIND, OPS, true>(pair, map, maps, job, sm_count, stream);
    return launch_one_tile<KIND, OPS, false>(pair, map, maps, job, sm_count, stream);
}

}  // namespace

cudaError_t read_linear_status(int* timed_out) {
    int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(timed_out, g_linear_timeout, sizeof(int));
    if (e != cudaSuccess) return e;
    if (*timed_out) e = cudaMemcpyToSymbol(g_linear_timeout, &zero, sizeof(int));
    return e;
}

// D[M, N] over K: operands given with their rows' strides in bytes (multiples of 16).  K-major operands are [M or N][K], MN-major ones [K][M or N].
cudaError_t launch_linear(int kind, int ops, const LinearPlan& p, long long M, int N, long long K, const void* a, long long stride_a, const void* b, long long stride_b,
                          const LinearEpilogue& epi, float* out, float* parts, float* a_parts, int sm_count, cudaStream_t stream) {
    const int ctas = p.pair ? 2 : 1, cols = p.bn / ctas, elem = ops != kOps16 ? 1 : 2;
    const bool a_mn = kind == kLinearWeights, b_mn = kind != kLinearForward;
    Maps maps;
    if (!encode_map(&maps.a, a, a_mn ? M : K, a_mn ? K : M, stride_a, elem, a_mn ? 64 : 128) ||
        !encode_map(&maps.b, b, b_mn ? N : K, b_mn ? K : N, stride_b, elem, b_mn ? 64 : cols))
        return cudaErrorInvalidValue;
    const void* in = kind == kLinearForward ? epi.residual : epi.z_in;
    const bool by_map = kind != kLinearWeights && p.splits == 1 && N % 8 == 0;
    maps.in = maps.in_up = maps.y = maps.z = maps.z_up = maps.a;
    // Two tiles a warp where the epilogue takes longer than the products: short sums with a residual or z_in to read or a costly activation.  One tile / two, us:
    // 550800 x 384 -> 1536, residual 802 / 760, silu 818 / 698, gelu with z 1078 / 1020, d_x of silu 1016 / 830; but z alone 798 / 850, e4m3 with gelu
    // 1029 / 1090; 131072 x 768 -> 768, d_x of gelu 183 / 203.
    const bool costly = in || epi.activation >= TERRA_ACT_SILU;
    const int tiles = ops == kOpsI8 && p.splits == 1 && p.k_blocks <= kI8TableBlocks ? 3 : by_map && p.pair && ops == kOps16 && p.k_blocks <= kTwoTilesBlocks && costly && !(in && epi.z) ? 2 : 1, wide = epi.z && tiles == 1 ? 64 : 128;
    if (by_map && ((in && !encode_map(&maps.in, in, N, M, 2ll * N, 2, 32, wide)) || !encode_map(&maps.y, epi.y, N, M, 2ll * N, 2, 32, wide) ||
                   (epi.z && !encode_map(&maps.z, epi.z, N, M, 2ll * N, 2, 32, wide))))
        return cudaErrorInvalidValue;
    Job job{};
    if (!set_job(job, p, p.bn, M, N, epi, parts)) return cudaErrorInvalidConfiguration;
    job.boxes_b = (cols + 63) / 64;
    job.bytes_b = b_mn ? job.boxes_b * (kOperand / 2) : cols * 128;
    job.idesc = ops == kOpsI8   ? make_idesc_i8(128 * ctas, p.bn)
              : ops == kOpsE4m3 ? make_idesc_f16(128 * ctas, p.bn, 0, 0)      // e4m3 has format number 0, as fp16 has in its kind
                                : make_idesc_elem(128 * ctas, p.bn, a_mn ? 1 : 0, b_mn ? 1 : 0);
    const int a_splits = epi.a_sums ? p.splits * p.n_tiles : 0;
    if (a_splits > 1) job.e.a_sums = a_parts;
    if (kind == kLinearWeights && p.splits == 1) job.e.sums = out;
    // (a part of a split sum goes neither way)
    const bool map = by_map || p.splits > 1;
    cudaError_t e;
    if (kind == kLinearForward && ops == kOpsI8) e = launch_kind<kLinearForward, kOpsI8>(p.pair, map, tiles, maps, job, sm_count, stream);
    else if (kind == kLinearForward && ops == kOpsE4m3) e = launch_kind<kLinearForward, kOpsE4m3>(p.pair, map, tiles, maps, job, sm_count, stream);
    else if (kind == kLinearForward) e = launch_kind<kLinearForward, kOps16>(p.pair, map, tiles, maps, job, sm_count, stream);
    else if (kind == kLinearInput) e = launch_kind<kLinearInput, kOps16>(p.pair, map, tiles, maps, job, sm_count, stream);
    else e = p.pair ? launch_one<true, kLinearWeights, kOps16, true, 1, false>(maps, job, sm_count, stream) : launch_one<false, kLinearWeights, kOps16, true, 1, false>(maps, job, sm_count, stream);
    if (e == cudaSuccess && p.splits == 1 && a_splits > 1) return launch_sum_partials(a_parts, a_splits, (int)M, epi.a_sums, stream);
    if (e != cudaSuccess || p.splits == 1) return e;
    const long long quads = M * ((N + 3) / 4);
    const float* ap = a_splits ? (const float*)a_parts : nullptr;
    prof_begin("linear_join_kernel", stream);
    if (splits_are_many(p.splits, quads)) {
        auto join = kind == kLinearWeights ? linear_join_small_kernel<kLinearWeights, false> : kind == kLinearInput ? linear_join_small_kernel<kLinearInput, false>
                  : ops == kOpsI8          ? linear_join_small_kernel<kLinearForward, true>  : linear_join_small_kernel<kLinearForward, false>;
        const unsigned blocks = (unsigned)((quads + 31) / 32);
        e = launch_dependent(join, blocks + (ap ? (unsigned)((M + 31) / 32) : 0u), 256u, 0, stream, epi, (const float*)parts, p.splits, M, N, out, ap, a_splits, (int)blocks);
    } else {
        auto join = kind == kLinearWeights ? linear_join_kernel<kLinearWeights, false> : kind == kLinearInput ? linear_join_kernel<kLinearInput, false>
                  : ops == kOpsI8          ? linear_join_kernel<kLinearForward, true>  : linear_join_kernel<kLinearForward, false>;
        const long long need = (quads + 255) / 256, fit = 8ll * sm_count;
        e = launch_dependent(join, (unsigned)(need < fit ? need : fit), 256u, 0, stream, epi, (const float*)parts, p.splits, M, N, out, ap, a_splits);
    }
    count_launch(stream);
    return e;
}

}  // namespace terra
