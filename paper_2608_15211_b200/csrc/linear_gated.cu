// The products around a gate (linear_tiles.cuh): y = act(g) u of [g, u] = x w' + bias in one kernel, and the input gradient of the product that follows
// through the gate, with the joining of their sums that are split.
//
// Forward: a tile of 256 accumulator columns is 128 gate columns and the 128 up columns that go with them, so that a thread of the epilogue has both of an
// output; of two CTAs on a tile one brings the gate's weights, the other the up rows.  Nothing but y (and z where it is kept) is written.  Backward: the tile
// is the gradient d of y; the epilogue reads g and u and writes d u act'(g) and d act(g) where z lies, so d itself never reaches memory.
//
// What bounds it, a call on a cool GPU (one after the other over seconds, under the power cap, in brackets): forward, the tensor pipe where the sum is long (32768 x 1024 -> 4096 337 us,
// busy in 92 % of the cycles, in 8-bit integers 184 us, 79 %; 156672 x 4096 -> 8192 in 8 bits 6.5 ms, 3240 TFLOP/s (7.5 ms)), the epilogue in 8 bits where it is short (550800 x 384 ->
// 1024 800 us, in 16 bits 715), writes where z is kept (550800 x 384 -> 1024 955 us (1.1 ms) for 3.4 GB); backward, operands and z that share the way into the SMs (156672 x 1024 -> 2752
// 925 us, with the weight gradient 1.6 ms (2.0), the pipe busy in 57 % of the cycles, HBM at 4.6 TB/s; 550800 x 384 -> 1024 905 us, 5.4 TB/s).
#include "linear_tiles.cuh"

#ifdef TERRA_ELEM_F16
#define launch_gated launch_gated_f16
#define launch_gated_input launch_gated_input_f16
#define read_gated_status read_gated_status_f16
#endif

namespace terra {
namespace {

// Joins the parts of a split product, in a fixed order: four neighbouring columns to 8 threads, which share the parts.  BWD: `parts` [splits][M][N] of d;
// forward [splits][2][M][N], gate and up.  WHOLE: parts in 32-bit integers.
constexpr int kJoinShare = 8, kJoinQuads = 32;
template <bool BWD, bool WHOLE>
__global__ void __launch_bounds__(kJoinShare * kJoinQuads) gated_join_kernel(const LinearEpilogue e, const float* parts, int splits, long long M, int N) {
    constexpr int H = BWD ? 1 : 2;
    typedef typename SumOf<WHOLE>::Type Sum;
    __shared__ Sum sums[kJoinShare][H][kJoinQuads][4];
    let_dependents_start();
    wait_for_prerequisites();
    const int sub = threadIdx.x / kJoinQuads, lane = threadIdx.x % kJoinQuads, per_row = (N + 3) / 4;
    const long long i = (long long)blockIdx.x * kJoinQuads + lane, part = M * N;
    const bool there = i < M * per_row;
    long long row = 0;
    int c4 = 0;
    if (there) split_item(i, per_row, row, c4);
    const int col = 4 * c4;
#pragma unroll
    for (int h = 0; h < H; ++h) {
        Sum v[4] = {0, 0, 0, 0};
        if (there)
#pragma unroll 4
            for (int s = sub; s < splits; s += kJoinShare) part4<WHOLE>(parts + ((long long)s * H + h) * part + row * N + col, col, N, v);
#pragma unroll
        for (int c = 0; c < 4; ++c) sums[sub][h][lane][c] = v[c];
    }
    __syncthreads();
    // a thread to a column
    if (sub >= 4 || !there || col + sub >= N) return;
    float v[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        Sum sum = 0;
#pragma unroll
        for (int s = 0; s < kJoinShare; ++s) sum += sums[s][h][lane][sub];
        v[h] = (float)sum;
    }
    const int n = col + sub;
    const long long g_at = row * 2 * N + n, u_at = g_at + N;
    with_act(e.activation, [&](auto tag) {
        constexpr int ACT = decltype(tag)::value;
        if constexpr (BWD) {
            const uint16_t* z = (const uint16_t*)e.z_in;
            const float g = elem2_to_float2(z[g_at]).x, u = elem2_to_float2(z[u_at]).x;
            Pair a2, s2;
            act_and_slope2<ACT>(both(g), a2, s2);
            float a, slope, ignore;
            split_pair(a2, a, ignore);
            split_pair(s2, slope, ignore);
            ((uint16_t*)e.y)[g_at] = (uint16_t)pack_elem(v[0] * u * slope, 0.f);
            ((uint16_t*)e.y)[u_at] = (uint16_t)pack_elem(v[0] * a, 0.f);
        } else {
            float z[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int f = n + h * N;
                const float b = e.bias ? e.bias[f] : 0.f;
                float ignore;
                if (e.x_scale) split_pair(scaled2(both(v[h]), both(e.x_scale[row]), both(e.w_scale[f]), both(b)), z[h], ignore);
                else z[h] = v[h] + b;
            }
            if (e.z) {
                ((uint16_t*)e.z)[g_at] = (uint16_t)pack_elem(z[0], 0.f);
                ((uint16_t*)e.z)[u_at] = (uint16_t)pack_elem(z[1], 0.f);
            }
            ((uint16_t*)e.y)[row * N + n] = (uint16_t)pack_elem(act<ACT>(z[0]) * z[1], 0.f);
        }
    });
}

template <int KIND, int OPS, bool MAP, int TILES>
cudaError_t launch_tiles(bool pair, const Maps& maps, Job& job, int sm_count, cudaStream_t stream) {
    if constexpr (OPS != kOpsI8)
        if (job.kb_per_split > kLinearLongChunk)
            return pair ? launch_one<true, KIND, OPS, MAP, TILES, true>(maps, job, sm_count, stream) : launch_one<false, KIND, OPS, MAP, TILES, true>(maps, job, sm_count, stream);
    return pair ? launch_one<true, KIND, OPS, MAP, TILES, false>(maps, job, sm_count, stream) : launch_one<false, KIND, OPS, MAP, TILES, false>(maps, job, sm_count, stream);
}

template <bool BWD>
cudaError_t join(cudaError_t e, int ops, const LinearPlan& p, const LinearEpilogue& epi, const float* parts, long long M, int N, cudaStream_t stream) {
    if (e != cudaSuccess || p.splits == 1) return e;
    prof_begin("gated_join_kernel", stream);
    e = launch_dependent(!BWD && ops == kOpsI8 ? gated_join_kernel<BWD, !BWD> : gated_join_kernel<BWD, false>, (unsigned)((M * ((N + 3) / 4) + kJoinQuads - 1) / kJoinQuads), (unsigned)(kJoinShare * kJoinQuads), 0, stream, epi, parts, p.splits,
                         M, N);
    count_launch(stream);
    return e;
}

// one half of rows of 2 N elements, for boxes of 32 columns x 32 rows
bool encode_half(CUtensorMap* map, const void* rows, int half, long long M, int N) {
    return encode_map(map, (const uint16_t*)rows + (size_t)half * N, N, M, 4ll * N, 2, 32, 64);
}

}  // namespace

cudaError_t read_gated_status(int* timed_out) {
    int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(timed_out, g_linear_timeout, sizeof(int));
    if (e != cudaSuccess) return e;
    if (*timed_out) e = cudaMemcpyToSymbol(g_linear_timeout, &zero, sizeof(int));
    return e;
}

// y [M][N] of operands x [M][K] and w [2 N][K], whose rows' strides are given in bytes (multiples of 16)
cudaError_t launch_gated(int ops, const LinearPlan& p, long long M, int N, long long K, const void* x, long long stride_x, const void* w, long long stride_w,
                         const LinearEpilogue& epi, float* parts, int sm_count, cudaStream_t stream) {
    const int ctas = p.pair ? 2 : 1, wide = p.bn / 2, elem = ops == kOps16 ? 2 : 1;
    const bool by_map = p.splits == 1 && N % 8 == 0;
    Maps maps;
    if (!encode_map(&maps.a, x, K, M, stride_x, elem, 128) || !encode_map(&maps.b, w, K, 2ll * N, stride_w, elem, wide)) return cudaErrorInvalidValue;
    maps.in = maps.in_up = maps.y = maps.z = maps.z_up = maps.a;
    if (by_map && (!encode_map(&maps.y, epi.y, N, M, 2ll * N, 2, 32, 64) || (epi.z && (!encode_half(&maps.z, epi.z, 0, M, N) || !encode_half(&maps.z_up, epi.z, 1, M, N)))))
        return cudaErrorInvalidValue;
    Job job{};
    if (!set_job(job, p, wide, M, N, epi, parts)) return cudaErrorInvalidConfiguration;
    job.boxes_b = 1;
    job.bytes_b = p.bn / ctas * 128;
    job.idesc = ops == kOpsI8 ? make_idesc_i8(128 * ctas, p.bn) : make_idesc_elem(128 * ctas, p.bn, 0, 0);
    // (a part of a split sum goes neither way)
    const bool map = by_map || p.splits > 1;
    cudaError_t e;
    if (ops == kOpsI8) e = map ? launch_tiles<kLinearGated, kOpsI8, true, 1>(p.pair, maps, job, sm_count, stream) : launch_tiles<kLinearGated, kOpsI8, false, 3>(p.pair, maps, job, sm_count, stream);
    else if (!map) e = launch_tiles<kLinearGated, kOps16, false, 3>(p.pair, maps, job, sm_count, stream);
    else if (epi.z && p.splits == 1) e = launch_tiles<kLinearGated, kOps16, true, 3>(p.pair, maps, job, sm_count, stream);
    else e = launch_tiles<kLinearGated, kOps16, true, 1>(p.pair, maps, job, sm_count, stream);
    return join<false>(e, ops, p, epi, parts, M, N, stream);
}

// [d u act'(g), d act(g)] with d = d_z w, of z_in = [g, u]; d_z [M][K], w [K][N], z_in and the result [M][2 N]
cudaError_t launch_gated_input(const LinearPlan& p, long long M, int N, long long K, const void* d_z, long long stride_z, const void* w, long long stride_w,
                               const LinearEpilogue& epi, float* parts, int sm_count, cudaStream_t stream) {
    const int ctas = p.pair ? 2 : 1, cols = p.bn / ctas;
    const bool by_map = p.splits == 1 && N % 8 == 0;
    Maps maps;
    if (!encode_map(&maps.a, d_z, K, M, stride_z, 2, 128) || !encode_map(&maps.b, w, N, K, stride_w, 2, 64)) return cudaErrorInvalidValue;
    maps.in = maps.in_up = maps.y = maps.z = maps.z_up = maps.a;
    if (by_map && (!encode_half(&maps.in, epi.z_in, 0, M, N) || !encode_half(&maps.in_up, epi.z_in, 1, M, N) || !encode_half(&maps.y, epi.y, 0, M, N) ||
                   !encode_half(&maps.z_up, epi.y, 1, M, N)))
        return cudaErrorInvalidValue;
    Job job{};
    if (!set_job(job, p, p.bn, M, N, epi, parts)) return cudaErrorInvalidConfiguration;
    job.boxes_b = (cols + 63) / 64;
    job.bytes_b = job.boxes_b * (kOperand / 2);
    job.idesc = make_idesc_elem(128 * ctas, p.bn, 0, 1);
    const cudaError_t e = by_map || p.splits > 1 ? launch_tiles<kLinearGatedInput, kOps16, true, 1>(p.pair, maps, job, sm_count, stream)
                                                 : launch_tiles<kLinearGatedInput, kOps16, false, 1>(p.pair, maps, job, sm_count, stream);
    return join<true>(e, kOps16, p, epi, parts, M, N, stream);
}

}  // namespace terra
