// Host-side launch interface between block_api.cu and the kernels of what stands around the attention in a Transformer block.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "swin_kernels.h"

namespace terra {

// n / d for 0 <= n < 2^31, d >= 1, by a multiplication: with 2^(l - 1) < d <= 2^l, m = floor(2^(31 + l) / d) + 1 is less than 2^32 and
// exceeds 2^(31 + l) / d by at most 1, so n m / 2^(31 + l) exceeds n / d by less than 2^-l <= 1 / d.
struct Divider {
    uint32_t d, m, shift;
    __host__ explicit Divider(uint32_t by) : d(by), m(0), shift(0) {
        uint32_t l = 0;
        while ((1ull << l) < by) ++l;
        if (by > 1) {
            m = (uint32_t)((1ull << (31 + l)) / by + 1);
            shift = l - 1;
        }
    }
    __device__ __forceinline__ void split(uint32_t n, uint32_t& quo, uint32_t& rem) const {
        quo = d > 1 ? __umulhi(n, m) >> shift : n;
        rem = n - quo * d;
    }
};

// What a product multiplies and a norm gives: the activations' type, e4m3, 8-bit integers.
constexpr int kOps16 = 0, kOpsE4m3 = 1, kOpsI8 = 2;

// ---- root-mean-square norm (norm.cu) ----------------------------------------------------------------------------
constexpr int kNormMaxChannels = 16384;
struct NormArgs {
    const void *x, *r;                 // backward: h, d_h
    const float* weight;
    const void* d_y;                   // backward only
    const float* rstd_in;
    void *h, *y;                       // forward; y: the type's or 8 bits, as `out` says.  Backward: y is dx
    float *rstd, *scale, *dweight;     // scale: of y in 8 bits
    float* partial;                    // backward: [blocks][channels]
    long long rows;
    int channels;
    int out;                           // forward: kOps* of y; in 8-bit integers without a weight: no norm, y = x
    float eps;
};
int norm_bwd_blocks(long long rows, int channels);      // rows of `partial` at most, whatever the device
cudaError_t launch_rms_norm_fwd(const NormArgs& a, int sm_count, cudaStream_t stream);
cudaError_t launch_rms_norm_fwd_f16(const NormArgs& a, int sm_count, cudaStream_t stream);
cudaError_t launch_rms_norm_bwd(const NormArgs& a, int sm_count, cudaStream_t stream);
cudaError_t launch_rms_norm_bwd_f16(const NormArgs& a, int sm_count, cudaStream_t stream);

// ---- group norm (group_norm.cu) ---------------------------------------------------------------------------------
struct GroupNormArgs {
    const void *x, *d_y;               // d_y: backward
    const float *weight, *bias;
    void* out;                         // y, or d_x
    float *stats, *d_weight, *d_bias;  // [samples][groups] mean and rstd
    void* workspace;
    long long tokens;
    int samples, channels, groups, activation;
    float eps;
};
struct GroupNormPlan {
    int elems, across, rows;           // channels of a thread; threads along the channels; tokens at a time
    int slab, slabs, pieces;           // channels of a block; blocks along the channels; of them to a group (1: whole groups)
    int chunks;                        // blocks along a sample's tokens
    int cluster, held;                 // blocks that hold a sample's slab in one launch (0: several launches), and vectors of a thread in shared memory (0: in registers)
    size_t smem;                       // shared memory of such a block
    bool backward;
    long long chunk;                   // tokens of a block
    size_t off_sums, bytes;            // workspace
};
GroupNormPlan plan_group_norm(int samples, long long tokens, int channels, int groups, bool backward);
cudaError_t launch_group_norm_fwd(const GroupNormArgs& a, const GroupNormPlan& plan, cudaStream_t stream);
cudaError_t launch_group_norm_fwd_f16(const GroupNormArgs& a, const GroupNormPlan& plan, cudaStream_t stream);
cudaError_t launch_group_norm_bwd(const GroupNormArgs& a, const GroupNormPlan& plan, cudaStream_t stream);
cudaError_t launch_group_norm_bwd_f16(const GroupNormArgs& a, const GroupNormPlan& plan, cudaStream_t stream);
cudaError_t read_group_norm_status(int* timed_out);       // after the stream has been synchronised
cudaError_t read_group_norm_status_f16(int* timed_out);

// ---- rotary positions (rotary.cu) -------------------------------------------------------------------------------
struct RotaryArgs {
    const void *q, *k;                 // k NULL: q alone
    void *q_out, *k_out;
    const double* freq;                // [rot / 2] radians a position
    const int* positions;              // [tokens][2] row and column, or NULL: the grid's in the shifted frame
    long long tokens;
    long long stride, stride_out;      // elements between tokens
    int H, W, sh, sw;
    int heads, d, rot, row_pairs;
    float scale;
    bool inverse, interleaved;
};
cudaError_t launch_rotary(const RotaryArgs& a, int sm_count, cudaStream_t stream);
cudaError_t launch_rotary_f16(const RotaryArgs& a, int sm_count, cudaStream_t stream);

// ---- products (linear.cu) ---------------------------------------------------------------------------------------
constexpr int kLinearForward = 0, kLinearInput = 1, kLinearWeights = 2, kLinearGated = 3, kLinearGatedInput = 4;
constexpr int kLinearMaxFeatures = 65536;
constexpr int kLinearChunk = 4;        // weight gradient: stages (of 64 rows) that are summed up in TMEM
constexpr int kLinearLongChunk = 32;   // the other products: stages (of 64 features, in e4m3 128) that are

// How a product is cut up.  Made for kPlanSms SMs whatever the device has, so that the workspace does not depend on it.
struct LinearPlan {
    bool pair;                         // tiles of 256 rows by two CTAs, else of 128 by one
    int bn;                            // columns of a tile
    int m_tiles, n_tiles, group;       // `group` rows of tiles are worked on together
    int splits, k_blocks, kb_per_split;
};
LinearPlan plan_linear(int kind, bool bytes, long long M, int N, long long K, size_t room = ~(size_t)0);      // room: bytes for the parts of a split sum, at most

// What stands for 64 columns' bias where there is none: read as 16-byte vectors.
struct alignas(16) NoBias { float values[64]; };

struct LinearEpilogue {
    const float *bias, *x_scale, *w_scale;
    const void *residual, *z_in;
    void *y, *z;
    float* a_sums;                     // weight gradient: the sums of A(m, .) over k, that is d_z over the rows; may be NULL
    float* sums;                       // set by launch_linear
    int activation;
};
// `parts`: splits x M x N floats where the plan splits the sum, `a_parts` splits x n_tiles x M where a_sums is asked for too; `out`: the weight gradient
cudaError_t launch_linear(int kind, int ops, const LinearPlan& p, long long M, int N, long long K, const void* a, long long stride_a, const void* b, long long stride_b,
                          const LinearEpilogue& epi, float* out, float* parts, float* a_parts, int sm_count, cudaStream_t stream);
cudaError_t launch_linear_f16(int kind, int ops, const LinearPlan& p, long long M, int N, long long K, const void* a, long long stride_a, const void* b, long long stride_b,
                              const LinearEpilogue& epi, float* out, float* parts, float* a_parts, int sm_count, cudaStream_t stream);
// the forward product for up to kFewRows rows (linear_few.cu): rows of any length, no workspace; gated: n_out gated outputs, w [2 n_out][n_in], z [rows][2 n_out]
constexpr int kFewRows = 8;
cudaError_t launch_linear_few(int ops, bool gated, int rows, int n_in, int n_out, const void* x, const void* w, const LinearEpilogue& epi, cudaStream_t stream);
cudaError_t launch_linear_few_f16(int ops, bool gated, int rows, int n_in, int n_out, const void* x, const void* w, const LinearEpilogue& epi, cudaStream_t stream);
cudaError_t read_linear_status(int* timed_out);       // after the stream has been synchronised
cudaError_t read_linear_status_f16(int* timed_out);

// ---- products around a gate (linear_gated.cu) -------------------------------------------------------------------
// `parts`: splits x M x N floats where the plan splits the sum, forward twice as many
cudaError_t launch_gated(int ops, const LinearPlan& p, long long M, int N, long long K, const void* x, long long stride_x, const void* w, long long stride_w,
                         const LinearEpilogue& epi, float* parts, int sm_count, cudaStream_t stream);
cudaError_t launch_gated_f16(int ops, const LinearPlan& p, long long M, int N, long long K, const void* x, long long stride_x, const void* w, long long stride_w,
                             const LinearEpilogue& epi, float* parts, int sm_count, cudaStream_t stream);
cudaError_t launch_gated_input(const LinearPlan& p, long long M, int N, long long K, const void* d_z, long long stride_z, const void* w, long long stride_w,
                               const LinearEpilogue& epi, float* parts, int sm_count, cudaStream_t stream);
cudaError_t launch_gated_input_f16(const LinearPlan& p, long long M, int N, long long K, const void* d_z, long long stride_z, const void* w, long long stride_w,
                                   const LinearEpilogue& epi, float* parts, int sm_count, cudaStream_t stream);
cudaError_t read_gated_status(int* timed_out);        // after the stream has been synchronised
cudaError_t read_gated_status_f16(int* timed_out);

// ---- around the products (linear_aux.cu) ------------------------------------------------------------------------
// rows of `bytes` into rows of `stride` bytes (a multiple of 16), zeros behind them; up to three tensors at once
struct PadJob { const void* src; void* dst; long long rows; int bytes, stride; };
struct PadJobs { PadJob job[3]; int count; };
cudaError_t launch_pad_rows(const PadJobs& jobs, int sm_count, cudaStream_t stream);
// out[c] = sum over the rows of x[., c]; rows of `stride` elements; `partial`: column_sum_blocks rows of `columns`
int column_sum_blocks(long long rows, int columns);
cudaError_t launch_column_sums(const void* x, long long rows, int columns, long long stride, float* partial, float* out, cudaStream_t stream);
cudaError_t launch_column_sums_f16(const void* x, long long rows, int columns, long long stride, float* partial, float* out, cudaStream_t stream);
// out[c] = sum over b of partial[b][c], in a fixed order
cudaError_t launch_sum_partials(const float* partial, int blocks, int columns, float* out, cudaStream_t stream);
// d_z = d_y act'(z), elementwise
cudaError_t launch_activation_bwd(const void* z, const void* d_y, void* d_z, long long n, int activation, int sm_count, cudaStream_t stream);
cudaError_t launch_activation_bwd_f16(const void* z, const void* d_y, void* d_z, long long n, int activation, int sm_count, cudaStream_t stream);

// the same through a gate: z = [g, u] and d_z of `rows` rows of 2 n, d_y of n: d_z = [d_y u act'(g), d_y act(g)]
cudaError_t launch_gated_activation_bwd(const void* z, const void* d_y, void* d_z, long long rows, int n, int activation, int sm_count, cudaStream_t stream);
cudaError_t launch_gated_activation_bwd_f16(const void* z, const void* d_y, void* d_z, long long rows, int n, int activation, int sm_count, cudaStream_t stream);

}  // namespace terra
