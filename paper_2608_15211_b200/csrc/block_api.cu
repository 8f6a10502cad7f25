// C ABI of what stands around the attention in a Transformer block: argument checks, plans, workspaces, launches.
#include <cmath>

#include "../../include/terra.h"
#include "block_kernels.h"

namespace terra {

int resolve_attention_geo(const terra_swin_desc* d, Geo* out);
int current_device_sm_count(int* sm_count);
int report_cuda_failure(cudaError_t e, const char* where);

namespace {

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
bool misaligned(std::initializer_list<const void*> ps) {
    uintptr_t any = 0;
    for (const void* p : ps) any |= reinterpret_cast<uintptr_t>(p);
    return (any & 15u) != 0;
}
bool known_dtype(int dtype) { return dtype == TERRA_DTYPE_BF16 || dtype == TERRA_DTYPE_F16; }
bool known_act(int a) { return a >= TERRA_ACT_NONE && a <= TERRA_ACT_GELU_TANH; }
int done(cudaError_t e, const char* where) { return e == cudaSuccess ? TERRA_OK : report_cuda_failure(e, where); }

int check_norm(const terra_norm_desc* d) {
    if (!d || d->rows < 1 || d->rows > (1ll << 40) || d->channels < 1 || !(d->eps >= 0.f) || std::isinf(d->eps) || !known_dtype(d->dtype)) return TERRA_ERR_INVALID_ARG;
    return d->channels > kNormMaxChannels ? TERRA_ERR_UNSUPPORTED : TERRA_OK;
}

int norm_fwd(const terra_norm_desc* d, const void* x, const void* residual, const float* weight, void* h, void* y, float* scale, float* rstd, bool e4m3, void* stream,
             const char* where) {
    int rc = check_norm(d);
    if (rc) return rc;
    if (!x || !weight || !y || (e4m3 && (!scale || y == x || y == residual)) || y == h) return TERRA_ERR_INVALID_ARG;
    if (misaligned({x, residual, weight, h, y, scale, rstd})) return TERRA_ERR_ALIGNMENT;
    int sms = 0;
    rc = current_device_sm_count(&sms);
    if (rc) return rc;
    NormArgs a = {};
    a.x = x; a.r = residual; a.weight = weight; a.h = h; a.y = y; a.rstd = rstd; a.scale = e4m3 ? scale : nullptr;
    a.rows = d->rows; a.channels = d->channels; a.eps = d->eps;
    return done(d->dtype == TERRA_DTYPE_F16 ? launch_rms_norm_fwd_f16(a, sms, (cudaStream_t)stream) : launch_rms_norm_fwd(a, sms, (cudaStream_t)stream), where);
}

// ---- products ---------------------------------------------------------------------------------------------------

int check_linear(const terra_linear_desc* d) {
    if (!d || d->rows < 1 || d->rows > 0x7fffffffll - 1023 || d->n_in < 1 || d->n_out < 1 || !known_act(d->activation) || !known_dtype(d->dtype)) return TERRA_ERR_INVALID_ARG;
    return d->n_in > kLinearMaxFeatures || d->n_out > kLinearMaxFeatures ? TERRA_ERR_UNSUPPORTED : TERRA_OK;
}

// What a call keeps in its workspace, from its start on.  (Offsets are multiples of 256 bytes.)
struct LinearSpace {
    size_t bytes = 0;
    size_t add(size_t n) {
        const size_t at = bytes;
        bytes += align_up(n, 256);
        return at;
    }
};
long long padded(long long bytes) { return (bytes + 15) / 16 * 16; }

struct LinearLayout {
    long long stride_x, stride_w, stride_z;      // bytes of a row as the products read it
    bool pad_x, pad_w, pad_z;
    size_t off_x, off_w, off_z, off_parts, off_sums;
    LinearPlan first, second;                    // forward or input gradient; weight gradient
    size_t bytes;
};

// (the kernel for few rows / the tiles of 128 rows, us, weights not in L2: 8 x 8192 -> 8192 26.5 / 33.1, 8 x 4096 -> 8192 15.9 / 19.0, 8 x 1024 -> 1024 4.3 / 7.6)
bool few_rows(const terra_linear_desc* d) { return d->rows <= kFewRows; }

LinearLayout layout_linear(const terra_linear_desc* d, int call) {
    LinearLayout l = {};
    LinearSpace s;
    const bool e4m3 = call == TERRA_LINEAR_FWD_E4M3, bwd = call == TERRA_LINEAR_BWD;
    if (!bwd && few_rows(d)) return l;
    const long long elem = e4m3 ? 1 : 2;
    l.stride_x = l.stride_w = padded(d->n_in * elem);
    l.stride_z = padded(d->n_out * elem);
    l.pad_x = l.pad_w = l.stride_x != d->n_in * elem;
    l.pad_z = bwd && l.stride_z != d->n_out * elem;
    if (l.pad_x) l.off_x = s.add((size_t)d->rows * l.stride_x);
    if (l.pad_w) l.off_w = s.add((size_t)d->n_out * l.stride_w);
    if (l.pad_z) l.off_z = s.add((size_t)d->rows * l.stride_z);
    size_t parts = 0;
    auto need = [&](const LinearPlan& p, size_t cells) {
        if (p.splits > 1 && p.splits * cells * sizeof(float) > parts) parts = p.splits * cells * sizeof(float);
    };
    if (bwd) {
        l.first = plan_linear(kLinearInput, false, d->rows, d->n_in, d->n_out);
        l.second = plan_linear(kLinearWeights, false, d->n_out, d->n_in, d->rows);
        need(l.first, (size_t)d->rows * d->n_in);
        need(l.second, (size_t)d->n_out * d->n_in);
        const size_t slices = column_sum_blocks(d->rows, d->n_out), splits = l.second.splits * l.second.n_tiles;        // without or with the weight gradient
        l.off_sums = s.add(sizeof(float) * (slices > splits ? slices : splits) * d->n_out);
    } else {
        l.first = plan_linear(kLinearForward, e4m3, d->rows, d->n_out, d->n_in);
        need(l.first, (size_t)d->rows * d->n_out);
    }
    l.off_parts = parts ? s.add(parts) : 0;
    l.bytes = s.bytes;
    return l;
}

// `p` is to be read with rows of `stride` bytes: where they are not, from a copy at `to`
void pad(PadJobs& jobs, const void*& p, bool wanted, char* to, long long rows, long long bytes, long long stride) {
    if (!wanted) return;
    jobs.job[jobs.count++] = {p, to, rows, (int)bytes, (int)stride};
    p = to;
}

int linear_fwd(const terra_linear_desc* d, bool e4m3, const void* x, const float* x_scale, const void* w, const float* w_scale, const float* bias, const void* residual,
               void* y, void* z, void* workspace, size_t workspace_bytes, void* stream, const char* where) {
    int rc = check_linear(d);
    if (rc) return rc;
    if (!x || !w || !y || (e4m3 && (!x_scale || !w_scale))) return TERRA_ERR_INVALID_ARG;
    if (y == z || y == x || y == w || (z && (z == x || z == w || z == residual))) return TERRA_ERR_INVALID_ARG;        // other threads still read those
    if (misaligned({x, w, x_scale, w_scale, bias, residual, y, z})) return TERRA_ERR_ALIGNMENT;
    const LinearLayout l = layout_linear(d, e4m3 ? TERRA_LINEAR_FWD_E4M3 : TERRA_LINEAR_FWD);
    if (l.bytes && (!workspace || workspace_bytes < l.bytes)) return TERRA_ERR_WORKSPACE;
    if (l.bytes && misaligned({workspace})) return TERRA_ERR_ALIGNMENT;
    int sms = 0;
    rc = current_device_sm_count(&sms);
    if (rc) return rc;
    char* ws = (char*)workspace;
    cudaStream_t st = (cudaStream_t)stream;
    const long long elem = e4m3 ? 1 : 2;
    LinearEpilogue epi = {};
    epi.bias = bias; epi.residual = residual; epi.y = y; epi.z = z; epi.activation = d->activation;
    epi.x_scale = e4m3 ? x_scale : nullptr;
    epi.w_scale = e4m3 ? w_scale : nullptr;
    if (few_rows(d)) {
        auto few = d->dtype == TERRA_DTYPE_F16 ? launch_linear_few_f16 : launch_linear_few;
        return done(few(e4m3, (int)d->rows, d->n_in, d->n_out, x, w, epi, st), where);
    }
    PadJobs jobs = {};
    pad(jobs, x, l.pad_x, ws + l.off_x, d->rows, d->n_in * elem, l.stride_x);
    pad(jobs, w, l.pad_w, ws + l.off_w, d->n_out, d->n_in * elem, l.stride_w);
    const cudaError_t e = jobs.count ? launch_pad_rows(jobs, sms, st) : cudaSuccess;
    if (e != cudaSuccess) return done(e, where);
    auto launch = d->dtype == TERRA_DTYPE_F16 ? launch_linear_f16 : launch_linear;
    return done(launch(kLinearForward, e4m3, l.first, d->rows, d->n_out, d->n_in, x, l.stride_x, w, l.stride_w, epi, nullptr, (float*)(ws + l.off_parts), nullptr, sms, st), where);
}

// ---- rotary positions -------------------------------------------------------------------------------------------

int rotary(const terra_swin_desc* desc, const terra_rotary_desc* r, const double* inv_freq, const int32_t* positions, const void* q, const void* k, void* q_out,
           void* k_out, bool packed, void* stream, const char* where) {
    Geo g;
    int rc = resolve_attention_geo(desc, &g);
    if (rc) return rc;
    if (!r || r->rot_dim < 2 || (r->rot_dim & 1) || r->rot_dim > g.d || (r->layout != TERRA_ROTARY_HALF && r->layout != TERRA_ROTARY_INTERLEAVED) ||
        r->row_pairs < 0 || r->row_pairs > r->rot_dim / 2 || !std::isfinite(r->scale))
        return TERRA_ERR_INVALID_ARG;
    if (!inv_freq || !q || !q_out || (!k != !k_out)) return TERRA_ERR_INVALID_ARG;
    if (misaligned({inv_freq, positions, q, k, q_out, k_out})) return TERRA_ERR_ALIGNMENT;
    if (k && (q_out == k || k_out == q || q_out == k_out)) return TERRA_ERR_INVALID_ARG;
    int sms = 0;
    rc = current_device_sm_count(&sms);
    if (rc) return rc;
    RotaryArgs a = {};
    a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out; a.freq = inv_freq; a.positions = positions;
    a.tokens = (long long)g.B * g.H * g.W;
    a.stride = a.stride_out = (long long)g.heads * g.d * (packed ? 3 : 1);
    a.H = g.H; a.W = g.W; a.sh = g.sh; a.sw = g.sw;
    a.heads = g.heads; a.d = g.d; a.rot = r->rot_dim; a.row_pairs = r->row_pairs;
    a.scale = r->scale;
    a.inverse = r->inverse != 0;
    a.interleaved = r->layout == TERRA_ROTARY_INTERLEAVED;
    return done(g.f16 ? launch_rotary_f16(a, sms, (cudaStream_t)stream) : launch_rotary(a, sms, (cudaStream_t)stream), where);
}

}  // namespace

// The tile, and into how many parts the sum is split, by an estimate of the time in SM cycles.
static LinearPlan make_plan(int kind, bool e4m3, long long M, int N, long long K) {
    const long long blocks = (K + (e4m3 ? 127 : 63)) / (e4m3 ? 128 : 64);
    LinearPlan best = {};
    double best_cost = 1e300;
    for (int pair = 0; pair < 2; ++pair) {
        const int ctas = pair ? 2 : 1, slots = kPlanSms / ctas;
        if (pair && M <= 128) continue;
        const long long m_tiles = (M + 128 * ctas - 1) / (128 * ctas);
        for (int bn = 32; bn <= 128 * ctas; bn += 32) {
            const int n_tiles = (N + bn - 1) / bn;
            if (bn % 64 && n_tiles > 1) continue;      // the epilogue's 64 columns would reach into the next tile
            if (bn > 32 && n_tiles == (n_tiles > 1 ? (N + bn - 65) / (bn - 64 > 0 ? bn - 64 : 1) : (N + bn - 33) / (bn - 32))) continue;        // a narrower tile does with as many
            const double operand = 128. * 128 + 128. * bn / ctas;
            const double step = 2. * bn > operand / 48 ? 2. * bn : operand / 48;
            for (int want = 1; want <= 64; ++want) {
                const long long per = (blocks + want - 1) / want;
                const int splits = (int)((blocks + per - 1) / per);
                if (splits != want) continue;
                if (kind != kLinearWeights && splits > 1 && m_tiles * n_tiles * (splits - 1) >= slots) break;
                const double units = (double)m_tiles * n_tiles * splits, waves = std::ceil(units / slots);
                const double write = splits > 1 || kind == kLinearWeights ? 2. : 1., epilogue = 400. + 900. * write * ((bn + 127) / 128);
                const double main = per * step + 200.;
                double cost = waves * (main > epilogue ? main : epilogue) + epilogue + 2500.;
                if (splits > 1) cost += 5000. + 8. * splits * (double)M * N / (20. * kPlanSms);
                if (cost < best_cost * 0.999) {
                    best_cost = cost;
                    best.pair = pair;
                    best.bn = bn;
                    best.m_tiles = (int)m_tiles;
                    best.n_tiles = n_tiles;
                    best.splits = splits;
                    best.k_blocks = (int)blocks;
                    best.kb_per_split = (int)per;
                }
            }
        }
    }
    // Rows of tiles that are worked on together: 8 (e4m3 156672 x 4096 -> 16384 over seconds, us: 8 8900, 4 9110; 4096 -> 4096 3892 / 3860), or down to 4
    // where that leaves no empty units in the last group: they would make a second round of one (550800 rows, weight gradient 384 x 1536: 572 -> 1009).
    best.group = best.m_tiles < 8 ? best.m_tiles : 0;
    for (int g = 8; !best.group && g >= 4; --g)
        if (best.m_tiles % g == 0) best.group = g;
    if (!best.group) best.group = (long long)best.m_tiles * best.n_tiles * best.splits > 16 * kPlanSms ? 8 : 1;
    return best;
}

// Each thread remembers the plans of its last few sizes: the search takes longer than a launch, and a call asks for its plans twice.
LinearPlan plan_linear(int kind, bool e4m3, long long M, int N, long long K) {
    struct Known { long long M = 0, K; int kind, N; bool e4m3; LinearPlan plan; };
    constexpr int kKnown = 32;
    static thread_local Known known[kKnown];
    static thread_local int next = 0;
    for (const Known& k : known)
        if (k.M == M && k.K == K && k.N == N && k.kind == kind && k.e4m3 == e4m3) return k.plan;
    Known& k = known[next];
    next = (next + 1) % kKnown;
    k.plan = make_plan(kind, e4m3, M, N, K);
    k.M = M; k.K = K; k.N = N; k.kind = kind; k.e4m3 = e4m3;
    return k.plan;
}

}  // namespace terra

using namespace terra;

extern "C" {

int terra_rms_norm_fwd(const terra_norm_desc* desc, const void* x, const void* residual, const float* weight, void* h, void* y, float* rstd, void* stream) {
    return norm_fwd(desc, x, residual, weight, h, y, nullptr, rstd, false, stream, "terra_rms_norm_fwd");
}

int terra_rms_norm_fwd_e4m3(const terra_norm_desc* desc, const void* x, const void* residual, const float* weight, void* h, void* y8, float* scale, float* rstd,
                            void* stream) {
    return norm_fwd(desc, x, residual, weight, h, y8, scale, rstd, true, stream, "terra_rms_norm_fwd_e4m3");
}

int terra_rms_norm_workspace_bytes(const terra_norm_desc* desc, size_t* bytes) {
    const int rc = check_norm(desc);
    if (rc) return rc;
    if (!bytes) return TERRA_ERR_INVALID_ARG;
    *bytes = align_up(sizeof(float) * (size_t)norm_bwd_blocks(desc->rows, desc->channels) * desc->channels, 256);
    return TERRA_OK;
}

int terra_rms_norm_bwd(const terra_norm_desc* desc, const void* h, const float* weight, const float* rstd, const void* d_y, const void* d_h, void* d_x, float* d_weight,
                       void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    int rc = terra_rms_norm_workspace_bytes(desc, &need);
    if (rc) return rc;
    if (!h || !weight || !rstd || !d_y || !d_x || !d_weight) return TERRA_ERR_INVALID_ARG;
    if (misaligned({h, weight, rstd, d_y, d_h, d_x, d_weight})) return TERRA_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < need) return TERRA_ERR_WORKSPACE;
    if (misaligned({workspace})) return TERRA_ERR_ALIGNMENT;
    int sms = 0;
    rc = current_device_sm_count(&sms);
    if (rc) return rc;
    NormArgs a = {};
    a.x = h; a.r = d_h; a.weight = weight; a.d_y = d_y; a.rstd_in = rstd; a.y = d_x; a.dweight = d_weight; a.partial = (float*)workspace;
    a.rows = desc->rows; a.channels = desc->channels;
    return done(desc->dtype == TERRA_DTYPE_F16 ? launch_rms_norm_bwd_f16(a, sms, (cudaStream_t)stream) : launch_rms_norm_bwd(a, sms, (cudaStream_t)stream),
                "terra_rms_norm_bwd");
}

int terra_linear_workspace_bytes(const terra_linear_desc* desc, int call, size_t* bytes) {
    const int rc = check_linear(desc);
    if (rc) return rc;
    if (!bytes || call < TERRA_LINEAR_FWD || call > TERRA_LINEAR_BWD) return TERRA_ERR_INVALID_ARG;
    *bytes = layout_linear(desc, call).bytes;
    return TERRA_OK;
}

int terra_linear_fwd(const terra_linear_desc* desc, const void* x, const void* w, const float* bias, const void* residual, void* y, void* z, void* workspace,
                     size_t workspace_bytes, void* stream) {
    return linear_fwd(desc, false, x, nullptr, w, nullptr, bias, residual, y, z, workspace, workspace_bytes, stream, "terra_linear_fwd");
}

int terra_linear_fwd_e4m3(const terra_linear_desc* desc, const void* x8, const float* x_scale, const void* w8, const float* w_scale, const float* bias,
                          const void* residual, void* y, void* workspace, size_t workspace_bytes, void* stream) {
    return linear_fwd(desc, true, x8, x_scale, w8, w_scale, bias, residual, y, nullptr, workspace, workspace_bytes, stream, "terra_linear_fwd_e4m3");
}

int terra_linear_bwd(const terra_linear_desc* desc, const void* x, const void* w, const void* d_z, const void* z_in, void* d_x, float* d_w, float* d_bias,
                     void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_linear(desc);
    if (rc) return rc;
    if (!d_z || (d_x && !w) || (d_w && !x) || (!d_x && !d_w && !d_bias)) return TERRA_ERR_INVALID_ARG;
    if (d_x && (d_x == d_z || d_x == w)) return TERRA_ERR_INVALID_ARG;
    if (misaligned({x, w, d_z, z_in, d_x, d_w, d_bias})) return TERRA_ERR_ALIGNMENT;
    const LinearLayout l = layout_linear(desc, TERRA_LINEAR_BWD);
    if (!workspace || workspace_bytes < l.bytes) return TERRA_ERR_WORKSPACE;
    if (misaligned({workspace})) return TERRA_ERR_ALIGNMENT;
    int sms = 0;
    rc = current_device_sm_count(&sms);
    if (rc) return rc;
    const char* where = "terra_linear_bwd";
    char* ws = (char*)workspace;
    float *parts = (float*)(ws + l.off_parts), *sums = (float*)(ws + l.off_sums);
    cudaStream_t st = (cudaStream_t)stream;
    const bool f16 = desc->dtype == TERRA_DTYPE_F16;
    auto launch = f16 ? launch_linear_f16 : launch_linear;
    PadJobs jobs = {};
    pad(jobs, d_z, l.pad_z, ws + l.off_z, desc->rows, 2ll * desc->n_out, l.stride_z);
    if (d_w) pad(jobs, x, l.pad_x, ws + l.off_x, desc->rows, 2ll * desc->n_in, l.stride_x);
    if (d_x) pad(jobs, w, l.pad_w, ws + l.off_w, desc->n_out, 2ll * desc->n_in, l.stride_w);
    cudaError_t e = jobs.count ? launch_pad_rows(jobs, sms, st) : cudaSuccess;
    if (e == cudaSuccess && d_w) {
        LinearEpilogue epi = {};
        epi.a_sums = d_bias;
        e = launch(kLinearWeights, false, l.second, desc->n_out, desc->n_in, desc->rows, d_z, l.stride_z, x, l.stride_x, epi, d_w, parts, sums, sms, st);
    } else if (e == cudaSuccess && d_bias) {
        e = f16 ? launch_column_sums_f16(d_z, desc->rows, desc->n_out, l.stride_z / 2, sums, d_bias, st)
                : launch_column_sums(d_z, desc->rows, desc->n_out, l.stride_z / 2, sums, d_bias, st);
    }
    if (e == cudaSuccess && d_x) {
        LinearEpilogue epi = {};
        epi.z_in = z_in; epi.y = d_x; epi.activation = z_in ? desc->activation : TERRA_ACT_NONE;
        e = launch(kLinearInput, false, l.first, desc->rows, desc->n_in, desc->n_out, d_z, l.stride_z, w, l.stride_w, epi, nullptr, parts, nullptr, sms, st);
    }
    return done(e, where);
}

int terra_activation_bwd(int64_t n, int32_t activation, int32_t dtype, const void* z, const void* d_y, void* d_z, void* stream) {
    if (n < 1 || n > (1ll << 46) || !known_act(activation) || !known_dtype(dtype) || !z || !d_y || !d_z) return TERRA_ERR_INVALID_ARG;
    if (misaligned({z, d_y, d_z})) return TERRA_ERR_ALIGNMENT;
    int sms = 0;
    const int rc = current_device_sm_count(&sms);
    if (rc) return rc;
    return done(dtype == TERRA_DTYPE_F16 ? launch_activation_bwd_f16(z, d_y, d_z, n, activation, sms, (cudaStream_t)stream)
                                         : launch_activation_bwd(z, d_y, d_z, n, activation, sms, (cudaStream_t)stream), "terra_activation_bwd");
}

int terra_rotary(const terra_swin_desc* desc, const terra_rotary_desc* r, const double* inv_freq, const int32_t* positions, const void* q, const void* k, void* q_out,
                 void* k_out, void* stream) {
    return rotary(desc, r, inv_freq, positions, q, k, q_out, k_out, false, stream, "terra_rotary");
}

int terra_rotary_packed(const terra_swin_desc* desc, const terra_rotary_desc* r, const double* inv_freq, const int32_t* positions, void* qkv, void* stream) {
    if (!desc || desc->heads <= 0 || desc->head_dim <= 0 || !qkv) return TERRA_ERR_INVALID_ARG;
    uint16_t *q = (uint16_t*)qkv, *k = q + (size_t)desc->heads * desc->head_dim;
    return rotary(desc, r, inv_freq, positions, q, k, q, k, true, stream, "terra_rotary_packed");
}

}  // extern "C"
