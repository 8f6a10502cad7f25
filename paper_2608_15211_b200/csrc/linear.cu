// Products of a Transformer block on the tcgen05 tensor cores, D[M, N] = sum over k of A(m, k) B(n, k), with what follows them in the epilogue:
//   forward          A = x [rows, n_in], B = w [n_out, n_in]: z = D (scales) + bias, y = act(z) + residual; 16-bit or e4m3 operands
//   input gradient   A = d_z [rows, n_out], B = w read along n_in: d_x = D act'(z_in)
//   weight gradient  A = d_z and B = x, both read along their features, summed over the rows: d_w = D in fp32
// An operand whose memory runs along k is "K-major", one that runs along m or n "MN-major"; TMA brings either in 128-byte-swizzled rows,
// and the shared-memory descriptors say which it is, so nothing is transposed.
//
// Persistent: a unit is one output tile (of one part of the sum, where it is split).  PAIR: two CTAs on neighbouring SMs work on a
// tile of 256 rows with tcgen05.mma.cta_group::2, each with its 128 rows of A and half of the columns of B; alone, a CTA has 128 rows.  Five
// stages of 64 k (128 in e4m3) each, two accumulators in TMEM, so that the epilogue of a tile runs under the products of the next.
// The epilogue turns a warp's 32 rows x 64 columns over in shared memory, so that all it reads and writes in global memory is runs of whole rows.
//
// The tensor cores' sum over k is not rounded to nearest, and its error grows with the number of steps.  The weight gradient, a sum over all
// rows that comes out in fp32, therefore leaves TMEM every kChunk stages and is added up in registers.
//
// Roles (384 threads): warp 0 copies, warp 1 issues the products, warp 2 has the TMEM, warps 4-11 the epilogue.
// Every mbarrier wait is bounded; on expiry the CTA raises an abort flag, all roles leave their loops, TMEM is released and the host reads
// the device status word.
#include <cuda.h>
#include <cstring>

#include "block_act.cuh"
#include "block_kernels.h"
#include "tc_common.cuh"

#ifdef TERRA_ELEM_F16
#define g_linear_timeout g_linear_timeout_f16
#define launch_linear launch_linear_f16
#define read_linear_status read_linear_status_f16
#endif

namespace terra {

__device__ int g_linear_timeout = 0;   // set when a bounded wait expired in any CTA of the kernel below

namespace {

using namespace tc;

constexpr int kThreads = 384;
constexpr int kEpiWarp0 = 4, kEpiWarps = 8;
constexpr int kStages = 5;
constexpr int kOperand = 128 * 128;                    // bytes of an operand's stage: 128 rows (or columns) x 128 bytes
constexpr int kTurn = 32 * 64 * 4;                     // a warp's 32 x 64 fp32
constexpr int kOffTurn = kStages * 2 * kOperand;
constexpr int kOffBars = kOffTurn + kEpiWarps * kTurn;
constexpr int kBFull = 0, kBEmpty = kStages, kBAccFull = 2 * kStages, kBAccEmpty = kBAccFull + 2, kBCount = kBAccEmpty + 2;
constexpr int kOffTmem = kOffBars + 8 * kBCount, kOffAbort = kOffTmem + 4;
constexpr int kSmem = kOffAbort + 4 + 1024;            // the base is rounded up to 1 KB
constexpr int kAccCols = 256;                          // TMEM columns between the two accumulators

// ---- two CTAs on one tile --------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cta_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t leaders(uint32_t addr) {       // the same place in the first CTA's shared memory
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;\n" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
template <bool PAIR>
__device__ __forceinline__ void load_box(uint32_t dst, const void* map, int x, int y, uint32_t bar) {
    if (PAIR)      // `bar` may lie in the other CTA of the pair
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        tma_load_2d(dst, map, x, y, bar);
}
template <bool PAIR, bool E4M3>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if (PAIR && E4M3)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else if (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else if (E4M3)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        mma_ss(d, a, b, idesc, accumulate);
}
// arrives on `bar`, at its place in both CTAs of a pair, once all products issued so far are complete
template <bool PAIR>
__device__ __forceinline__ void commit(uint32_t bar) {
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        mma_commit(bar);
}
template <bool PAIR>
__device__ __forceinline__ void arrive_leader(uint32_t bar) {
    if (PAIR)
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(leaders(bar)) : "memory");
    else
        mbar_arrive(bar);
}

struct Maps { CUtensorMap a, b; };

struct Job {
    long long M;
    int N;
    int bn;                                    // columns of a tile: a multiple of 32
    int m_tiles, n_tiles, group;               // tiles are walked through in groups of `group` rows of tiles
    int splits, k_blocks, kb_per_split;
    int bytes_b;                               // of a CTA's share of B in a stage
    int boxes_b;                               // MN-major: boxes of 64 columns
    uint32_t idesc;
    LinearEpilogue e;
};

struct Unit { long long m0; int n0, k0, k1, split; };

__device__ __forceinline__ Unit unit_at(const Job& j, long long u, int tile_rows) {
    const int per_split = j.m_tiles * j.n_tiles;
    long long split, rest;
    int tile;
    split_item(u, per_split, split, tile);
    const int per_group = j.group * j.n_tiles, g = tile / per_group, first = g * j.group, rows = min(j.group, j.m_tiles - first);
    rest = tile - g * per_group;
    const int n = (int)rest / rows, m = first + (int)rest - n * rows;
    Unit r;
    r.m0 = (long long)m * tile_rows;
    r.n0 = n * j.bn;
    r.split = (int)split;
    r.k0 = r.split * j.kb_per_split;
    r.k1 = min(j.k_blocks, r.k0 + j.kb_per_split);
    return r;
}

__device__ __forceinline__ float4 elems4(uint2 v) {
    const float2 a = elem2_to_float2(v.x), b = elem2_to_float2(v.y);
    return make_float4(a.x, a.y, b.x, b.y);
}

// What is made of four neighbouring columns of D.  `r`, `z`: the residual's or the activation input's four elements.
template <int KIND, int ACT>
__device__ __forceinline__ void finish4(float (&v)[4], const float4& bias, const float4& ws, float xs, const float4& in, bool scaled, float (&z)[4]) {
    const float b[4] = {bias.x, bias.y, bias.z, bias.w}, w[4] = {ws.x, ws.y, ws.z, ws.w}, t[4] = {in.x, in.y, in.z, in.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (KIND == kLinearForward) {
            z[i] = scaled ? fmaf(v[i] * xs, w[i], b[i]) : v[i] + b[i];
            v[i] = act<ACT>(z[i]) + t[i];
        } else {
            v[i] *= act_slope<ACT>(t[i]);
        }
    }
}

// One warp's rows x 64 columns, out of its turned-over tile (`v4(i)`: columns 4 j .. 4 j + 3 of row 2 i + lane / 16, j = lane % 16) to global memory.
// `row0`: the row of i = 0, lane 0; `col0`: the column of j = 0; columns from `cols` on belong to others.
template <int KIND, int ACT, class V>
__device__ __forceinline__ void write_rows(const LinearEpilogue& e, long long M, int N, long long row0, int col0, int cols, int lane, V v4) {
    const int j = lane & 15, col = col0 + 4 * j;
    const long long row_a = row0 + (lane >> 4);
    const bool in_col = 4 * j < cols && col < N;
    const uint16_t* extra = (const uint16_t*)(KIND == kLinearForward ? e.residual : e.z_in);
    float4 bias = make_float4(0.f, 0.f, 0.f, 0.f), ws = bias;
    if ((N & 3) == 0) {
        if (in_col && KIND == kLinearForward && e.bias) bias = *reinterpret_cast<const float4*>(e.bias + col);
        if (in_col && KIND == kLinearForward && e.w_scale) ws = *reinterpret_cast<const float4*>(e.w_scale + col);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint2 in[8];
            float xs[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const long long row = row_a + 2 * (8 * half + i);
                in[i] = make_uint2(0, 0);
                xs[i] = 1.f;
                if (in_col && row < M) {
                    if (extra) in[i] = *reinterpret_cast<const uint2*>(extra + row * N + col);
                    if (KIND == kLinearForward && e.x_scale) xs[i] = e.x_scale[row];
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const long long row = row_a + 2 * (8 * half + i);
                float v[4], z[4];
                v4(8 * half + i, v);
                if (!in_col || row >= M) continue;
                finish4<KIND, ACT>(v, bias, ws, xs[i], elems4(in[i]), e.w_scale != nullptr, z);
                if (KIND == kLinearForward && e.z)
                    *reinterpret_cast<uint2*>((uint16_t*)e.z + row * N + col) = make_uint2(pack_elem(z[0], z[1]), pack_elem(z[2], z[3]));
                *reinterpret_cast<uint2*>((uint16_t*)e.y + row * N + col) = make_uint2(pack_elem(v[0], v[1]), pack_elem(v[2], v[3]));
            }
        }
        return;
    }
    // rows that are not multiples of 8 bytes
    float b[4] = {0.f, 0.f, 0.f, 0.f}, w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (in_col && col + c < N && KIND == kLinearForward) {
            if (e.bias) b[c] = e.bias[col + c];
            if (e.w_scale) w[c] = e.w_scale[col + c];
        }
    bias = make_float4(b[0], b[1], b[2], b[3]);
    ws = make_float4(w[0], w[1], w[2], w[3]);
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
        const long long row = row_a + 2 * i;
        float v[4], z[4], t[4] = {0.f, 0.f, 0.f, 0.f};
        v4(i, v);
        if (!in_col || row >= M) continue;
        if (extra)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (col + c < N) t[c] = elem2_to_float2(extra[row * N + col + c]).x;
        finish4<KIND, ACT>(v, bias, ws, KIND == kLinearForward && e.x_scale ? e.x_scale[row] : 1.f, make_float4(t[0], t[1], t[2], t[3]), e.w_scale != nullptr, z);
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (col + c < N) {
                if (KIND == kLinearForward && e.z) ((uint16_t*)e.z)[row * N + col + c] = (uint16_t)pack_elem(z[c], 0.f);
                ((uint16_t*)e.y)[row * N + col + c] = (uint16_t)pack_elem(v[c], 0.f);
            }
    }
}

// The same for sums that stay in fp32: parts of a split product, and the weight gradient
template <class V>
__device__ __forceinline__ void write_sums(float* out, long long M, int N, long long row0, int col0, int cols, int lane, V v4) {
    const int j = lane & 15, col = col0 + 4 * j;
    const long long row_a = row0 + (lane >> 4);
    const bool in_col = 4 * j < cols && col < N;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const long long row = row_a + 2 * i;
        float v[4];
        v4(i, v);
        if (!in_col || row >= M) continue;
        float* p = out + row * N + col;
        if ((N & 3) == 0) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (col + c < N) p[c] = v[c];
        }
    }
}

template <bool PAIR, int KIND, bool E4M3>
__global__ void __launch_bounds__(kThreads, 1) linear_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Job job) {
    constexpr int CTAS = PAIR ? 2 : 1;
    constexpr int kTileRows = 128 * CTAS;
    constexpr bool A_MN = KIND == kLinearWeights, B_MN = KIND != kLinearForward;
    constexpr int kBK = E4M3 ? 128 : 64;               // elements of a stage along k
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - smem_u32(smem_raw));
    volatile int* cta_abort = reinterpret_cast<volatile int*>(smem + kOffAbort);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = PAIR ? cta_rank() : 0;
    auto bar = [&](int i) { return base + kOffBars + 8 * i; };
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(bar(kBFull + s), 1);
            mbar_init(bar(kBEmpty + s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(bar(kBAccFull + b), 1);
            mbar_init(bar(kBAccEmpty + b), kEpiWarps * CTAS);
        }
        *cta_abort = 0;
        fence_barrier_init();
    }
    if (warp == 2) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(base + kOffTmem), "r"(2 * kAccCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
        } else {
            tmem_alloc(base + kOffTmem, 2 * kAccCols);
            tmem_relinquish();
        }
    }
    let_dependents_start();
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem + kOffTmem);
    wait_for_prerequisites();

    const long long units = (long long)job.m_tiles * job.n_tiles * job.splits;
    const long long first = blockIdx.x / CTAS, step = gridDim.x / CTAS;
    if (warp == 0) {
        if (lane == 0) {
            const int cols = job.bn / CTAS;            // this CTA's share of B
            const uint32_t bytes = CTAS * (kOperand + job.bytes_b);
            uint32_t it = 0;
            bool ok = true;
            for (long long u = first; u < units && ok; u += step) {
                const Unit x = unit_at(job, u, kTileRows);
                const int m = (int)x.m0 + 128 * (int)rank, n = x.n0 + cols * (int)rank;
                for (int kb = x.k0; kb < x.k1 && ok; ++kb, ++it) {
                    const uint32_t s = it % kStages, use = it / kStages;
                    ok = mbar_wait<0>(bar(kBEmpty + s), (use & 1) ^ 1u, cta_abort);
                    if (!ok) break;
                    const uint32_t full = PAIR ? leaders(bar(kBFull + s)) : bar(kBFull + s), a = base + s * 2 * kOperand, b = a + kOperand;
                    if (rank == 0) mbar_arrive_expect_tx(bar(kBFull + s), bytes);
                    if (A_MN) {
                        load_box<PAIR>(a, &maps.a, m, kb * kBK, full);
                        load_box<PAIR>(a + kOperand / 2, &maps.a, m + 64, kb * kBK, full);
                    } else {
                        load_box<PAIR>(a, &maps.a, kb * kBK, m, full);
                    }
                    if (B_MN) {
                        for (int i = 0; i < job.boxes_b; ++i) load_box<PAIR>(b + i * (kOperand / 2), &maps.b, n + 64 * i, kb * kBK, full);
                    } else {
                        load_box<PAIR>(b, &maps.b, kb * kBK, n, full);
                    }
                }
            }
            // after an expired wait: the copies in flight are waited for, so that none lands in memory that is no longer this CTA's
            if (!ok && rank == 0) {
                volatile int ignore = 0;
                for (uint32_t i = it > kStages ? it - kStages : 0; i < it; ++i)
                    mbar_wait<0>(bar(kBFull + i % kStages), (i / kStages) & 1, &ignore, 200000000LL);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            uint32_t it = 0, done = 0;
            bool ok = true;
            for (long long u = first; u < units && ok; u += step) {
                const Unit x = unit_at(job, u, kTileRows);
                for (int kb = x.k0; kb < x.k1 && ok;) {
                    const int end = KIND == kLinearWeights ? min(x.k1, kb + kLinearChunk) : x.k1;
                    const uint32_t buf = done & 1, acc = tmem + buf * kAccCols;
                    ok = mbar_wait<0>(bar(kBAccEmpty + buf), ((done >> 1) & 1) ^ 1u, cta_abort);
                    if (!ok) break;
                    tc_fence_after();
                    uint32_t accumulate = 0;
                    for (; kb < end; ++kb, ++it) {
                        const uint32_t s = it % kStages;
                        ok = mbar_wait<0>(bar(kBFull + s), (it / kStages) & 1, cta_abort);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t a = base + s * 2 * kOperand, b = a + kOperand;
                        // 32 bytes along k a step, 16 rows of 128 bytes where k is the slow axis
                        const uint64_t da = make_sdesc_sw128(a, A_MN ? kOperand / 2 : 16), db = make_sdesc_sw128(b, B_MN ? kOperand / 2 : 16);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            mma<PAIR, E4M3>(acc, da + k * (A_MN ? 2048 / 16 : 2), db + k * (B_MN ? 2048 / 16 : 2), job.idesc, accumulate);
                            accumulate = 1;
                        }
                        commit<PAIR>(bar(kBEmpty + s));
                    }
                    if (!ok) break;
                    commit<PAIR>(bar(kBAccFull + buf));
                    ++done;
                }
            }
        }
        __syncwarp();
    } else if (warp >= kEpiWarp0) {
        const int quarter = warp & 3, half = (warp - kEpiWarp0) >> 2;
        uint8_t* turn = smem + kOffTurn + (warp - kEpiWarp0) * kTurn;
        const uint32_t turn_a = smem_u32(turn);
        const uint32_t lane_tmem = tmem + ((uint32_t)(quarter * 32) << 16);
        // this thread's row, 16 columns from 16 part on; the 16-byte places of a row are exchanged by the row's number against bank conflicts
        auto put16 = [&](int part, const float* v) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t at = turn_a + lane * 256 + (((4 * part + c) ^ (lane & 7)) << 4);
                asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};\n" ::"r"(at), "f"(v[4 * c]), "f"(v[4 * c + 1]), "f"(v[4 * c + 2]), "f"(v[4 * c + 3]) : "memory");
            }
        };
        auto get4 = [&](int i, float (&v)[4]) {
            const int r = 2 * i + (lane >> 4);
            const uint32_t at = turn_a + r * 256 + (((lane & 15) ^ (r & 7)) << 4);
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];\n" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(at) : "memory");
        };
        uint32_t done = 0;
        bool ok = true;
        for (long long u = first; u < units && ok; u += step) {
            const Unit x = unit_at(job, u, kTileRows);
            const long long row0 = x.m0 + 128 * rank + 32 * quarter;
            float* sums = job.e.sums ? job.e.sums + (size_t)x.split * job.M * job.N : nullptr;
            if constexpr (KIND == kLinearWeights) {
                float acc[2][64];
#pragma unroll
                for (int i = 0; i < 64; ++i) acc[0][i] = acc[1][i] = 0.f;
                for (int kb = x.k0; kb < x.k1 && ok; kb += kLinearChunk, ++done) {
                    const uint32_t buf = done & 1;
                    ok = mbar_wait_all(bar(kBAccFull + buf), (done >> 1) & 1, cta_abort);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int p = 0; p < 4; ++p) {
                            const int col = 64 * (2 * c + half) + 16 * p;
                            if (col < job.bn) {
                                uint32_t t[16];
                                tmem_ld16(lane_tmem + buf * kAccCols + col, t);
                                tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 16; ++i) acc[c][16 * p + i] += __uint_as_float(t[i]);
                            }
                        }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_leader<PAIR>(bar(kBAccEmpty + buf));
                }
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int col0 = 64 * (2 * c + half);
                    if (col0 < job.bn) {
#pragma unroll
                        for (int p = 0; p < 4; ++p) put16(p, &acc[c][16 * p]);
                        __syncwarp();
                        write_sums(sums, job.M, job.N, row0, x.n0 + col0, min(64, job.bn - col0), lane, get4);
                        __syncwarp();
                    }
                }
            } else {
                const uint32_t buf = done & 1;
                ok = mbar_wait_all(bar(kBAccFull + buf), (done >> 1) & 1, cta_abort);
                if (!ok) break;
                tc_fence_after();
                ++done;
                for (int col0 = 64 * half; col0 < job.bn; col0 += 128) {
                    const int cols = min(64, job.bn - col0);
                    uint32_t t[32];
                    tmem_ld32(lane_tmem + buf * kAccCols + col0, t);
                    tmem_ld_wait();
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        float f[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(t[16 * p + i]);
                        put16(p, f);
                    }
                    if (cols > 32) {
                        tmem_ld32(lane_tmem + buf * kAccCols + col0 + 32, t);
                        tmem_ld_wait();
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            float f[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(t[16 * p + i]);
                            put16(2 + p, f);
                        }
                    }
                    if (col0 + 128 >= job.bn) {        // the accumulator has been read
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) arrive_leader<PAIR>(bar(kBAccEmpty + buf));
                    }
                    __syncwarp();
                    if (sums) {
                        write_sums(sums, job.M, job.N, row0, x.n0 + col0, cols, lane, get4);
                    } else {
                        with_act(job.e.activation, [&](auto tag) {
                            write_rows<KIND, decltype(tag)::value>(job.e, job.M, job.N, row0, x.n0 + col0, cols, lane, get4);
                        });
                    }
                    __syncwarp();
                }
                if (64 * half >= job.bn && lane == 0) arrive_leader<PAIR>(bar(kBAccEmpty + buf));      // a narrow tile has no columns for this warp
            }
        }
    }

    // teardown: every role ends up here, also after an expired wait
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();           // the other CTA's arrivals and copies on this one's barriers are done
    tc_fence_after();
    if (warp == 2) {
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(2 * kAccCols) : "memory");
        else tmem_dealloc(tmem, 2 * kAccCols);
    }
    if (tid == 0 && *cta_abort) atomicExch(&g_linear_timeout, 1);
}

// Joins the parts of a split product: the sum over the splits, then the epilogue.
template <int KIND>
__global__ void __launch_bounds__(256) linear_join_kernel(const LinearEpilogue e, const float* __restrict__ parts, int splits, long long M, int N, float* out) {
    let_dependents_start();
    wait_for_prerequisites();
    const int per_row = (N + 3) / 4;
    const long long total = M * per_row;
    const bool wide = (N & 3) == 0;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        long long row;
        int c4;
        split_item(i, per_row, row, c4);
        const int col = 4 * c4;
        const size_t at = (size_t)row * N + col, part = (size_t)M * N;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (wide) {
#pragma unroll 8
            for (int s = 0; s < splits; ++s) {
                const float4 t = *reinterpret_cast<const float4*>(parts + s * part + at);
                v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
            }
        } else {
            for (int s = 0; s < splits; ++s)
                for (int c = 0; c < 4; ++c)
                    if (col + c < N) v[c] += parts[s * part + at + c];
        }
        if (KIND == kLinearWeights) {
            if (wide) *reinterpret_cast<float4*>(out + at) = make_float4(v[0], v[1], v[2], v[3]);
            else
                for (int c = 0; c < 4; ++c)
                    if (col + c < N) out[at + c] = v[c];
            continue;
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
        with_act(e.activation, [&](auto tag) {
            finish4<KIND, decltype(tag)::value>(v, make_float4(b[0], b[1], b[2], b[3]), make_float4(w[0], w[1], w[2], w[3]),
                                                KIND == kLinearForward && e.x_scale ? e.x_scale[row] : 1.f, make_float4(t[0], t[1], t[2], t[3]), e.w_scale != nullptr, z);
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
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_tiled_fn() {
    static EncodeTiledFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiledFn>(p);
    }();
    return fn;
}

// [slow][fast] with rows of `stride` bytes, boxes of 128 bytes x box_rows; beyond the tensor zeros are read
bool encode_map(CUtensorMap* map, const void* base, long long fast, long long slow, long long stride, int elem_bytes, int box_rows) {
    EncodeTiledFn enc = encode_tiled_fn();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)fast, (cuuint64_t)slow};
    const cuuint64_t strides[1] = {(cuuint64_t)stride};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / elem_bytes), (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1u, 1u};
    return enc(map, elem_bytes == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool PAIR, int KIND, bool E4M3>
cudaError_t launch_one(const Maps& maps, const Job& job, int sm_count, cudaStream_t stream) {
    auto kern = linear_kernel<PAIR, KIND, E4M3>;
    cudaError_t e = prepare_kernel((const void*)kern, kSmem);
    if (e != cudaSuccess) return e;
    const long long units = (long long)job.m_tiles * job.n_tiles * job.splits, fit = sm_count / (PAIR ? 2 : 1);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = PAIR ? 2 : 1;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(units < fit ? units : fit) * (PAIR ? 2 : 1));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = PAIR ? 2 : 1;
    prof_begin("linear_kernel", stream);
    e = cudaLaunchKernelEx(&cfg, kern, maps, job);
    count_launch(stream);
    return e;
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
cudaError_t launch_linear(int kind, bool e4m3, const LinearPlan& p, long long M, int N, long long K, const void* a, long long stride_a, const void* b, long long stride_b,
                          const LinearEpilogue& epi, float* out, float* parts, int sm_count, cudaStream_t stream) {
    const int ctas = p.pair ? 2 : 1, cols = p.bn / ctas, elem = e4m3 ? 1 : 2;
    const bool a_mn = kind == kLinearWeights, b_mn = kind != kLinearForward;
    Maps maps;
    if (!encode_map(&maps.a, a, a_mn ? M : K, a_mn ? K : M, stride_a, elem, a_mn ? 64 : 128) ||
        !encode_map(&maps.b, b, b_mn ? N : K, b_mn ? K : N, stride_b, elem, b_mn ? 64 : cols))
        return cudaErrorInvalidValue;
    Job job;
    job.M = M;
    job.N = N;
    job.bn = p.bn;
    job.m_tiles = p.m_tiles;
    job.n_tiles = p.n_tiles;
    job.group = p.group;
    job.splits = p.splits;
    job.k_blocks = p.k_blocks;
    job.kb_per_split = p.kb_per_split;
    job.boxes_b = (cols + 63) / 64;
    job.bytes_b = b_mn ? job.boxes_b * (kOperand / 2) : cols * 128;
    job.idesc = e4m3 ? make_idesc_f16(128 * ctas, p.bn, 0, 0)            // e4m3 has format number 0, as fp16 has in its kind
                     : make_idesc_elem(128 * ctas, p.bn, a_mn ? 1 : 0, b_mn ? 1 : 0);
    job.e = epi;
    job.e.sums = p.splits > 1 ? parts : kind == kLinearWeights ? out : nullptr;
    cudaError_t e;
    if (kind == kLinearForward && e4m3) e = p.pair ? launch_one<true, kLinearForward, true>(maps, job, sm_count, stream) : launch_one<false, kLinearForward, true>(maps, job, sm_count, stream);
    else if (kind == kLinearForward) e = p.pair ? launch_one<true, kLinearForward, false>(maps, job, sm_count, stream) : launch_one<false, kLinearForward, false>(maps, job, sm_count, stream);
    else if (kind == kLinearInput) e = p.pair ? launch_one<true, kLinearInput, false>(maps, job, sm_count, stream) : launch_one<false, kLinearInput, false>(maps, job, sm_count, stream);
    else e = p.pair ? launch_one<true, kLinearWeights, false>(maps, job, sm_count, stream) : launch_one<false, kLinearWeights, false>(maps, job, sm_count, stream);
    if (e != cudaSuccess || p.splits == 1) return e;
    const long long quads = M * ((N + 3) / 4), need = (quads + 255) / 256, fit = 8ll * sm_count;
    const unsigned grid = (unsigned)(need < fit ? need : fit);
    prof_begin("linear_join_kernel", stream);
    auto join = kind == kLinearForward ? linear_join_kernel<kLinearForward> : kind == kLinearInput ? linear_join_kernel<kLinearInput> : linear_join_kernel<kLinearWeights>;
    e = launch_dependent(join, grid, 256u, 0, stream, epi, (const float*)parts, p.splits, M, N, out);
    count_launch(stream);
    return e;
}

}  // namespace terra
