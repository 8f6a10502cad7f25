// Products of a Transformer block on the tcgen05 tensor cores, D[M, N] = sum over k of A(m, k) B(n, k), with what follows them in the epilogue:
//   forward          A = x [rows, n_in], B = w [n_out, n_in]: z = D (scales) + bias, y = act(z) + residual; operands of 16 bits, e4m3 or 8-bit integers
//   gated forward    B = the gate's rows of w and as many up rows: [g, u] = D (scales) + bias, y = act(g) u; operands of 16 bits or 8-bit integers
//   input gradient   A = d_z [rows, n_out], B = w read along n_in: d_x = D act'(z_in), or through a gate z_in = [g, u]: [D u act'(g), D act(g)]
//   weight gradient  A = d_z and B = x, both read along their features, summed over the rows: d_w = D in fp32
// An operand whose memory runs along k is "K-major", one that runs along m or n "MN-major"; TMA brings either in 128-byte-swizzled rows,
// and the shared-memory descriptors say which it is, so nothing is transposed.
//
// Persistent: a unit is one output tile (of one part of the sum, where it is split).  PAIR: two CTAs on neighbouring SMs work on a
// tile of 256 rows with tcgen05.mma.cta_group::2, each with its 128 rows of A and half of the columns of B; alone, a CTA has 128 rows.  Five
// (or four, or three) stages of 64 k (128 of 8 bits) each, two accumulators in TMEM, so that the epilogue of a tile runs under the products of the next.
// The epilogue works on a warp's 32 rows x 64 columns at a time, a row to a thread, two columns to an instruction; the residual comes and the
// results go as tiles in shared memory that the copy engine moves (rows that are no multiples of 16 bytes: the warp itself, in whole rows).
//
// Sums of 8-bit integers are exact.  The tensor cores' sum in fp32 over k is cut off, not rounded to nearest, and its error grows with the number of steps, four a stage: 1.9e-8 of the 2-norm a step
// on N(0, 1), 1.05e-7 where all terms have one sign.  The weight gradient, a sum over all rows that comes out in fp32, therefore leaves TMEM every kLinearChunk
// stages and is added up in registers (156672 rows of N(0, 1) in fp16: 3.6e-7 off in the 2-norm, with 16 stages 1.2e-6, at the same time).  The other products,
// whose results are rounded to 16 bits, leave it every kLinearLongChunk stages: terms of one sign are then 1.3e-5 off at most, a fortieth of fp16's half
// step.  (4096 features in one go 2.6e-5, 65536 4.3e-4.  156672 x 4096 -> 4096 takes 3399 us instead of 3367 so, with a residual 3538 instead of 3505.)
//
// What bounds it, a call on a cool GPU: the tensor pipe where the sum is long (156672 x 4096 -> 4096 3.40 ms, 1546 TFLOP/s, the pipe busy in 89 % of the cycles; e4m3 to 16384 with
// GELU 7.2 ms, 2920 TFLOP/s), over seconds the power cap (4.1 and 9.0 ms); the epilogue where it is short (550800 x 384 -> 1536 with GELU 0.85 ms, two
// reciprocals or exponentials an output in a unit that takes 16 a clock and SM, busy in half the cycles), with z besides the writes: 3.4 GB, of which HBM
// takes 3.9 GB a ms (0.98 ms).  Rows that are no multiples of 16 bytes: the warps' copies (2203200 x 256 -> 372 0.64 ms, -> 384 0.56).
//
// Roles (640 threads): warp 0 copies, warp 1 issues the products, warp 2 has the TMEM, warps 4-19 the epilogue; weight gradient: warps 2 and 3 the
// sums of d_z.
// Every mbarrier wait is bounded; on expiry the CTA raises an abort flag, all roles leave their loops, TMEM is released and the host reads
// the device status word.
#pragma once
#include <cuda.h>
#include <cstring>

#include "block_act.cuh"
#include "block_kernels.h"
#include "tc_common.cuh"

namespace terra {

static __device__ int g_linear_timeout = 0;   // set when a bounded wait expired in any CTA of the kernel below

namespace {

using namespace tc;

constexpr int kGroups = 4;                             // groups of four epilogue warps, one for each 32 lanes of TMEM
constexpr int kEpiWarp0 = 4, kEpiWarps = 4 * kGroups;
constexpr int kThreads = 32 * (kEpiWarp0 + kEpiWarps);
constexpr int kRegsLaunch = 96, kRegsEpi = 104, kRegsOther = 64;      // of a thread at launch, in the epilogue and elsewhere
static_assert(kEpiWarps * kRegsEpi + kEpiWarp0 * kRegsOther <= (kEpiWarps + kEpiWarp0) * kRegsLaunch, "register hand-over does not balance");
constexpr int kOperand = 128 * 128;                    // bytes of an operand's stage: 128 rows (or columns) x 128 bytes
constexpr int kTile = 32 * 128;                        // a warp's 32 rows x 64 columns of 16-bit elements, or 32 columns of 32-bit ones
// Shared memory: five stages and a tile for each epilogue warp, or, for short sums whose epilogue is the longer part, three stages and two tiles
// or four stages and one and a half: for the three results of a gated product that keeps its z, and for a product of 8-bit integers with the bias and scales of
// a chunk's columns behind its tile
template <int TILES> struct Stages { static constexpr int value = TILES == 2 ? 3 : TILES == 3 ? 4 : 5, tile = TILES == 2 ? 2 * kTile : TILES == 3 ? 3 * kTile / 2 : kTile; };
constexpr int kMostStages = 5;
constexpr int kOffBars = kMostStages * 2 * kOperand + kEpiWarps * kTile;
static_assert(Stages<2>::value * 2 * kOperand + kEpiWarps * Stages<2>::tile <= kOffBars && Stages<3>::value * 2 * kOperand + kEpiWarps * Stages<3>::tile <= kOffBars,
              "the layouts share their end");
constexpr int kBFull = 0, kBEmpty = kMostStages, kBAccFull = 2 * kMostStages, kBAccEmpty = kBAccFull + 2, kBIn = kBAccEmpty + 2,
              kBUsed = kBIn + 2 * kEpiWarps, kBCount = kBUsed + kMostStages;
constexpr int kOffTmem = kOffBars + 8 * kBCount, kOffAbort = kOffTmem + 4;
constexpr int kSmem = kOffAbort + 4 + 1024;            // the base is rounded up to 1 KB
constexpr int kTwoTilesBlocks = 8;
constexpr int kI8TableBlocks = 16;     // the longest sums of 8-bit integers (in stages of 128) whose epilogue counts: 156672 x 4096 -> 4096, 32 of them, 1640 us with and without the table
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
// D[tmem] (+)= A B; descriptors as their low words (start address and leading dimension) and the high words that all of a kind share
#define TERRA_MMA(GROUP, KIND)                                                                                                       \
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\tsetp.ne.b32 p, %5, 0;\n\t" \
                 "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], da, db, %4, p;\n\t}\n" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate) : "memory")
template <bool PAIR, int OPS>
__device__ __forceinline__ void mma(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
    if (PAIR && OPS == kOpsI8) TERRA_MMA("2", "i8");
    else if (PAIR && OPS == kOpsE4m3) TERRA_MMA("2", "f8f6f4");
    else if (PAIR) TERRA_MMA("2", "f16");
    else if (OPS == kOpsI8) TERRA_MMA("1", "i8");
    else if (OPS == kOpsE4m3) TERRA_MMA("1", "f8f6f4");
    else TERRA_MMA("1", "f16");
}
#undef TERRA_MMA
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
        // (relaxed: what the arrival is about, reads of TMEM, has been waited for; a release would wait for all of the warp's stores, 2000 cycles)
        asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(leaders(bar)) : "memory");
    else
        mbar_arrive(bar);
}

// For roles that wait most of the time: they sleep between polls, which take issue slots from the epilogue's warps.
__device__ __forceinline__ bool wait_asleep(uint32_t bar, uint32_t parity, volatile int* cta_abort) {
    return __all_sync(0xffffffffu, mbar_wait<64>(bar, parity, cta_abort));
}

struct Maps { CUtensorMap a, b, in, in_up, y, z, z_up; };      // in: the residual or z_in; in_up, z_up: the second halves of gated rows
__device__ __forceinline__ void store_box(const void* map, int x, int y, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];\n" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;\n" ::"n"(N) : "memory"); }   // all but the last N

struct Digits { int m, n, g, split; };      // of a unit's number, see Units

struct Job {
    long long M;
    int N;
    int bn;                                    // columns of a tile: a multiple of 32
    int wide;                                  // columns of the output that it is for: bn, or half of it where gate and up columns make one output
    int m_tiles, n_tiles, group, groups;       // tiles are walked through in groups of `group` rows of tiles
    Divider by_group{1}, by_n_tiles{1}, by_groups{1};
    Digits step;                               // of the number of tiles that are worked on at a time
    int splits, k_blocks, kb_per_split;
    int bytes_b;                               // of a CTA's share of B in a stage
    int boxes_b;                               // MN-major: boxes of 64 columns
    uint32_t idesc;
    LinearEpilogue e;
};

// A unit as digits: the row of tiles within its group (fastest), the column of tiles, the group, the part of the sum.  Going `step` units on adds the
// step's digits with carries.  (Divisions, in every role for every tile, cost each tile 700 cycles, 64-bit ones 1500.)  The last group
// may have fewer rows than the others: its units beyond are there and empty.
__device__ __forceinline__ Digits digits_of(const Job& j, uint32_t u) {
    uint32_t m, n, g, split;
    j.by_group.split(u, u, m);
    j.by_n_tiles.split(u, u, n);
    j.by_groups.split(u, split, g);
    return {(int)m, (int)n, (int)g, (int)split};
}
struct Units {
    const Job& j;
    Digits at, step;
    __device__ __forceinline__ Units(const Job& job, uint32_t first) : j(job), at(digits_of(job, first)), step(job.step) {}
    __device__ __forceinline__ bool there() const { return at.split < j.splits; }
    __device__ __forceinline__ bool empty() const { return at.g * j.group + at.m >= j.m_tiles; }
    __device__ __forceinline__ void advance() {
        at.m += step.m;
        int carry = at.m >= j.group;
        at.m -= carry ? j.group : 0;
        at.n += step.n + carry;
        carry = at.n >= j.n_tiles;
        at.n -= carry ? j.n_tiles : 0;
        at.g += step.g + carry;
        carry = at.g >= j.groups;
        at.g -= carry ? j.groups : 0;
        at.split += step.split + carry;
    }
    __device__ __forceinline__ void next() {           // the next one that is not empty, or the end
        do advance();
        while (there() && empty());
    }
    __device__ __forceinline__ void settle() {         // from an empty first one on
        if (there() && empty()) next();
    }
    __device__ __forceinline__ long long m0(int tile_rows) const { return (long long)(at.g * j.group + at.m) * tile_rows; }
    __device__ __forceinline__ int n0() const { return at.n * j.wide; }
    __device__ __forceinline__ int k0() const { return at.split * j.kb_per_split; }
    __device__ __forceinline__ int k1() const { return min(j.k_blocks, (at.split + 1) * j.kb_per_split); }
};

// The scales one after the other, as for few rows: their product may lie below fp32's normal numbers where the result does not.
__device__ __forceinline__ Pair scaled2(Pair d, Pair x_scale, Pair w_scale, Pair bias) { return pfma(pmul(d, x_scale), w_scale, bias); }
// Two neighbouring columns of D to z and y.  `in`: the residual's or the activation input's two elements.
template <int KIND, int ACT, bool SCALED>
__device__ __forceinline__ Pair finish2(Pair d, Pair bias, Pair x_scale, Pair w_scale, Pair in, Pair& z) {
    if (KIND == kLinearInput) return pmul(d, act_slope2<ACT>(in));
    z = SCALED ? scaled2(d, x_scale, w_scale, bias) : padd(d, bias);
    return padd(act2<ACT>(z), in);
}
__device__ __forceinline__ Pair elems2(uint32_t v) { const float2 t = elem2_to_float2(v); return pair_of(t.x, t.y); }
// A sum as the matrix instructions leave it: fp32, of 8-bit integers 32-bit ones (exact: at most 2^16 products of at most 2^14), rounded to fp32 here.
// Parts of a split sum keep their form and are added up in it: SumOf.
template <int OPS>
__device__ __forceinline__ float sum_value(uint32_t v) { return OPS == kOpsI8 ? __int2float_rn((int)v) : __uint_as_float(v); }
template <bool WHOLE> struct SumOf { typedef float Type; typedef float4 Four; };
template <> struct SumOf<true> { typedef int Type; typedef int4 Four; };
// Adds a part's four columns from `col` of N on.
template <bool WHOLE>
__device__ __forceinline__ void part4(const float* p, int col, int N, typename SumOf<WHOLE>::Type (&v)[4]) {
    if ((N & 3) == 0) {
        const typename SumOf<WHOLE>::Four t = *reinterpret_cast<const typename SumOf<WHOLE>::Four*>(p);
        v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (col + c < N) v[c] += reinterpret_cast<const typename SumOf<WHOLE>::Type*>(p)[c];
    }
}
__device__ __forceinline__ uint32_t pack2(Pair p) { float a, b; split_pair(p, a, b); return pack_elem(a, b); }

__device__ __forceinline__ void prefetch_l1(const float* p) { asm volatile("prefetch.global.L1 [%0];\n" ::"l"(p)); }

__device__ NoBias g_no_bias;

// p[col .. col + 15], the same for all threads of a warp; from the n-th value on some that is there.  (Plain loads, here and wherever a kernel reads behind
// wait_for_prerequisites(): the launch before may write these values while this kernel is already resident, so they are not read-only for its lifetime.)
__device__ __forceinline__ void row_values(const float* p, int col, int n, float (&v)[16]) {
    if (col + 16 <= n) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 t = reinterpret_cast<const float4*>(p + col)[q];
            v[4 * q] = t.x; v[4 * q + 1] = t.y; v[4 * q + 2] = t.z; v[4 * q + 3] = t.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = p[min(col + i, n - 1)];
    }
}

// Where a warp's tile keeps 16 bytes: rows of 128 bytes (64 columns) or 64 (32 columns), whose 16-byte places are exchanged by the row's
// number, as the copy engine does it.
__device__ __forceinline__ uint32_t place(int row, int at, bool narrow) {
    return narrow ? row * 64 + ((at ^ ((row >> 1) & 3)) << 4) : row * 128 + ((at ^ (row & 7)) << 4);
}

__device__ __forceinline__ void lds(uint32_t at, unsigned long long& v) { asm volatile("ld.shared.b64 %0, [%1];\n" : "=l"(v) : "r"(at) : "memory"); }
__device__ __forceinline__ void lds(uint32_t at, uint32_t& v) { asm volatile("ld.shared.b32 %0, [%1];\n" : "=r"(v) : "r"(at) : "memory"); }
__device__ __forceinline__ void lds(uint32_t at, uint16_t& v) { asm volatile("ld.shared.b16 %0, [%1];\n" : "=h"(v) : "r"(at) : "memory"); }
__device__ __forceinline__ void sts(uint32_t at, unsigned long long v) { asm volatile("st.shared.b64 [%0], %1;\n" ::"r"(at), "l"(v) : "memory"); }
__device__ __forceinline__ void sts(uint32_t at, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;\n" ::"r"(at), "r"(v) : "memory"); }
__device__ __forceinline__ void sts(uint32_t at, uint16_t v) { asm volatile("st.shared.b16 [%0], %1;\n" ::"r"(at), "h"(v) : "memory"); }

// A warp's tile <-> `rows` rows of global memory from g on (its first row and column; rows of `stride` elements), the first `cols` columns, in units
// of T: for rows that are no multiples of 16 bytes.  Eight rows (of 8-byte units sixteen) are read before they are written; their exchanged places
// differ by constants, so that a unit costs a read, a write and a step of the address (2203200 x 256 -> 372 707 -> 638 us).
template <bool OUT, bool NARROW, typename T>
__device__ __forceinline__ void copy_tile_units(uint32_t tile, uint16_t* g, long long stride, int rows, int cols, int lane) {
    constexpr int kUnit = sizeof(T) / 2, kAcross = 64 / kUnit, kLanes = kAcross < 32 ? kAcross : 32, kDown = 32 / kLanes, kPitch = NARROW ? 64 : 128;
    const int sub = lane / kLanes;
    const long long step = kDown * stride * 2;
#pragma unroll 1
    for (int col = (lane % kLanes) * kUnit; col < cols; col += kLanes * kUnit) {
        char* p = (char*)(g + sub * stride + col);
        uint32_t at = tile + place(sub, col >> 3, NARROW) + (col & 7) * 2;
#pragma unroll 1
        for (int left = rows - sub; left > 0; left -= 8 * kDown, at += 8 * kDown * kPitch) {
            T v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            char* q = p;
#pragma unroll
            for (int i = 0; i < 8; ++i) {              // (sub is 0, or 1 where kDown is 2: the row's number is sub ^ kDown i as well)
                const uint32_t here = (at ^ place(kDown * i, 0, NARROW) % kPitch) + kDown * i * kPitch;
                if (OUT) {
                    lds(here, v[i]);
                } else {
                    if (kDown * i < left) v[i] = *reinterpret_cast<const T*>(q);
                    q += step;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t here = (at ^ place(kDown * i, 0, NARROW) % kPitch) + kDown * i * kPitch;
                if (!OUT) {
                    sts(here, v[i]);
                } else {
                    if (kDown * i < left) *reinterpret_cast<T*>(q) = v[i];
                    q += step;
                }
            }
            p = q;
        }
    }
}
template <bool OUT, bool NARROW>
__device__ __forceinline__ void copy_tile(uint32_t tile, uint16_t* g, long long stride, int rows, int cols, int lane) {
    if (((stride | cols) & 3) == 0) copy_tile_units<OUT, NARROW, unsigned long long>(tile, g, stride, rows, cols, lane);
    else if (((stride | cols) & 1) == 0) copy_tile_units<OUT, NARROW, uint32_t>(tile, g, stride, rows, cols, lane);
    else copy_tile_units<OUT, NARROW, uint16_t>(tile, g, stride, rows, cols, lane);
}
template <bool OUT>
__device__ __forceinline__ void copy_tile(uint32_t tile, bool narrow, uint16_t* g, long long stride, int rows, int cols, int lane) {
    if (narrow) copy_tile<OUT, true>(tile, g, stride, rows, cols, lane);
    else copy_tile<OUT, false>(tile, g, stride, rows, cols, lane);
}

// 32 columns of a thread's row: out of TMEM (`acc`), through the epilogue, into the warp's tile from its 16-byte place `first` on.
// IN: the places that take y hold the residual or z_in before.  Z: z goes 2 KB behind, or (WIDE) into the next tile.
// READY: scales and bias have been applied.  TABLE: they come from the chunk's table, from these columns' on: 64 of the bias, 64 scales.
template <int KIND, int ACT, int OPS, bool IN, bool Z, bool WIDE, bool READY, bool TABLE = false>
__device__ __forceinline__ void finish32(const uint32_t (&acc)[32], const LinearEpilogue& e, int n, int col, int first, int lane, float x_scale, uint32_t tile,
                                         const float* table = nullptr) {
    constexpr bool SCALED = OPS != kOps16;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        float b[16], w[16];
        if (TABLE) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 s = reinterpret_cast<const float4*>(table + 16 * part)[i], t = reinterpret_cast<const float4*>(table + 64 + 16 * part)[i];
                b[4 * i] = s.x; b[4 * i + 1] = s.y; b[4 * i + 2] = s.z; b[4 * i + 3] = s.w;
                w[4 * i] = t.x; w[4 * i + 1] = t.y; w[4 * i + 2] = t.z; w[4 * i + 3] = t.w;
            }
        } else if (KIND == kLinearForward && !READY) {
            row_values(e.bias ? e.bias : g_no_bias.values, e.bias ? col + 16 * part : 0, e.bias ? n : 64, b);
            if (SCALED) row_values(e.w_scale, col + 16 * part, n, w);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {                  // 8 columns: one 16-byte place
            const uint32_t at = tile + place(lane, first + 2 * part + h, Z && !WIDE);
            uint32_t in[4] = {0, 0, 0, 0}, y[4], z[4];
            if (IN) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(in[0]), "=r"(in[1]), "=r"(in[2]), "=r"(in[3]) : "r"(at) : "memory");
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = 8 * h + 2 * i, k = 16 * part + c;
                const Pair d = pair_of(sum_value<OPS>(acc[k]), sum_value<OPS>(acc[k + 1]));
                if (KIND == kLinearInput) {
                    y[i] = pack2(IN ? pmul(d, act_slope2<ACT>(elems2(in[i]))) : d);
                } else {
                    const Pair bias = READY ? 0 : pair_of(b[c], b[c + 1]);
                    const Pair zz = READY ? d : SCALED ? scaled2(d, both(x_scale), pair_of(w[c], w[c + 1]), bias) : padd(d, bias), a = act2<ACT>(zz);
                    y[i] = pack2(IN ? padd(a, elems2(in[i])) : a);
                    if (Z) z[i] = pack2(zz);
                }
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
            if (KIND == kLinearForward && Z)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at + (WIDE ? kTile : kTile / 2)), "r"(z[0]), "r"(z[1]), "r"(z[2]), "r"(z[3]) : "memory");
        }
    }
}

// The same of 64 sums in place, four columns at a time.
template <bool SCALED>
__device__ __forceinline__ void scale_and_add(float (&sum)[64], const LinearEpilogue& e, int n, int col, float x_scale) {
    auto four = [&](const float* p, int at, float (&v)[4]) {
        if (at + 4 <= n) {
            const float4 t = *reinterpret_cast<const float4*>(p + at);
            v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = p[min(at + i, n - 1)];
        }
    };
#pragma unroll
    for (int k = 0; k < 64; k += 4) {
        float b[4] = {0.f, 0.f, 0.f, 0.f}, w[4];
        if (e.bias) four(e.bias, col + k, b);
        if (SCALED) four(e.w_scale, col + k, w);
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const Pair d = pair_of(sum[k + i], sum[k + i + 1]), bias = pair_of(b[i], b[i + 1]);
            split_pair(SCALED ? scaled2(d, both(x_scale), pair_of(w[i], w[i + 1]), bias) : padd(d, bias), sum[k + i], sum[k + i + 1]);
        }
    }
}

// The same for both halves (32 columns of each at most, in narrow tiles 2 KB apart) of gated rows of 2 n elements, whose halves lie n elements apart: 16 units are
// read before they are written.
template <bool OUT, typename T>
__device__ __forceinline__ void copy_halves_units(uint32_t tile, uint16_t* g, long long n, int rows, int cols, int lane) {
    constexpr int kUnit = sizeof(T) / 2, kAcross = 32 / kUnit, kDown = 32 / kAcross, kBatch = 8;
    const int sub = lane / kAcross, col = lane % kAcross * kUnit;
    if (col >= cols) return;
    char* p = (char*)(g + sub * 2 * n + col);
    const long long step = kDown * 4 * n, half = 2 * n;            // in bytes
#pragma unroll 1
    for (int row = sub; row < rows; row += kBatch * kDown) {
        T v[2][kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v[h][i] = 0;
                const int r = row + kDown * i;
                if (OUT) lds(tile + h * (kTile / 2) + place(r, col >> 3, true) + (col & 7) * 2, v[h][i]);
                else if (r < rows) v[h][i] = *reinterpret_cast<const T*>(p + i * step + h * half);
            }
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = row + kDown * i;
                if (!OUT) sts(tile + h * (kTile / 2) + place(r, col >> 3, true) + (col & 7) * 2, v[h][i]);
                else if (r < rows) *reinterpret_cast<T*>(p + i * step + h * half) = v[h][i];
            }
        p += kBatch * step;
    }
}
template <bool OUT>
__device__ __forceinline__ void copy_halves(uint32_t tile, uint16_t* g, long long n, int rows, int cols, int lane) {
    if (((n | cols) & 3) == 0) copy_halves_units<OUT, unsigned long long>(tile, g, n, rows, cols, lane);
    else if (((n | cols) & 1) == 0) copy_halves_units<OUT, uint32_t>(tile, g, n, rows, cols, lane);
    else copy_halves_units<OUT, uint16_t>(tile, g, n, rows, cols, lane);
}

// 2 N of p's values from `col` on, in pairs, of one half of a gated row of values, n apart: 16 bytes at a time only where both halves are aligned.
template <int N>
__device__ __forceinline__ void half_values(const float* p, int col, int n, int half, Pair (&v)[N]) {
    const float* q = p + (long long)half * n;
    if ((n & 3) == 0 && col + 2 * N <= n) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float4 t = *reinterpret_cast<const float4*>(q + col + 2 * i);
            v[i] = pair_of(t.x, t.y);
            v[i + 1] = pair_of(t.z, t.w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = pair_of(q[min(col + 2 * i, n - 1)], q[min(col + 2 * i + 1, n - 1)]);
    }
}

// 16 outputs act(g) u of a thread's row, from column `col` of n on, into the tile from its 16-byte place `first` on; Z: g 2 KB and u 4 KB behind.  Bias and scales
// come from `table` (columns `first` x 8 on of the chunk's 32: the gate's bias, up's, and their scales), or, where there is no room for one, from memory.
template <int ACT, int OPS, bool Z, bool LONG, bool TABLE>
__device__ __forceinline__ void gate16(const uint32_t (&g)[16], const uint32_t (&u)[16], const LinearEpilogue& e, int n, int col, int first, int lane, float x_scale,
                                       uint32_t tile, const float* table) {
    constexpr bool SCALED = OPS != kOps16;
    // (from memory the values of all 16 columns at once: by four columns each wait for them is its own, 16 bits, 550800 x 384 -> 1024 955 -> 1085 us)
    constexpr int kWidth = TABLE || LONG ? 8 : 16;
#pragma unroll
    for (int s = 0; s < 16; s += kWidth) {
        Pair bias[2][kWidth / 2] = {}, scale[2][kWidth / 2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (TABLE) {
                const float4* t = reinterpret_cast<const float4*>(table + 32 * h + 8 * first + s);
#pragma unroll
                for (int i = 0; i < kWidth / 2; i += 2) {
                    const float4 b = t[i / 2];
                    bias[h][i] = pair_of(b.x, b.y);
                    bias[h][i + 1] = pair_of(b.z, b.w);
                    if (SCALED) {
                        const float4 w = t[16 + i / 2];
                        scale[h][i] = pair_of(w.x, w.y);
                        scale[h][i + 1] = pair_of(w.z, w.w);
                    }
                }
            } else if (e.bias) {
                half_values(e.bias, col + s, n, h, bias[h]);
            }
        }
#pragma unroll
        for (int q = 0; q < kWidth / 8; ++q) {         // 8 columns: one 16-byte place
            const uint32_t at = tile + place(lane, first + s / 8 + q, true);
            uint32_t y[4], zg[4], zu[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = 4 * q + i, c = s + 2 * k;
                Pair z[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const Pair d = pair_of(sum_value<OPS>(h ? u[c] : g[c]), sum_value<OPS>(h ? u[c + 1] : g[c + 1]));
                    z[h] = SCALED ? scaled2(d, both(x_scale), scale[h][k], bias[h][k]) : padd(d, bias[h][k]);
                }
                y[i] = pack2(pmul(act2<ACT>(z[0]), z[1]));
                if (Z) {
                    zg[i] = pack2(z[0]);
                    zu[i] = pack2(z[1]);
                }
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
            if (Z) {
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at + kTile / 2), "r"(zg[0]), "r"(zg[1]), "r"(zg[2]), "r"(zg[3]) : "memory");
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at + kTile), "r"(zu[0]), "r"(zu[1]), "r"(zu[2]), "r"(zu[3]) : "memory");
            }
        }
    }
}

// 32 columns of a thread's row: g and u in the tile give way to their gradients, of act(g) u whose gradient d is.
template <int ACT>
__device__ __forceinline__ void through_gate32(const uint32_t (&d)[32], int lane, uint32_t tile) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t at = tile + place(lane, q, true);
        uint32_t g[4], u[4];
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(g[0]), "=r"(g[1]), "=r"(g[2]), "=r"(g[3]) : "r"(at) : "memory");
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]) : "r"(at + kTile / 2) : "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            Pair a, slope;
            const Pair dd = pair_of(__uint_as_float(d[8 * q + 2 * i]), __uint_as_float(d[8 * q + 2 * i + 1]));
            act_and_slope2<ACT>(elems2(g[i]), a, slope);
            g[i] = pack2(pmul(pmul(dd, elems2(u[i])), slope));
            u[i] = pack2(pmul(dd, a));
        }
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at), "r"(g[0]), "r"(g[1]), "r"(g[2]), "r"(g[3]) : "memory");
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at + kTile / 2), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]) : "memory");
    }
}

// Sums that stay in fp32 (parts of a split product, the weight gradient): 32 columns of a thread's row into the warp's tile, and the tile, in
// whole rows, to global memory.  Rows of 128 bytes, places exchanged by the row's number.
__device__ __forceinline__ void put_sums(uint32_t tile, int lane, int part, const float* v) {        // 16 columns
#pragma unroll
    for (int c = 0; c < 4; ++c)
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};\n" ::"r"(tile + place(lane, 4 * part + c, false)), "f"(v[4 * c]), "f"(v[4 * c + 1]), "f"(v[4 * c + 2]),
                     "f"(v[4 * c + 3]) : "memory");
}
__device__ __forceinline__ void write_sums(uint32_t tile, float* out, long long M, int N, long long row0, int col0, int lane) {
    const int j = lane & 7, col = col0 + 4 * j;
    if (col >= N) return;
#pragma unroll 4
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 3);
        float v[4];
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];\n" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(tile + place(r, j, false)) : "memory");
        if (row0 + r >= M) continue;
        float* p = out + (row0 + r) * N + col;
        if ((N & 3) == 0) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (col + c < N) p[c] = v[c];
        }
    }
}

// MAP: the rows of the outputs (and of the residual or z_in) are multiples of 16 bytes and the copy engine moves them; else the warps do.  (One kernel with
// both spilled registers around the warps' copies: 2203200 x 256 -> 384 558 -> 1032 us.  The 16-bit kernels of sums that are not LONG spill none, e4m3's up to
// 56 bytes a thread, the weight gradient's 76 with two CTAs and 100 with one.)
// LONG: the sum leaves TMEM every kLinearLongChunk stages, for sums that have more.  (An instantiation of its own: the 64 sums that a thread holds spill
// registers around the epilogue, and what is spilled takes the way to memory that the products' operands take.  Scales and bias go to the sums in place, four
// columns at a time: with 16 of them in registers, as elsewhere, 4096 -> 4096 took 4 % longer, 8448 -> 4096 in e4m3 8 %.)
template <bool PAIR, int KIND, int OPS, bool MAP, int TILES, bool LONG>
__global__ void __launch_bounds__(kThreads, 1) linear_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Job job) {
    static_assert(!LONG || TILES != 2, "two tiles a warp are for short sums");
    static_assert(!LONG || OPS != kOpsI8, "whole numbers are summed up exactly, however many");
    constexpr bool SCALED = OPS != kOps16;             // operands of 8 bits
    constexpr bool kInChunks = LONG || KIND == kLinearWeights;
    constexpr int kChunk = KIND == kLinearWeights ? kLinearChunk : kLinearLongChunk;
    constexpr int CTAS = PAIR ? 2 : 1;
    constexpr int kStages = Stages<TILES>::value, kOffTiles = kStages * 2 * kOperand;
    constexpr int kTileRows = 128 * CTAS;
    constexpr bool GATED = KIND == kLinearGated;        // (N: the outputs; B has as many gate rows and, behind them, up rows)
    constexpr bool A_MN = KIND == kLinearWeights, B_MN = KIND != kLinearForward && !GATED;
    constexpr int kBK = SCALED ? 128 : 64;               // elements of a stage along k
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
            mbar_init(bar(kBEmpty + s), KIND == kLinearWeights ? 2 : 1);
            mbar_init(bar(kBUsed + s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(bar(kBAccFull + b), 1);
            mbar_init(bar(kBAccEmpty + b), kEpiWarps * CTAS);
        }
        for (int w = 0; w < 2 * kEpiWarps; ++w) mbar_init(bar(kBIn + w), 1);
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

    Units at(job, blockIdx.x / CTAS);
    at.settle();
    if (warp < kEpiWarp0) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kRegsOther));
    // (Warps 0 and 1 run their loops as whole warps and elect a thread for the instructions alone: what the loops count stays in the uniform
    // registers that those instructions take their operands from.  By one thread, a stage's products took 500 cycles to issue.)
    if (warp == 0) {
        const int cols = job.bn / CTAS;                // this CTA's share of B
        const uint32_t bytes = CTAS * (kOperand + job.bytes_b);
        uint32_t s = 0, phase = 1, it = 0;
        bool ok = true;
        for (; at.there() && ok; at.next()) {
            const int m = (int)at.m0(kTileRows) + 128 * (int)rank, n = at.n0() + (GATED ? job.N : cols) * (int)rank, k1 = at.k1();
            for (int kb = at.k0(); kb < k1; ++kb, ++it) {
                ok = wait_asleep(bar(kBEmpty + s), phase, cta_abort);
                if (!ok) break;
                const uint32_t full = PAIR ? leaders(bar(kBFull + s)) : bar(kBFull + s), a = base + s * 2 * kOperand, b = a + kOperand;
                if (elect_one()) {
                    if (rank == 0) mbar_arrive_expect_tx(bar(kBFull + s), bytes);
                    if (A_MN) {
                        load_box<PAIR>(a, &maps.a, m, kb * kBK, full);
                        load_box<PAIR>(a + kOperand / 2, &maps.a, m + 64, kb * kBK, full);
                    } else {
                        load_box<PAIR>(a, &maps.a, kb * kBK, m, full);
                    }
                    if (B_MN) {
                        load_box<PAIR>(b, &maps.b, n, kb * kBK, full);
                        if (job.boxes_b > 1) load_box<PAIR>(b + kOperand / 2, &maps.b, n + 64, kb * kBK, full);
                    } else {
                        load_box<PAIR>(b, &maps.b, kb * kBK, n, full);
                        if (GATED && !PAIR) load_box<PAIR>(b + job.wide * 128, &maps.b, kb * kBK, job.N + n, full);
                    }
                }
                __syncwarp();
                if (++s == kStages) { s = 0; phase ^= 1; }
            }
        }
        // after an expired wait: the copies in flight are waited for, so that none lands in memory that is no longer this CTA's
        if (!ok && rank == 0 && lane == 0) {
            volatile int ignore = 0;
            for (uint32_t i = it > kStages ? it - kStages : 0; i < it; ++i)
                mbar_wait<0>(bar(kBFull + i % kStages), (i / kStages) & 1, &ignore, 200000000LL);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            // 32 bytes along k a step, 16 rows of 128 bytes where k is the slow axis
            const uint64_t da = make_sdesc_sw128(base, A_MN ? kOperand / 2 : 16), db = make_sdesc_sw128(base + kOperand, B_MN ? kOperand / 2 : 16);
            const uint32_t hi = sdesc_hi(da), a0 = sdesc_lo(da), b0 = sdesc_lo(db);
            constexpr uint32_t kStageLo = 2 * kOperand / 16, kALo = A_MN ? 2048 / 16 : 2, kBLo = B_MN ? 2048 / 16 : 2;
            uint32_t s = 0, phase = 0, done = 0;
            bool ok = true;
            for (; at.there() && ok; at.next()) {
                const int k1 = at.k1();
                for (int kb = at.k0(); kb < k1 && ok;) {
                    const int end = kInChunks ? min(k1, kb + kChunk) : k1;
                    const uint32_t buf = done & 1, acc = tmem + buf * kAccCols;
                    ok = wait_asleep(bar(kBAccEmpty + buf), ((done >> 1) & 1) ^ 1u, cta_abort);
                    if (!ok) break;
                    tc_fence_after();
                    uint32_t accumulate = 0;
                    for (; kb < end; ++kb) {
                        ok = mbar_wait_all(bar(kBFull + s), phase, cta_abort);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t a = a0 + s * kStageLo, b = b0 + s * kStageLo;
                        if (elect_one()) {
                            mma<PAIR, OPS>(acc, a, b, hi, job.idesc, accumulate);
#pragma unroll
                            for (int k = 1; k < 4; ++k) mma<PAIR, OPS>(acc, a + k * kALo, b + k * kBLo, hi, job.idesc, 1);
                            commit<PAIR>(bar((KIND == kLinearWeights ? kBUsed : kBEmpty) + s));
                        }
                        __syncwarp();
                        accumulate = 1;
                        if (++s == kStages) { s = 0; phase ^= 1; }
                    }
                    if (!ok) break;
                    if (elect_one()) commit<PAIR>(bar(kBAccFull + buf));
                    __syncwarp();
                    ++done;
                }
            }
        }
        __syncwarp();
    } else if (warp < kEpiWarp0) {
        if constexpr (KIND == kLinearWeights) {
            // Warps 2 and 3 hand the stages that the products have used back to the copies; on the way they add up the rows of A, 64 columns of d_z
            // each: the bias's gradient.  The tiles of a row share the stages, every n_tiles-th to each.  (A pass over d_z of its own took 67 us of 935 at
            // 156672 x 1024; all stages by the row's first tile made those tiles, and the kernel, 18 % slower.)
            uint32_t s = 0, phase = 0;
            bool ok = true;
            for (; at.there() && ok; at.next()) {
                float all[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                const int k1 = at.k1();
                uint32_t round, turn;                  // of this row's tiles, whose stage it is
                job.by_n_tiles.split((uint32_t)at.k0(), round, turn);
                for (int kb = at.k0(); kb < k1; ++kb) {
                    ok = mbar_wait_all(bar(kBUsed + s), phase, cta_abort);
                    if (!ok) break;
                    if (job.e.a_sums && (int)turn == at.at.n) {
                        const uint32_t box = base + s * 2 * kOperand + (warp - 2) * (kOperand / 2);
                        float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
                        for (int i = 0; i < 16; ++i) {
                            const int row = 4 * i + (lane >> 3);
                            uint32_t v[4];
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                                         : "r"(box + place(row, lane & 7, false)) : "memory");
#pragma unroll
                            for (int q = 0; q < 4; ++q) add_elems(sum[2 * q], sum[2 * q + 1], v[q]);
                        }
#pragma unroll
                        for (int c = 0; c < 8; ++c) all[c] += sum[c];
                    }
                    if ((int)++turn == job.n_tiles) turn = 0;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(kBEmpty + s));
                    if (++s == kStages) { s = 0; phase ^= 1; }
                }
                if (!ok || !job.e.a_sums) continue;
                const long long m = at.m0(kTileRows) + 128 * rank + 64 * (warp - 2) + 8 * (lane & 7);
                float* out = job.e.a_sums + ((size_t)at.at.split * job.n_tiles + at.at.n) * job.M;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    all[c] += __shfl_xor_sync(0xffffffffu, all[c], 8);
                    all[c] += __shfl_xor_sync(0xffffffffu, all[c], 16);
                    if (lane < 8 && m + c < job.M) out[m + c] = all[c];
                }
            }
        }
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kRegsEpi));
        // A chunk is 64 columns of the warp's 32 rows.  The chunks of all tiles go to the groups of four warps in turn: a warp has one of a tile,
        // or none of a narrow one.  (Every warp waits for every accumulator and gives it back, so that none falls behind by a phase.)
        const int quarter = warp & 3, group = (warp - kEpiWarp0) >> 2, chunks = (job.bn + 63) >> 6;
        const uint32_t tile = base + kOffTiles + (warp - kEpiWarp0) * Stages<TILES>::tile;
        const uint32_t lane_tmem = tmem + ((uint32_t)(quarter * 32) << 16);
        uint32_t done = 0;
        bool ok = true;
        int first_chunk = group;                       // of this tile's, this group's first: the tiles' chunks are counted through
        auto next_chunk = [&] {
            first_chunk -= chunks;
            while (first_chunk < 0) first_chunk += kGroups;
        };
        auto give_back = [&](uint32_t buf) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_leader<PAIR>(bar(kBAccEmpty + buf));
        };
        // column p of a chunk in the accumulator (gated: 32 of the gate, then 32 of up)
        auto column = [&](int col0, int p) { return !GATED ? col0 + p : p < 32 ? (col0 >> 1) + p : job.wide + (col0 >> 1) + p - 32; };
        // a unit's sum over all of its chunks along k, this warp's 64 columns from col0 on (none: the warp only keeps in step)
        auto add_up = [&](float (&acc)[64], int col0, bool some) {
            const int k1 = at.k1();
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = 0.f;
            for (int kb = at.k0(); kb < k1; kb += kChunk, ++done) {
                const uint32_t buf = done & 1;
                ok = wait_asleep(bar(kBAccFull + buf), (done >> 1) & 1, cta_abort);
                if (!ok) break;
                tc_fence_after();
                if (some)
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        if (col0 + 16 * p < job.bn) {
                            uint32_t t[16];
                            tmem_ld16(lane_tmem + buf * kAccCols + column(col0, 16 * p), t);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) acc[16 * p + i] += __uint_as_float(t[i]);
                        }
                give_back(buf);
            }
        };
        if (kInChunks && (KIND == kLinearWeights || job.e.sums)) {
            for (; at.there() && ok; at.next(), next_chunk()) {
                const long long row0 = at.m0(kTileRows) + 128 * rank + 32 * quarter;
                const int n0 = at.n0();
                const int chunk = first_chunk, col0 = 64 * chunk;          // (as many groups as chunks: a group has one at most)
                float acc[64];
                add_up(acc, col0, chunk < chunks);
                if (!ok || chunk >= chunks) continue;
                float* sums = job.e.sums + (size_t)at.at.split * job.M * job.N * (GATED ? 2 : 1);      // (gated: gate and up columns apart)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (col0 + 32 * h < job.bn) {
                        put_sums(tile, lane, 0, &acc[32 * h]);
                        put_sums(tile, lane, 1, &acc[32 * h + 16]);
                        __syncwarp();
                        if (GATED) write_sums(tile, sums + h * (size_t)job.M * job.N, job.M, job.N, row0, n0 + (col0 >> 1), lane);
                        else write_sums(tile, sums, job.M, job.N, row0, n0 + col0 + 32 * h, lane);
                        __syncwarp();
                    }
            }
        } else if (!kInChunks && job.e.sums) {
            for (; at.there() && ok; at.next(), ++done) {        // parts of a split sum
                const long long row0 = at.m0(kTileRows) + 128 * rank + 32 * quarter;
                const int n0 = at.n0();
                const uint32_t buf = done & 1;
                ok = wait_asleep(bar(kBAccFull + buf), (done >> 1) & 1, cta_abort);
                if (!ok) break;
                tc_fence_after();
                for (int chunk = first_chunk; chunk < chunks; chunk += kGroups) {
#pragma unroll 1
                    for (int c = 64 * chunk; c < min(job.bn, 64 * chunk + 64); c += 32) {
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            uint32_t t[16];
                            float f[16];
                            tmem_ld16(lane_tmem + buf * kAccCols + (GATED ? column(64 * chunk, c - 64 * chunk) : c) + 16 * p, t);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(t[i]);         // (whole numbers stay what they are)
                            put_sums(tile, lane, p, f);
                        }
                        __syncwarp();
                        if (GATED)
                            write_sums(tile, job.e.sums + (2 * (size_t)at.at.split + (c - 64 * chunk) / 32) * job.M * job.N, job.M, job.N, row0, n0 + 32 * chunk, lane);
                        else write_sums(tile, job.e.sums + (size_t)at.at.split * job.M * job.N, job.M, job.N, row0, n0 + c, lane);
                        __syncwarp();
                    }
                }
                give_back(buf);
                next_chunk();
            }
        } else if constexpr (GATED) {
            // A chunk is 32 outputs of the warp's 32 rows, 2 KB, and as much of the gate's and of the up columns where z is kept.
            const bool has_z = OPS == kOps16 && !(MAP && TILES == 1) && job.e.z != nullptr;
            // Bias and scales of the chunk's columns, a lane to a column, come while the accumulator is waited for; every thread reads them out of the tile's second
            // 2 KB, where no z has them.  (Read from memory by every thread: 550800 x 384 -> 1024 in 8 bits 1860 us instead of 800, in 16 bits 898 instead of 715.)
            constexpr bool TABLE = OPS == kOpsI8 || (MAP && TILES == 1);
            float* table = reinterpret_cast<float*>(smem + (tile - base) + kTile / 2);
            for (; at.there() && ok; at.next(), done += LONG ? 0 : 1) {
                const long long row0 = at.m0(kTileRows) + 128 * rank + 32 * quarter;
                const int n0 = at.n0(), chunk = first_chunk, col = n0 + 32 * chunk;        // (as many groups as chunks: a group has one at most)
                const uint32_t buf = done & 1, acc = lane_tmem + buf * kAccCols;
                const int rows = (int)min(32ll, job.M - row0), own = min(32, job.N - col);
                const bool mine = chunk < chunks && own > 0 && rows > 0;
                float sum[LONG ? 64 : 1];
                if (TABLE && mine) {
                    const int c = min(col + lane, job.N - 1);
                    table[lane] = job.e.bias ? job.e.bias[c] : 0.f;
                    table[32 + lane] = job.e.bias ? job.e.bias[job.N + c] : 0.f;
                    if (SCALED) {
                        table[64 + lane] = job.e.w_scale[c];
                        table[96 + lane] = job.e.w_scale[job.N + c];
                    }
                } else if (mine && lane < 2 && job.e.bias) {
                    prefetch_l1(job.e.bias + col + lane * job.N);
                }
                if constexpr (LONG) add_up(sum, 64 * chunk, mine);
                else ok = wait_asleep(bar(kBAccFull + buf), (done >> 1) & 1, cta_abort);
                if (!ok) break;
                tc_fence_after();
                if (mine) {
                    if (MAP && lane == 0) stores_read<0>();        // what was there has been read
                    __syncwarp();
                    float x_scale = 1.f;
                    if (SCALED && lane < rows) x_scale = job.e.x_scale[row0 + lane];
#pragma unroll 1
                    for (int part = 0; part < 2; ++part) {
                        uint32_t g[16], u[16];
                        if constexpr (LONG) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                g[i] = __float_as_uint(sum[i]);
                                u[i] = __float_as_uint(sum[32 + i]);
                                sum[i] = sum[16 + i];
                                sum[32 + i] = sum[48 + i];
                            }
                        } else {
                            tmem_ld16(acc + 32 * chunk + 16 * part, g);
                            tmem_ld16(acc + job.wide + 32 * chunk + 16 * part, u);
                            tmem_ld_wait();
                            if (part) give_back(buf);  // the accumulator has been read
                        }
                        with_act(job.e.activation, [&](auto tag) {
                            constexpr int ACT = decltype(tag)::value;
                            if constexpr (!TABLE) {
                                if (has_z) {
                                    gate16<ACT, OPS, true, LONG, false>(g, u, job.e, job.N, col + 16 * part, 2 * part, lane, x_scale, tile, nullptr);
                                    return;
                                }
                            }
                            gate16<ACT, OPS, false, LONG, TABLE>(g, u, job.e, job.N, col + 16 * part, 2 * part, lane, x_scale, tile, table);
                        });
                    }
                    if (MAP) {
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) {
                            store_box(&maps.y, col, (int)row0, tile);
                            if (has_z) {
                                store_box(&maps.z, col, (int)row0, tile + kTile / 2);
                                store_box(&maps.z_up, col, (int)row0, tile + kTile);
                            }
                            stores_commit();
                        }
                    } else {
                        __syncwarp();
                        copy_tile<true>(tile, true, (uint16_t*)job.e.y + row0 * job.N + col, job.N, rows, own, lane);
                        if (has_z) copy_halves<true>(tile + kTile / 2, (uint16_t*)job.e.z + row0 * 2 * job.N + col, job.N, rows, own, lane);
                        __syncwarp();
                    }
                } else if (!LONG) {
                    give_back(buf);                    // a warp without a chunk here
                }
                next_chunk();
            }
            if (lane == 0) stores_read<0>();
            __syncwarp();
        } else if constexpr (KIND == kLinearGatedInput) {
            // The gradient d of the gated values x = act(g) u comes out of TMEM, 32 columns at a time; the warp's tile takes g and u of such a piece, 2 KB each, and
            // their gradients d u act'(g) and d act(g) over them.  As soon as the copy engine has read those, it is asked for the next piece.  (550800 x 384 -> 1024
            // 905 us; asked once the tile's accumulator is waited for 994.  Two tiles a warp and three stages: 1000, and 156672 x 1024 -> 2752 925 -> 1060 us: the more
            // of z is under way, the longer the products wait for their operands.  Prefetched into L2 a unit ahead 1236.)
            uint32_t taken = 0, asked = 0;
            const uint32_t in_bar = bar(kBIn + warp - kEpiWarp0);
            Units ahead = at;                          // the unit, the chunk and the column in it of the next piece to ask for
            int ahead_chunk = first_chunk, ahead_p0 = 0;
            auto columns = [&](const Units& u, int chunk) { return u.m0(kTileRows) + 128 * rank + 32 * quarter < job.M ? min(64, min(job.bn - 64 * chunk, job.N - u.n0() - 64 * chunk)) : 0; };
            auto ask = [&] {                           // by one lane; the tile is free
                while (ahead.there() && ahead_p0 >= columns(ahead, ahead_chunk)) {
                    ahead.next();
                    ahead_p0 = 0;
                    ahead_chunk -= chunks;
                    while (ahead_chunk < 0) ahead_chunk += kGroups;
                }
                if (!ahead.there()) return;
                const int row = (int)ahead.m0(kTileRows) + 128 * (int)rank + 32 * quarter, col = ahead.n0() + 64 * ahead_chunk + ahead_p0;
                mbar_arrive_expect_tx(in_bar, kTile);
                tma_load_2d(tile, &maps.in, col, row, in_bar);
                tma_load_2d(tile + kTile / 2, &maps.in_up, col, row, in_bar);
                ++asked;
                ahead_p0 += 32;
            };
            auto landed = [&](volatile int* abort, long long limit) { return mbar_wait<0>(in_bar, taken & 1, abort, limit); };
            if (MAP && lane == 0) ask();
            __syncwarp();
            for (; at.there() && ok; at.next(), done += LONG ? 0 : 1) {
                const long long row0 = at.m0(kTileRows) + 128 * rank + 32 * quarter;
                const int chunk = first_chunk, col0 = 64 * chunk, col = at.n0() + col0, cols = columns(at, chunk);        // (as many groups as chunks: a group has one at most)
                const uint32_t buf = done & 1, acc = lane_tmem + buf * kAccCols;
                const int rows = (int)min(32ll, job.M - row0);
                float sum[LONG ? 64 : 1];
                uint16_t *in = (uint16_t*)job.e.z_in + row0 * 2 * job.N + col, *out = (uint16_t*)job.e.y + row0 * 2 * job.N + col;
                if (!MAP && cols > 0) copy_halves<false>(tile, in, job.N, rows, min(32, cols), lane);      // while the accumulator is waited for
                if constexpr (LONG) add_up(sum, col0, cols > 0);
                else ok = wait_asleep(bar(kBAccFull + buf), (done >> 1) & 1, cta_abort);
                if (!ok) break;
                tc_fence_after();
                bool given = LONG;
#pragma unroll 1
                for (int p0 = 0; p0 < cols; p0 += 32) {
                    const int own = min(32, cols - p0);
                    if (MAP) {
                        ok = __all_sync(0xffffffffu, landed(cta_abort, 4000000000LL));
                        if (!ok) break;
                        ++taken;
                    } else {
                        if (p0) copy_halves<false>(tile, in + p0, job.N, rows, own, lane);
                        __syncwarp();
                    }
                    uint32_t d[32];
                    if constexpr (LONG) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            d[i] = __float_as_uint(sum[i]);
                            sum[i] = sum[i + 32];
                        }
                    } else {
                        tmem_ld32(acc + col0 + p0, d);
                        tmem_ld_wait();
                        if (p0 + 32 >= cols) {         // the accumulator has been read
                            give_back(buf);
                            given = true;
                        }
                    }
                    with_act(job.e.activation, [&](auto tag) { through_gate32<decltype(tag)::value>(d, lane, tile); });
                    if (MAP) {
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) {
                            store_box(&maps.y, col + p0, (int)row0, tile);
                            store_box(&maps.z_up, col + p0, (int)row0, tile + kTile / 2);
                            stores_commit();
                            stores_read<0>();
                            ask();
                        }
                        __syncwarp();
                    } else {
                        __syncwarp();
                        copy_halves<true>(tile, out + p0, job.N, rows, own, lane);
                        __syncwarp();
                    }
                }
                if (ok && !given) give_back(buf);      // a warp without a chunk here
                next_chunk();
            }
            if (MAP && lane == 0)                      // after an expired wait: what was asked for lands before this CTA ends
                for (volatile int ignore = 0; taken < asked; ++taken) landed(&ignore, 200000000LL);
            __syncwarp();
        } else if constexpr (KIND != kLinearWeights) {
            // A tile takes the residual (or z_in) first and y over it, each thread its row.  One tile: with z a chunk goes in two pieces of 32 columns, y in
            // the first 2 KB of the tile and z in the others.  Two tiles: z has the second, or else the chunks take them in turn, and the next chunk's
            // residual comes while this one is worked on.
            const void* in = KIND == kLinearForward ? job.e.residual : job.e.z_in;
            const bool has_in = in != nullptr, has_z = KIND == kLinearForward && !SCALED && job.e.z != nullptr;
            const bool fetched = MAP && has_in;
            // Bias and scales of the chunk's columns, a lane to two of them, come while the accumulator is waited for.  (Read from memory by every thread, 8-bit
            // integers, us: 550800 x 384 -> 1152 397 instead of 345, 131072 x 768 -> 3000 with GELU 630 instead of 470.)
            constexpr bool TABLE = OPS == kOpsI8 && TILES == 3;
            float* table = reinterpret_cast<float*>(smem + (tile - base) + kTile);
            const int width = TILES == 1 && has_z ? 32 : 64;
            uint32_t taken = 0;                        // tiles that took a residual by the copy engine; two tiles: chunks
            bool ahead = false;                        // the chunk's residual is under way
            // by one lane: waits until the tile is free and asks for the residual
            auto prepare = [&](long long row0, int col, uint32_t t) {
                if (TILES == 2 && !has_in && !has_z) stores_read<1>();
                else stores_read<0>();
                if (fetched) {
                    const uint32_t b = bar(kBIn + (TILES == 2 ? 2 : 1) * (warp - kEpiWarp0) + (int)t);
                    mbar_arrive_expect_tx(b, 64 * width);
                    tma_load_2d(tile + t * kTile, &maps.in, col, (int)row0, b);
                }
            };
            auto landed = [&](uint32_t t, volatile int* abort, long long limit) {
                return mbar_wait<0>(bar(kBIn + (TILES == 2 ? 2 : 1) * (warp - kEpiWarp0) + (int)t), (TILES == 2 ? taken >> 1 : taken) & 1, abort, limit);
            };
            // whether this group has a chunk of a unit
            auto has_chunk = [&](const Units& u, int chunk) { return chunk < chunks && u.n0() + 64 * chunk < job.N && u.m0(kTileRows) + 128 * rank + 32 * quarter < job.M; };
            for (; at.there() && ok; at.next(), done += LONG ? 0 : 1) {
                const long long row0 = at.m0(kTileRows) + 128 * rank + 32 * quarter;
                const int n0 = at.n0();
                const uint32_t buf = done & 1, acc = lane_tmem + buf * kAccCols;
                float sum[LONG ? 64 : 1];
                const int rows = (int)min(32ll, job.M - row0);
                const uint32_t t = TILES == 2 && !has_z ? taken & 1 : 0, to = tile + t * kTile;
                const bool mine = has_chunk(at, first_chunk);
                if (mine) {                            // the residual comes while the accumulator is waited for
                    const int c = n0 + 64 * first_chunk;
                    if (lane == 0 && !ahead) prepare(row0, c, t);
                    // (the bias of the chunk: from HBM, it took longer than the rest of a small product's epilogue)
                    if (TABLE) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int n = min(c + 32 * h + lane, job.N - 1);
                            table[32 * h + lane] = job.e.bias ? job.e.bias[n] : 0.f;
                            table[64 + 32 * h + lane] = job.e.w_scale[n];
                        }
                    } else if (KIND == kLinearForward && lane < 2 && c + 32 * lane < job.N) {
                        if (job.e.bias) prefetch_l1(job.e.bias + c + 32 * lane);
                        if (SCALED) prefetch_l1(job.e.w_scale + c + 32 * lane);
                    }
                }
                if constexpr (LONG) add_up(sum, 64 * first_chunk, mine);
                else ok = wait_asleep(bar(kBAccFull + buf), (done >> 1) & 1, cta_abort);
                if (!ok) {
                    if (mine && fetched && lane == 0) {        // it lands before this CTA ends
                        volatile int ignore = 0;
                        landed(t, &ignore, 200000000LL);
                    }
                    break;
                }
                tc_fence_after();
                bool given = LONG;
                if (const int chunk = first_chunk; mine) {     // (as many groups as chunks: a group has one at most)
                    const int col0 = 64 * chunk, col = n0 + col0, cols = min(64, job.bn - col0), own = min(cols, job.N - col);
                    float x_scale = 1.f;
                    if (SCALED && lane < rows) x_scale = job.e.x_scale[row0 + lane];
                    if constexpr (LONG && KIND == kLinearForward) scale_and_add<SCALED>(sum, job.e, job.N, col, x_scale);
                    auto shift = [&] {                 // the sums of the next 32 columns take the place of those that are done
                        if constexpr (LONG)
#pragma unroll
                            for (int i = 0; i < 32; ++i) sum[i] = sum[i + 32];
                    };
#pragma unroll 1
                    for (int p0 = 0; p0 < cols; p0 += 32, shift()) {
                        if (p0 == 0 || width == 32) {          // a new tile
                            if (lane == 0 && p0 > 0) prepare(row0, col + p0, t);
                            __syncwarp();
                            if (fetched) {
                                ok = __all_sync(0xffffffffu, landed(t, cta_abort, 4000000000LL));
                                if (!ok) {
                                    volatile int ignore = 0;
                                    if (lane == 0) landed(t, &ignore, 200000000LL);
                                    break;
                                }
                                if (TILES != 2) ++taken;
                            } else if (!MAP && has_in) {
                                if (own > p0) copy_tile<false>(to, width == 32, (uint16_t*)in + row0 * job.N + col + p0, job.N, rows, min(width, own - p0), lane);
                                __syncwarp();
                            }
                            if (TILES == 2 && fetched) {       // the next chunk's
                                Units next = at;
                                int c = first_chunk;
                                do {
                                    next.next();
                                    c -= chunks;
                                    while (c < 0) c += kGroups;
                                } while (next.there() && !has_chunk(next, c));
                                ahead = next.there();
                                ++taken;
                                if (ahead && lane == 0) prepare(next.m0(kTileRows) + 128 * rank + 32 * quarter, next.n0() + 64 * c, t ^ 1);
                            }
                        }
                        uint32_t cur[32];
                        if constexpr (LONG) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) cur[i] = __float_as_uint(sum[i]);
                        } else {
                            tmem_ld32(acc + col0 + p0, cur);
                            tmem_ld_wait();
                            if (p0 + 32 >= cols) {     // the accumulator has been read
                                give_back(buf);
                                given = true;
                            }
                        }
                        with_act(job.e.activation, [&](auto tag) {
                            constexpr int ACT = decltype(tag)::value;
                            constexpr bool W = TILES == 2;
                            if (TILES == 1 && has_z && has_in) finish32<KIND, ACT, OPS, true, true, W, LONG>(cur, job.e, job.N, col + p0, 0, lane, x_scale, to);
                            else if (has_z) finish32<KIND, ACT, OPS, false, true, W, LONG>(cur, job.e, job.N, col + p0, W ? p0 >> 3 : 0, lane, x_scale, to);
                            else if (has_in) finish32<KIND, ACT, OPS, true, false, W, LONG, TABLE>(cur, job.e, job.N, col + p0, p0 >> 3, lane, x_scale, to, table + p0);
                            else finish32<KIND, ACT, OPS, false, false, W, LONG, TABLE>(cur, job.e, job.N, col + p0, p0 >> 3, lane, x_scale, to, table + p0);
                        });
                        if (width == 64 && p0 + 32 < cols) continue;
                        const int at0 = width == 32 ? p0 : 0;  // the tile's first column
                        if (MAP) {
                            fence_proxy_async();
                            __syncwarp();
                            if (lane == 0) {
                                store_box(&maps.y, col + at0, (int)row0, to);
                                if (has_z) store_box(&maps.z, col + at0, (int)row0, to + (TILES == 2 ? kTile : kTile / 2));
                                stores_commit();
                            }
                        } else {
                            __syncwarp();
                            if (own > at0) {
                                const long long where = row0 * job.N + col + at0;
                                copy_tile<true>(to, width == 32, (uint16_t*)job.e.y + where, job.N, rows, min(width, own - at0), lane);
                                if (has_z) copy_tile<true, true>(to + kTile / 2, (uint16_t*)job.e.z + where, job.N, rows, min(width, own - at0), lane);
                            }
                            __syncwarp();
                        }
                    }
                    if (TILES == 2 && !fetched) ++taken;
                }
                if (ok && !given) give_back(buf);      // a warp without a chunk here
                next_chunk();
            }
            if (!ok && ahead && lane == 0) {           // what was asked for ahead lands before this CTA ends
                volatile int ignore = 0;
                landed(taken & 1, &ignore, 200000000LL);
            }
            if (lane == 0) stores_read<0>();
            __syncwarp();
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

// [slow][fast] with rows of `stride` bytes, boxes of box_bytes (128 or 64, swizzled over as many) x box_rows; beyond the tensor zeros are read
bool encode_map(CUtensorMap* map, const void* base, long long fast, long long slow, long long stride, int elem_bytes, int box_rows, int box_bytes = 128) {
    EncodeTiledFn enc = encode_tiled_fn();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)fast, (cuuint64_t)slow};
    const cuuint64_t strides[1] = {(cuuint64_t)stride};
    const cuuint32_t box[2] = {(cuuint32_t)(box_bytes / elem_bytes), (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1u, 1u};
    return enc(map, elem_bytes == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, box_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool PAIR, int KIND, int OPS, bool MAP, int TILES, bool LONG>
cudaError_t launch_one(const Maps& maps, Job& job, int sm_count, cudaStream_t stream) {
    auto kern = linear_kernel<PAIR, KIND, OPS, MAP, TILES, LONG>;
    cudaError_t e = prepare_kernel((const void*)kern, kSmem);
    if (e != cudaSuccess) return e;
    const unsigned units = (unsigned)(job.groups * job.group * job.n_tiles * job.splits), fit = (unsigned)sm_count / (PAIR ? 2 : 1), at_a_time = units < fit ? units : fit;
    job.step = {(int)(at_a_time % job.group), (int)(at_a_time / job.group % job.n_tiles), (int)(at_a_time / job.group / job.n_tiles % job.groups),
                (int)(at_a_time / job.group / job.n_tiles / job.groups)};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = PAIR ? 2 : 1;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(at_a_time * (PAIR ? 2 : 1));
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

// What a kernel's job takes from its plan; `wide`: columns of the output of a tile.  Whether its units can be numbered.
inline bool set_job(Job& job, const LinearPlan& p, int wide, long long M, int N, const LinearEpilogue& epi, float* parts) {
    job.M = M;
    job.N = N;
    job.bn = p.bn;
    job.wide = wide;
    job.m_tiles = p.m_tiles;
    job.n_tiles = p.n_tiles;
    job.group = p.group < p.m_tiles ? p.group : p.m_tiles;
    job.groups = (p.m_tiles + job.group - 1) / job.group;
    job.by_group = Divider((uint32_t)job.group);
    job.by_n_tiles = Divider((uint32_t)p.n_tiles);
    job.by_groups = Divider((uint32_t)job.groups);
    job.splits = p.splits;
    job.k_blocks = p.k_blocks;
    job.kb_per_split = p.kb_per_split;
    job.e = epi;
    job.e.sums = p.splits > 1 ? parts : nullptr;
    return (long long)job.groups * job.group * p.n_tiles * p.splits <= 0x3fffffffLL;
}

}  // namespace
}  // namespace terra
