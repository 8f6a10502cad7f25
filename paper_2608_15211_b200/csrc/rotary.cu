// Rotary positions of queries and keys: the first `rot` channels of each head are rot / 2 pairs, and pair p is turned by position x freq[p]
//   a' = a cos - b sin,  b' = a sin + b cos   (both times `scale`; the inverse turn has -sin),
// where the pair is channels (p, p + rot / 2) or (2 p, 2 p + 1).  The first row_pairs pairs go by the token's row, the others by its column, in the
// frame that the windows tile ((u - shift) mod H: the tokens of a window that lies over the seam have consecutive positions), or by given positions.
//
// A block takes a few tokens: first the angles of all their pairs (in fp64: position 10^7 times a frequency leaves fp32 no digit behind
// the point; reduced to half a turn, then cos and sin in fp32) into shared memory, once for all heads of q and k, then the heads by 16-byte
// accesses.  A thread reads all that it writes before it writes, so the outputs may be the inputs.
// What bounds it: HBM (510 x 1080 tokens, 12 x 32, 257 us, 6.6 TB/s; 288 x 544, 32 x 128, half of the channels interleaved, 850 us, 6.0 TB/s).
#include "block_kernels.h"

#ifdef TERRA_ELEM_F16
#define launch_rotary launch_rotary_f16
#endif

namespace terra {
namespace {

constexpr int kBlock = 256;
constexpr int kMaxTokens = 64, kMaxAngles = 2048;     // of a block
constexpr int kMaxHeads = 128;                        // of a block: more go to other blocks

__device__ __forceinline__ void floats(const uint4& r, float (&f)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 t = elem2_to_float2(w[i]); f[2 * i] = t.x; f[2 * i + 1] = t.y; }
}
__device__ __forceinline__ uint4 words(const float (&f)[8]) {
    return make_uint4(pack_elem(f[0], f[1]), pack_elem(f[2], f[3]), pack_elem(f[4], f[5]), pack_elem(f[6], f[7]));
}

// Eight consecutive channels, the first n of them, from an address that is a multiple of A elements
template <int A>
__device__ __forceinline__ uint4 read8(const uint16_t* p, int n) {
    if (A == 8 && n == 8) return *reinterpret_cast<const uint4*>(p);
    uint32_t w[4] = {0, 0, 0, 0};
    if (A >= 2 && n == 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int A>
__device__ __forceinline__ void write8(uint16_t* p, int n, const uint4& v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if (A == 8 && n == 8) {
        *reinterpret_cast<uint4*>(p) = v;
    } else if (A >= 2 && n == 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(p)[i] = w[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
}

struct Deal {                      // how a block's work is cut up
    int tokens, heads;             // of a block
    int turned;                    // items of a head: the first `turned` are turned, the others copied
    int copied_from;               // first channel of the copied items
    Divider per_token, per_head, pairs;
};

// An item is 8 channels and, for HALF, the 8 channels rot / 2 further on, which start at a multiple of A elements.  What lies between the turned
// channels and the next 16 bytes goes with the last turned item.
template <int A, bool HALF>
__global__ void __launch_bounds__(kBlock) rotary_kernel(const RotaryArgs a, const Deal deal) {
    __shared__ float2 turn[kMaxAngles];
    const int pairs = a.rot >> 1;
    const long long token0 = (long long)blockIdx.x * deal.tokens;
    const int nt = (int)min((long long)deal.tokens, a.tokens - token0);
    const int head0 = blockIdx.y * deal.heads, nh = min(deal.heads, a.heads - head0);
    const uint32_t total = (uint32_t)nt * deal.per_token.d;
    constexpr int B = HALF ? 2 : 4;          // items in flight: 4 loads either way
    uint4 lo[B], hi[B];
    const uint16_t* src[B];
    uint16_t* dst[B];
    int angle0[B], n[B];                 // n: pairs to be turned; 0 a copy, -1 nothing
    auto fetch = [&](uint32_t i0) {
#pragma unroll
        for (int k = 0; k < B; ++k) {
            const uint32_t i = i0 + k * kBlock;
            n[k] = -1;
            if (i < total) {
                uint32_t t, rem, th, j;
                deal.per_token.split(i, t, rem);
                deal.per_head.split(rem, th, j);
                const bool key = (int)th >= deal.heads;
                const int head = (int)th - (key ? deal.heads : 0);
                if (head < nh) {
                    const bool turned = (int)j < deal.turned;
                    const int ch = (turned ? (int)j * 8 : deal.copied_from + ((int)j - deal.turned) * 8) + (head0 + head) * a.d;
                    src[k] = (const uint16_t*)(key ? a.k : a.q) + (token0 + t) * a.stride + ch;
                    dst[k] = (uint16_t*)(key ? a.k_out : a.q_out) + (token0 + t) * a.stride_out + ch;
                    const int first = (int)j * (HALF ? 8 : 4);       // pair
                    n[k] = turned ? min(HALF ? 8 : 4, pairs - first) : 0;
                    angle0[k] = (int)t * pairs + first;
                    if (HALF && n[k] > 0) {
                        lo[k] = read8<8>(src[k], A == 8 ? 8 : n[k]);
                        hi[k] = read8<A>(src[k] + pairs, A == 8 ? 8 : n[k]);
                    } else {
                        lo[k] = read8<8>(src[k], 8);
                    }
                }
            }
        }
    };
    // the first items' reads are under way while the angles are worked out (510 x 1080 x 12 x 32: 264 -> 257 us; interleaved it is slower, 309 -> 343)
    if (HALF) fetch(threadIdx.x);
    const long long grid = (long long)a.H * a.W;
    for (uint32_t i = threadIdx.x; i < (uint32_t)(nt * pairs); i += kBlock) {
        uint32_t t, p;
        deal.pairs.split(i, t, p);
        const long long token = token0 + t;
        int pos;
        if (a.positions) {
            pos = a.positions[2 * token + ((int)p < a.row_pairs ? 0 : 1)];
        } else {
            const int at = (int)(token % grid), u = at / a.W, v = at - u * a.W;
            if ((int)p < a.row_pairs) pos = u >= a.sh ? u - a.sh : u - a.sh + a.H;
            else pos = v >= a.sw ? v - a.sw : v - a.sw + a.W;
        }
        const double turns = (double)pos * a.freq[p] * 0.15915494309189535;       // 1 / (2 pi)
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        turn[i] = make_float2(c * a.scale, (a.inverse ? -s : s) * a.scale);
    }
    __syncthreads();
    for (uint32_t i0 = threadIdx.x; i0 < total;) {
        if (!HALF) fetch(i0);
#pragma unroll
        for (int k = 0; k < B; ++k) {
            if (n[k] < 0) continue;
            if (n[k] == 0) {
                write8<8>(dst[k], 8, lo[k]);
                continue;
            }
            float x[8];
            floats(lo[k], x);
            if (HALF) {
                float y[8];
                floats(hi[k], y);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 cs = turn[angle0[k] + (A == 8 ? e : min(e, n[k] - 1))];
                    const float p = x[e], q = y[e];
                    x[e] = p * cs.x - q * cs.y;
                    y[e] = p * cs.y + q * cs.x;
                }
                write8<8>(dst[k], A == 8 ? 8 : n[k], words(x));
                write8<A>(dst[k] + pairs, A == 8 ? 8 : n[k], words(y));
                if (A < 8 && src[k] != dst[k] && n[k] == pairs - (angle0[k] % pairs)) {          // the last turned item: up to the copied ones
                    const int at = angle0[k] % pairs;                                            // its first channel in the head
                    for (int c = a.rot; c < deal.copied_from; ++c) dst[k][c - at] = src[k][c - at];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    if (e / 2 < n[k]) {      // (the last vector may hold channels behind the turned ones)
                        const float2 cs = turn[angle0[k] + e / 2];
                        const float p = x[e], q = x[e + 1];
                        x[e] = p * cs.x - q * cs.y;
                        x[e + 1] = p * cs.y + q * cs.x;
                    }
                }
                write8<8>(dst[k], 8, words(x));
            }
        }
        i0 += B * kBlock;
        if (HALF && i0 < total) fetch(i0);
    }
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, int sm_count, cudaStream_t stream) {
    const int pairs = a.rot / 2;
    const bool in_place = a.q == a.q_out && a.stride == a.stride_out && (!a.k || a.k == a.k_out);
    const int turned = a.interleaved ? (a.rot + 7) / 8 : (pairs + 7) / 8, copied_from = (a.rot + 7) / 8 * 8, copied = in_place ? 0 : (a.d - copied_from) / 8;
    const int tensors = a.k ? 2 : 1, heads = a.heads < kMaxHeads ? a.heads : kMaxHeads;
    const int head_blocks = (a.heads + heads - 1) / heads;
    // tokens of a block: as many as give each thread two batches of loads, fewer where that leaves SMs without a block
    const int per_token = tensors * heads * (turned + copied);
    long long tokens = (2 * 4 * kBlock + per_token - 1) / per_token;
    const long long spread = a.tokens * head_blocks / (2 * sm_count);
    if (tokens > spread) tokens = spread;
    if (tokens > kMaxTokens) tokens = kMaxTokens;
    if (tokens > kMaxAngles / pairs) tokens = kMaxAngles / pairs;
    if (tokens < 1) tokens = 1;
    const Deal deal{(int)tokens, heads, turned, copied_from, Divider((uint32_t)per_token), Divider((uint32_t)(turned + copied)), Divider((uint32_t)pairs)};
    const long long blocks = (a.tokens + tokens - 1) / tokens;
    if (blocks > 0x7fffffffLL || head_blocks > 65535) return cudaErrorInvalidConfiguration;
    auto kern = a.interleaved ? rotary_kernel<8, false> : pairs % 8 == 0 ? rotary_kernel<8, true> : pairs % 2 == 0 ? rotary_kernel<2, true> : rotary_kernel<1, true>;
    prof_begin("rotary_kernel", stream);
    kern<<<dim3((unsigned)blocks, (unsigned)head_blocks), kBlock, 0, stream>>>(a, deal);
    count_launch(stream);
    return cudaGetLastError();
}

}  // namespace terra
