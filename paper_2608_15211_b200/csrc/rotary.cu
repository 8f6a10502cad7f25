// Rotary positions of queries and keys: the first `rot` channels of each head are rot / 2 pairs, and pair p is turned by position x freq[p]
//   a' = a cos - b sin,  b' = a sin + b cos   (both times `scale`; the inverse turn has -sin),
// where the pair is channels (p, p + rot / 2) or (2 p, 2 p + 1).  The first row_pairs pairs go by the token's row, the others by its column, in the
// frame that the windows tile ((u - shift) mod H: the tokens of a window that lies over the seam have consecutive positions), or by given positions.
//
// A block takes a few tokens: first the angles of all their pairs (in fp64: position 10^7 times a frequency leaves fp32 no digit behind
// the point; reduced to half a turn, then cos and sin in fp32) into shared memory, once for all heads of q and k, then the heads by 16-byte
// accesses.  A thread reads all that it writes before it writes, so the outputs may be the inputs.
// What bounds it: HBM.
#include "block_kernels.h"

#ifdef TERRA_ELEM_F16
#define launch_rotary launch_rotary_f16
#endif

namespace terra {
namespace {

constexpr int kBlock = 256;
constexpr int kMaxTokens = 64, kMaxAngles = 2048;     // of a block
constexpr int kMaxHeads = 128;                        // of a block: more go to other blocks

template <int E> struct Words;                        // E elements as they lie in memory
template <> struct Words<8> { uint4 v; };
template <> struct Words<2> { uint32_t v; };
template <> struct Words<1> { uint16_t v; };

__device__ __forceinline__ void floats(const Words<8>& r, float (&f)[8]) {
    const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 t = elem2_to_float2(w[i]); f[2 * i] = t.x; f[2 * i + 1] = t.y; }
}
__device__ __forceinline__ void floats(const Words<2>& r, float (&f)[2]) { const float2 t = elem2_to_float2(r.v); f[0] = t.x; f[1] = t.y; }
__device__ __forceinline__ void floats(const Words<1>& r, float (&f)[1]) { f[0] = elem2_to_float2(r.v).x; }
__device__ __forceinline__ Words<8> words(const float (&f)[8]) {
    return {make_uint4(pack_elem(f[0], f[1]), pack_elem(f[2], f[3]), pack_elem(f[4], f[5]), pack_elem(f[6], f[7]))};
}
__device__ __forceinline__ Words<2> words(const float (&f)[2]) { return {pack_elem(f[0], f[1])}; }
__device__ __forceinline__ Words<1> words(const float (&f)[1]) { return {(uint16_t)pack_elem(f[0], 0.f)}; }

struct Deal {                      // how a block's work is cut up
    int tokens, heads;             // of a block
    int turned, items;             // items of a head: the first `turned` are turned, the others copied
    int tensors;
    Divider per_token, per_head, pairs;
};

// An item is E channels and, for HALF, the E channels rot / 2 further on (one run of E to be copied behind the turned ones).
template <int E, bool HALF>
__global__ void __launch_bounds__(kBlock) rotary_kernel(const RotaryArgs a, const Deal deal) {
    __shared__ float2 turn[kMaxAngles];
    const int pairs = a.rot >> 1;
    const long long token0 = (long long)blockIdx.x * deal.tokens;
    const int nt = (int)min((long long)deal.tokens, a.tokens - token0);
    const int head0 = blockIdx.y * deal.heads, nh = min(deal.heads, a.heads - head0);
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
    const uint32_t total = (uint32_t)nt * deal.per_token.d;
    constexpr int B = HALF ? 2 : 4;          // items in flight: 4 loads either way
    for (uint32_t i0 = threadIdx.x; i0 < total; i0 += B * kBlock) {
        Words<E> lo[B], hi[B];
        uint16_t* dst[B];
        int angle0[B], job[B];               // job: 0 nothing, 1 copy, 2 turn; interleaved: 2 + the first pair
#pragma unroll
        for (int k = 0; k < B; ++k) {
            const uint32_t i = i0 + k * kBlock;
            job[k] = 0;
            if (i < total) {
                uint32_t t, rem, th, j;
                deal.per_token.split(i, t, rem);
                deal.per_head.split(rem, th, j);
                const bool key = (int)th >= deal.heads;
                const int head = (int)th - (key ? deal.heads : 0);
                if (head < nh) {
                    const bool turned = (int)j < deal.turned;
                    const int ch = (HALF && !turned ? a.rot + ((int)j - deal.turned) * E : (int)j * E) + (head0 + head) * a.d;
                    const uint16_t* src = (const uint16_t*)(key ? a.k : a.q) + (token0 + t) * a.stride + ch;
                    dst[k] = (uint16_t*)(key ? a.k_out : a.q_out) + (token0 + t) * a.stride_out + ch;
                    job[k] = turned ? 2 : 1;
                    angle0[k] = (int)t * pairs + (int)j * (HALF ? E : E / 2);
                    if (!HALF) job[k] = turned ? 2 + (int)j * (E / 2) : 1;
                    lo[k] = *reinterpret_cast<const Words<E>*>(src);
                    if (HALF && turned) hi[k] = *reinterpret_cast<const Words<E>*>(src + pairs);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < B; ++k) {
            if (job[k] == 0) continue;
            if (job[k] == 1) {
                *reinterpret_cast<Words<E>*>(dst[k]) = lo[k];
                continue;
            }
            float x[E];
            floats(lo[k], x);
            if (HALF) {
                float y[E];
                floats(hi[k], y);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float2 cs = turn[angle0[k] + e];
                    const float p = x[e], q = y[e];
                    x[e] = p * cs.x - q * cs.y;
                    y[e] = p * cs.y + q * cs.x;
                }
                *reinterpret_cast<Words<E>*>(dst[k]) = words(x);
                *reinterpret_cast<Words<E>*>(dst[k] + pairs) = words(y);
            } else {
#pragma unroll
                for (int e = 0; e + 1 < E; e += 2) {
                    if (job[k] - 2 + e / 2 < pairs) {        // the last turned vector may hold channels behind the turned ones
                        const float2 cs = turn[angle0[k] + e / 2];
                        const float p = x[e], q = x[e + 1];
                        x[e] = p * cs.x - q * cs.y;
                        x[e + 1] = p * cs.y + q * cs.x;
                    }
                }
                *reinterpret_cast<Words<E>*>(dst[k]) = words(x);
            }
        }
    }
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, int sm_count, cudaStream_t stream) {
    const int pairs = a.rot / 2;
    const int E = a.interleaved || pairs % 8 == 0 ? 8 : pairs % 2 == 0 ? 2 : 1;
    const bool in_place = a.q == a.q_out && a.stride == a.stride_out && (!a.k || a.k == a.k_out);
    const int turned = a.interleaved ? (a.rot + 7) / 8 : pairs / E;
    const int copied = in_place ? 0 : a.interleaved ? a.d / 8 - turned : (a.d - a.rot) / E;
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
    const Deal deal{(int)tokens, heads, turned, turned + copied, tensors, Divider((uint32_t)per_token), Divider((uint32_t)(turned + copied)),
                    Divider((uint32_t)pairs)};
    const long long blocks = (a.tokens + tokens - 1) / tokens;
    if (blocks > 0x7fffffffLL || head_blocks > 65535) return cudaErrorInvalidConfiguration;
    auto kern = a.interleaved ? rotary_kernel<8, false> : E == 8 ? rotary_kernel<8, true> : E == 2 ? rotary_kernel<2, true> : rotary_kernel<1, true>;
    prof_begin("rotary_kernel", stream);
    kern<<<dim3((unsigned)blocks, (unsigned)head_blocks), kBlock, 0, stream>>>(a, deal);
    count_launch(stream);
    return cudaGetLastError();
}

}  // namespace terra
