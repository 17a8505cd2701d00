// New keys and values into a paged cache, queries and keys normed by head and rotated on the way, by positions of one axis or of several: kernel.
#pragma once
#include "cache_append.hpp"
#include "wave_topk.hpp"

namespace dba {

// Weights of the heads' elements: in the data's type or in fp32.
struct WeightsAt {
    const unsigned char *data;         // nullptr: 1 everywhere
    int64_t head;                      // elements; 0: one for all
};

struct NormedParams {
    AppendParams a;                    // position [B, n, axes]
    WeightsAt qw, kw;
    const int32_t *axis;               // of each pair; nullptr: 0
    float eps, per_element;            // 1 / D
    int axes;
    int lanes, lane_bits;              // of a head: a power of two
    int q_units, k_units;              // waves' worths of queries, of keys and of values
};

constexpr int kNormedTokens = 4, kNormedThreads = 256;   // of a workgroup, where there are many

// Sixteen bytes' worth of a head's elements as weights.
template <int FMT, bool WIDE>
struct Weights {
    static constexpr int N = 16 / (int)sizeof(typename Elem<FMT>::type);
    typedef typename Elem<WIDE ? 0 : FMT>::type W;
    struct alignas(16) Vec { W e[N]; } v;
    __device__ __forceinline__ void load(const unsigned char *data, int64_t at) { v = *reinterpret_cast<const Vec *>(reinterpret_cast<const W *>(data) + at); }
    __device__ __forceinline__ void all(float x)
    {
#pragma unroll
        for (int e = 0; e < N; ++e) v.e[e] = (W)x;
    }
    __device__ __forceinline__ float operator[](int e) const { return (float)v.e[e]; }
};

// Over the lanes of a head.
__device__ __forceinline__ float sum_over_lanes(float v, int lanes)
{
    if (lanes > 1) v += __uint_as_float(xor_lane_u32<1, true>(__float_as_uint(v)));
    if (lanes > 2) v += __uint_as_float(xor_lane_u32<2, true>(__float_as_uint(v)));
    if (lanes > 4) v += __uint_as_float(xor_lane_u32<4, true>(__float_as_uint(v)));
    if (lanes > 8) v += __uint_as_float(xor_lane_u32<8, true>(__float_as_uint(v)));
    if (lanes > 16) v += __uint_as_float(xor_lane_u32<16, true>(__float_as_uint(v)));
    return v;
}
__device__ __forceinline__ float max_over_lanes(float v, int lanes)
{
    if (lanes > 1) v = fmaxf(v, __uint_as_float(xor_lane_u32<1, true>(__float_as_uint(v))));
    if (lanes > 2) v = fmaxf(v, __uint_as_float(xor_lane_u32<2, true>(__float_as_uint(v))));
    if (lanes > 4) v = fmaxf(v, __uint_as_float(xor_lane_u32<4, true>(__float_as_uint(v))));
    if (lanes > 8) v = fmaxf(v, __uint_as_float(xor_lane_u32<8, true>(__float_as_uint(v))));
    if (lanes > 16) v = fmaxf(v, __uint_as_float(xor_lane_u32<16, true>(__float_as_uint(v))));
    return v;
}

// y = x / sqrt(mean x^2 + eps) w over a head's D elements, then pairs of y turn as in dba_append_kernel; y stays in fp32 until it is rounded once.
// Squares are added up in fp32, and once more without a power of two that is taken out of all elements where a head's sum leaves the range in which
// that is as good (fp32 and bf16 have elements whose squares pass fp32's range at either end).
//
// A thread has two chunks of 16 bytes at a time (partners of the rotation, or neighbours), a head a power of two of lanes, which add up their squares
// without a trip through LDS.  A wave has queries, keys or values of some heads, so that what differs between them is the same for all of its
// lanes; lanes that have nothing to do read what another one reads.  It goes through the workgroup's TOKENS tokens with the next ones' loads under way: one where there
// are few, for the shortest chain of loads, else several, whose angles the workgroup works out together and which share a wave's weights and addresses.
//
// Bound: HBM; with few tokens the chain of loads and the call.  23000 tokens of 32 + 8 + 8 heads of 128 in fp16 (and 8800 rows of queries that become 0) take 130 us, 4.9 TB/s read and
// written, where torch's copy of as much reaches 5.3; with 1, 2 and 8 tokens a workgroup 165, 169 and 140.  1280 tokens take 11.7 us; with six waves a token
// instead of three, which then do not all find room, 20.9.
template <int FMT, bool NORM, bool WIDE, int TOKENS, bool INTERLEAVED>
__global__ __launch_bounds__(kNormedThreads) void dba_append_normed_kernel(NormedParams np)
{
    typedef typename Elem<FMT>::type E;
    constexpr int N = 16 / (int)sizeof(E);
    struct alignas(16) Vec { E e[N]; };
    __shared__ float2 s_turn[TOKENS][128];
    __shared__ int64_t s_slot[TOKENS];
    const AppendParams &p = np.a;
    const int b = (int)blockIdx.y, i0 = (int)blockIdx.x * TOKENS, t = (int)threadIdx.x, T = (int)blockDim.x;
    const int lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), waves = T >> 6;
    const int chunks = p.D / N, pairs = (chunks + 1) / 2, half = p.rot / 2;
    const int tokens = min(TOKENS, p.n - i0), there = min(tokens, p.count ? max(p.count[b], 0) - i0 : tokens);     // of which the first ones are there
    const int units = np.q_units + 2 * np.k_units, pair = lane & (np.lanes - 1);
#pragma unroll 1
    for (int unit = wave; unit < units; unit += waves) {
        const int kind = unit < np.q_units ? 0 : unit < np.q_units + np.k_units ? 1 : 2;       // queries, keys, values
        const int first = ((unit - (kind == 0 ? 0 : kind == 1 ? np.q_units : np.q_units + np.k_units)) * 64 + lane) >> np.lane_bits;
        const int most = (kind == 0 ? p.q_heads : p.heads) - 1, h = min(first, most);
        const ChunkPair c = chunk_pair(min(pair, pairs - 1), chunks, p.rot / N, INTERLEAVED || kind == 2);
        const bool one = pair < pairs, two = one && c.b >= 0, mine = one && first <= most, turns = kind < 2 && c.a * N < p.rot;    // (and then the second chunk does, too: rot is a multiple of 16)
        const int cb = c.b < 0 ? c.a : c.b;
        const HeadsAt &from = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
        const E *src = reinterpret_cast<const E *>(from.data) + ((int64_t)b * from.sent + (int64_t)i0 * from.token + (int64_t)h * from.head);
        E *to = kind == 0 ? reinterpret_cast<E *>(p.q_out.data) + ((int64_t)b * p.q_out.sent + (int64_t)i0 * p.q_out.token + (int64_t)h * p.q_out.head)
                          : reinterpret_cast<E *>(kind == 1 ? p.k_pages : p.v_pages) + (int64_t)h * p.cache.head_stride;
        Vec next[2] = {};
        if (there > 0) {
            next[0] = *reinterpret_cast<const Vec *>(src + c.a * N);
            next[1] = *reinterpret_cast<const Vec *>(src + cb * N);
        }
        Weights<FMT, WIDE> w[2];
        const WeightsAt &of = kind == 0 ? np.qw : np.kw;
        const bool weighted = NORM && kind < 2 && of.data;
        if (weighted) {
            w[0].load(of.data, h * of.head + c.a * N);
            w[1].load(of.data, h * of.head + cb * N);
        } else {
            w[0].all(1.0f);
            w[1].all(1.0f);
        }
        if (unit == wave) {                             // what all units need
#pragma unroll 1
            for (int x = t; x < half * there; x += T) {
                const int token = TOKENS == 1 ? 0 : x / half, j = x - token * half;
                const int axis = np.axis ? np.axis[j] : 0;
                const int64_t i = (int64_t)i0 + token;
                if ((uint32_t)axis < (uint32_t)np.axes)
                    s_turn[token][j] = turn_of(p.position ? p.position[((int64_t)b * p.n + i) * np.axes + axis] : p.first[b] + i, p.inv_freq[j]);
                else s_turn[token][j] = make_float2(1.0f, 0.0f);
            }
            if (t < TOKENS) s_slot[t] = t < there ? token_offset(p.cache, b, (int64_t)p.first[b] + i0 + t) : -1;
            __syncthreads();
        }
#pragma unroll 1
        for (int token = 0; token < tokens; ++token) {
            Vec raw[2] = {next[0], next[1]};
            src += from.token;
            if (token + 1 < there) {
                next[0] = *reinterpret_cast<const Vec *>(src + c.a * N);
                next[1] = *reinterpret_cast<const Vec *>(src + cb * N);
            }
            if (token >= there) {                       // no such token: its queries are 0
                if (kind != 0) break;
                raw[0] = raw[1] = Vec{};
            } else if (kind < 2) {
                float y[2][N];
#pragma unroll
                for (int z = 0; z < 2; ++z)
#pragma unroll
                    for (int e = 0; e < N; ++e) y[z][e] = (float)raw[z].e[e];
                if constexpr (NORM) {
                    float sum[2] = {0.0f, 0.0f};
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        sum[0] = fmaf(y[0][e], y[0][e], sum[0]);
                        sum[1] = fmaf(y[1][e], y[1][e], sum[1]);
                    }
                    const float all = sum_over_lanes((one ? sum[0] : 0.0f) + (two ? sum[1] : 0.0f), np.lanes);
                    const float mean = fmaf(all, np.per_element, np.eps);
                    float f = __builtin_amdgcn_rsqf(mean);  // good to a step of fp32
                    if constexpr (FMT != 1) {           // (squares of fp16 stay well inside)
                        if (__any(!((all > 1e-30f && all < 1e36f) || all == 0.0f))) {      // rare: a power of two is taken out first
                            float most_of = 0.0f;
#pragma unroll
                            for (int e = 0; e < N; ++e) most_of = fmaxf(most_of, fmaxf(fabsf(y[0][e]), fabsf(y[1][e])));
                            most_of = max_over_lanes(most_of, np.lanes);
                            const int exponent = min(max((int)(__float_as_uint(most_of) >> 23), 1), 253);
                            const float g = __uint_as_float((uint32_t)(254 - exponent) << 23);
                            sum[0] = sum[1] = 0.0f;
#pragma unroll
                            for (int e = 0; e < N; ++e) {
                                y[0][e] *= g;
                                y[1][e] *= g;
                                sum[0] = fmaf(y[0][e], y[0][e], sum[0]);
                                sum[1] = fmaf(y[1][e], y[1][e], sum[1]);
                            }
                            const float scaled = sum_over_lanes((one ? sum[0] : 0.0f) + (two ? sum[1] : 0.0f), np.lanes);
                            f = (float)__builtin_amdgcn_rsq((double)scaled * np.per_element + (double)np.eps * g * g);     // (an infinity leaves 0 of the others)
                        }
                    }
#pragma unroll
                    for (int z = 0; z < 2; ++z)
#pragma unroll
                        for (int e = 0; e < N; ++e) y[z][e] = y[z][e] * f * w[z][e];
                }
                if (turns && !INTERLEAVED) {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float2 r = s_turn[token][c.a * N + e];
                        const float y0 = y[0][e], y1 = y[1][e];
                        y[0][e] = y0 * r.x - y1 * r.y;
                        y[1][e] = y1 * r.x + y0 * r.y;
                    }
                } else if (turns) {
#pragma unroll
                    for (int x = 0; x < 2 * N; x += 2) {
                        const float2 r = s_turn[token][(c.a * N + x) / 2];
                        const float y0 = y[x / N][x % N], y1 = y[x / N][x % N + 1];
                        y[x / N][x % N] = y0 * r.x - y1 * r.y;
                        y[x / N][x % N + 1] = y1 * r.x + y0 * r.y;
                    }
                }
#pragma unroll
                for (int z = 0; z < 2; ++z)
#pragma unroll
                    for (int e = 0; e < N; ++e) raw[z].e[e] = (E)y[z][e];
            }
            const int64_t slot = kind == 0 ? 0 : s_slot[token];
            E *const at = to + slot;
            if (mine && slot >= 0) {
                *reinterpret_cast<Vec *>(at + c.a * N) = raw[0];
                if (two) *reinterpret_cast<Vec *>(at + c.b * N) = raw[1];
            }
            if (kind == 0) to += p.q_out.token;
        }
    }
}

}  // namespace dba
