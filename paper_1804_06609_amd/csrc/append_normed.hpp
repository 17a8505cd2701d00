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
    double eps;
    int axes;
    int lanes, lane_bits;              // of a head: a power of two
};

template <int FMT, bool WIDE>
__device__ __forceinline__ void load_weights(float (&w)[16 / sizeof(typename Elem<FMT>::type)], const unsigned char *data, int64_t at)
{
    constexpr int N = 16 / (int)sizeof(typename Elem<FMT>::type);
    typedef float f32x4_t __attribute__((ext_vector_type(4)));
    if constexpr (WIDE || FMT == 0) {
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const f32x4_t v = *reinterpret_cast<const f32x4_t *>(reinterpret_cast<const float *>(data) + at + e);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[e + j] = v[j];
        }
    } else {
        typedef typename Elem<FMT>::type E;
        struct alignas(16) Vec { E e[N]; };
        const Vec v = *reinterpret_cast<const Vec *>(reinterpret_cast<const E *>(data) + at);
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = (float)v.e[e];
    }
}

template <int J>
__device__ __forceinline__ double xor_lane_double(double v) { return __longlong_as_double((long long)xor_lane_t<u64, J, true>((u64)__double_as_longlong(v))); }

// y = x / sqrt(mean x^2 + eps) w over a head's D elements, then pairs of y turn as in dba_append_kernel; y stays in fp32 until it is rounded once.
// Squares are added up in 64 bits: those of fp32 and bf16 pass fp32's range, and none of it shows (memory bounds).
//
// One workgroup per token, a thread for every two chunks of 16 bytes (partners of the rotation, or neighbours), and a power of two of lanes
// a head, which add up their squares without a trip through LDS.
template <int FMT, bool NORM, bool WIDE>
__global__ __launch_bounds__(kAppendThreads) void dba_append_normed_kernel(NormedParams np)
{
    typedef typename Elem<FMT>::type E;
    constexpr int N = 16 / (int)sizeof(E), U = 2;      // pairs a thread has under way
    struct alignas(16) Vec { E e[N]; };
    __shared__ float2 s_turn[128];
    const AppendParams &p = np.a;
    const int b = (int)blockIdx.y, i = (int)blockIdx.x, t = (int)threadIdx.x, T = (int)blockDim.x;
    const bool there = !p.count || i < p.count[b];
    const int64_t at = (int64_t)p.first[b] + i;
    const int64_t slot = there ? token_offset(p.cache, b, at) : -1;
    const int chunks = p.D / N, pairs = (chunks + 1) / 2, half = p.rot / 2, heads = p.q_heads + 2 * p.heads;
    const int items = heads << np.lane_bits;
    for (int x0 = 0; x0 < items; x0 += U * T) {
        Vec raw[U][2];
        float w[U][2][N];
        E *to[U];
        ChunkPair c[U];
        bool turns[U], norms[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = x0 + u * T + t, head = x >> np.lane_bits, pair = x & (np.lanes - 1);
            to[u] = nullptr;
            raw[u][0] = raw[u][1] = Vec{};
            c[u] = {0, -1};
            turns[u] = norms[u] = false;
            if (x >= items || pair >= pairs) continue;
            const bool is_q = head < p.q_heads, is_v = head >= p.q_heads + p.heads;
            const int h = is_q ? head : is_v ? head - p.q_heads - p.heads : head - p.q_heads;
            const HeadsAt &from = is_q ? p.q : is_v ? p.v : p.k;
            c[u] = chunk_pair(pair, chunks, p.rot / N, p.interleaved || is_v);
            turns[u] = there && !is_v && c[u].a * N < p.rot;
            norms[u] = NORM && there && !is_v;
            if (is_q) to[u] = reinterpret_cast<E *>(p.q_out.data) + ((int64_t)b * p.q_out.sent + (int64_t)i * p.q_out.token + (int64_t)h * p.q_out.head);
            else if (slot >= 0) to[u] = reinterpret_cast<E *>(is_v ? p.v_pages : p.k_pages) + (slot + (int64_t)h * p.cache.head_stride);
            if (!there) continue;
            const E *src = reinterpret_cast<const E *>(from.data) + ((int64_t)b * from.sent + (int64_t)i * from.token + (int64_t)h * from.head);
            raw[u][0] = *reinterpret_cast<const Vec *>(src + c[u].a * N);
            if (c[u].b >= 0) raw[u][1] = *reinterpret_cast<const Vec *>(src + c[u].b * N);
            if constexpr (NORM) {
                const WeightsAt &weights = is_q ? np.qw : np.kw;
#pragma unroll
                for (int e = 0; e < N; ++e) w[u][0][e] = w[u][1][e] = 1.0f;
                if (!is_v && weights.data) {
                    load_weights<FMT, WIDE>(w[u][0], weights.data, h * weights.head + c[u].a * N);
                    if (c[u].b >= 0) load_weights<FMT, WIDE>(w[u][1], weights.data, h * weights.head + c[u].b * N);
                }
            }
        }
        if (x0 == 0) {
            if (there)
                for (int j = t; j < half; j += T) {
                    const int axis = np.axis ? np.axis[j] : 0;
                    if ((uint32_t)axis < (uint32_t)np.axes)
                        s_turn[j] = turn_of(p.position ? p.position[((int64_t)b * p.n + i) * np.axes + axis] : at, p.inv_freq[j]);
                    else s_turn[j] = make_float2(1.0f, 0.0f);
                }
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float y[2][N];
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
                for (int e = 0; e < N; ++e) y[z][e] = (float)raw[u][z].e[e];
            if constexpr (NORM) {
                double sum[2] = {0.0, 0.0};
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    sum[0] = fma((double)y[0][e], (double)y[0][e], sum[0]);
                    sum[1] = fma((double)y[1][e], (double)y[1][e], sum[1]);
                }
                double all = sum[0] + sum[1];
                if (np.lanes > 1) all += xor_lane_double<1>(all);
                if (np.lanes > 2) all += xor_lane_double<2>(all);
                if (np.lanes > 4) all += xor_lane_double<4>(all);
                if (np.lanes > 8) all += xor_lane_double<8>(all);
                if (np.lanes > 16) all += xor_lane_double<16>(all);
                if (norms[u]) {
                    const double mean = all / p.D + np.eps;
                    double r = __builtin_amdgcn_rsq(mean);      // good to 2^-23; one step of Newton's squares that
                    if (mean < 1e300) r = r * (1.5 - 0.5 * mean * r * r);      // (an infinity among them leaves 0 of the others)
                    const bool large = mean > 0x1p120;          // there r would leave fp32's normal numbers
                    const float f = (float)(large ? r * 0x1p64 : r), g = large ? 0x1p-64f : 1.0f;
#pragma unroll
                    for (int z = 0; z < 2; ++z)
#pragma unroll
                        for (int e = 0; e < N; ++e) y[z][e] = y[z][e] * g * f * w[u][z][e];
                }
            }
            if (!to[u]) continue;
            if (turns[u] && !p.interleaved) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float2 r = s_turn[c[u].a * N + e];
                    const float y0 = y[0][e], y1 = y[1][e];
                    y[0][e] = y0 * r.x - y1 * r.y;
                    y[1][e] = y1 * r.x + y0 * r.y;
                }
            } else if (turns[u]) {
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const int chunk = z ? c[u].b : c[u].a;
                    if (chunk < 0 || chunk * N >= p.rot) continue;
#pragma unroll
                    for (int e = 0; e < N; e += 2) {
                        const float2 r = s_turn[(chunk * N + e) / 2];
                        const float y0 = y[z][e], y1 = y[z][e + 1];
                        y[z][e] = y0 * r.x - y1 * r.y;
                        y[z][e + 1] = y1 * r.x + y0 * r.y;
                    }
                }
            }
            if (turns[u] || norms[u]) {
#pragma unroll
                for (int z = 0; z < 2; ++z)
#pragma unroll
                    for (int e = 0; e < N; ++e) raw[u][z].e[e] = (E)y[z][e];
            }
            *reinterpret_cast<Vec *>(to[u] + c[u].a * N) = raw[u][0];
            if (c[u].b >= 0) *reinterpret_cast<Vec *>(to[u] + c[u].b * N) = raw[u][1];
        }
    }
}

}  // namespace dba
