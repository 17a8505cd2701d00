// New keys and values into a paged cache, rotated on the way: kernel.
#pragma once
#include "paged.hpp"

namespace dba {

template <int FMT> struct Elem;
template <> struct Elem<0> { typedef float type; };
template <> struct Elem<1> { typedef _Float16 type; };
template <> struct Elem<2> { typedef __bf16 type; };

struct HeadsAt {
    unsigned char *data;
    int64_t sent, token, head;         // elements
};

struct AppendParams {
    Paged cache;
    unsigned char *k_pages, *v_pages;
    HeadsAt q, q_out, k, v;
    const int32_t *first, *count, *position;
    const float *inv_freq;
    int n, heads, q_heads, D, rot, interleaved;
};

constexpr int kAppendThreads = 256;

// cos and sin of position * inv_freq.  The angle in turns is formed and reduced in 64 bits: a position of a million leaves an fp32
// angle no better than 0.06 radians.
__device__ __forceinline__ float2 turn_of(int64_t position, float inv_freq)
{
    const double turns = (double)position * ((double)inv_freq * 0.159154943091895335768883763);
    const float x = (float)(2.0 * (turns - rint(turns)));      // in half turns
    float s, c;
    sincospif(x, &s, &c);
    return make_float2(c, s);
}

// Two chunks of 16 bytes of one head, which one thread moves: partners of the rotation, or neighbours.
struct ChunkPair {
    int a, b;                          // -1: none
};
__device__ __forceinline__ ChunkPair chunk_pair(int i, int chunks, int rotated, bool neighbours)
{
    if (!neighbours && i < rotated / 2) return {i, i + rotated / 2};
    return {2 * i, 2 * i + 1 < chunks ? 2 * i + 1 : -1};
}

// One workgroup per token: its angles once, then all its heads.  Bound: HBM; at few tokens the chain of loads.  What a thread moves is
// asked for before the angles are worked out (1280 tokens of 32 + 8 + 8 heads of 128 in bf16: 21.6 -> 9.5 us; prompts of 23000 tokens in
// fp16, 139 -> 120 us, 4.8 TB/s read and written; torch's copy of as much reaches 5.4).
template <int FMT>
__global__ __launch_bounds__(kAppendThreads) void dba_append_kernel(AppendParams p)
{
    typedef typename Elem<FMT>::type E;
    constexpr int N = 16 / (int)sizeof(E), U = 2;      // pairs a thread has under way
    struct alignas(16) Vec { E e[N]; };
    __shared__ float2 s_turn[128];
    const int b = (int)blockIdx.y, i = (int)blockIdx.x, t = (int)threadIdx.x, T = (int)blockDim.x;
    const bool there = !p.count || i < p.count[b];
    const int64_t at = (int64_t)p.first[b] + i;
    const int64_t position = p.position ? p.position[(int64_t)b * p.n + i] : at;       // (first + i may pass 2^31: such a token has no place, but a query)
    const int64_t slot = there ? token_offset(p.cache, b, at) : -1;
    const int chunks = p.D / N, pairs = (chunks + 1) / 2, half = p.rot / 2, heads = p.q_heads + 2 * p.heads;
    const int items = heads * pairs;
    for (int x0 = 0; x0 < items; x0 += U * T) {
        Vec lo[U], hi[U];
        E *to[U];
        ChunkPair c[U];
        bool rotates[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = x0 + u * T + t, head = x / pairs;
            to[u] = nullptr;
            lo[u] = hi[u] = Vec{};
            c[u] = {0, -1};
            rotates[u] = false;
            if (x >= items) continue;
            const bool is_q = head < p.q_heads, is_v = head >= p.q_heads + p.heads;
            const int h = is_q ? head : is_v ? head - p.q_heads - p.heads : head - p.q_heads;
            const HeadsAt &from = is_q ? p.q : is_v ? p.v : p.k;
            c[u] = chunk_pair(x - head * pairs, chunks, p.rot / N, p.interleaved || is_v);
            rotates[u] = there && !is_v && c[u].a * N < p.rot;
            if (is_q) to[u] = reinterpret_cast<E *>(p.q_out.data) + ((int64_t)b * p.q_out.sent + (int64_t)i * p.q_out.token + (int64_t)h * p.q_out.head);
            else if (slot >= 0) to[u] = reinterpret_cast<E *>(is_v ? p.v_pages : p.k_pages) + (slot + (int64_t)h * p.cache.head_stride);
            if (!there) continue;
            const E *src = reinterpret_cast<const E *>(from.data) + ((int64_t)b * from.sent + (int64_t)i * from.token + (int64_t)h * from.head);
            lo[u] = *reinterpret_cast<const Vec *>(src + c[u].a * N);
            if (c[u].b >= 0) hi[u] = *reinterpret_cast<const Vec *>(src + c[u].b * N);
        }
        if (x0 == 0) {
            if (there)
                for (int j = t; j < half; j += T) s_turn[j] = turn_of(position, p.inv_freq[j]);
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!to[u]) continue;
            if (rotates[u] && !p.interleaved) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float2 r = s_turn[c[u].a * N + e];
                    const float x0f = (float)lo[u].e[e], x1f = (float)hi[u].e[e];
                    lo[u].e[e] = (E)(x0f * r.x - x1f * r.y);
                    hi[u].e[e] = (E)(x1f * r.x + x0f * r.y);
                }
            } else if (rotates[u]) {
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    const float2 r = s_turn[(c[u].a * N + e) / 2];
                    const float x0f = (float)lo[u].e[e], x1f = (float)lo[u].e[e + 1];
                    lo[u].e[e] = (E)(x0f * r.x - x1f * r.y);
                    lo[u].e[e + 1] = (E)(x1f * r.x + x0f * r.y);
                    if (c[u].b >= 0 && c[u].b * N < p.rot) {
                        const float2 s = s_turn[(c[u].b * N + e) / 2];
                        const float y0 = (float)hi[u].e[e], y1 = (float)hi[u].e[e + 1];
                        hi[u].e[e] = (E)(y0 * s.x - y1 * s.y);
                        hi[u].e[e + 1] = (E)(y1 * s.x + y0 * s.y);
                    }
                }
            }
            *reinterpret_cast<Vec *>(to[u] + c[u].a * N) = lo[u];
            if (c[u].b >= 0) *reinterpret_cast<Vec *>(to[u] + c[u].b * N) = hi[u];
        }
    }
}

}  // namespace dba
