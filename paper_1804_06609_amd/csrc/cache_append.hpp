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
__device__ __forceinline__ float2 turn_of(int position, float inv_freq)
{
    const double turns = (double)position * ((double)inv_freq * 0.159154943091895335768883763);
    const float x = (float)(2.0 * (turns - rint(turns)));      // in half turns
    float s, c;
    sincospif(x, &s, &c);
    return make_float2(c, s);
}

// One workgroup per token: its angles once, then all its heads, 16 bytes at a time.  Bound: HBM.
template <int FMT>
__global__ __launch_bounds__(kAppendThreads) void dba_append_kernel(AppendParams p)
{
    typedef typename Elem<FMT>::type E;
    constexpr int N = 16 / (int)sizeof(E);
    struct alignas(16) Vec { E e[N]; };
    __shared__ float2 s_turn[128];
    const int b = (int)blockIdx.y, i = (int)blockIdx.x;
    const int t = (int)threadIdx.x;
    const bool there = !p.count || i < p.count[b];
    const int64_t at = (int64_t)p.first[b] + i;
    const int position = p.position ? p.position[(int64_t)b * p.n + i] : (int)at;
    const int64_t slot = there ? token_offset(p.cache, b, at) : -1;
    const int half = p.rot / 2;
    if (there)
        for (int j = t; j < half; j += kAppendThreads) s_turn[j] = turn_of(position, p.inv_freq[j]);
    __syncthreads();
    const int per_head = p.D / N, items = (p.q_heads + 2 * p.heads) * per_head;
    for (int x = t; x < items; x += kAppendThreads) {
        const int head = x / per_head, c = x - head * per_head;
        const E *src;
        E *dst;
        bool rotates = true;
        if (head < p.q_heads) {
            src = reinterpret_cast<const E *>(p.q.data) + (b * p.q.sent + i * p.q.token + head * p.q.head);
            dst = reinterpret_cast<E *>(p.q_out.data) + (b * p.q_out.sent + i * p.q_out.token + head * p.q_out.head);
        } else {
            const bool is_v = head >= p.q_heads + p.heads;
            const int h = head - p.q_heads - (is_v ? p.heads : 0);
            const HeadsAt &a = is_v ? p.v : p.k;
            if (slot < 0) continue;
            src = reinterpret_cast<const E *>(a.data) + (b * a.sent + i * a.token + h * a.head);
            dst = reinterpret_cast<E *>(is_v ? p.v_pages : p.k_pages) + (slot + h * p.cache.head_stride);
            rotates = !is_v;
        }
        const int d0 = c * N;
        if (!rotates || d0 >= p.rot || !there) {
            Vec v{};
            if (there) v = *reinterpret_cast<const Vec *>(src + d0);
            *reinterpret_cast<Vec *>(dst + d0) = v;
        } else if (p.interleaved) {
            Vec v = *reinterpret_cast<const Vec *>(src + d0);
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                const float2 r = s_turn[(d0 + e) / 2];
                const float x0 = (float)v.e[e], x1 = (float)v.e[e + 1];
                v.e[e] = (E)(x0 * r.x - x1 * r.y);
                v.e[e + 1] = (E)(x1 * r.x + x0 * r.y);
            }
            *reinterpret_cast<Vec *>(dst + d0) = v;
        } else if (d0 < half) {
            // (half is a multiple of 8, so a chunk of 16 bytes has one partner; q_out may be q: both are read before either is written)
            Vec lo = *reinterpret_cast<const Vec *>(src + d0), hi = *reinterpret_cast<const Vec *>(src + d0 + half);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float2 r = s_turn[d0 + e];
                const float x0 = (float)lo.e[e], x1 = (float)hi.e[e];
                lo.e[e] = (E)(x0 * r.x - x1 * r.y);
                hi.e[e] = (E)(x1 * r.x + x0 * r.y);
            }
            *reinterpret_cast<Vec *>(dst + d0) = lo;
            *reinterpret_cast<Vec *>(dst + d0 + half) = hi;
        }
    }
}

}  // namespace dba
