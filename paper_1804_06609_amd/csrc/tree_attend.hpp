// Attention of a tree's nodes over a paged cache: kernels.
#pragma once
#include "cache_append.hpp"
#include "paged.hpp"

namespace dba {

struct AttendParams {
    Paged cache;
    const unsigned char *k_pages, *v_pages;
    HeadsAt q, out;
    const int32_t *prefix, *tree;
    const unsigned long long *mask;
    float *lse;
    int n, q_heads, heads, D, mask_words, max_len;
    float scale;
};

// One query head of one node a workgroup, a token a wave at a time, the running maximum and sum of the softmax in fp32.
template <int FMT>
__global__ __launch_bounds__(256) void dba_attend_simple_kernel(AttendParams p)
{
    typedef typename Elem<FMT>::type E;
    __shared__ float s_m[4], s_l[4], s_o[4][256];
    const int t = (int)threadIdx.x, lane = t & 63, wave = t >> 6;
    const int h = (int)blockIdx.x % p.q_heads, i = (int)blockIdx.x / p.q_heads, b = (int)blockIdx.y;
    const int64_t kv_head = (int64_t)(h / (p.q_heads / p.heads)) * p.cache.head_stride;
    const Span span = span_of(p.prefix[b], p.tree ? p.tree[b] : 0, p.max_len);
    const int tree = p.tree ? max(p.tree[b], 0) : 0;
    const E *q = reinterpret_cast<const E *>(p.q.data) + (b * p.q.sent + i * p.q.token + h * p.q.head);
    float x[4], o[4] = {0.0f, 0.0f, 0.0f, 0.0f}, m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = lane + 64 * j < p.D ? (float)q[lane + 64 * j] * p.scale : 0.0f;
    for (int tok = wave; tok < span.end; tok += 4) {
        if (tok >= span.prefix) {
            const int j = tok - span.prefix;
            if (!p.mask) {
                if (j > tree - p.n + i) continue;
            } else if (j >= 64 * p.mask_words || !((p.mask[((int64_t)b * p.n + i) * p.mask_words + (j >> 6)] >> (j & 63)) & 1)) {
                continue;
            }
        }
        const int64_t at = token_offset(p.cache, b, tok);
        if (at < 0) continue;
        const E *k = reinterpret_cast<const E *>(p.k_pages) + (at + kv_head), *v = reinterpret_cast<const E *>(p.v_pages) + (at + kv_head);
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (lane + 64 * j < p.D) s += x[j] * (float)k[lane + 64 * j];
#pragma unroll
        for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
        const float m1 = fmaxf(m, s);
        const float keep = m1 == m ? 1.0f : __expf(m - m1), w = __expf(s - m1);
        m = m1;
        l = l * keep + w;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (lane + 64 * j < p.D) o[j] = o[j] * keep + w * (float)v[lane + 64 * j];
    }
    if (lane == 0) {
        s_m[wave] = m;
        s_l[wave] = l;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) s_o[wave][lane + 64 * j] = o[j];
    __syncthreads();
    float top = -INFINITY, sum = 0.0f, y = 0.0f;
    for (int w = 0; w < 4; ++w) top = fmaxf(top, s_m[w]);
    for (int w = 0; w < 4; ++w) {
        const float f = s_l[w] != 0.0f ? __expf(s_m[w] - top) : 0.0f;     // (a NaN is not nothing)
        sum += s_l[w] * f;
        if (t < p.D && f != 0.0f) y += s_o[w][t] * f;
    }
    E *out = reinterpret_cast<E *>(p.out.data) + (b * p.out.sent + i * p.out.token + h * p.out.head);
    if (t < p.D) out[t] = (E)(sum != 0.0f ? y / sum : 0.0f);
    if (t == 0 && p.lse) p.lse[((int64_t)b * p.n + i) * p.q_heads + h] = sum != 0.0f ? top + __logf(sum) : -INFINITY;
}

}  // namespace dba
