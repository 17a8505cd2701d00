// Attention behind a prefix that all sentences of a batch have in common: the rows of all sentences together over that prefix, each sentence's own over its
// cache, and the join of both.
#pragma once
#include "tree_attend.hpp"

namespace dba {

struct SharedParams {
    AttendParams common;               // one sentence with the nodes of all: nodes b * n + i
    AttendParams own;
    int common_tile, own_tile;         // tokens of a tile
    int own_shift;                     // log2 of own.tile_rows
};

// Joins a row's parts, of both kinds: 2^(m_s - m) O_s and 2^(m_s - m) l_s added up, as dba_attend_join_kernel does for one kind.  Every row has one part
// of each kind at least.
template <int FMT, int Q>
__global__ __launch_bounds__(256) void dba_shared_join_kernel(SharedParams sp)
{
    typedef typename Elem<FMT>::type E;
    const AttendParams &p = sp.own;
    const int lane = (int)threadIdx.x & 63, b = (int)blockIdx.z, head = (int)blockIdx.y;
    const int G = p.q_heads / p.heads, rows = p.n * G;
    const int r0 = ((int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)) * Q;
    if (r0 >= rows) return;
    int tree_all;
    const Span span = span_of_rows(p, b, r0 >> sp.own_shift, G, tree_all);
    const int tiles = (span.prefix + sp.own_tile - 1) / sp.own_tile + (span.end - span.prefix + sp.own_tile - 1) / sp.own_tile;
    const int ctiles = (span_of(sp.common.prefix[0], 0, sp.common.max_len).prefix + sp.common_tile - 1) / sp.common_tile;
    const int own = max(1, (tiles + p.chunk - 1) / p.chunk), parts = own + max(1, (ctiles + sp.common.chunk - 1) / sp.common.chunk);
    const int all = sp.common.n * G;                   // rows of a part of the common prefix
    const size_t own_at = ((size_t)b * p.heads + head) * p.splits * rows + r0;
    const size_t common_at = (size_t)head * sp.common.splits * all + (size_t)b * rows + r0;
    const int across = p.D <= 32 ? 8 : p.D <= 64 ? 16 : p.D <= 128 ? 32 : 64, side = 64 / across;   // lanes of a part, parts side by side
    const int d = lane % across * 4;
    float top[Q], sum[Q];
    f32x4 v[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        top[q] = -INFINITY;
        sum[q] = 0.0f;
        v[q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (int s0 = 0; s0 < parts; s0 += 64) {
        const int n = min(64, parts - s0);
        float w[Q];
        const int mine = s0 + lane;
        const float *ml = mine < own ? p.part_ml + (own_at + (size_t)mine * rows) * 2 : sp.common.part_ml + (common_at + (size_t)(mine - own) * all) * 2;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            float ms = -INFINITY, ls = 0.0f;
            if (lane < n && r0 + q < rows) {
                const float2 x = *reinterpret_cast<const float2 *>(ml + q * 2);
                ms = x.x;
                ls = x.y;
            }
            const float top1 = fmaxf(top[q], wave_max_float(ms));
            const float keep = top[q] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top[q] - top1);
            w[q] = ls == 0.0f ? 0.0f : ms == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ms - top1);
            top[q] = top1;
            sum[q] = sum[q] * keep + wave_sum_float(ls * w[q]);
            v[q] *= keep;
        }
        constexpr int U = 4 / Q > 0 ? 4 / Q : 1;       // parts of a row that a lane has under way
        for (int s1 = 0; s1 < n; s1 += U * side) {
            f32x4 y[Q][U];
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int s = s1 + x * side + lane / across, part = s0 + s;
                const float *at = part < own ? p.part_o + (own_at + (size_t)part * rows) * p.D + d : sp.common.part_o + (common_at + (size_t)(part - own) * all) * p.D + d;
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    y[q][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                    if (s < n && d < p.D && r0 + q < rows) y[q][x] = *reinterpret_cast<const f32x4 *>(at + q * p.D);
                }
            }
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int s = s1 + x * side + lane / across;
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    const float f = __shfl(w[q], s & 63);
                    v[q] += y[q][x] * (s < n && d < p.D ? f : 0.0f);
                }
            }
        }
    }
    int node = r0 / G, h = r0 - node * G;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        if (r0 + q >= rows) return;
        for (int x = across; x < 64; x *= 2)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[q][i] += __shfl_xor(v[q][i], x);
        if (lane == 0 && p.lse) p.lse[((int64_t)b * p.n + node) * p.q_heads + head * G + h] = sum[q] != 0.0f ? (top[q] + __builtin_amdgcn_logf(sum[q])) * kLn2f : -INFINITY;
        if (lane < across && d < p.D) {
            v[q] *= sum[q] != 0.0f ? 1.0f / sum[q] : 0.0f;
            E *to = reinterpret_cast<E *>(p.out.data) + ((int64_t)b * p.out.sent + (int64_t)node * p.out.token + (int64_t)(head * G + h) * p.out.head + d);
            if constexpr (FMT == 0) *reinterpret_cast<f32x4 *>(to) = v[q];
            else *reinterpret_cast<uint2 *>(to) = make_uint2(pack2<FMT>(v[q][0], v[q][1]), pack2<FMT>(v[q][2], v[q][3]));
        }
        if (++h == G) {
            h = 0;
            ++node;
        }
    }
}

template <int FMT> hipError_t shared_launch(const SharedParams &p, const AttendPlan &own, const AttendPlan &common, int B, hipStream_t stream);

}  // namespace dba
