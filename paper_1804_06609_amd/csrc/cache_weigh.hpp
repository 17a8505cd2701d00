// How much attention each token of a paged cache has had: kernel.
#pragma once
#include "tree_attend.hpp"

namespace dba {

struct WeighParams {
    Paged cache;
    const unsigned char *k_pages;
    HeadsAt q;
    const float *lse;                  // [B, n, q_heads]
    const int32_t *prefix, *tree, *count;
    const unsigned long long *mask;
    const float *score;                // [B, 1 or heads, ..]
    float *out;
    int64_t score_sent, score_head, out_sent, out_head;
    int n, q_heads, heads, D, mask_words, max_len;
    int width;                         // tokens that out has; those that nobody asks about are taken over
    int by_head;
    float scale;
};

// How a workgroup works: its four waves have TW tokens each, whose keys stay in registers, and go through the rows (a node's query heads of one head of
// the cache, as in attention) together, RQ of them in LDS at a time.
template <int FMT, int DP>
struct WeighShape {
    static constexpr int ES = FMT == 0 ? 4 : 2;
    static constexpr int KS = DP / 32;
    static constexpr int FC = Frag<FMT>::C;
    static constexpr int NT = 64 / (KS * 4 * FC) < 4 ? 64 / (KS * 4 * FC) : 4;    // 16-token tiles of a wave: 64 registers of keys
    static constexpr int TW = 16 * NT, TG = 4 * TW;
    static constexpr int ROW = DP * ES, CH = ROW / 16;
    static constexpr int RQ = ROW <= 256 ? 64 : ROW <= 512 ? 32 : 16;
    static constexpr int PER = RQ * CH / 256;           // chunks of the next rows that a thread holds
    static constexpr int RK = CH >= 16 ? 1 : 16 / CH;   // rows that share 256 bytes
    // 16 lanes that read one chunk of 16 rows meet all 64 banks
    static __device__ __forceinline__ int at(int row, int chunk) { return row * ROW + ((chunk + (row % 16) / RK) & (CH - 1)) * 16; }
};

// out[t] = score[t] + sum over the rows r that see token t of exp(scale q_r . k_t - lse_r).  S = Q K^T leaves lane (g, c) with rows 4g .. 4g+3 of token c, so that
// a token's sum is four additions a lane and, at the very end, two exchanges.  Each token belongs to one wave, which adds up in the order of the
// rows: nothing is added atomically, and results do not vary.
//
// Bound: memory with few rows (the keys, read once), the exponentials and what is around them with many.
template <int FMT, int DP>
__global__ __launch_bounds__(256) void dba_weigh_kernel(WeighParams p)
{
    typedef WeighShape<FMT, DP> W;
    typedef typename Elem<FMT>::type E;
    constexpr int KS = W::KS, FC = W::FC, NT = W::NT, NE = 16 / W::ES;
    __shared__ __align__(16) unsigned char s_q[W::RQ * W::ROW];
    __shared__ float s_lse[W::RQ];                      // in powers of two; +inf: the row counts for nothing
    __shared__ unsigned long long s_seen[W::RQ][4];     // which of a wave's tokens a row sees
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int b = (int)blockIdx.z, head0 = p.by_head ? (int)blockIdx.y : 0, head1 = p.by_head ? head0 + 1 : p.heads;
    const int t0 = (int)blockIdx.x * W::TG, mine = t0 + wave * W::TW;
    const int G = p.q_heads / p.heads;
    const int tree_all = p.tree ? max(p.tree[b], 0) : 0;
    const Span span = span_of(p.prefix[b], tree_all, p.max_len);
    const int n = p.count ? min(max(p.count[b], 0), p.n) : p.n;
    const int rows = n * G;
    // of a chain, the first node that sees any of these tokens
    const int node0 = p.mask ? 0 : (int)max((int64_t)0, min((int64_t)n, (int64_t)t0 - span.prefix - tree_all + p.n));
    const int first = node0 * G / W::RQ * W::RQ;
    float acc[NT];
    bool there[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = 0.0f;
    int64_t at[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int pos = mine + t * 16 + c;
        const int64_t off = pos < span.end ? token_offset(p.cache, b, pos) : -1;
        there[t] = off >= 0;
        at[t] = there[t] ? off : 0;
    }
    const uint32_t sign = p.scale < 0.0f ? (FMT == 0 ? 0x80000000u : 0x80008000u) : 0u;
    const float sl2 = fabsf(p.scale) * kLog2e;
    if (t0 < span.end && first < rows) {
        for (int head = head0; head < head1; ++head) {
            u32x4 next[W::PER];
            auto ask = [&](int row0) {                  // the rows from row0 on; elements behind the head's end, rows behind the last: 0
#pragma unroll
                for (int x = 0; x < W::PER; ++x) {
                    const int chunk = (x * 256 + (int)threadIdx.x) % W::CH, r = row0 + (x * 256 + (int)threadIdx.x) / W::CH;
                    next[x] = u32x4{0, 0, 0, 0};
                    if (r < rows && chunk * NE < p.D && p.scale != 0.0f) {
                        const int node = r / G, h = head * G + r % G;
                        next[x] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const E *>(p.q.data) + ((int64_t)b * p.q.sent + (int64_t)node * p.q.token + (int64_t)h * p.q.head) + chunk * NE) ^ sign;
                    }
                }
            };
            ask(first);
            Frag<FMT> k[NT][KS];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const E *src = reinterpret_cast<const E *>(p.k_pages) + (at[t] + (int64_t)head * p.cache.head_stride);
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int f = 0; f < FC; ++f) {
                        const int d = s * 32 + g * 8 + f * NE;
                        k[t][s].c[f] = *reinterpret_cast<const u32x4 *>(src + (d < p.D ? d : 0));
                    }
            }
            for (int row0 = first; row0 < rows; row0 += W::RQ) {
                __syncthreads();                        // (nobody reads the last ones any more)
#pragma unroll
                for (int x = 0; x < W::PER; ++x)
                    *reinterpret_cast<u32x4 *>(s_q + W::at((x * 256 + (int)threadIdx.x) / W::CH, (x * 256 + (int)threadIdx.x) % W::CH)) = next[x];
                if ((int)threadIdx.x < W::RQ * 4) {
                    const int i = (int)threadIdx.x >> 2, w = (int)threadIdx.x & 3, r = row0 + i;
                    unsigned long long seen = 0;
                    if (r < rows) {
                        const int node = r / G, j0 = t0 + w * W::TW - span.prefix, end = span.end - span.prefix - j0;      // (tokens from j0 on; end of them)
                        const float lse = p.lse[((int64_t)b * p.n + node) * p.q_heads + head * G + r % G];
                        if (fabsf(lse) < INFINITY) {
                            if (p.mask) {
                                const unsigned long long *words = p.mask + ((int64_t)b * p.n + node) * p.mask_words;
                                if (j0 < 0) {           // tokens of the prefix first
                                    seen = j0 <= -64 ? ~0ull : (1ull << -j0) - 1;
                                    if (j0 > -64 && p.mask_words > 0) seen |= words[0] << -j0;
                                } else {
                                    const int word = j0 >> 6, bit = j0 & 63;
                                    if (word < p.mask_words) seen = words[word] >> bit;
                                    if (bit && word + 1 < p.mask_words) seen |= words[word + 1] << (64 - bit);
                                }
                            } else {
                                const int64_t last = (int64_t)tree_all - p.n + node - j0;
                                seen = last < 0 ? 0 : last >= 63 ? ~0ull : (2ull << last) - 1;
                                if (j0 < 0) seen |= j0 <= -64 ? ~0ull : (1ull << -j0) - 1;
                            }
                            if (end < 64) seen &= end <= 0 ? 0 : (1ull << end) - 1;
                        }
                        if (w == 0) s_lse[i] = lse * kLog2e;
                    } else if (w == 0) {
                        s_lse[i] = INFINITY;
                    }
                    s_seen[i][w] = seen;
                }
                __syncthreads();
                ask(row0 + W::RQ);
                for (int r16 = 0; r16 < W::RQ && row0 + r16 < rows; r16 += 16) {
                    Frag<FMT> q[KS];
#pragma unroll
                    for (int s = 0; s < KS; ++s)
#pragma unroll
                        for (int f = 0; f < FC; ++f) q[s].c[f] = *reinterpret_cast<const u32x4 *>(s_q + W::at(r16 + c, (s * 4 + g) * FC + f));
                    const f32x4 lse = *reinterpret_cast<const f32x4 *>(s_lse + r16 + g * 4);
                    unsigned long long seen[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) seen[i] = s_seen[r16 + g * 4 + i][wave];
                    constexpr unsigned long long kAll = W::TW == 64 ? ~0ull : (1ull << (W::TW & 63)) - 1;
                    const bool all = !__any((seen[0] & seen[1] & seen[2] & seen[3] & kAll) != kAll);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        f32x4 s = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int x = 0; x < KS; ++x) s = mfma32<FMT>(q[x], k[t][x], s);
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], sl2, -lse[i]));
                        if (!all) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (!((seen[i] >> (t * 16 + c)) & 1)) s[i] = 0.0f;
                        }
                        acc[t] += (s[0] + s[1]) + (s[2] + s[3]);
                    }
                }
            }
        }
    }
    const int64_t from = (int64_t)b * p.score_sent + (int64_t)head0 * p.score_head, to = (int64_t)b * p.out_sent + (int64_t)head0 * p.out_head;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float sum = sum_over_groups(acc[t]);
        const int pos = mine + t * 16 + c;
        if (g == 0 && pos < p.width && (there[t] || p.out != p.score)) p.out[to + pos] = p.score[from + pos] + (there[t] ? sum : 0.0f);
    }
}

}  // namespace dba
