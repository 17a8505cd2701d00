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
    const float *score;                // [B, 1 or heads, ..]; nullptr: sums are left for another launch
    float *out;                        // [B, 1 or heads, ..], or those sums [B, heads, splits, max_len]
    int64_t score_sent, score_head, out_sent, out_head;
    int n, q_heads, heads, D, mask_words, max_len;
    int width;                         // tokens that out has; those that nobody asks about are taken over
    int chunk;                         // of few rows: tokens of a workgroup
    int splits, split_rows;            // of many: workgroups along them, rows of each
    float scale;
};

// What of its sentence's tree a node sees.
struct WeighMask {
    const unsigned long long *words;   // of the sentence; nullptr: a chain
    int mask_words, prefix, end, last; // last: tree token that node 0 of a chain sees at most, or so many before the tree
};
// Which of the 64 tokens from t0 on `node` sees: two words of its mask, and what they say.
struct WeighWords {
    unsigned long long lo, hi;
};
// (Read whether they are wanted or not: how many loads are under way is then known, and those that are can be waited for alone.  `any` is what can be read where there is
// no mask.)
__device__ __forceinline__ WeighWords weigh_words(const WeighMask &m, const void *any, int node, int t0)
{
    const int word = (t0 - m.prefix) >> 6;             // (rounded down; in front of the tree all are set)
    const bool none = !m.words || m.mask_words == 0;
    const unsigned long long *row = none ? static_cast<const unsigned long long *>(any) : m.words + (int64_t)node * m.mask_words;
    const int last = none ? 0 : m.mask_words - 1;
    const unsigned long long lo = row[min(max(word, 0), last)], hi = row[min(max(word + 1, 0), last)];
    return {word < 0 ? ~0ull : word >= m.mask_words ? 0 : lo, word + 1 < 0 ? ~0ull : word + 1 >= m.mask_words ? 0 : hi};
}
__device__ __forceinline__ unsigned long long weigh_seen(const WeighMask &m, const WeighWords &w, int node, int t0)
{
    const int j0 = t0 - m.prefix, end = m.end - t0;
    if (end <= 0) return 0;
    unsigned long long seen;
    if (m.words) {
        seen = w.lo >> (j0 & 63) | (w.hi << 1) << (63 - (j0 & 63));
    } else {
        const int64_t last = max((int64_t)m.last + node, (int64_t)-1) - j0;    // (the prefix is always seen)
        seen = last < 0 ? 0 : last >= 63 ? ~0ull : (2ull << last) - 1;
    }
    return end < 64 ? seen & ((1ull << end) - 1) : seen;
}

// The same number, of which the compiler does not know that it is: what follows from it is worked out where it is used, and not kept in registers around a loop.
__device__ __forceinline__ int anew(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}
// r / G and the rest, for r below 2^23.
struct NodeOf {
    int G;
    float per;
    __device__ __forceinline__ int node(int r) const
    {
        const int q = (int)((float)r * per), rest = r - q * G;
        return q + (rest >= G) - (rest < 0);
    }
};
// Offset in elements of a sentence's token; of one that is not there, or from `limit` on, that of one that is.
__device__ __forceinline__ int64_t weigh_offset(const Paged &c, const int32_t *table, int pos, int limit, bool &there)
{
    const int32_t page = table[min(pos >> c.page_shift, c.max_pages - 1)];
    there = pos < limit && (pos >> c.page_shift) < c.max_pages && (uint32_t)page < (uint32_t)c.n_pages;
    return there ? (int64_t)page * c.page_stride + (int64_t)(pos & ((1 << c.page_shift) - 1)) * c.token_stride : 0;
}

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
// Rows are split where there are few tokens; sums of splits are added up in their order by another launch.
// Bound: waits.  All of 8 prompts of 1500 tokens, 32 heads on 8 of 128: 418 us, in which a SIMD has 0.94 waves on average, whose steps are chains of reads from LDS, four products that need each other
// and sixteen exponentials; the VALU is at work for 25 % of the clocks, the matrix units for 9.  Workgroups are too few (384, not split), and in a chain the first tile of tokens has all rows and the last a seventh of them.
template <int FMT, int DP, bool FULL>
__global__ __launch_bounds__(256, 2) void dba_weigh_kernel(WeighParams p)
{
    typedef WeighShape<FMT, DP> W;
    typedef typename Elem<FMT>::type E;
    constexpr int KS = W::KS, FC = W::FC, NT = W::NT, NE = 16 / W::ES;
    __shared__ __align__(16) unsigned char s_q[W::RQ * W::ROW];
    __shared__ float s_lse[W::RQ];                      // in powers of two; +inf: the row counts for nothing
    __shared__ unsigned long long s_seen[W::RQ][4];     // which of a wave's tokens a row sees
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int b = (int)blockIdx.z, head = (int)blockIdx.y / p.splits, split = (int)blockIdx.y - head * p.splits;
    const int t0 = (int)blockIdx.x * W::TG, mine = t0 + wave * W::TW;
    const int G = p.q_heads / p.heads;
    const NodeOf of = {G, 1.0f / (float)G};
    const int tree_all = p.tree ? max(p.tree[b], 0) : 0;
    const Span span = span_of(p.prefix[b], tree_all, p.max_len);
    const int n = p.count ? min(max(p.count[b], 0), p.n) : p.n;
    const int r0 = split * p.split_rows, rows = min(n * G, r0 + p.split_rows);     // this workgroup's
    const WeighMask mask = {p.mask ? p.mask + (int64_t)b * p.n * p.mask_words : nullptr, p.mask_words, span.prefix, span.end, tree_all - p.n};
    // of a chain, the first node that sees any of these tokens
    const int node0 = p.mask || t0 < span.prefix ? 0 : (int)max((int64_t)0, min((int64_t)n, (int64_t)t0 - span.prefix - tree_all + p.n));
    const int first = max(r0, node0 * G / W::RQ * W::RQ);
    float acc[NT];
    bool there[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = 0.0f;
    int64_t at[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        at[t] = weigh_offset(p.cache, p.cache.table + (int64_t)b * p.cache.table_stride, mine + t * 16 + c, span.end, there[t]);
    }
    const uint32_t sign = p.scale < 0.0f ? (FMT == 0 ? 0x80000000u : 0x80008000u) : 0u;
    const float sl2 = fabsf(p.scale) * kLog2e;
    if (t0 < span.end && first < rows) {
        u32x4 next[W::PER];
        auto ask = [&](int row0) {                  // the rows from row0 on; elements behind the head's end, rows behind the last: 0
            const int t = anew((int)threadIdx.x);
#pragma unroll
            for (int x = 0; x < W::PER; ++x) {
                const int chunk = (x * 256 + t) % W::CH, r = row0 + (x * 256 + t) / W::CH;
                next[x] = u32x4{0, 0, 0, 0};
                if (r < rows && (FULL || chunk * NE < p.D) && p.scale != 0.0f) {
                    const int node = of.node(r), h = head * G + r - node * G;
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
                    k[t][s].c[f] = *reinterpret_cast<const u32x4 *>(src + (FULL || d < p.D ? d : 0));
                }
        }
        for (int row0 = first; row0 < rows; row0 += W::RQ) {
            __syncthreads();                        // (nobody reads the last ones any more)
            const int tid = anew((int)threadIdx.x);
#pragma unroll
            for (int x = 0; x < W::PER; ++x)
                *reinterpret_cast<u32x4 *>(s_q + W::at((x * 256 + tid) / W::CH, (x * 256 + tid) % W::CH)) = next[x];
            if (tid < W::RQ * 4) {
                const int i = tid >> 2, w = tid & 3, r = row0 + i;
                unsigned long long seen = 0;
                if (r < rows) {
                    const int node = of.node(r);
                    const float lse = p.lse[((int64_t)b * p.n + node) * p.q_heads + head * G + r - node * G];
                    if (fabsf(lse) < INFINITY) seen = weigh_seen(mask, weigh_words(mask, p.k_pages, node, t0 + w * W::TW), node, t0 + w * W::TW);
                    if (w == 0) s_lse[i] = lse * kLog2e;
                } else if (w == 0) {
                    s_lse[i] = INFINITY;
                }
                s_seen[i][w] = seen;
            }
            __syncthreads();
            ask(row0 + W::RQ);
#pragma unroll 1
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
    const int64_t from = (int64_t)b * p.score_sent + (int64_t)head * p.score_head, to = (int64_t)b * p.out_sent + (int64_t)blockIdx.y * p.out_head;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float sum = sum_over_groups(acc[t]);
        const int pos = mine + t * 16 + c;
        if (g == 0 && pos < p.width && (there[t] || p.out != p.score)) p.out[to + pos] = (p.score ? p.score[from + pos] : 0.0f) + (there[t] ? sum : 0.0f);
    }
}

// The same with so few rows that they lie in LDS together: then the waves go through tokens, TF of them at a time and each on its own, with the next ones'
// keys under way.  What the next tile needs of tables and masks is asked for before those keys: loads come back in order, so waiting for it would be
// waiting for them.
//
// FULL: heads have DP elements.  SR: rows in sixty-fours, whose masks the lanes look after.
// Bound: memory and waits, each key is read once: 64 sentences of 20 branches over 900 to 1500 tokens, 16 heads of 64, 48 us (3.5 TB/s, the VALU at work for 45 % of the clocks; attention, which reads the same layout for
// two heads a workgroup, reaches 4.8, and that has not been tried here), 128 rows of 128 over 16 x 3000 to 16000 tokens, 8 heads, 93 (3.4 TB/s; the VALU 47 %, the matrix units 21, the exponentials alone are 28 us).
// The 16-bit instances with SR = 2 have 8 to 10 registers in scratch (36 to 44 bytes a lane), some of them read again within the loop, which then waits for the next tile's keys as well; without that the second case has not been measured.
template <int FMT, int DP>
struct WeighFew {
    typedef WeighShape<FMT, DP> W;
    static constexpr int NT = FMT != 0 && DP == 64 ? 4 : DP == 128 && FMT != 0 ? 2 : 1;
    static constexpr int TF = 16 * NT;
    static constexpr int MOST = 32768 / W::ROW < 128 ? 32768 / W::ROW : 128;       // rows
    static __host__ __device__ int lds(int rows, int chunk)     // queries, normalisers, what a row sees of a wave's tile, sums (of whole turns of the waves)
    {
        const int r = (rows + 15) / 16 * 16;
        return r * (W::ROW + 4 + 32) + chunk * 4;
    }
};

template <int FMT, int DP, bool FULL, int SR>
__global__ __launch_bounds__(256, (DP == 256 || FMT == 0 ? 2 : 4)) void dba_weigh_few_kernel(WeighParams p)
{
    typedef WeighShape<FMT, DP> W;
    typedef WeighFew<FMT, DP> F;
    typedef typename Elem<FMT>::type E;
    constexpr int KS = W::KS, FC = W::FC, NT = F::NT, TF = F::TF, NE = 16 / W::ES;
    extern __shared__ __align__(16) unsigned char s_mem[];
    __shared__ int s_dead[4];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const int b = (int)blockIdx.z, head = (int)blockIdx.y;
    const int G = p.q_heads / p.heads;
    const NodeOf of = {G, 1.0f / (float)G};
    const int most = (p.n * G + 15) / 16 * 16;          // rows that there is room for
    unsigned char *const s_q = s_mem;
    float *const s_lse = reinterpret_cast<float *>(s_mem + most * W::ROW);
    unsigned long long *const s_seen = reinterpret_cast<unsigned long long *>(s_mem + most * (W::ROW + 4)) + wave * most;
    float *const s_sum = reinterpret_cast<float *>(s_mem + most * (W::ROW + 36));
    const int tree_all = p.tree ? max(p.tree[b], 0) : 0;
    const Span span = span_of(p.prefix[b], tree_all, p.max_len);
    const int rows = (p.count ? min(max(p.count[b], 0), p.n) : p.n) * G, padded = (rows + 15) / 16 * 16;
    const int t0 = (int)blockIdx.x * p.chunk, t1 = min(span.end, t0 + p.chunk), last = min(p.width, t0 + p.chunk);     // this workgroup's tokens
    const float *const score = p.score ? p.score + ((int64_t)b * p.score_sent + (int64_t)head * p.score_head) : nullptr;
    float *const out = p.out + ((int64_t)b * p.out_sent + (int64_t)head * p.out_head);
    if (p.out != p.score)                               // tokens that nobody asks about
        for (int t = max(t0, rows > 0 ? span.end : t0) + (int)threadIdx.x; t < last; t += 256) out[t] = score ? score[t] : 0.0f;
    if (t0 >= t1 || rows == 0) return;
    const uint32_t sign = p.scale < 0.0f ? (FMT == 0 ? 0x80000000u : 0x80008000u) : 0u;
    const float sl2 = fabsf(p.scale) * kLog2e;
    const int32_t *const table = p.cache.table + (int64_t)b * p.cache.table_stride;
    const E *const keys = reinterpret_cast<const E *>(p.k_pages) + (int64_t)head * p.cache.head_stride;
    const WeighMask mask = {p.mask ? p.mask + (int64_t)b * p.n * p.mask_words : nullptr, p.mask_words, span.prefix, span.end, tree_all - p.n};
    const int first = t0 + wave * TF, step = 4 * TF;
    auto page_of = [&](int u) -> int {                 // of token u + lane; -1: no such token
        const int pos = u + min(lane, TF - 1);
        const int32_t page = table[min(pos >> p.cache.page_shift, p.cache.max_pages - 1)];
        return pos < t1 && (uint32_t)page < (uint32_t)p.cache.n_pages ? page : -1;     // (tokens before t1 are in the table: max_len is)
    };
    Frag<FMT> k[NT][KS];
    auto load = [&](int u, int pages) {                // of a token that is not there: of the pool's first one
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int pos = u + t * 16 + c, page = __shfl(pages, t * 16 + c);
            const int64_t at = page < 0 ? 0 : (int64_t)page * p.cache.page_stride + (int64_t)(pos & ((1 << p.cache.page_shift) - 1)) * p.cache.token_stride;
            const E *src = keys + at;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int f = 0; f < FC; ++f) {
                    const int d = s * 32 + g * 8 + f * NE;
                    k[t][s].c[f] = *reinterpret_cast<const u32x4 *>(src + (FULL || d < p.D ? d : 0));
                }
        }
    };
    const int page = page_of(first);
    int page_next = page_of(first + step);
    WeighWords words[SR];
    bool dead = false;
    {
        const E *const q_b = reinterpret_cast<const E *>(p.q.data) + (int64_t)b * p.q.sent;
        const float *const lse_b = p.lse + (int64_t)b * p.n * p.q_heads;
#pragma unroll 1
        for (int x = anew((int)threadIdx.x); x < padded * W::CH; x += 256) {
            const int chunk = x % W::CH, r = x / W::CH;
            u32x4 v = u32x4{0, 0, 0, 0};
            if (r < rows && (FULL || chunk * NE < p.D) && p.scale != 0.0f) {
                const int node = of.node(r), h = head * G + r - node * G;
                v = *reinterpret_cast<const u32x4 *>(q_b + ((int64_t)node * p.q.token + (int64_t)h * p.q.head) + chunk * NE) ^ sign;
            }
            *reinterpret_cast<u32x4 *>(s_q + W::at(r, chunk)) = v;
        }
        const int r = (int)threadIdx.x;                 // (there are fewer than threads)
        if (r < padded) {
            float lse = INFINITY;
            if (r < rows) {
                const int node = of.node(r);
                lse = lse_b[(int64_t)node * p.q_heads + head * G + r - node * G];
                if (!(fabsf(lse) < INFINITY)) {
                    lse = INFINITY;
                    dead = true;
                }
            }
            s_lse[r] = lse * kLog2e;
        }
    }
#pragma unroll
    for (int x = 0; x < SR; ++x) words[x] = weigh_words(mask, p.k_pages, of.node(min(lane + x * 64, rows - 1)), first);
    load(first, page);
    dead = __any(dead);
    if (lane == 0) s_dead[wave] = dead;
    __syncthreads();
    // rows that count for nothing, and those behind the last, have weights of 0, unless their products are not finite
    dead = s_dead[0] | s_dead[1] | s_dead[2] | s_dead[3] | (rows != padded);
#pragma unroll 1
    for (int u = first; u < t1; u += step) {
        const bool masked = dead || u + TF > span.prefix;
        if (masked) {
#pragma unroll
            for (int x = 0; x < SR; ++x) {
                const int r = lane + x * 64;
                if (r < padded) s_seen[r] = r < rows && s_lse[r] < INFINITY ? weigh_seen(mask, words[x], of.node(r), u) : 0;
            }
        }
        if (u + step + TF > span.prefix)
#pragma unroll
            for (int x = 0; x < SR; ++x) words[x] = weigh_words(mask, p.k_pages, of.node(min(lane + x * 64, rows - 1)), u + step);
        const int pages = page_next;
        page_next = page_of(u + 2 * step);
        Frag<FMT> now[NT][KS];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s) now[t][s] = k[t][s];
        if (u + step < t1) load(u + step, pages);
        float acc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t] = 0.0f;
#pragma unroll 1
        for (int r16 = 0; r16 < padded; r16 += 16) {
            Frag<FMT> q[KS];
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int f = 0; f < FC; ++f) q[s].c[f] = *reinterpret_cast<const u32x4 *>(s_q + W::at(r16 + c, (s * 4 + g) * FC + f));
            const f32x4 lse = *reinterpret_cast<const f32x4 *>(s_lse + r16 + g * 4);
            f32x4 s[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                s[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int x = 0; x < KS; ++x) s[t] = mfma32<FMT>(q[x], now[t][x], s[t]);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], sl2, -lse[i]));
            }
            if (masked) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned long long seen = s_seen[r16 + g * 4 + i] >> c;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        if (!((seen >> (t * 16)) & 1)) s[t][i] = 0.0f;
                }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] += (s[t][0] + s[t][1]) + (s[t][2] + s[t][3]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float sum = sum_over_groups(acc[t]);
            if (g == 0) s_sum[u - t0 + t * 16 + c] = sum;      // (scores are read at the end: here they would be waited for, and with them the next tile)
        }
    }
    __syncthreads();
    for (int t = t0 + (int)threadIdx.x; t < t1; t += 256) {
        const bool there = token_offset(p.cache, b, t) >= 0;
        if (there || p.out != p.score) out[t] = (score ? score[t] : 0.0f) + (there ? s_sum[t - t0] : 0.0f);
    }
}

// Sums of heads (one score for all: parts are those of all heads) or of a head's rows, added up in their order.
__global__ __launch_bounds__(256) void dba_weigh_join_kernel(WeighParams p, const float *sums, int parts)
{
    const int b = (int)blockIdx.z, row = (int)blockIdx.y, t = (int)blockIdx.x * 256 + (int)threadIdx.x;
    if (t >= p.width) return;
    const Span span = span_of(p.prefix[b], p.tree ? p.tree[b] : 0, p.max_len);
    const bool there = t < span.end && token_offset(p.cache, b, t) >= 0;
    if (!there && p.out == p.score) return;
    float sum = 0.0f;
    if (there)
        for (int x = 0; x < parts; ++x) sum += sums[(((int64_t)b * gridDim.y + row) * parts + x) * p.max_len + t];
    p.out[(int64_t)b * p.out_sent + (int64_t)row * p.out_head + t] = p.score[(int64_t)b * p.score_sent + (int64_t)row * p.score_head + t] + sum;
}

}  // namespace dba
