// Attention of a tree's nodes over a paged cache: kernels.
//
// For one sentence and one head of the cache, the queries that read it are rows: row r is node r / G, query head r % G of the
// G that share the head.  With x = scale log2 e (q . k), a row's output is sum 2^(x_t - m) v_t / sum 2^(x_t - m) over the tokens it
// sees, m being about the running maximum; parts of the token axis are joined by their m and sums.
//
// Both products run on the matrix units, transposed: S^T = K Q^T leaves lane (g, c) of a wave (c = lane % 16, g = lane / 16) with
// four consecutive tokens 4g .. 4g+3 of row c, which is what the second product O^T = V^T P^T takes as its right operand: the
// probabilities never leave the registers, the softmax's statistics are one number a lane, and joining a row's
// lanes takes two exchanges.  V^T, its left operand, comes out of LDS through the transposing read.  The order of tokens
// inside a product's sum is arbitrary as long as both sides have the same.
#pragma once
#include "cache_append.hpp"
#include "paged.hpp"
#include "wave_topk.hpp"

namespace dba {

struct AttendParams {
    Paged cache;
    const unsigned char *k_pages, *v_pages;
    HeadsAt q, out;
    const int32_t *prefix, *tree;
    const unsigned long long *mask;
    float *lse;
    float *part_o, *part_ml;           // of split launches: [B, heads, splits, rows, D] and [.., 2]
    int n, q_heads, heads, D, mask_words, max_len;
    int row_tiles, tile_rows;          // workgroups along the rows, rows of each
    int splits, chunk;                 // workgroups along the token axis, tiles of each
    int pairs, groups;                 // sentences times heads, or pairs of them; times splits
    int per;                           // with PARTS: nodes that q has side by side; the next ones lie a sentence further on
    float scale;
};

// Tokens of a sentence that the workgroup of row r looks at: of a chain those up to tree - n + its last node.
__device__ __forceinline__ Span span_of_rows(const AttendParams &p, int b, int row_tile, int G, int &tree_all)
{
    tree_all = p.tree ? max(p.tree[b], 0) : 0;
    return p.mask ? span_of(p.prefix[b], tree_all, p.max_len)
                  : span_of_chain(p.prefix[b], tree_all, p.n, (min((row_tile + 1) * p.tile_rows, p.n * G) - 1) / G, p.max_len);
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2f = 0.69314718055994530942f;

// A row's weights are 2^(x - m) with m kept kWeightBits below the maximum that it was set by, and set anew where a tile's maximum passes that
// by more than kWeightRoom (which few tiles do; by any amount every third tile did, at 64 multiplications for two rows of 128).  fp16, whose
// exponents end at 2^-14 and 2^15, has its weights near the upper end, or a long tail of small ones would be lost from the product and not from the sum.
template <int FMT> constexpr float kWeightBits = FMT == 1 ? 12.0f : 0.0f;
template <int FMT> constexpr float kWeightRoom = FMT == 1 ? 3.5f : 8.0f;

// Eight elements of a row along the contraction: 16 bytes, or 32 in fp32.
template <int FMT> struct Frag {
    static constexpr int C = FMT == 0 ? 2 : 1;
    u32x4 c[C];
};

// c += a b^T of 16 rows each over 32 elements; lane (g, i) gives elements 8g .. 8g+7 of row i of a and of b.  In fp32 the products come four
// at a time, one of each lane's eight.
template <int FMT>
__device__ __forceinline__ f32x4 mfma32(const Frag<FMT> &a, const Frag<FMT> &b, f32x4 c)
{
    if constexpr (FMT == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.c[j / 4][j % 4]), __uint_as_float(b.c[j / 4][j % 4]), c, 0, 0, 0);
        return c;
    } else if constexpr (FMT == 1) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.c[0]), __builtin_bit_cast(f16x8, b.c[0]), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.c[0]), __builtin_bit_cast(bf16x8, b.c[0]), c, 0, 0, 0);
    }
}

template <int FMT>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (FMT == 1) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        const h2 v = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, v);
    } else {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        const b2 v = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, v);
    }
}

// What is left of a and b where pack2 has made `both` of them, packed alike.  The differences are exact; an instruction each, which takes its half of `both` as it is.
// (In assembly for fp16.  Whatever wrote a and b has been waited for by the instruction that made `both`.)
template <int FMT>
__device__ __forceinline__ uint32_t rest2(float a, float b, uint32_t both)
{
    if constexpr (FMT == 1) {
        float x, y;
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[0,0,0] op_sel_hi:[1,0,0]" : "=v"(x) : "v"(both), "v"(a));
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(y) : "v"(both), "v"(b));
        return pack2<FMT>(x, y);
    } else {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        uint32_t low = 0x0000BF80u, high = 0xBF800000u;     // (-1, 0) and (0, -1); kept from the compiler, which makes the first an inline constant that is read as another number
        asm("" : "+s"(low), "+s"(high));
        const b2 v = __builtin_bit_cast(b2, both);
        return pack2<FMT>(__builtin_amdgcn_fdot2_f32_bf16(v, __builtin_bit_cast(b2, low), a, false), __builtin_amdgcn_fdot2_f32_bf16(v, __builtin_bit_cast(b2, high), b, false));
    }
}

template <int FMT>
__device__ __forceinline__ float low_half(uint32_t w)
{
    if constexpr (FMT == 1) return (float)__builtin_bit_cast(_Float16, (uint16_t)w);
    else return __uint_as_float(w << 16);
}
template <int FMT>
__device__ __forceinline__ float high_half(uint32_t w)
{
    if constexpr (FMT == 1) return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16));
    else return __uint_as_float(w & 0xFFFF0000u);
}

// Elements that are not finite are made 0.
template <int FMT>
__device__ __forceinline__ uint32_t finite_of(uint32_t w)
{
    if constexpr (FMT == 0) {
        return (w & 0x7F800000u) == 0x7F800000u ? 0u : w;
    } else {
        constexpr uint32_t E = FMT == 1 ? 0x7C00u : 0x7F80u;
        w = (w & E) == E ? w & 0xFFFF0000u : w;
        return (w & (E << 16)) == (E << 16) ? w & 0xFFFFu : w;
    }
}

template <int FMT>
__device__ __forceinline__ u32x4 finite_of(u32x4 c)
{
    return u32x4{finite_of<FMT>(c.x), finite_of<FMT>(c.y), finite_of<FMT>(c.z), finite_of<FMT>(c.w)};
}

// Where the exponent of an element of `w` is all ones, so that it is not finite, the bit of its sign is set (others may be, too).
template <int FMT> constexpr uint32_t kSignBits = FMT == 0 ? 0x80000000u : 0x80008000u;
template <int FMT>
__device__ __forceinline__ uint32_t not_finite(uint32_t w)
{
    constexpr uint32_t E = FMT == 0 ? 0x7F800000u : FMT == 1 ? 0x7C007C00u : 0x7F807F80u, LEAST = FMT == 0 ? 0x00800000u : FMT == 1 ? 0x04000400u : 0x00800080u;
    return (w & E) + LEAST;
}

// Elements as what they do to a sum: 1 for an infinity, 128 for a negative one, 129 for a NaN, 0 for all else.  Of up to 64 elements, a sum of these tells
// what theirs is.
template <int FMT>
__device__ __forceinline__ uint32_t effect_of(uint32_t w)
{
    if constexpr (FMT == 0) {
        const float x = __uint_as_float(w);
        return __float_as_uint(x != x ? 129.0f : x == INFINITY ? 1.0f : x == -INFINITY ? 128.0f : 0.0f);
    } else {
        constexpr uint32_t E = FMT == 1 ? 0x7C00u : 0x7F80u, ONE = FMT == 1 ? 0x3C00u : 0x3F80u, MANY = FMT == 1 ? 0x5800u : 0x4300u, BOTH = FMT == 1 ? 0x5808u : 0x4301u;
        auto half = [](uint32_t h) { return (h & E) != E ? 0u : (h & 0x7FFFu) != E ? BOTH : h >> 15 ? MANY : ONE; };
        return half(w & 0xFFFFu) | half(w >> 16) << 16;
    }
}
__device__ __forceinline__ float sum_of_effects(float effects)
{
    const uint32_t n = (uint32_t)effects;
    return n == 0 ? 0.0f : n < 128 ? INFINITY : n & 127 ? NAN : -INFINITY;
}

// Over a wave, without a trip through LDS.
template <int J> __device__ __forceinline__ float xor_lane_float(float v) { return __uint_as_float(xor_lane_u32<J, true>(__float_as_uint(v))); }
__device__ __forceinline__ float wave_max_float(float v)
{
    v = fmaxf(v, xor_lane_float<1>(v));
    v = fmaxf(v, xor_lane_float<2>(v));
    v = fmaxf(v, xor_lane_float<4>(v));
    v = fmaxf(v, xor_lane_float<8>(v));
    v = fmaxf(v, xor_lane_float<16>(v));
    return fmaxf(v, xor_lane_float<32>(v));
}
__device__ __forceinline__ float wave_sum_float(float v)
{
    v += xor_lane_float<1>(v);
    v += xor_lane_float<2>(v);
    v += xor_lane_float<4>(v);
    v += xor_lane_float<8>(v);
    v += xor_lane_float<16>(v);
    return v + xor_lane_float<32>(v);
}

// Over the four lanes of a row, without a trip through LDS.
__device__ __forceinline__ float max_over_groups(float v)
{
    v = fmaxf(v, __uint_as_float(xor16_valu_u32(__float_as_uint(v))));
    return fmaxf(v, __uint_as_float(xor32_u32(__float_as_uint(v))));
}
__device__ __forceinline__ float sum_over_groups(float v)
{
    v += __uint_as_float(xor16_valu_u32(__float_as_uint(v)));
    return v + __uint_as_float(xor32_u32(__float_as_uint(v)));
}

// Tokens a wave takes at a time where it has tiles of its own: 16 KB of keys and values where there are registers for that.
template <int FMT, int DP, int QT> constexpr int attend_tile = (FMT == 0 ? 16 : 32) * (DP == 64 && QT <= 2 ? 2 : 1);

// How a kernel's LDS is laid out.  ROWS: the four waves have rows of their own and share tiles of 64 tokens, keys and values both in LDS;
// else they have all rows and tiles of their own, keys straight in registers, values in LDS.
template <int FMT, int DP, int QT, bool ROWS>
struct AttendShape {
    static constexpr int ES = FMT == 0 ? 4 : 2;
    static constexpr int KS = DP / 32;                  // steps of 32 elements
    static constexpr int DT = DP / 16;                  // tiles of 16 elements
    static constexpr int NT = ROWS ? 1 : attend_tile<FMT, DP, QT> / 16;     // 16-token tiles a wave loads at a time
    static constexpr int CT = ROWS ? 4 : NT;            // and works on at a time
    static constexpr int TT = 16 * CT;
    static constexpr int ROW = DP * ES;                 // bytes
    static constexpr int CH = ROW / 16;
    static constexpr int RK = CH >= 16 ? 1 : 16 / CH;   // tokens whose rows share 256 bytes
    static constexpr int TILE = TT * ROW;
    static constexpr int BUFS = ROWS ? (4 * TILE <= 131072 ? 2 : 1) : 1;
    static constexpr int LOOP = ROWS ? 2 * TILE * BUFS : 4 * TILE;
    static constexpr int JOIN = ROWS ? 0 : 4 * QT * (DT / 4) * 1024;
    static constexpr int LDS = LOOP > JOIN ? LOOP : JOIN;
    static constexpr int REGS = QT * (DT * 4 + KS * 4 * (FMT == 0 ? 2 : 1)) + 2 * NT * KS * 4 * (FMT == 0 ? 2 : 1) + CT * QT * 4;
    static constexpr int PER_SIMD = REGS <= 190 ? 2 : 1;

    // Weights of 16 bits leave an output 1.4 times as far from the exact one as its own rounding does (2.3e-3 against 1.66e-3 in bf16, 2.9e-4 against 2.07e-4 in
    // fp16).  In attention over a sentence's own cache (PARTS, below, has the product throughout), where memory is what bounds, what the rounding leaves of a weight goes through a second product, and they do not: 64 sentences of 20 branches 65.4 us instead of
    // 64.1, 4 of 57000 tokens 192.6 either way.  Where the matrix units and the VALU do, they are left at that: with the second product 36 rows of 64 a head would take 45.7 us instead of 42.9,
    // 64 of 128 106 instead of 96, 32 drafts of 63 nodes 156 instead of 122, 8 prompts of 1500 tokens 346 instead of 277.
    static constexpr bool REST = FMT != 0 && !ROWS && QT <= 2;

    // A row's chunks are rotated, so that 16 lanes that read one chunk of 16 rows (keys), or 32 lanes that read 32 bytes of eight
    // rows (values; 64 of four in fp32), meet all 64 banks.
    static __device__ __forceinline__ int key_at(int token, int chunk)
    {
        return token * ROW + ((chunk + (token % 16) / RK) & (CH - 1)) * 16;
    }
    static __device__ __forceinline__ int value_at(int token, int chunk)
    {
        if constexpr (FMT == 0) return token * ROW + (((chunk >> 2) + (token >> 2)) & (CH / 4 - 1)) * 64 + (chunk & 3) * 16;
        else return token * ROW + (((chunk >> 1) + (token % 16) / RK) & (CH / 2 - 1)) * 32 + (chunk & 1) * 16;
    }
};

// Bound: without ROWS memory; each token is read once.  A pool with the heads of a token side by side gives 128 or 256 bytes at a time (64 sentences of
// 20 branches, heads of 64: 65.7 us, 4.8 TB/s; 4 of 57000 tokens, heads of 128: 186 us, 5.1 TB/s), one with a head's tokens side by side
// more (the second and its join 172 us instead of 193).  With ROWS the issue slots: a tile of 64 tokens and 32 rows of 128 takes a wave 64 matrix instructions
// and 340 others of the VALU (32 sentences of 500 to 4000 tokens, 63 nodes of 32 heads: 125 us, 0.6 PFLOP/s of fp16).
//
// SIDE: heads of a workgroup.  With two, waves 0 and 2 have the first, 1 and 3 the second: a longer stretch of memory where the heads of a token lie
// side by side, and twice the tiles a wave for the same start and end (when this was chosen, a call of the first case above took 83 -> 75 us, with four heads 106).
//
// Workgroups come to the eight XCDs in turn.  The row tiles of one part of one head, which read the same tokens, are put behind each
// other on one XCD, whose L2 then serves all but the first (63 nodes, 8 query heads to one, 32 sentences of 500 to 4000 tokens:
// 225 -> 140 us when this was chosen).  There the parts of the token axis vary slowest, so that what is left of short sentences comes last; where
// tokens are read once they vary fastest (4 sentences of 50000 and more: 186 instead of 199 us).
//
// PARTS: results are always left as parts, for another join; and the nodes of several sentences may be taken for those of one.  What the rounding leaves of weights goes through a second
// product whatever the form (64 sentences of 80 rows of 128, 8 heads, over 900 to 1500 tokens: 115 to 122 us instead of 101; 128 of 64 rows over 110 to 160, 4 heads: 26.5 either way).
template <int FMT, int DP, int QT, bool ROWS, int SIDE, bool PARTS = false>
__global__ __launch_bounds__(256, (AttendShape<FMT, DP, QT, ROWS>::PER_SIMD)) void dba_attend_kernel(AttendParams p)
{
    typedef AttendShape<FMT, DP, QT, ROWS> A;
    typedef typename Elem<FMT>::type E;
    constexpr int KS = A::KS, DT = A::DT, NT = A::NT, CT = A::CT, TT = A::TT, FC = Frag<FMT>::C, NE = 16 / A::ES;
    constexpr bool REST = A::REST || (PARTS && FMT != 0);
    extern __shared__ __align__(16) unsigned char s_mem[];
    __shared__ float s_ml[4][16 * QT][2];
    __shared__ unsigned long long s_live[2][4];
    __shared__ int s_bad[2][4];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x, turn = id / 8;
    const uint32_t group = turn / (uint32_t)p.row_tiles * 8 + id % 8;
    if (group >= (uint32_t)p.groups) return;
    const int row_tile = (int)(turn % (uint32_t)p.row_tiles);
    int split, pair;
    if (ROWS) {
        split = (int)(group / (uint32_t)p.pairs);
        pair = (int)(group % (uint32_t)p.pairs);
    } else {
        pair = (int)(group / (uint32_t)p.splits);
        split = (int)((group + (uint32_t)pair * (uint32_t)p.splits / 8) % (uint32_t)p.splits);    // (an XCD gets all kinds of parts)
    }
    const int heads_at = p.heads / SIDE;
    const int b = pair / heads_at, head0 = pair % heads_at * SIDE, head = head0 + wave % SIDE;
    const int G = p.q_heads / p.heads, rows = p.n * G;
    const int row0 = (ROWS ? row_tile * 4 + wave : row_tile) * 16 * QT;

    int tree_all;
    const Span span = span_of_rows(p, b, row_tile, G, tree_all);
    const int tree = span.end - span.prefix;           // (max_len leaves room for a few tiles more before 2^31)
    const int prefix_tiles = (span.prefix + TT - 1) / TT, tiles = prefix_tiles + (tree + TT - 1) / TT;
    const int u0 = split * p.chunk, u1 = min(tiles, u0 + p.chunk);
    if (u0 >= tiles && split > 0) return;              // (the join does not ask for it; the first split is always there)

    // the queries, and what rows they are
    Frag<FMT> q[QT][KS];
    const unsigned long long *mask_row[QT];
    int chain[QT];                                     // the last tree token a row of a chain sees
    const uint32_t sign = p.scale < 0.0f ? (FMT == 0 ? 0x80000000u : 0x80008000u) : 0u;    // a negative scale turns the queries round
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int r = row0 + t * 16 + c, node = min(r, rows - 1) / G, h = head * G + min(r, rows - 1) % G;
        const int sent = PARTS ? b + node / p.per : b, token = PARTS ? node % p.per : node;
        const E *src = reinterpret_cast<const E *>(p.q.data) + ((int64_t)sent * p.q.sent + (int64_t)token * p.q.token + (int64_t)h * p.q.head);
        mask_row[t] = p.mask ? p.mask + ((int64_t)b * p.n + node) * p.mask_words : nullptr;
        chain[t] = tree_all - p.n + node;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
#pragma unroll
            for (int f = 0; f < FC; ++f) {
                const int d = k * 32 + g * 8 + f * NE;
                u32x4 v = u32x4{0, 0, 0, 0};
                if (r < rows && d < p.D && p.scale != 0.0f) v = *reinterpret_cast<const u32x4 *>(src + d);
                q[t][k].c[f] = v ^ sign;
            }
        }
    }
    const float sl2 = p.scale != 0.0f ? fabsf(p.scale) * kLog2e : 1.0f;    // (without a scale the queries are 0)

    // tokens of tile u that this wave loads: 16 * (ROWS ? wave : 0) + 16 t + c
    const int load0 = ROWS ? wave * 16 : 0;
    const int step = ROWS ? 1 : 4 / SIDE, first = ROWS ? u0 : u0 + wave / SIDE;
    auto page_of = [&](int u, int t) -> int {          // -1: no such token
        const bool in_tree = u >= prefix_tiles;
        const int pos = (in_tree ? span.prefix + (u - prefix_tiles) * TT : u * TT) + load0 + t * 16 + c;
        const int lim = in_tree ? span.prefix + tree : span.prefix;
        int page = -1;
        if (u < u1 && pos < lim) page = p.cache.table[(int64_t)b * p.cache.table_stride + (pos >> p.cache.page_shift)];
        return (uint32_t)page < (uint32_t)p.cache.n_pages ? page : -1;
    };
    const int64_t head_at = (int64_t)head * p.cache.head_stride;
    auto offset_of = [&](int u, int t, int page) -> int64_t {      // of a token that is not there: of one that is
        if (page < 0) return head_at;
        const int pos = (u >= prefix_tiles ? span.prefix + (u - prefix_tiles) * TT : u * TT) + load0 + t * 16 + c;
        return (int64_t)page * p.cache.page_stride + (int64_t)(pos & ((1 << p.cache.page_shift) - 1)) * p.cache.token_stride + head_at;
    };
    bool met = false;                                  // this wave has met a value of the tree that is not finite
    u32x4 kr[NT][KS][FC], vr[NT][KS][FC];
    // a chunk behind the head's end is read as its first: the queries have 0 there, and nobody asks for those outputs
    auto load = [&](const unsigned char *pool, u32x4 (&to)[KS][FC], int64_t at) {
        const E *src = reinterpret_cast<const E *>(pool) + at;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int f = 0; f < FC; ++f) {
                const int d = k * 32 + g * 8 + f * NE;
                to[k][f] = *reinterpret_cast<const u32x4 *>(src + (d < p.D ? d : 0));
            }
    };

    auto any_not_finite = [&](const u32x4 (&v)[KS][FC]) {      // of a wave's 16 tokens
        uint32_t bits = 0;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int f = 0; f < FC; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) bits |= not_finite<FMT>(v[k][f][i]);
        return __any((bits & kSignBits<FMT>) != 0);
    };

    // which rows see which tokens of tile u (bit t: token t)
    auto seen_of = [&](int u, int t) -> unsigned long long {
        if (u < prefix_tiles || u >= u1) return ~0ull;
        const int j0 = (u - prefix_tiles) * TT;
        if (p.mask) return (j0 >> 6) < p.mask_words ? mask_row[t][j0 >> 6] >> (j0 & 63) : 0;
        const int last = chain[t] - j0;
        return last < 0 ? 0 : last >= 63 ? ~0ull : (2ull << last) - 1;
    };
    unsigned long long seen[QT], seen_next[QT];

    f32x4 o[QT][DT];
    float m[QT], l[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m[t] = -INFINITY;
        l[t] = 0.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    unsigned char *const s_v = s_mem + (ROWS ? A::TILE * A::BUFS : wave * A::TILE);
    int page[NT], page_next[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        page[t] = page_of(first, t);
        page_next[t] = page_of(first + step, t);
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) seen_next[t] = seen_of(first, t);
    if (first < u1) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int64_t at = offset_of(first, t, page[t]);
            load(p.k_pages, kr[t], at);
            load(p.v_pages, vr[t], at);
        }
    }

    int buf = 0;
    for (int u = first; u < u1; u += step) {
        const bool in_tree = u >= prefix_tiles;
        unsigned char *const kb = s_mem + buf * A::TILE, *const vb = s_v + (ROWS ? buf * A::TILE : 0);
        // this wave's tokens of the tile: values into LDS, where those that are not there, and in the tree what is not finite, become 0
        unsigned long long live = 0;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const unsigned long long here = __ballot(page[t] >= 0) & 0xFFFF;
            live |= here << (load0 + t * 16);
            if (here != 0xFFFF) {
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int f = 0; f < FC; ++f)
                        if (page[t] < 0) vr[t][k][f] = u32x4{0, 0, 0, 0};
            }
            if (in_tree && any_not_finite(vr[t])) {
                met = true;
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int f = 0; f < FC; ++f) vr[t][k][f] = finite_of<FMT>(vr[t][k][f]);
            }
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int f = 0; f < FC; ++f) {
                    const int token = load0 + t * 16 + c, chunk = (k * 4 + g) * FC + f;
                    *reinterpret_cast<u32x4 *>(vb + A::value_at(token, chunk)) = vr[t][k][f];
                    if constexpr (ROWS) *reinterpret_cast<u32x4 *>(kb + A::key_at(token, chunk)) = kr[t][k][f];
                }
        }
        if constexpr (ROWS) {
            if (lane == 0) s_live[buf][wave] = live;
            __syncthreads();
            live = s_live[buf][0] | s_live[buf][1] | s_live[buf][2] | s_live[buf][3];
        }
        // The next tile's mask and values, and in this form its keys, are asked for now, and before them the pages of the one
        // behind: loads come back in order, so waiting for a tile is waiting for all that the next steps need.
        int64_t at[NT];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            seen[t] = seen_next[t];
            seen_next[t] = seen_of(u + step, t);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            page[t] = page_next[t];
            at[t] = offset_of(u + step, t, page[t]);
            page_next[t] = page_of(u + 2 * step, t);
            load(p.v_pages, vr[t], at[t]);
            if constexpr (ROWS) load(p.k_pages, kr[t], at[t]);
        }
        // S^T
        f32x4 s[CT][QT];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
#pragma unroll
            for (int j = 0; j < QT; ++j) s[t][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                Frag<FMT> kf;
#pragma unroll
                for (int f = 0; f < FC; ++f) {
                    if constexpr (ROWS) kf.c[f] = *reinterpret_cast<const u32x4 *>(kb + A::key_at(t * 16 + c, (k * 4 + g) * FC + f));
                    else kf.c[f] = kr[t][k][f];
                }
#pragma unroll
                for (int j = 0; j < QT; ++j) s[t][j] = mfma32<FMT>(kf, q[j][k], s[t][j]);
            }
        }
        if constexpr (!ROWS) {
#pragma unroll
            for (int t = 0; t < NT; ++t) load(p.k_pages, kr[t], at[t]);
        }
        // softmax, one row a lane
        constexpr unsigned long long kAll = TT == 64 ? ~0ull : (1ull << (TT & 63)) - 1;
#pragma unroll
        for (int j = 0; j < QT; ++j) {
            const unsigned long long sees = seen[j] & live;
            if (__any((sees & kAll) != kAll)) {
#pragma unroll
                for (int t = 0; t < CT; ++t) {
                    const uint32_t four = (uint32_t)(sees >> (t * 16 + g * 4));
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!((four >> i) & 1)) s[t][j][i] = -INFINITY;
                }
            }
            float top = s[0][j][0];
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][j][i]);
            top = fmaf(max_over_groups(top), sl2, -kWeightBits<FMT>);
            if (__any(top > m[j] + kWeightRoom<FMT>)) {
                const float m1 = top > m[j] + kWeightRoom<FMT> ? top : m[j];       // (a row's own: what others of the wave see is nothing to it)
                const float keep = m1 == m[j] ? 1.0f : __builtin_amdgcn_exp2f(m[j] - m1);
                m[j] = m1;
                l[j] *= keep;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[j][d] *= keep;
            }
            const float base = m[j] == -INFINITY ? 0.0f : m[j];
            float sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[t][j][i] = __builtin_amdgcn_exp2f(fmaf(s[t][j][i], sl2, -base));
                    sum[i & 1] += s[t][j][i];
                }
            l[j] += sum[0] + sum[1];
        }
        // O^T += V^T P^T
        if constexpr (FMT == 0) {
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float v = *reinterpret_cast<const float *>(vb + A::value_at(t * 16 + 4 * g + i, d * 4 + (c >> 2)) + (c & 3) * 4);
#pragma unroll
                        for (int j = 0; j < QT; ++j) o[j][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[t][j][i], o[j][d], 0, 0, 0);
                    }
        } else {
            typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
#pragma unroll
            for (int t = 0; t < CT; t += 2) {
                // weights in 16 bits, as the matrix units take them: each is off by half a step of itself, either way, and with REST what that
                // leaves is multiplied too
                Frag<FMT> w[QT], rest[QT];
#pragma unroll
                for (int j = 0; j < QT; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float w0 = s[t + i / 2][j][i % 2 * 2], w1 = s[t + i / 2][j][i % 2 * 2 + 1];
                        const uint32_t both = pack2<FMT>(w0, w1);
                        w[j].c[0][i] = both;
                        if constexpr (REST && PARTS) rest[j].c[0][i] = rest2<FMT>(w0, w1, both);
                        else if constexpr (REST) rest[j].c[0][i] = pack2<FMT>(w0 - low_half<FMT>(both), w1 - high_half<FMT>(both));
                    }
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    // lane (g, i) of 16 points at elements 4 (i % 4) .. of token 4g + i / 4 and receives element i of tokens 4g .. 4g+3
                    struct { i16x4 lo, hi; } v;
                    const int token = 4 * g + (c >> 2), in = (c & 3) * 8;
                    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(vb + A::value_at(t * 16 + token, d * 2 + (in >> 4)) + (in & 15)));
                    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(vb + A::value_at(t * 16 + 16 + token, d * 2 + (in >> 4)) + (in & 15)));
                    Frag<FMT> vf;
                    vf.c[0] = __builtin_bit_cast(u32x4, v);
#pragma unroll
                    for (int j = 0; j < QT; ++j) {
                        o[j][d] = mfma32<FMT>(vf, w[j], o[j][d]);
                        if constexpr (REST) o[j][d] = mfma32<FMT>(vf, rest[j], o[j][d]);
                    }
                }
            }
        }
        if constexpr (ROWS) {
            if (A::BUFS == 1) __syncthreads();
            else buf ^= 1;
        }
    }

    // Values of the tree that are not finite have been left out, since a weight of 0 would not keep them out of a product.  Whatever its weight, such a
    // value makes an element of the rows that see it an infinity or a NaN.  So where there were any, the tree's tiles are gone through once more, their values as
    // what they do to a sum, times 1 where they are seen.  (16 prompts of 500 to 2000 tokens asked for as 2000, 32 heads on 8 of 128 in bf16: 0.96 ms with zeros
    // behind them, 1.45 to 1.56 with infinities, NaN or any bits.)
    if constexpr (ROWS) {
        if (lane == 0) s_bad[0][wave] = met;
        __syncthreads();                               // (and nobody reads the last tiles any more)
        met = __builtin_amdgcn_readfirstlane(s_bad[0][0] | s_bad[0][1] | s_bad[0][2] | s_bad[0][3]);
    }
    if (__builtin_expect(met, 0)) {
        constexpr uint32_t ONE = FMT == 1 ? 0x3C00u : 0x3F80u;     // in 16 bits
        // (What is used here is worked out anew: registers in which it were kept are wanted by the loop above.  32 drafts of 63 nodes 130 -> 122 us.)
        const int lane1 = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0)), c1 = lane1 & 15, g1 = lane1 >> 4;
        for (int u = first + (max(prefix_tiles - first, 0) + step - 1) / step * step; u < u1; u += step) {
            unsigned long long live = 0;
            bool bad = false;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int x = (u - prefix_tiles) * TT + load0 + t * 16 + c1;
                const int64_t at = x < tree ? token_offset(p.cache, b, span.prefix + x) : -1;
                const E *src = reinterpret_cast<const E *>(p.v_pages) + (max(at, (int64_t)0) + head_at);
                live |= (__ballot(at >= 0) & 0xFFFF) << (load0 + t * 16);
                u32x4 v[KS][FC];
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int f = 0; f < FC; ++f) {
                        const int d = k * 32 + g1 * 8 + f * NE;
                        v[k][f] = *reinterpret_cast<const u32x4 *>(src + (d < p.D ? d : 0));
                    }
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int f = 0; f < FC; ++f) {
                        if (at < 0) v[k][f] = u32x4{0, 0, 0, 0};
                        *reinterpret_cast<u32x4 *>(s_v + A::value_at(load0 + t * 16 + c1, (k * 4 + g1) * FC + f)) = v[k][f];
                    }
                bad |= any_not_finite(v);
            }
            if constexpr (ROWS) {
                if (lane1 == 0) {
                    s_live[0][wave] = live;
                    s_bad[1][wave] = bad;
                }
                __syncthreads();
                live = s_live[0][0] | s_live[0][1] | s_live[0][2] | s_live[0][3];
                bad = __builtin_amdgcn_readfirstlane(s_bad[1][0] | s_bad[1][1] | s_bad[1][2] | s_bad[1][3]);
            }
            if (bad) {
                unsigned long long sees[QT];
                const int j0 = (u - prefix_tiles) * TT;
#pragma unroll
                for (int j = 0; j < QT; ++j) {
                    const int node = min(row0 + j * 16 + c1, rows - 1) / G, last = tree_all - p.n + node - j0;
                    const unsigned long long *words = p.mask + ((int64_t)b * p.n + node) * p.mask_words;
                    sees[j] = live & (p.mask ? ((j0 >> 6) < p.mask_words ? words[j0 >> 6] >> (j0 & 63) : 0) : last < 0 ? 0 : last >= 63 ? ~0ull : (2ull << last) - 1);
                }
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    f32x4 e[QT];
#pragma unroll
                    for (int j = 0; j < QT; ++j) e[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
                    for (int t = 0; t < CT; t += FMT == 0 ? 1 : 2) {
                        if constexpr (FMT == 0) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t x = *reinterpret_cast<const uint32_t *>(s_v + A::value_at(t * 16 + 4 * g1 + i, d * 4 + (c1 >> 2)) + (c1 & 3) * 4);
#pragma unroll
                                for (int j = 0; j < QT; ++j)
                                    e[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(effect_of<FMT>(x)), (sees[j] >> (t * 16 + g1 * 4 + i)) & 1 ? 1.0f : 0.0f, e[j], 0, 0, 0);
                            }
                        } else {
                            typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
                            struct { i16x4 lo, hi; } v;
                            const int token = t * 16 + 4 * g1 + (c1 >> 2), in = (c1 & 3) * 8;
                            v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(s_v + A::value_at(token, d * 2 + (in >> 4)) + (in & 15)));
                            v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(s_v + A::value_at(token + 16, d * 2 + (in >> 4)) + (in & 15)));
                            Frag<FMT> vf, w;
                            vf.c[0] = __builtin_bit_cast(u32x4, v);
#pragma unroll
                            for (int i = 0; i < 4; ++i) vf.c[0][i] = effect_of<FMT>(vf.c[0][i]);
#pragma unroll
                            for (int j = 0; j < QT; ++j) {
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const uint32_t two = (uint32_t)(sees[j] >> ((t + i / 2) * 16 + g1 * 4 + i % 2 * 2));
                                    w.c[0][i] = (two & 1 ? ONE : 0) | (two & 2 ? ONE << 16 : 0);
                                }
                                e[j] = mfma32<FMT>(vf, w, e[j]);
                            }
                        }
                    }
#pragma unroll
                    for (int j = 0; j < QT; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[j][d][i] += sum_of_effects(e[j][i]);
                }
            }
            if constexpr (ROWS) __syncthreads();
        }
    }

    // results: [rows, D] of the output, or this split's part
    const bool whole = !PARTS && tiles <= p.chunk;     // no other part has anything
    auto part_of = [&](int hd) { return (((size_t)b * p.heads + hd) * p.splits + split) * rows; };
    auto put_row = [&](int hd, int r, float mm, float ll) {        // statistics of a row
        if (!whole) {
            p.part_ml[(part_of(hd) + r) * 2] = mm;
            p.part_ml[(part_of(hd) + r) * 2 + 1] = ll;
        } else if (p.lse) {
            p.lse[((int64_t)b * p.n + r / G) * p.q_heads + hd * G + r % G] = ll != 0.0f ? (mm + __builtin_amdgcn_logf(ll)) * kLn2f : -INFINITY;
        }
    };
    auto put = [&](int hd, int r, int d, float ll, f32x4 v) {      // four elements of a row
        if (!whole) {
            *reinterpret_cast<f32x4 *>(p.part_o + (part_of(hd) + r) * p.D + d) = v;
            return;
        }
        const float f = ll != 0.0f ? 1.0f / ll : 0.0f; // (a sum that is not a number is not nothing)
        E *to = reinterpret_cast<E *>(p.out.data) + ((int64_t)b * p.out.sent + (int64_t)(r / G) * p.out.token + (int64_t)(hd * G + r % G) * p.out.head + d);
        v *= f;
        if constexpr (FMT == 0) *reinterpret_cast<f32x4 *>(to) = v;
        else *reinterpret_cast<uint2 *>(to) = make_uint2(pack2<FMT>(v[0], v[1]), pack2<FMT>(v[2], v[3]));
    };
#pragma unroll
    for (int j = 0; j < QT; ++j) l[j] = sum_over_groups(l[j]);
    if constexpr (ROWS) {
#pragma unroll
        for (int j = 0; j < QT; ++j) {
            const int r = row0 + j * 16 + c;
            if (r >= rows) continue;
            if (g == 0) put_row(head, r, m[j], l[j]);
#pragma unroll
            for (int d = 0; d < DT; ++d)
                if (d * 16 + g * 4 < p.D) put(head, r, d * 16 + g * 4, l[j], o[j][d]);
        }
    } else {
        // the four waves' parts: each on the common maximum, then added up from LDS
        if (g == 0)
#pragma unroll
            for (int j = 0; j < QT; ++j) {
                s_ml[wave][j * 16 + c][0] = m[j];
                s_ml[wave][j * 16 + c][1] = l[j];
            }
        __syncthreads();                               // (and nobody reads values any more)
        float sum[SIDE][QT], f[QT];                       // of each head of this workgroup
#pragma unroll
        for (int hh = 0; hh < SIDE; ++hh) {
#pragma unroll
            for (int j = 0; j < QT; ++j) {
                float top = -INFINITY;
                sum[hh][j] = 0.0f;
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    if (w % SIDE == hh) top = fmaxf(top, s_ml[w][j * 16 + c][0]);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    if (w % SIDE != hh) continue;
                    const float mw = s_ml[w][j * 16 + c][0], lw = s_ml[w][j * 16 + c][1];
                    sum[hh][j] += mw == -INFINITY ? lw : lw * __builtin_amdgcn_exp2f(mw - top);
                }
                if (wave % SIDE == hh) f[j] = m[j] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[j] - top);
                const int r = row0 + j * 16 + c;
                if (wave == hh && g == 0 && r < rows) put_row(head, r, top, sum[hh][j]);
            }
        }
        f32x4 *const s_o = reinterpret_cast<f32x4 *>(s_mem);       // [wave][j][d of this round][lane]
        constexpr int DR = DT / 4;
#pragma unroll
        for (int round = 0; round < 4; ++round) {
            if (round) __syncthreads();
#pragma unroll
            for (int j = 0; j < QT; ++j)
#pragma unroll
                for (int d = 0; d < DR; ++d) s_o[((wave * QT + j) * DR + d) * 64 + lane] = o[j][round * DR + d] * f[j];
            __syncthreads();
#pragma unroll
            for (int hh = 0; hh < SIDE; ++hh) {
#pragma unroll
                for (int j = 0; j < QT; ++j)
#pragma unroll
                    for (int d = 0; d < DR; ++d) {
                        if (((hh * QT + j) * DR + d) % 4 != wave) continue;
                        f32x4 v = s_o[((hh * QT + j) * DR + d) * 64 + lane];
#pragma unroll
                        for (int w = 1; w < 4; ++w)
                            if (w > hh && w % SIDE == hh) v += s_o[((w * QT + j) * DR + d) * 64 + lane];
                        const int r = row0 + j * 16 + c, e = (round * DR + d) * 16 + g * 4;
                        if (r < rows && e < p.D) put(head0 + hh, r, e, sum[hh][j], v);
                    }
            }
        }
    }
}

// Joins the parts of a row: 2^(m_s - m) O_s and 2^(m_s - m) l_s added up over its parts s.  Of a part, a lane takes four elements, and as many parts
// are taken at a time as there are lanes for.  A wave has Q rows of one row tile: where there are a great many rows, what is done once a wave
// (addresses, divisions) is what the VALU's time goes to (64500 rows of 128, half of them in two parts: 25 us with a row a wave, 15 with four); with few, the chain of loads
// counts, and a row a wave is best (1024 rows in 16 parts: 6.9 against 12 us).  Rows with one part have been written already.
template <int FMT, int Q>
__global__ __launch_bounds__(256) void dba_attend_join_kernel(AttendParams p, int tile, int tile_shift)
{
    typedef typename Elem<FMT>::type E;
    const int lane = (int)threadIdx.x & 63, b = (int)blockIdx.z, head = (int)blockIdx.y;
    const int G = p.q_heads / p.heads, rows = p.n * G;
    const int r0 = ((int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)) * Q;
    if (r0 >= rows) return;
    int tree_all;
    const Span span = span_of_rows(p, b, r0 >> tile_shift, G, tree_all);
    const int tiles = (span.prefix + tile - 1) / tile + (span.end - span.prefix + tile - 1) / tile;
    if (tiles <= p.chunk) return;
    const int parts = (tiles + p.chunk - 1) / p.chunk;
    const size_t part = ((size_t)b * p.heads + head) * p.splits * rows + r0;
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
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            float ms = -INFINITY, ls = 0.0f;
            if (lane < n && r0 + q < rows) {
                const float2 ml = *reinterpret_cast<const float2 *>(p.part_ml + (part + (size_t)(s0 + lane) * rows + q) * 2);
                ms = ml.x;
                ls = ml.y;
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
                const int s = s1 + x * side + lane / across;
                const float *at = p.part_o + (part + (size_t)(s0 + s) * rows) * p.D + d;
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

// The most 16-row tiles a wave has registers for where it holds all rows of a head.
template <int FMT, int DP> constexpr int kAttendWidest = DP == 64 ? 4 : DP == 128 ? (FMT == 0 ? 2 : 4) : 1;

// How a call is laid out: which kernel, how many workgroups along the rows and the token axis.
struct AttendPlan {
    int DP, QT;
    int side;                          // heads of a workgroup whose waves have tiles of their own: 1 or 2
    bool shared;                       // the waves have rows of their own (ROWS)
    int tile, tile_rows, row_tiles, splits, chunk;
    bool dense = false;                // rows that all see all tokens, and many of them: dba_common_kernel
};

template <int FMT> hipError_t attend_launch(const AttendParams &p, const AttendPlan &plan, int B, hipStream_t stream);

}  // namespace dba
