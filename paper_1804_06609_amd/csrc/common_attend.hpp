// Attention of a great many rows over the same tokens, all of which every row sees: kernel.
#pragma once
#include <type_traits>

#include "tree_attend.hpp"

namespace dba {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// c += a b^T of 32 rows each over 16 elements; lane (h, i) of two 32s gives elements 8h .. 8h+7 of row i of a and of b, and has rows 8 (x / 4) + 4h + x % 4 of
// column i.
template <int FMT>
__device__ __forceinline__ f32x16 mfma16(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (FMT == 1) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// (In assembly, as the compiler would first make b and c canonical.  It does not know that this reads them: where a matrix instruction has written them, `a` has to come from an
// ordinary instruction that read another element of the same result, and so has waited for all of it.)
__device__ __forceinline__ float max_of_3(float a, float b, float c)
{
    float d;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

// 64 bytes' worth of lanes put 16 bytes each from where they point into LDS, one behind the other, without a register; done when the wave's loads are.
__device__ __forceinline__ void load_to_lds(const void *from, void *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) unsigned int *)from, (__attribute__((address_space(3))) unsigned int *)to, 16, 0, 0);
}

// Four waves of 32 rows each, tiles of 64 tokens in LDS twice.  Of a token's 16-byte chunks, which a wave's lanes put side by side, each reads one of another place, so
// that 16 lanes that read a chunk of 16 keys, or 32 that read 64 bytes of four tokens' values, meet all 64 banks.
template <int DP>
struct CommonShape {
    static constexpr int TT = 64, ROW = DP * 2, CH = ROW / 16;
    static constexpr int KS = DP / 16, DB = DP / 32;
    static constexpr int TILE = TT * ROW, LDS = 4 * TILE;
    static constexpr int PER = 64 / CH, LOADS = TT / 4 / PER;       // tokens of a wave's load, and loads of its 16 tokens
    static __device__ __forceinline__ int key_swap(int token) { return (token / (16 / CH)) & (CH - 1); }
    static __device__ __forceinline__ int value_swap(int token) { return CH == 16 ? (token & 3) << 2 : ((token >> 1) & 1) << 2; }
};

// As in dba_attend_kernel both products are transposed and the weights stay in registers: S^T = K Q^T leaves a lane with 16 tokens of one row for each 32 of them, which in
// their order are what O^T = V^T P^T takes, V^T coming out of LDS through the transposing read.  The path of a tile that is all there has no branch but the one around
// new maxima.
//
// Weights are rounded to 16 bits for the matrix units, and what that leaves of them goes through a second product with the same values: outputs are then as far from the exact ones as their own
// rounding (1.66e-3 in bf16, 2.07e-4 in fp16) and no further, as they would be without it (2.3e-3, 2.9e-4).  It costs half as many matrix instructions again and 48 others a tile, and nothing of LDS: 8192
// rows of 128 over 8000 tokens, 4 heads: 224 us instead of 173 to 181; 5120 over 1500, 8 heads: 77 instead of 65.
//
// Bound: no unit alone.  In the first of these the matrix units are at work for 49 % of the clocks, the VALU for 39, LDS, whose reads take 64 bytes a clock, for 68; with two waves a SIMD the first two hardly
// overlap (0.60 PFLOP/s, each product counted once).  64 rows a wave would halve what is read of LDS, but have not the registers (when the kernel had one product and 173 us: a wave alone on its SIMD 209, two with
// a half of each tile's tokens for either, whose 35 spilled registers make every tile wait for the next one's loads, 267).
template <int FMT, int DP>
__global__ __launch_bounds__(256, 2) void dba_common_kernel(AttendParams p)
{
    typedef CommonShape<DP> A;
    typedef typename Elem<FMT>::type E;
    constexpr int KS = A::KS, DB = A::DB, TT = A::TT;
    extern __shared__ __align__(16) unsigned char s_mem[];
    __shared__ unsigned s_live[2][4];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int i = lane & 31, h = lane >> 5;
    // workgroups come to the eight XCDs in turn: those of one part of one head, which read the same tokens, are put on one where that leaves them all as much
    int group, row_tile;
    if (p.groups % 8 == 0) {
        const uint32_t turn = blockIdx.x / 8;
        group = (int)(turn / (uint32_t)p.row_tiles * 8 + blockIdx.x % 8);
        row_tile = (int)(turn % (uint32_t)p.row_tiles);
    } else {
        group = (int)(blockIdx.x % (uint32_t)p.groups);
        row_tile = (int)(blockIdx.x / (uint32_t)p.groups);
    }
    const int head = group % p.heads, split = group / p.heads;
    const int G = p.q_heads / p.heads, rows = p.n * G, r = row_tile * p.tile_rows + wave * 32 + i;
    const int len = span_of(p.prefix[0], 0, p.max_len).prefix, tiles = (len + TT - 1) / TT;
    const int u0 = split * p.chunk, u1 = min(tiles, u0 + p.chunk);
    if (u0 >= tiles && split > 0) return;              // (the join does not ask for it; the first split is always there)

    u32x4 q[KS];
    const uint32_t sign = p.scale < 0.0f ? 0x80008000u : 0u;    // a negative scale turns the queries round
    {
        const int node = min(r, rows - 1) / G, hq = head * G + min(r, rows - 1) % G;
        const E *src = reinterpret_cast<const E *>(p.q.data) + ((int64_t)(node / p.per) * p.q.sent + (int64_t)(node % p.per) * p.q.token + (int64_t)hq * p.q.head);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int d = k * 16 + h * 8;
            u32x4 v = u32x4{0, 0, 0, 0};
            if (r < rows && d < p.D && p.scale != 0.0f) v = *reinterpret_cast<const u32x4 *>(src + d);
            q[k] = v ^ sign;
        }
    }
    const float sl2 = p.scale != 0.0f ? fabsf(p.scale) * kLog2e : 1.0f;

    // loading: this wave's tokens 16 wave + PER j + lane / CH of a tile, which lie in one page (pages have 16 tokens at least): where from there a lane reads
    uint32_t key_from[A::LOADS], value_from[A::LOADS];
#pragma unroll
    for (int j = 0; j < A::LOADS; ++j) {
        const int x = j * A::PER + lane / A::CH, token = wave * 16 + x, at = lane % A::CH;
        const int a = (at ^ A::key_swap(token)) * 8, b = (at ^ A::value_swap(token)) * 8;
        key_from[j] = (uint32_t)(x * p.cache.token_stride + (a < p.D ? a : 0)) * 2;       // (behind the head's end: its first elements)
        value_from[j] = (uint32_t)(x * p.cache.token_stride + (b < p.D ? b : 0)) * 2;
    }
    auto ask_page = [&](int u) -> int { return p.cache.table[min((u * TT + wave * 16) >> p.cache.page_shift, p.cache.max_pages - 1)]; };
    const unsigned char *const keys = p.k_pages + (int64_t)head * p.cache.head_stride * 2, *const values = p.v_pages + (int64_t)head * p.cache.head_stride * 2;
    auto ask_tile = [&](int u, int buf, int page_of) { // (of tokens that are not there: ones that are)
        const int pos = u * TT + wave * 16, page = __builtin_amdgcn_readfirstlane(page_of);
        const bool there = (uint32_t)page < (uint32_t)p.cache.n_pages && pos < len;
        const int64_t at = there ? ((int64_t)page * p.cache.page_stride + (int64_t)(pos & ((1 << p.cache.page_shift) - 1)) * p.cache.token_stride) * 2 : 0;
        unsigned char *const to = s_mem + buf * 2 * A::TILE + wave * 16 * A::ROW;
#pragma unroll
        for (int j = 0; j < A::LOADS; ++j) {
            load_to_lds(keys + at + key_from[j], to + j * A::PER * A::ROW);
            load_to_lds(values + at + value_from[j], to + j * A::PER * A::ROW + A::TILE);
        }
        if (lane == 0) s_live[buf][wave] = !there ? 0 : len - pos >= 16 ? 0xFFFFu : (1u << (len - pos)) - 1;
    };

    f32x16 o[DB];
    float m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = f32x16{};
    int key_at[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) key_at[k] = i * A::ROW + ((k * 2 + h) ^ A::key_swap(i)) * 16;     // (tokens 32 on have the same places)
    // lane (g, x) of 16 points at elements 4 (x % 4) .. of token 4h + x / 4, 16 (g % 2) elements on
    const int vt = 4 * h + ((lane & 15) >> 2), vc = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    int value_at[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) value_at[d] = A::TILE + vt * A::ROW + ((d * 4 + vc) ^ A::value_swap(vt)) * 16 + (lane & 1) * 8;

    auto work = [&](int u, auto buf_of, int page_next) {
        constexpr int buf = decltype(buf_of)::value;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // this wave's loads into LDS, which a barrier does not wait for
        __syncthreads();                               // the tile has come, and nobody reads the last one any more
        constexpr int kb = buf * 2 * A::TILE;
        const unsigned long long live = (unsigned long long)(s_live[buf][0] | s_live[buf][1] << 16) | (unsigned long long)(s_live[buf][2] | s_live[buf][3] << 16) << 32;
        const bool all = __builtin_amdgcn_readfirstlane(live == ~0ull);
        if (__builtin_expect(!all, 0)) {               // values that are not there become 0, which no weight of 0 would make them
            for (int x = lane; x < 16 * A::CH; x += 64)
                if (!((live >> (wave * 16 + x / A::CH)) & 1)) *reinterpret_cast<u32x4 *>(s_mem + kb + A::TILE + (wave * 16 + x / A::CH) * A::ROW + x % A::CH * 16) = u32x4{0, 0, 0, 0};
            __syncthreads();
        }
        if (u + 1 < u1) ask_tile(u + 1, buf ^ 1, page_next);
        // S^T
        f32x16 s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const u32x4 kf = *reinterpret_cast<const u32x4 *>(s_mem + key_at[k] + (kb + b * 32 * A::ROW));
                s[b] = mfma16<FMT>(kf, q[k], k == 0 ? f32x16{} : s[b]);
            }
        // softmax, one row a lane and a half
        if (__builtin_expect(!all, 0)) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    if (!((live >> (b * 32 + x / 4 * 8 + h * 4 + x % 4)) & 1)) s[b][x] = -INFINITY;
        }
        const float seed = fmaxf(s[0][0], s[1][0]);
        float top = max_of_3(seed, s[0][1], s[1][1]), top1 = max_of_3(seed, s[0][2], s[1][2]);
#pragma unroll
        for (int x = 3; x < 15; x += 2) {
            top = max_of_3(top, s[0][x], s[1][x]);
            top1 = max_of_3(top1, s[0][x + 1], s[1][x + 1]);
        }
        top = max_of_3(top, s[0][15], s[1][15]);
        top = fmaxf(top, top1);
        top = fmaxf(top, __uint_as_float(xor32_u32(__float_as_uint(top))));
        top = fmaf(top, sl2, -kWeightBits<FMT>);
        if (__any(top > m + kWeightRoom<FMT>)) {
            const float m1 = top > m + kWeightRoom<FMT> ? top : m;
            const float keep = m1 == m ? 1.0f : __builtin_amdgcn_exp2f(m - m1);
            m = m1;
            l *= keep;
#pragma unroll
            for (int d = 0; d < DB; ++d) o[d] *= keep;
        }
        const float base = m == -INFINITY ? 0.0f : m;
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                s[b][x] = __builtin_amdgcn_exp2f(fmaf(s[b][x], sl2, -base));
                sum[x & 1] += s[b][x];
            }
        l += sum[0] + sum[1];
        // O^T += V^T P^T
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                u32x4 w, rest;                         // weights in 16 bits, and what that leaves of them
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float w0 = s[b][y * 8 + 2 * x], w1 = s[b][y * 8 + 2 * x + 1];
                    w[x] = pack2<FMT>(w0, w1);
                    rest[x] = rest2<FMT>(w0, w1, w[x]);
                }
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
                    struct { i16x4 lo, hi; } v;
                    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(s_mem + value_at[d] + (kb + (b * 32 + y * 16) * A::ROW)));
                    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(s_mem + value_at[d] + (kb + (b * 32 + y * 16 + 8) * A::ROW)));
                    o[d] = mfma16<FMT>(__builtin_bit_cast(u32x4, v), w, o[d]);
                    o[d] = mfma16<FMT>(__builtin_bit_cast(u32x4, v), rest, o[d]);
                }
            }
    };
    if (u0 < u1) ask_tile(u0, 0, ask_page(u0));
    int page = ask_page(u0 + 1);                       // of the next tile
#pragma unroll 1
    for (int u = u0; u < u1; u += 2) {
        const int page1 = ask_page(u + 2);
        work(u, std::integral_constant<int, 0>{}, page);
        if (u + 1 == u1) break;
        page = ask_page(u + 3);
        work(u + 1, std::integral_constant<int, 1>{}, page1);
    }

    // this part's results: [rows, D] and the statistics
    const size_t part = ((size_t)head * p.splits + split) * rows;
    l += __uint_as_float(xor32_u32(__float_as_uint(l)));
    if (r >= rows) return;
    if (h == 0) *reinterpret_cast<float2 *>(p.part_ml + (part + r) * 2) = make_float2(m, l);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int e = d * 32 + x * 8 + h * 4;
            if (e < p.D) *reinterpret_cast<f32x4 *>(p.part_o + (part + r) * p.D + e) = f32x4{o[d][x * 4], o[d][x * 4 + 1], o[d][x * 4 + 2], o[d][x * 4 + 3]};
        }
}

}  // namespace dba
