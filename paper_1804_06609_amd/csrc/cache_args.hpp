// What the entry points around a paged cache share: checks of their arguments, and how attention is laid out.  Host only.
#pragma once
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "../../include/dba_beam.h"
#include "entry.hpp"
#include "places.hpp"
#include "tree_attend.hpp"

namespace dba {

extern template hipError_t attend_launch<0>(const AttendParams &, const AttendPlan &, int, hipStream_t);
extern template hipError_t attend_launch<1>(const AttendParams &, const AttendPlan &, int, hipStream_t);
extern template hipError_t attend_launch<2>(const AttendParams &, const AttendPlan &, int, hipStream_t);

constexpr size_t align256(size_t x) { return (x + 255) / 256 * 256; }
constexpr int kMostRows = 1 << 22;          // tokens, or heads of tokens, of one sentence in a call
constexpr int kMostLength = INT32_MAX - 1023;   // tokens that attention looks at: positions of the tiles behind them are ints, too

inline int launched(const char *who, hipError_t e)
{
    return e == hipSuccess ? DBA_OK : set_error(DBA_EHIP, "%s: launch failed: %s", who, hipGetErrorString(e));
}

// ---- caches -------------------------------------------------------------------------------------------------------

inline const char *cache_fault(const dba_cache *c)
{
    if (!c) return "the cache is NULL";
    if (!format_ok(c->format)) return "unknown format";
    if (!c->k || !c->v || !c->table) return "a pointer of the cache is NULL";
    if (c->heads < 1 || c->heads > 1024) return "1 <= heads <= 1024";
    if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8) return "head_dim must be a multiple of 8, 8 to 256";
    if (c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return "page_size must be a power of two, at most 65536";
    if (c->n_pages < 1 || c->max_pages < 1) return "n_pages and max_pages must be at least 1";
    if ((int64_t)c->max_pages * c->page_size > INT32_MAX) return "max_pages * page_size must be below 2^31";
    if (c->table_stride < c->max_pages) return "table_stride is less than max_pages";
    const int unit = 16 / (int)elem_bytes(c->format);
    if (misaligned(c->k, 16) || misaligned(c->v, 16) || c->page_stride % unit || c->token_stride % unit || c->head_stride % unit ||
        c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0)
        return "k, v and the strides of pages, tokens and heads must be multiples of 16 bytes, none negative";
    return nullptr;
}

inline const char *heads_fault(const dba_heads *h, int format)
{
    if (!h || !h->data) return "a tensor is NULL";
    const int unit = 16 / (int)elem_bytes(format);
    if (misaligned(h->data, 16) || h->sent_stride % unit || h->token_stride % unit || h->head_stride % unit || h->sent_stride < 0 ||
        h->token_stride < 0 || h->head_stride < 0)
        return "tensors and their strides must be multiples of 16 bytes, none negative";
    return nullptr;
}

inline Paged paged_of(const dba_cache &c)
{
    Paged p;
    p.table = c.table;
    p.table_stride = c.table_stride;
    p.page_stride = c.page_stride;
    p.token_stride = c.token_stride;
    p.head_stride = c.head_stride;
    p.n_pages = c.n_pages;
    p.page_shift = __builtin_ctz((unsigned)c.page_size);
    p.max_pages = c.max_pages;
    return p;
}

// What a tensor [B, n, heads, head_dim], and a pool of pages, take up.
inline Places places_of(const dba_heads &h, int B, int n, int heads, const dba_cache &c)
{
    const int64_t e = elem_bytes(c.format);
    return Places(h.data, c.head_dim * e).axis(B, h.sent_stride * e).axis(n, h.token_stride * e).axis(heads, h.head_stride * e);
}
inline Places places_of(const void *pool, const dba_cache &c)
{
    const int64_t e = elem_bytes(c.format);
    return Places(pool, c.head_dim * e).axis(c.n_pages, c.page_stride * e).axis(c.page_size, c.token_stride * e).axis(c.heads, c.head_stride * e);
}
inline bool same(const dba_heads &a, const dba_heads &b)
{
    return a.data == b.data && a.sent_stride == b.sent_stride && a.token_stride == b.token_stride && a.head_stride == b.head_stride;
}

inline HeadsAt heads_of(const dba_heads *h)
{
    if (!h) return HeadsAt{nullptr, 0, 0, 0};
    return HeadsAt{static_cast<unsigned char *>(h->data), h->sent_stride, h->token_stride, h->head_stride};
}

// Rows (nodes times the query heads of a cache head) decide the form.  Up to 64, a wave holds them all and the waves share out the tokens,
// which are then read once; with more, or without registers for so many, the waves have rows of their own and share the tokens' tiles
// (when this was chosen, 504 rows of 128 took 145 us against 246 with row tiles of 64 that each read the tokens; 40 to 48 rows of 128: 175 and 197 us against
// 182 and 184 with shared tiles).  The token axis is cut into as many parts as fill the GPU once: each part costs a start-up of several
// trips to memory, and twice as many were slower (one sentence of 29000 tokens 59 against 43 us, five of 21600 56 against 39),
// but for shared tiles, whose sentences' lengths matter more than that.  There the first part of a sentence has a quarter more than an even share, so that
// fewer sentences have rows to join and what comes last is short (when this was chosen, 32 sentences of 500 to 4000 tokens, 63 nodes of 32 heads: 127 us; even parts
// 144, half as much again 135, one part a sentence 147, three 153).  Parts have four tiles at least, three with heads of 256, or joining costs more than
// they save (11 sentences of 930 tokens, 32 nodes, parts of 1, 2, 4, 8 tiles: 34, 28, 25, 29 us; one of 4000 tokens, fp32: 82, 83, 59, 93).
// Two heads a workgroup (SIDE) halve the workgroups, then: 1024 heads of 64 in two rounds of 512 or in one 83 and 75 us, of 128 81 and 74, 1024 of 256 in four rounds or
// two 122 and 116, 2048 of 32 66 and 62; but 1200 of 80, in three rounds or in two of which the second is nearly empty, 75 and 82, and 512 of 128, which then need
// parts to fill the GPU, 110 and 117.
inline AttendPlan attend_plan(int B, int n, int q_heads, const dba_cache &c, int max_len)
{
    AttendPlan a;
    const int rows = n * (q_heads / c.heads);
    const bool f32 = c.format == DBA_LOGP_F32;
    a.DP = c.head_dim <= 64 ? 64 : c.head_dim <= 128 ? 128 : 256;
    const int widest = a.DP == 64 ? kAttendWidest<1, 64> : a.DP == 256 ? kAttendWidest<1, 256> : f32 ? kAttendWidest<0, 128> : kAttendWidest<1, 128>;
    a.shared = rows > 16 * widest;
    a.QT = a.shared ? (a.DP <= 128 ? 2 : 1) : rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    a.tile_rows = (a.shared ? 64 : 16) * a.QT;
    a.row_tiles = (rows + a.tile_rows - 1) / a.tile_rows;
    a.tile = a.shared ? 64
           : a.DP == 64 && a.QT <= 2 ? (f32 ? attend_tile<0, 64, 2> : attend_tile<1, 64, 2>) : f32 ? attend_tile<0, 256, 1> : attend_tile<1, 256, 1>;
    const int tiles = (max_len + a.tile - 1) / a.tile + 1;         // (the prefix and the tree each end in a tile of their own)
    const int resident = a.DP == 256 || (a.DP == 128 && (a.QT == 4 || (f32 && a.QT == 2))) ? 256 : 512;
    // two heads a workgroup where that leaves no more of the last round of workgroups empty
    const int64_t pairs = (int64_t)B * c.heads;
    const auto rounds = [&](int64_t n) { return (n + resident - 1) / resident; };
    a.side = !a.shared && c.heads % 2 == 0 && pairs >= 2 * resident && 2 * rounds(pairs / 2) * 19 <= rounds(pairs) * 20 ? 2 : 1;
    const int64_t groups = pairs / a.side * a.row_tiles;
    const int64_t parts = std::max<int64_t>(1, resident * (a.shared ? 2 : 1) / groups);
    const int64_t even = (tiles + parts - 1) / parts;
    const int64_t chunk = a.shared ? std::max<int64_t>(a.DP == 256 ? 3 : 4, even * 5 / 4) : std::max<int64_t>(4 / a.side, (even + 3) / 4 * 4);
    a.chunk = (int)chunk;
    a.splits = (int)((tiles + chunk - 1) / chunk);
    return a;
}

inline const char *attend_fault(int B, int n, int q_heads, const dba_cache *cache, int max_len)
{
    const char *fault = cache_fault(cache);
    if (fault) return fault;
    if (B < 1 || B > 65535 || n < 1 || q_heads < 1 || q_heads > 8192 || (int64_t)n * q_heads > kMostRows)
        return "need 1 <= B <= 65535, 1 <= q_heads <= 8192, n >= 1, n * q_heads <= 2^22";
    if (q_heads % cache->heads) return "q_heads must be a multiple of the cache's heads";
    if (max_len < 1 || max_len > cache->max_pages * cache->page_size || max_len > kMostLength)
        return "need 1 <= max_len <= max_pages * page_size, max_len <= 2^31 - 1024";
    if ((int64_t)B * cache->heads * (((int64_t)n * (q_heads / cache->heads) + 15) / 16) > (1 << 28))
        return "need B * heads * (n * q_heads / heads, in sixteens) <= 2^28";
    return nullptr;
}

inline size_t attend_rows_of(int B, int n, int q_heads, const AttendPlan &a) { return (size_t)B * n * q_heads * a.splits; }

}  // namespace dba
