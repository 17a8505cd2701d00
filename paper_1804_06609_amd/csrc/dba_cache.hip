// libdba: the operators around a long paged cache (see include/dba_beam.h), host side.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/dba_beam.h"
#include "append_normed.hpp"
#include "cache_args.hpp"
#include "cache_evict.hpp"
#include "cache_weigh.hpp"
#include "shared_attend.hpp"

using namespace dba;

namespace dba {
extern template hipError_t shared_launch<0>(const SharedParams &, const AttendPlan &, const AttendPlan &, int, hipStream_t);
extern template hipError_t shared_launch<1>(const SharedParams &, const AttendPlan &, const AttendPlan &, int, hipStream_t);
extern template hipError_t shared_launch<2>(const SharedParams &, const AttendPlan &, const AttendPlan &, int, hipStream_t);
}  // namespace dba

namespace {

constexpr int kMostTokens = 1 << 28;        // of a sentence, that are weighed or chosen from
constexpr int64_t kMostSharedRows = 1 << 26;

// ---- appending ----------------------------------------------------------------------------------------------------

const char *weights_fault(const void *data, int64_t stride, int format)
{
    if (!data) return nullptr;
    const int unit = 16 / (int)elem_bytes(format);
    return misaligned(data, 16) || stride < 0 || stride % unit ? "weights of norms and their stride must be multiples of 16 bytes, not negative" : nullptr;
}

template <int FMT, int TOKENS, bool INTERLEAVED>
hipError_t normed_tokens(const NormedParams &p, bool norm, bool wide, int B, unsigned threads, hipStream_t stream)
{
    const auto kernel = !norm ? dba_append_normed_kernel<FMT, false, false, TOKENS, INTERLEAVED>
                      : wide ? dba_append_normed_kernel<FMT, true, true, TOKENS, INTERLEAVED> : dba_append_normed_kernel<FMT, true, false, TOKENS, INTERLEAVED>;
    return launch(kernel, dim3((unsigned)((p.a.n + TOKENS - 1) / TOKENS), (unsigned)B), dim3(threads), 0, stream, p);
}

// A wave for each unit where there are few tokens; several tokens a workgroup where that leaves workgroups enough.
template <int FMT>
hipError_t normed_launch(const NormedParams &p, bool norm, bool wide, int B, hipStream_t stream)
{
    const int units = p.q_units + 2 * p.k_units, most = kNormedThreads / 64, turns = (units + most - 1) / most;
    const unsigned threads = 64u * (unsigned)((units + turns - 1) / turns);
    const bool many = (int64_t)p.a.n * B >= 1024 * kNormedTokens && p.a.n >= kNormedTokens;
    const auto go = p.a.interleaved ? many ? normed_tokens<FMT, kNormedTokens, true> : normed_tokens<FMT, 1, true>
                                    : many ? normed_tokens<FMT, kNormedTokens, false> : normed_tokens<FMT, 1, false>;
    return go(p, norm, wide, B, threads, stream);
}

// ---- attention behind a common prefix ------------------------------------------------------------------------------

struct SharedPlan {
    AttendPlan own, common;
    size_t own_o, own_ml, common_o, common_ml, total;      // where the parts are in the workspace
};

const char *shared_fault(int B, int n, int q_heads, const dba_cache *cache, int shared_pages, int max_shared, int max_len)
{
    const char *fault = attend_fault(B, n, q_heads, cache, max_len);
    if (fault) return fault;
    if (shared_pages < 1 || (int64_t)shared_pages * cache->page_size > INT32_MAX) return "need shared_pages >= 1, shared_pages * page_size below 2^31";
    if (max_shared < 1 || max_shared > shared_pages * cache->page_size || max_shared > kMostLength)
        return "need 1 <= max_shared <= shared_pages * page_size, max_shared <= 2^31 - 1024";
    if ((int64_t)B * n * q_heads > kMostSharedRows) return "need B * n * q_heads <= 2^26";
    return nullptr;
}

// Many rows over common tokens: how many parts of the token axis.  A part costs about kPartTiles tiles to begin with and to write and join; workgroups come in rounds of `resident`, two a compute unit.
// (64 x 20 branches, 32 heads on 8 of 128, over 1500 tokens: 199 us a call, with 0 and 8 for kPartTiles 240 and 204, with 1, 2 and 5 the same; 128 x 8, 32 heads on 4, over 8000: 236 to 242, with rounds of 256
// 279, of 1024 253; 8 x 16, 32 on 8, over 16000: 86, 97, 100; but 16 x 8, 16 on 2 of 64, over 4000: 34, 28, 37.)
constexpr int kPartTiles = 3;

AttendPlan common_plan(int nodes, int q_heads, const dba_cache &c, int max_shared)
{
    AttendPlan a = attend_plan(1, nodes, q_heads, c, max_shared);
    if (!a.shared || c.format == DBA_LOGP_F32 || a.DP > 128 || c.page_size < 16 || c.token_stride >= 1 << 25) return a;     // (a wave's 16 tokens lie in a page, within 2^31 bytes)
    const int rows = nodes * (q_heads / c.heads);
    a.dense = true;
    a.side = 1;
    a.tile = 64;
    a.tile_rows = 128;
    a.row_tiles = (rows + a.tile_rows - 1) / a.tile_rows;
    const int tiles = (int)(((int64_t)max_shared + 63) / 64), resident = 512;
    const int64_t units = (int64_t)a.row_tiles * c.heads;
    int64_t best = INT64_MAX;
    for (int splits = 1; splits <= 64 && splits <= tiles; ++splits) {
        const int chunk = (tiles + splits - 1) / splits;
        const int64_t cost = (units * splits + resident - 1) / resident * (chunk + kPartTiles);
        if (cost < best) {
            best = cost;
            a.chunk = chunk;
            a.splits = (tiles + chunk - 1) / chunk;
        }
    }
    return a;
}

SharedPlan shared_plan(int B, int n, int q_heads, const dba_cache &c, int max_shared, int max_len)
{
    SharedPlan s;
    s.own = attend_plan(B, n, q_heads, c, max_len);
    s.common = common_plan(B * n, q_heads, c, max_shared);
    const size_t own = attend_rows_of(B, n, q_heads, s.own), common = attend_rows_of(B, n, q_heads, s.common);
    s.own_o = 0;
    s.own_ml = s.own_o + align256(own * c.head_dim * 4);
    s.common_o = s.own_ml + align256(own * 8);
    s.common_ml = s.common_o + align256(common * c.head_dim * 4);
    s.total = s.common_ml + align256(common * 8);
    return s;
}

void lay_out(AttendParams &p, const AttendPlan &plan, int B, const dba_cache &c)
{
    p.row_tiles = plan.row_tiles;
    p.tile_rows = plan.tile_rows;
    p.splits = plan.splits;
    p.chunk = plan.chunk;
    p.pairs = B * (c.heads / plan.side);
    p.groups = p.pairs * plan.splits;
}

// ---- weighing -------------------------------------------------------------------------------------------------------

// Up to WeighFew::MOST rows a head the waves go through tokens, else through rows.  Of the former a workgroup has as few tokens as fill the GPU
// (kWeighGroups workgroups, about three rounds: 32 rows, 32 heads on 8 of 128, 16 x 3000 to 16000 tokens 100 us, with 2048 workgroups 125, 4096 123; 20 rows, 16 heads of 64, 64 x 900 to 1500 tokens 51, with 2048 56; five other
// sizes within 0.6 us but for one, 31 and with 2048 33), but two tiles a wave at least, and sums that fit into LDS.  Of the latter rows are split where tokens alone leave GPU empty, two
// turns of rows in LDS at least to a workgroup (one sentence of 300 tokens, 2400 rows: 18 us a call instead of 108; one of 4000 tokens, 16000 rows for each of 8 heads: 324 instead of 979).
constexpr int kWeighGroups = 3200, kWeighChunk = 2048, kWeighRowGroups = 512;

struct WeighPlan {
    bool few;
    int chunk, splits, split_rows;
};

template <int FMT, int DP>
WeighPlan weigh_plan_of(int B, int heads, int rows, int tokens)
{
    typedef WeighShape<FMT, DP> W;
    typedef WeighFew<FMT, DP> F;
    static_assert(F::MOST % 16 == 0, "rows come in sixteens");
    WeighPlan w;
    w.few = rows <= F::MOST;
    w.splits = 1;
    w.split_rows = rows;
    const int64_t pairs = (int64_t)B * heads;
    if (w.few) {
        constexpr int turn = 4 * F::TF;
        const int64_t groups = std::max<int64_t>(1, kWeighGroups / pairs), even = (tokens + groups - 1) / groups;
        w.chunk = (int)std::min<int64_t>(kWeighChunk / turn * turn, std::max<int64_t>(2 * turn, (even + turn - 1) / turn * turn));
    } else {
        w.chunk = W::TG;
        const int64_t groups = pairs * ((tokens + W::TG - 1) / W::TG), turns = (rows + W::RQ - 1) / W::RQ;
        const int64_t per = std::max<int64_t>(2, turns / std::max<int64_t>(1, kWeighRowGroups / groups));       // turns of a workgroup
        w.splits = (int)((turns + per - 1) / per);
        w.split_rows = (int)(per * W::RQ);
    }
    return w;
}
WeighPlan weigh_plan(int B, const dba_cache &c, int rows, int tokens)
{
    const auto plan = c.format == DBA_LOGP_F32 ? c.head_dim <= 64 ? weigh_plan_of<0, 64> : c.head_dim <= 128 ? weigh_plan_of<0, 128> : weigh_plan_of<0, 256>
                                               : c.head_dim <= 64 ? weigh_plan_of<1, 64> : c.head_dim <= 128 ? weigh_plan_of<1, 128> : weigh_plan_of<1, 256>;
    return plan(B, c.heads, rows, tokens);
}

template <int FMT, int DP, bool FULL>
hipError_t weigh_one(WeighParams p, int B, int tokens, hipStream_t stream)
{
    const int rows = p.n * (p.q_heads / p.heads);
    const WeighPlan w = weigh_plan_of<FMT, DP>(B, p.heads, rows, p.max_len);        // (laid out for max_len, as the workspace is)
    p.chunk = w.chunk;
    p.splits = w.splits;
    p.split_rows = w.split_rows;
    const dim3 grid((unsigned)((tokens + w.chunk - 1) / w.chunk), (unsigned)(p.heads * w.splits), (unsigned)B);
    if (!w.few) return launch(dba_weigh_kernel<FMT, DP, FULL>, grid, dim3(256), 0, stream, p);
    const auto kernel = rows <= 64 || WeighFew<FMT, DP>::MOST <= 64 ? dba_weigh_few_kernel<FMT, DP, FULL, 1> : dba_weigh_few_kernel<FMT, DP, FULL, WeighFew<FMT, DP>::MOST <= 64 ? 1 : 2>;
    return launch(kernel, grid, dim3(256), (size_t)WeighFew<FMT, DP>::lds(rows, w.chunk), stream, p);
}
template <int FMT>
hipError_t weigh_launch(const WeighParams &p, int B, int tokens, hipStream_t stream)
{
    const auto go = p.D == 64 ? weigh_one<FMT, 64, true> : p.D < 64 ? weigh_one<FMT, 64, false> : p.D == 128 ? weigh_one<FMT, 128, true>
                  : p.D < 128 ? weigh_one<FMT, 128, false> : p.D == 256 ? weigh_one<FMT, 256, true> : weigh_one<FMT, 256, false>;
    return go(p, B, tokens, stream);
}

// Rows of scores [B, heads_s, width].
const char *scores_fault(const float *data, int64_t sent, int64_t head)
{
    return !data ? "a pointer of scores is NULL" : misaligned(data, 4) || sent < 0 || head < 0 ? "scores must be aligned to 4 bytes, with strides that are not negative" : nullptr;
}
Places places_of(const float *scores, int B, int heads_s, int width, int64_t sent, int64_t head)
{
    return scores ? Places(scores, (int64_t)width * 4).axis(B, sent * 4).axis(heads_s, head * 4) : Places();
}

}  // namespace

extern "C" {

DBA_API int dba_cache_append_normed(int B, int n, const dba_cache *cache, const dba_heads *k, const dba_heads *v, int q_heads, const dba_heads *q,
                                    const dba_heads *q_out, const dba_norms *norms, const int32_t *first_dev, const int32_t *count_dev,
                                    const int32_t *position_dev, int axes, const int32_t *axis_dev, const float *inv_freq_dev, int rot_dim,
                                    int interleaved, void *hip_stream)
{
    static const char *const who = "dba_cache_append_normed";
    const char *fault = cache_fault(cache);
    if (fault) return set_error(DBA_EINVAL, "%s: %s", who, fault);
    if (B < 1 || B > 65535 || n < 1 || n > kMostRows) return set_error(DBA_EINVAL, "%s: need 1 <= B <= 65535, 1 <= n <= 2^22", who);
    if ((fault = heads_fault(k, cache->format)) || (fault = heads_fault(v, cache->format))) return set_error(DBA_EINVAL, "%s: %s", who, fault);
    if ((q != nullptr) != (q_out != nullptr)) return set_error(DBA_EINVAL, "%s: q and q_out go together", who);
    if (q) {
        if ((fault = heads_fault(q, cache->format)) || (fault = heads_fault(q_out, cache->format))) return set_error(DBA_EINVAL, "%s: %s", who, fault);
        if (q_heads < 1 || q_heads > 8192) return set_error(DBA_EINVAL, "%s: 1 <= q_heads <= 8192", who);
        if (q->data == q_out->data && !same(*q, *q_out)) return set_error(DBA_EINVAL, "%s: q is rotated in place with two sets of strides", who);
    }
    if (!first_dev) return set_error(DBA_EINVAL, "%s: first_dev is NULL", who);
    if (rot_dim < 0 || rot_dim > cache->head_dim || rot_dim % 16) return set_error(DBA_EINVAL, "%s: rot_dim must be a multiple of 16, at most head_dim", who);
    if (rot_dim && !inv_freq_dev) return set_error(DBA_EINVAL, "%s: inv_freq_dev is NULL", who);
    if (axes < 1 || axes > 65536 || (axis_dev && !position_dev) || (!axis_dev && axes != 1))
        return set_error(DBA_EINVAL, "%s: need 1 <= axes <= 65536; axis_dev needs position_dev, and more than one axis axis_dev", who);
    if (norms) {
        if (!(norms->eps >= 1e-37f && norms->eps < INFINITY)) return set_error(DBA_EINVAL, "%s: eps must be a number of 1e-37 or more", who);
        if (!format_ok(norms->format) || (norms->format != cache->format && norms->format != DBA_LOGP_F32))
            return set_error(DBA_EINVAL, "%s: weights of norms are of the cache's format or fp32", who);
        if ((fault = weights_fault(norms->q_weight, norms->q_stride, norms->format)) || (fault = weights_fault(norms->k_weight, norms->k_stride, norms->format)))
            return set_error(DBA_EINVAL, "%s: %s", who, fault);
    }
    if (!places_of(cache->k, *cache).nested()) return set_error(DBA_EINVAL, "%s: tokens of the cache overlap", who);
    if (q) {
        const Places to = places_of(*q_out, B, n, q_heads, *cache);
        if (!to.nested()) return set_error(DBA_EINVAL, "%s: pieces of q_out overlap", who);
        if ((!same(*q, *q_out) && meet(to, places_of(*q, B, n, q_heads, *cache))) || meet(to, places_of(*k, B, n, cache->heads, *cache)) ||
            meet(to, places_of(*v, B, n, cache->heads, *cache)))
            return set_error(DBA_EINVAL, "%s: q_out overlaps k, v or a part of q", who);
        const Places small[] = {{first_dev, (int64_t)B * 4}, {count_dev, count_dev ? (int64_t)B * 4 : 0}, {position_dev, position_dev ? (int64_t)B * n * axes * 4 : 0},
                                {axis_dev, axis_dev ? rot_dim * 2 : 0}, {inv_freq_dev, rot_dim * 2}};
        for (const Places &x : small)
            if (meet(to, x)) return set_error(DBA_EINVAL, "%s: q_out overlaps counts, positions or frequencies", who);
        if (norms) {
            const int64_t len = (int64_t)cache->head_dim * elem_bytes(norms->format), e = elem_bytes(norms->format);
            if ((norms->q_weight && meet(to, Places(norms->q_weight, len).axis(q_heads, norms->q_stride * e))) ||
                (norms->k_weight && meet(to, Places(norms->k_weight, len).axis(cache->heads, norms->k_stride * e))))
                return set_error(DBA_EINVAL, "%s: q_out overlaps weights of norms", who);
        }
    }
    NormedParams p;
    p.a.cache = paged_of(*cache);
    p.a.k_pages = static_cast<unsigned char *>(cache->k);
    p.a.v_pages = static_cast<unsigned char *>(cache->v);
    p.a.q = heads_of(q);
    p.a.q_out = heads_of(q_out);
    p.a.k = heads_of(k);
    p.a.v = heads_of(v);
    p.a.first = first_dev;
    p.a.count = count_dev;
    p.a.position = position_dev;
    p.a.inv_freq = inv_freq_dev;
    p.a.n = n;
    p.a.heads = cache->heads;
    p.a.q_heads = q ? q_heads : 0;
    p.a.D = cache->head_dim;
    p.a.rot = rot_dim;
    p.a.interleaved = interleaved != 0;
    p.qw = WeightsAt{norms ? static_cast<const unsigned char *>(norms->q_weight) : nullptr, norms ? norms->q_stride : 0};
    p.kw = WeightsAt{norms ? static_cast<const unsigned char *>(norms->k_weight) : nullptr, norms ? norms->k_stride : 0};
    p.axis = axis_dev;
    p.axes = axes;
    p.eps = norms ? norms->eps : 0.0f;
    p.per_element = 1.0f / (float)cache->head_dim;
    const int pairs = (p.a.D * (int)elem_bytes(cache->format) / 16 + 1) / 2;
    p.lane_bits = 0;
    while ((1 << p.lane_bits) < pairs) ++p.lane_bits;
    p.lanes = 1 << p.lane_bits;
    p.q_units = ((p.a.q_heads << p.lane_bits) + 63) / 64;
    p.k_units = ((p.a.heads << p.lane_bits) + 63) / 64;
    const bool wide = norms && norms->format != cache->format;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = cache->format == DBA_LOGP_F32 ? normed_launch<0>(p, norms, false, B, stream)
                       : cache->format == DBA_LOGP_F16 ? normed_launch<1>(p, norms, wide, B, stream) : normed_launch<2>(p, norms, wide, B, stream);
    return launched(who, e);
}

DBA_API size_t dba_shared_attend_workspace_bytes(int B, int n, int q_heads, const dba_cache *cache, int shared_pages, int max_shared, int max_len)
{
    return shared_fault(B, n, q_heads, cache, shared_pages, max_shared, max_len) ? 0 : shared_plan(B, n, q_heads, *cache, max_shared, max_len).total;
}

DBA_API int dba_shared_attend(int B, int n, int q_heads, const dba_heads *q, const dba_cache *cache, const int32_t *shared_table_dev, int shared_pages,
                              const int32_t *shared_len_dev, int max_shared, const int32_t *prefix_dev, const int32_t *tree_dev,
                              const uint64_t *mask_dev, int mask_words, int max_len, float scale, const dba_heads *out, float *out_lse_dev,
                              void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    static const char *const who = "dba_shared_attend";
    const char *fault = shared_fault(B, n, q_heads, cache, shared_pages, max_shared, max_len);
    if (fault) return set_error(DBA_EINVAL, "%s: %s", who, fault);
    if ((fault = heads_fault(q, cache->format)) || (fault = heads_fault(out, cache->format))) return set_error(DBA_EINVAL, "%s: %s", who, fault);
    if (!shared_table_dev || !shared_len_dev || !prefix_dev) return set_error(DBA_EINVAL, "%s: shared_table_dev, shared_len_dev or prefix_dev is NULL", who);
    if (mask_words < 0 || (mask_dev && !tree_dev)) return set_error(DBA_EINVAL, "%s: a mask needs tree_dev and mask_words >= 0", who);
    if (!(fabsf(scale) <= 1e30f)) return set_error(DBA_EINVAL, "%s: scale is not a number between -1e30 and 1e30", who);
    const SharedPlan plan = shared_plan(B, n, q_heads, *cache, max_shared, max_len);
    if (!workspace_dev || misaligned(workspace_dev, 256)) return set_error(DBA_EINVAL, "%s: workspace_dev must be 256-byte aligned", who);
    if (workspace_bytes < plan.total) return set_error(DBA_ENOMEM, "%s: workspace has %zu bytes, %zu needed", who, workspace_bytes, plan.total);
    const Places to = places_of(*out, B, n, q_heads, *cache), from = places_of(*q, B, n, q_heads, *cache);
    const Places lse(out_lse_dev, out_lse_dev ? (int64_t)B * n * q_heads * 4 : 0), room(workspace_dev, (int64_t)plan.total);
    if (!to.nested()) return set_error(DBA_EINVAL, "%s: pieces of out overlap", who);
    if (!same(*q, *out) && meet(to, from)) return set_error(DBA_EINVAL, "%s: out overlaps a part of q", who);
    if (meet(lse, to) || meet(lse, from)) return set_error(DBA_EINVAL, "%s: out_lse_dev lies in out or q", who);
    if (meet(room, to) || meet(room, from) || meet(room, lse)) return set_error(DBA_EINVAL, "%s: q, out or out_lse_dev lies in the workspace", who);
    unsigned char *const ws = static_cast<unsigned char *>(workspace_dev);
    SharedParams p;
    AttendParams &a = p.own, &c = p.common;
    a.cache = paged_of(*cache);
    a.k_pages = static_cast<const unsigned char *>(cache->k);
    a.v_pages = static_cast<const unsigned char *>(cache->v);
    a.q = heads_of(q);
    a.out = heads_of(out);
    a.prefix = prefix_dev;
    a.tree = tree_dev;
    a.mask = reinterpret_cast<const unsigned long long *>(mask_dev);
    a.lse = out_lse_dev;
    a.n = a.per = n;
    a.q_heads = q_heads;
    a.heads = cache->heads;
    a.D = cache->head_dim;
    a.mask_words = mask_words;
    a.max_len = max_len;
    a.scale = scale;
    c = a;
    lay_out(a, plan.own, B, *cache);
    a.part_o = reinterpret_cast<float *>(ws + plan.own_o);
    a.part_ml = reinterpret_cast<float *>(ws + plan.own_ml);
    c.cache.table = shared_table_dev;
    c.cache.table_stride = 0;
    c.cache.max_pages = shared_pages;
    c.prefix = shared_len_dev;
    c.tree = nullptr;
    c.mask = nullptr;
    c.mask_words = 0;
    c.lse = nullptr;
    c.n = B * n;
    c.max_len = max_shared;
    lay_out(c, plan.common, 1, *cache);
    c.part_o = reinterpret_cast<float *>(ws + plan.common_o);
    c.part_ml = reinterpret_cast<float *>(ws + plan.common_ml);
    p.common_tile = plan.common.tile;
    p.own_tile = plan.own.tile;
    p.own_shift = __builtin_ctz((unsigned)plan.own.tile_rows);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = cache->format == DBA_LOGP_F32 ? shared_launch<0>(p, plan.own, plan.common, B, stream)
                       : cache->format == DBA_LOGP_F16 ? shared_launch<1>(p, plan.own, plan.common, B, stream) : shared_launch<2>(p, plan.own, plan.common, B, stream);
    return launched(who, e);
}

DBA_API size_t dba_cache_weigh_workspace_bytes(int B, int n, int q_heads, const dba_cache *cache, int by_head, int max_len)
{
    if (attend_fault(B, n, q_heads, cache, max_len) || max_len > kMostTokens) return 0;
    const int splits = weigh_plan(B, *cache, n * (q_heads / cache->heads), max_len).splits;
    return splits == 1 && (by_head || cache->heads == 1) ? 0 : align256((size_t)B * cache->heads * splits * max_len * 4);
}

DBA_API int dba_cache_weigh(int B, int n, int q_heads, const dba_heads *q, const float *lse_dev, const dba_cache *cache, const int32_t *prefix_dev,
                            const int32_t *tree_dev, const uint64_t *mask_dev, int mask_words, const int32_t *count_dev, int max_len, float scale,
                            int by_head, const float *score_dev, int64_t score_sent, int64_t score_head, float *out_dev, int64_t out_sent,
                            int64_t out_head, int width, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    static const char *const who = "dba_cache_weigh";
    const char *fault = attend_fault(B, n, q_heads, cache, max_len);
    if (fault || (fault = heads_fault(q, cache->format)) || (fault = scores_fault(score_dev, score_sent, score_head)) || (fault = scores_fault(out_dev, out_sent, out_head)))
        return set_error(DBA_EINVAL, "%s: %s", who, fault);
    if (!lse_dev || misaligned(lse_dev, 4) || !prefix_dev) return set_error(DBA_EINVAL, "%s: lse_dev or prefix_dev is NULL or not aligned", who);
    if (mask_words < 0 || (mask_dev && !tree_dev)) return set_error(DBA_EINVAL, "%s: a mask needs tree_dev and mask_words >= 0", who);
    if (!(fabsf(scale) <= 1e30f)) return set_error(DBA_EINVAL, "%s: scale is not a number between -1e30 and 1e30", who);
    if (width < max_len || width > kMostTokens) return set_error(DBA_EINVAL, "%s: need max_len <= width <= 2^28", who);
    const int heads_s = by_head ? cache->heads : 1;
    const bool in_place = score_dev == out_dev;
    if (in_place && ((B > 1 && score_sent != out_sent) || (heads_s > 1 && score_head != out_head)))
        return set_error(DBA_EINVAL, "%s: scores are added to in place with two sets of strides", who);
    const Places was = places_of(score_dev, B, heads_s, width, score_sent, score_head), to = places_of(out_dev, B, heads_s, width, out_sent, out_head);
    if (!to.nested()) return set_error(DBA_EINVAL, "%s: rows of out_dev overlap", who);
    if (!in_place && meet(to, was)) return set_error(DBA_EINVAL, "%s: out_dev overlaps a part of score_dev", who);
    if (meet(to, places_of(*q, B, n, q_heads, *cache)) || meet(to, Places(lse_dev, (int64_t)B * n * q_heads * 4)) ||
        (mask_dev && meet(to, Places(mask_dev, (int64_t)B * n * mask_words * 8))) || meet(to, places_of(cache->k, *cache)))
        return set_error(DBA_EINVAL, "%s: out_dev lies in q, lse_dev, mask_dev or the cache", who);
    const size_t need = dba_cache_weigh_workspace_bytes(B, n, q_heads, cache, by_head, max_len);
    if (need) {
        if (!workspace_dev || misaligned(workspace_dev, 256)) return set_error(DBA_EINVAL, "%s: workspace_dev must be 256-byte aligned", who);
        if (workspace_bytes < need) return set_error(DBA_ENOMEM, "%s: workspace has %zu bytes, %zu needed", who, workspace_bytes, need);
        const Places room(workspace_dev, (int64_t)need);
        if (meet(room, was) || meet(room, to) || meet(room, places_of(*q, B, n, q_heads, *cache)) || meet(room, Places(lse_dev, (int64_t)B * n * q_heads * 4)))
            return set_error(DBA_EINVAL, "%s: scores, q or lse_dev lie in the workspace", who);
    }
    WeighParams p;
    p.cache = paged_of(*cache);
    p.k_pages = static_cast<const unsigned char *>(cache->k);
    p.q = heads_of(q);
    p.lse = lse_dev;
    p.prefix = prefix_dev;
    p.tree = tree_dev;
    p.count = count_dev;
    p.mask = reinterpret_cast<const unsigned long long *>(mask_dev);
    p.score = score_dev;
    p.out = out_dev;
    p.score_sent = score_sent;
    p.score_head = score_head;
    p.out_sent = out_sent;
    p.out_head = out_head;
    p.n = n;
    p.q_heads = q_heads;
    p.heads = cache->heads;
    p.D = cache->head_dim;
    p.mask_words = mask_words;
    p.max_len = max_len;
    p.width = width;
    p.scale = scale;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const auto go = cache->format == DBA_LOGP_F32 ? weigh_launch<0> : cache->format == DBA_LOGP_F16 ? weigh_launch<1> : weigh_launch<2>;
    if (!need) return launched(who, go(p, B, in_place ? max_len : width, stream));
    const int splits = weigh_plan(B, *cache, n * (q_heads / cache->heads), max_len).splits;
    WeighParams sums = p;
    sums.score = nullptr;
    sums.out = static_cast<float *>(workspace_dev);
    sums.out_sent = (int64_t)cache->heads * splits * max_len;
    sums.out_head = max_len;
    sums.width = max_len;
    hipError_t e = go(sums, B, max_len, stream);
    if (e == hipSuccess) e = launch(dba_weigh_join_kernel, dim3((unsigned)((width + 255) / 256), (unsigned)heads_s, (unsigned)B), dim3(256), 0, stream, p,
                                     static_cast<const float *>(workspace_dev), cache->heads / heads_s * splits);
    return launched(who, e);
}

// The workspace: lists, and for long rows counts of digits, bars, and what is there and stays.
struct EvictPlan {
    int parts;                         // 0: rows are short
    size_t hist_at, found_at, counts_at, tally_at, total;
};
constexpr int kShortRow = 16384;

static EvictPlan evict_plan(int B, int heads_s, int keep, int max_len)
{
    EvictPlan e;
    const size_t rows = (size_t)B * heads_s;
    e.parts = max_len <= kShortRow ? 0 : (max_len + kEvictPart - 1) / kEvictPart;
    e.hist_at = align256(rows * std::min(keep, max_len) * 4);
    e.found_at = e.hist_at + align256(rows * e.parts * kDigits * 4);
    e.counts_at = e.found_at + (e.parts ? align256(rows * 8) : 0);
    e.tally_at = e.counts_at + (e.parts ? align256((size_t)B * 8) : 0);
    e.total = e.tally_at + align256(rows * e.parts * 8);
    return e;
}

static const char *evict_fault(int B, const dba_cache *cache, int keep, int max_len)
{
    const char *fault = cache_fault(cache);
    if (fault) return fault;
    if (B < 1 || B > 65535 || keep < 1) return "need 1 <= B <= 65535, keep >= 1";
    if (max_len < 1 || max_len > cache->max_pages * cache->page_size || max_len > kMostTokens) return "need 1 <= max_len <= max_pages * page_size, max_len <= 2^28";
    return nullptr;
}

DBA_API size_t dba_cache_evict_workspace_bytes(int B, const dba_cache *cache, int by_head, int keep, int max_len)
{
    return evict_fault(B, cache, keep, max_len) ? 0 : evict_plan(B, by_head ? cache->heads : 1, keep, max_len).total;
}

DBA_API int dba_cache_evict(int B, const dba_cache *cache, const int32_t *new_table_dev, int64_t new_table_stride, int new_max_pages, int by_head,
                            const float *score_dev, int64_t score_sent, int64_t score_head, const int32_t *prefix_dev, const int32_t *tree_dev, int keep,
                            const int32_t *budget_dev, int sinks, int recent, int max_len, int32_t *new_prefix_dev, float *new_score_dev,
                            int64_t new_sent, int64_t new_head, int width, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    static const char *const who = "dba_cache_evict";
    const char *fault = evict_fault(B, cache, keep, max_len);
    if (fault || (fault = scores_fault(score_dev, score_sent, score_head)) || (new_score_dev && (fault = scores_fault(new_score_dev, new_sent, new_head))))
        return set_error(DBA_EINVAL, "%s: %s", who, fault);
    if (!new_table_dev || !prefix_dev || !new_prefix_dev) return set_error(DBA_EINVAL, "%s: new_table_dev, prefix_dev or new_prefix_dev is NULL", who);
    if (new_max_pages < 1 || (int64_t)new_max_pages * cache->page_size > INT32_MAX || new_table_stride < new_max_pages)
        return set_error(DBA_EINVAL, "%s: need new_max_pages >= 1, new_max_pages * page_size below 2^31, new_table_stride >= new_max_pages", who);
    if (sinks < 0 || recent < 0) return set_error(DBA_EINVAL, "%s: sinks and recent must not be negative", who);
    if (width < max_len || width > kMostTokens) return set_error(DBA_EINVAL, "%s: need max_len <= width <= 2^28", who);
    const size_t need = dba_cache_evict_workspace_bytes(B, cache, by_head, keep, max_len);
    if (!workspace_dev || misaligned(workspace_dev, 256)) return set_error(DBA_EINVAL, "%s: workspace_dev must be 256-byte aligned", who);
    if (workspace_bytes < need) return set_error(DBA_ENOMEM, "%s: workspace has %zu bytes, %zu needed", who, workspace_bytes, need);
    const int heads_s = by_head ? cache->heads : 1;
    const Places was = places_of(score_dev, B, heads_s, width, score_sent, score_head), to = places_of(new_score_dev, B, heads_s, width, new_sent, new_head);
    const Places room(workspace_dev, (int64_t)need), stay(new_prefix_dev, (int64_t)B * 4);
    const Places table = Places(cache->table, (int64_t)cache->max_pages * 4).axis(B, cache->table_stride * 4);
    const Places new_table = Places(new_table_dev, (int64_t)new_max_pages * 4).axis(B, new_table_stride * 4);
    const Places small[] = {{prefix_dev, (int64_t)B * 4}, {tree_dev, tree_dev ? (int64_t)B * 4 : 0}, {budget_dev, budget_dev ? (int64_t)B * 4 : 0}, table, new_table, was};
    if (!places_of(cache->k, *cache).nested()) return set_error(DBA_EINVAL, "%s: tokens of the cache overlap", who);
    if (!to.nested()) return set_error(DBA_EINVAL, "%s: rows of new_score_dev overlap", who);
    if (meet(to, stay) || meet(to, room) || meet(stay, room)) return set_error(DBA_EINVAL, "%s: results or the workspace overlap", who);
    const Places keys = places_of(cache->k, *cache), values = places_of(cache->v, *cache);
    for (const Places &x : small)
        if (meet(x, to) || meet(x, stay) || meet(x, room)) return set_error(DBA_EINVAL, "%s: a result or the workspace overlaps what is read", who);
    for (const Places &x : {to, stay, room, was})
        if (meet(x, keys) || meet(x, values)) return set_error(DBA_EINVAL, "%s: scores, a result or the workspace lie in the cache", who);
    EvictParams p;
    p.from = p.to = paged_of(*cache);
    p.to.table = new_table_dev;
    p.to.table_stride = new_table_stride;
    p.to.max_pages = new_max_pages;
    p.k_pages = static_cast<unsigned char *>(cache->k);
    p.v_pages = static_cast<unsigned char *>(cache->v);
    p.score = score_dev;
    p.new_score = new_score_dev;
    p.score_sent = score_sent;
    p.score_head = score_head;
    p.new_sent = new_sent;
    p.new_head = new_head;
    p.prefix = prefix_dev;
    p.tree = tree_dev;
    p.budget = budget_dev;
    p.new_prefix = new_prefix_dev;
    p.list = static_cast<int32_t *>(workspace_dev);
    p.cap = std::min(keep, max_len);
    p.keep = keep;
    p.sinks = sinks;
    p.recent = recent;
    p.max_len = max_len;
    p.width = width;
    p.heads = cache->heads;
    p.heads_s = heads_s;
    p.elem = (int)elem_bytes(cache->format);
    p.chunks = cache->head_dim * p.elem / 16;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const EvictPlan plan = evict_plan(B, heads_s, keep, max_len);
    hipError_t e;
    if (!plan.parts) {
        const auto kernel = max_len <= 1024 ? dba_evict_choose_kernel<4, 4> : max_len <= 4096 ? dba_evict_choose_kernel<8, 8> : dba_evict_choose_kernel<16, 16>;
        e = launch(kernel, dim3((unsigned)heads_s, (unsigned)B), dim3(max_len <= 1024 ? 256u : max_len <= 4096 ? 512u : 1024u), 0, stream, p);
    } else {
        unsigned char *const ws = static_cast<unsigned char *>(workspace_dev);
        const EvictLong l = {reinterpret_cast<uint32_t *>(ws + plan.hist_at), reinterpret_cast<uint32_t *>(ws + plan.found_at), reinterpret_cast<int2 *>(ws + plan.counts_at),
                             reinterpret_cast<uint2 *>(ws + plan.tally_at), plan.parts};
        const dim3 parts((unsigned)plan.parts, (unsigned)heads_s, (unsigned)B), threads(64 * kEvictWaves);
        e = launch(dba_evict_there_kernel, dim3((unsigned)B), threads, 0, stream, p, l);
        if (e == hipSuccess) e = launch(dba_evict_count_kernel, parts, threads, 0, stream, p, l);
        if (e == hipSuccess) e = launch(dba_evict_bar_kernel, dim3((unsigned)heads_s, (unsigned)B), threads, 0, stream, p, l);
        if (e == hipSuccess) e = launch(dba_evict_tally_kernel, parts, threads, 0, stream, p, l);
        if (e == hipSuccess) e = launch(dba_evict_list_kernel, parts, threads, 0, stream, p, l);
    }
    if (e == hipSuccess) {
        // (without a tree no more than keep tokens are moved; scores are written for all of a row)
        const int64_t items = (int64_t)(tree_dev ? max_len : p.cap) * p.heads * p.chunks, turn = kMoveThreads * kMoveItems;
        const int64_t scores = new_score_dev ? (int64_t)heads_s * width : 0, score_turn = kMoveThreads * kMoveScores;
        const int64_t most = std::max<int64_t>(1, 8192 / B), wanted = std::max((items + turn - 1) / turn, (scores + score_turn - 1) / score_turn);
        e = launch(dba_evict_move_kernel, dim3((unsigned)std::min(wanted, most), (unsigned)B), dim3(kMoveThreads), 0, stream, p);
    }
    return launched(who, e);
}

}  // extern "C"
