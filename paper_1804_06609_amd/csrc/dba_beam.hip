// libdba: the operators next to the selection step (see include/dba_beam.h), host side.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <memory>
#include <new>

#include "../../include/dba_beam.h"
#include "beam_reorder.hpp"
#include "beam_select.hpp"
#include "cache_args.hpp"
#include "cache_append.hpp"
#include "entry.hpp"

using namespace dba;

namespace {

// ---- selection ----------------------------------------------------------------------------------------------------

struct SelectPlan {
    int nparts, part_chunks, cap;
    size_t keys_at, total;
};

bool select_shape_ok(int B, int k_in, int k_out, int V, int format)
{
    return B >= 1 && B <= 65535 && k_in >= 1 && k_in <= DBA_MAX_BEAM && k_out >= 1 && k_out <= DBA_MAX_BEAM && V >= 1 &&
           V <= (1 << 24) && format_ok(format);
}

SelectPlan select_plan(int B, int k_in, int k_out, int V, int format)
{
    SelectPlan s;
    const int per_chunk = 16 / (int)elem_bytes(format);
    const int chunks = (V + per_chunk - 1) / per_chunk;
    const int most = kSelectThreads * kSelectChunks;
    s.nparts = (chunks + most - 1) / most;
    // whole rounds of the workgroup, where that leaves no part without a chunk
    s.part_chunks = (chunks + s.nparts - 1) / s.nparts;
    s.part_chunks = (s.part_chunks + kSelectThreads - 1) / kSelectThreads * kSelectThreads;
    s.nparts = (chunks + s.part_chunks - 1) / s.part_chunks;
    s.cap = std::max(32, 2 * k_out);
    const size_t lists = (size_t)B * k_in * s.nparts;
    s.keys_at = align256(lists * sizeof(SelectPart));
    s.total = align256(s.keys_at + lists * s.cap * sizeof(u64));
    return s;
}

// the two launches of a selection
template <int FMT>
hipError_t select_launch(const SelectParams &p, int B, const void *logits, hipStream_t stream)
{
    hipError_t e = launch(dba_select_part_kernel<FMT>, dim3((unsigned)p.nparts, (unsigned)p.k_in, (unsigned)B), dim3(kSelectThreads), 0, stream, logits, p);
    if (e != hipSuccess) return e;
    return p.k_in * p.nparts <= 32 ? launch(dba_select_sentence_kernel<256>, dim3((unsigned)B), dim3(256), 0, stream, p)
                                             : launch(dba_select_sentence_kernel<1024>, dim3((unsigned)B), dim3(1024), 0, stream, p);
}

}  // namespace

extern "C" {

DBA_API size_t dba_beam_select_workspace_bytes(int B, int k_in, int k_out, int V, int logits_format)
{
    return select_shape_ok(B, k_in, k_out, V, logits_format) ? select_plan(B, k_in, k_out, V, logits_format).total : 0;
}

DBA_API int dba_beam_select(int B, int k_in, int k_out, int V, int eos_id, int pad_id, const void *logits_dev, int logits_format,
                            int64_t sent_stride, int64_t row_stride, const float *score_dev, const uint8_t *flags_dev,
                            int32_t *out_token_dev, int32_t *out_backptr_dev, float *out_score_dev, uint8_t *out_flags_dev,
                            void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    if (!select_shape_ok(B, k_in, k_out, V, logits_format))
        return set_error(DBA_EINVAL, "dba_beam_select: need 1 <= B <= 65535, 1 <= k_in, k_out <= %d, 1 <= V <= 2^24 and a known format",
                         DBA_MAX_BEAM);
    if (pad_id < 0 || pad_id >= V || eos_id < -1 || eos_id >= V || eos_id == pad_id)
        return set_error(DBA_EINVAL, "dba_beam_select: eos_id/pad_id must be distinct ids in [0,V) (eos_id may be -1)");
    if (!logits_dev || !score_dev || !out_token_dev || !out_backptr_dev || !out_score_dev || !out_flags_dev)
        return set_error(DBA_EINVAL, "dba_beam_select: a pointer is NULL");
    if (misaligned(logits_dev, elem_bytes(logits_format)))
        return set_error(DBA_EINVAL, "dba_beam_select: logits_dev must be aligned to its element size");
    if ((k_in > 1 && row_stride < V) || (B > 1 && sent_stride < 0))
        return set_error(DBA_EINVAL, "dba_beam_select: row_stride must be at least V and sent_stride not negative");
    const SelectPlan plan = select_plan(B, k_in, k_out, V, logits_format);
    if (!workspace_dev || misaligned(workspace_dev, 256))
        return set_error(DBA_EINVAL, "dba_beam_select: workspace_dev must be 256-byte aligned");
    if (workspace_bytes < plan.total)
        return set_error(DBA_ENOMEM, "dba_beam_select: workspace has %zu bytes, %zu needed", workspace_bytes, plan.total);
    // the new beam is written while the old one is still read, its arrays and the workspace while each other are
    const int64_t rows_in = (int64_t)B * k_in, rows_out = (int64_t)B * k_out, e = elem_bytes(logits_format);
    const Places score(score_dev, rows_in * 4), flags(flags_dev, flags_dev ? rows_in : 0);
    const Places logits = Places(logits_dev, V * e).axis(B, sent_stride * e).axis(k_in, row_stride * e), room(workspace_dev, (int64_t)plan.total);
    const Places outs[] = {{out_token_dev, rows_out * 4}, {out_backptr_dev, rows_out * 4}, {out_score_dev, rows_out * 4}, {out_flags_dev, rows_out}};
    for (const Places &o : outs)
        if (meet(o, score) || meet(o, flags))
            return set_error(DBA_EINVAL, "dba_beam_select: the new beam lies in the old one's scores or flags");
    for (const Places &o : outs) {
        if (meet(o, logits)) return set_error(DBA_EINVAL, "dba_beam_select: the new beam lies in the logits");
        if (meet(o, room)) return set_error(DBA_EINVAL, "dba_beam_select: the new beam lies in the workspace");
        for (const Places *other = outs; other != &o; ++other)
            if (meet(o, *other)) return set_error(DBA_EINVAL, "dba_beam_select: two arrays of the new beam overlap");
    }
    if (meet(room, score) || meet(room, flags) || meet(room, logits)) return set_error(DBA_EINVAL, "dba_beam_select: an input lies in the workspace");
    SelectParams p;
    p.score = score_dev;
    p.flags = flags_dev;
    p.out_token = out_token_dev;
    p.out_backptr = out_backptr_dev;
    p.out_score = out_score_dev;
    p.out_flags = out_flags_dev;
    p.parts = static_cast<SelectPart *>(workspace_dev);
    p.keys = reinterpret_cast<u64 *>(static_cast<unsigned char *>(workspace_dev) + plan.keys_at);
    p.sent_stride = sent_stride;
    p.row_stride = row_stride;
    p.k_in = k_in;
    p.k_out = k_out;
    p.V = V;
    p.nparts = plan.nparts;
    p.cap = plan.cap;
    p.part_chunks = plan.part_chunks;
    p.eos = eos_id;
    p.pad = pad_id;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const hipError_t done = logits_format == DBA_LOGP_F32 ? select_launch<0>(p, B, logits_dev, stream)
                          : logits_format == DBA_LOGP_F16 ? select_launch<1>(p, B, logits_dev, stream) : select_launch<2>(p, B, logits_dev, stream);
    return launched("dba_beam_select", done);
}

DBA_API int dba_beam_reorder(int B, int k, const int32_t *backptr_dev, const dba_state *states_host, int n_states, void *hip_stream)
{
    if (B < 1 || B > 65535 || k < 1 || k > DBA_MAX_BEAM || n_states < 0)
        return set_error(DBA_EINVAL, "dba_beam_reorder: need 1 <= B <= 65535, 1 <= k <= %d, n_states >= 0", DBA_MAX_BEAM);
    if (!backptr_dev || (n_states > 0 && !states_host)) return set_error(DBA_EINVAL, "dba_beam_reorder: a pointer is NULL");
    // everything is looked at before anything is launched
    struct Moved {
        Places dst, src;
        bool in_place, any;
    };
    Moved few[kReorderStates];
    std::unique_ptr<Moved[]> many(n_states > kReorderStates ? new (std::nothrow) Moved[n_states] : nullptr);
    if (n_states > kReorderStates && !many) return set_error(DBA_ENOMEM, "dba_beam_reorder: no host memory to look at %d states", n_states);
    Moved *const moved = many ? many.get() : few;
    for (int i = 0; i < n_states; ++i) {
        const dba_state &s = states_host[i];
        if (s.segs < 0 || s.seg_bytes < 0) return set_error(DBA_EINVAL, "dba_beam_reorder: state %d has a negative size", i);
        Moved &m = moved[i];
        m.any = s.segs != 0 && s.seg_bytes != 0;
        if (!m.any) continue;
        if (!s.dst || !s.src) return set_error(DBA_EINVAL, "dba_beam_reorder: a pointer of state %d is NULL", i);
        m.dst = Places(s.dst, s.seg_bytes).axis(B, s.dst_sent).axis(k, s.dst_row).axis(s.segs, s.dst_seg);
        m.src = Places(s.src, s.seg_bytes).axis(B, s.src_sent).axis(k, s.src_row).axis(s.segs, s.src_seg);
        m.in_place = s.dst == s.src;
        if (!m.dst.nested()) return set_error(DBA_EINVAL, "dba_beam_reorder: pieces of state %d's dst overlap", i);
        if (m.src.axes && m.src.stride[m.src.axes - 1] < 0) return set_error(DBA_EINVAL, "dba_beam_reorder: state %d has a negative stride", i);
        if (!m.dst.fits() || !m.src.fits()) return set_error(DBA_EINVAL, "dba_beam_reorder: state %d is larger than memory", i);
        if (m.in_place) {
            if ((B > 1 && s.dst_sent != s.src_sent) || (k > 1 && s.dst_row != s.src_row) || (s.segs > 1 && s.dst_seg != s.src_seg))
                return set_error(DBA_EINVAL, "dba_beam_reorder: state %d is reordered in place with two sets of strides", i);
        } else if (meet(m.dst, m.src)) {
            return set_error(DBA_EINVAL, "dba_beam_reorder: dst and src of state %d overlap", i);
        }
        if ((__int128)s.segs * s.seg_bytes > ((__int128)1 << 31))
            return set_error(DBA_EINVAL, "dba_beam_reorder: a row of state %d has more than 2 GB", i);
    }
    // states are moved at the same time, in any order
    const Places back(backptr_dev, (int64_t)B * k * 4);
    for (int i = 0; i < n_states; ++i) {
        if (!moved[i].any) continue;
        if (meet(moved[i].dst, back)) return set_error(DBA_EINVAL, "dba_beam_reorder: backptr_dev lies in state %d's dst", i);
        for (int j = 0; j < i; ++j)
            if (moved[j].any && (meet(moved[i].dst, moved[j].dst) || (!moved[j].in_place && meet(moved[i].dst, moved[j].src)) ||
                                 (!moved[i].in_place && meet(moved[j].dst, moved[i].src))))
                return set_error(DBA_EINVAL, "dba_beam_reorder: states %d and %d overlap where one is written", j, i);
    }
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    ReorderParams p;
    p.back = backptr_dev;
    p.k = k;
    p.n_states = 0;
    uint32_t blocks = 0;
    const auto flush = [&]() -> int {
        if (!p.n_states) return DBA_OK;
        const dim3 grid(blocks, (unsigned)B);
        const auto kernel = k <= 4 ? dba_reorder_kernel<4> : k <= 8 ? dba_reorder_kernel<8> : k <= 16 ? dba_reorder_kernel<16>
                          : k <= 32 ? dba_reorder_kernel<32> : dba_reorder_kernel<64>;
        const hipError_t e = launch(kernel, grid, dim3(kReorderThreads), 0, stream, p);
        p.n_states = 0;
        blocks = 0;
        return launched("dba_beam_reorder", e);
    };
    for (int i = 0; i < n_states; ++i) {
        dba_state s = states_host[i];
        if (s.segs == 0 || s.seg_bytes == 0) continue;
        if (s.segs > 1 && s.dst_seg == s.seg_bytes && s.src_seg == s.seg_bytes) {
            s.seg_bytes *= s.segs;
            s.segs = 1;
        }
        uintptr_t bits = reinterpret_cast<uintptr_t>(s.dst) | reinterpret_cast<uintptr_t>(s.src) | (uintptr_t)s.seg_bytes;
        if (B > 1) bits |= (uintptr_t)(s.dst_sent | s.src_sent);
        if (k > 1) bits |= (uintptr_t)(s.dst_row | s.src_row);
        if (s.segs > 1) bits |= (uintptr_t)(s.dst_seg | s.src_seg);
        const uint32_t widest = k > 32 ? 8 : 16;       // 64 columns of 16 bytes are more than a thread has registers for
        const uint32_t col = std::min<uint32_t>(widest, (uint32_t)(bits & (~bits + 1)) ? (uint32_t)std::min<uintptr_t>(bits & (~bits + 1), 16) : 16u);
        const uint64_t columns = (uint64_t)(s.segs * s.seg_bytes) / col;
        const uint32_t more = (uint32_t)((columns + kReorderThreads - 1) / kReorderThreads);
        if (p.n_states == kReorderStates || (uint64_t)blocks + more > (1u << 23)) {
            const int rc = flush();
            if (rc != DBA_OK) return rc;
        }
        ReorderState &r = p.s[p.n_states++];
        r.dst = static_cast<unsigned char *>(s.dst);
        r.src = static_cast<const unsigned char *>(s.src);
        r.dst_sent = s.dst_sent;
        r.dst_row = s.dst_row;
        r.dst_seg = s.dst_seg;
        r.src_sent = s.src_sent;
        r.src_row = s.src_row;
        r.src_seg = s.src_seg;
        r.segs = (uint32_t)s.segs;
        r.per_seg = (uint32_t)(s.seg_bytes / col);
        r.col_bytes = col;
        r.first_block = blocks;
        blocks += more;
    }
    return flush();
}

DBA_API int dba_cache_append(int B, int n, const dba_cache *cache, const dba_heads *k, const dba_heads *v, int q_heads, const dba_heads *q,
                             const dba_heads *q_out, const int32_t *first_dev, const int32_t *count_dev, const int32_t *position_dev,
                             const float *inv_freq_dev, int rot_dim, int interleaved, void *hip_stream)
{
    const char *fault = cache_fault(cache);
    if (fault) return set_error(DBA_EINVAL, "dba_cache_append: %s", fault);
    if (B < 1 || B > 65535 || n < 1 || n > kMostRows) return set_error(DBA_EINVAL, "dba_cache_append: need 1 <= B <= 65535, 1 <= n <= 2^22");
    if ((fault = heads_fault(k, cache->format)) || (fault = heads_fault(v, cache->format)))
        return set_error(DBA_EINVAL, "dba_cache_append: %s", fault);
    if ((q != nullptr) != (q_out != nullptr)) return set_error(DBA_EINVAL, "dba_cache_append: q and q_out go together");
    if (q) {
        if ((fault = heads_fault(q, cache->format)) || (fault = heads_fault(q_out, cache->format)))
            return set_error(DBA_EINVAL, "dba_cache_append: %s", fault);
        if (q_heads < 1 || q_heads > 8192) return set_error(DBA_EINVAL, "dba_cache_append: 1 <= q_heads <= 8192");
        if (q->data == q_out->data && (q->sent_stride != q_out->sent_stride || q->token_stride != q_out->token_stride || q->head_stride != q_out->head_stride))
            return set_error(DBA_EINVAL, "dba_cache_append: q is rotated in place with two sets of strides");
    }
    if (!first_dev) return set_error(DBA_EINVAL, "dba_cache_append: first_dev is NULL");
    if (rot_dim < 0 || rot_dim > cache->head_dim || rot_dim % 16) return set_error(DBA_EINVAL, "dba_cache_append: rot_dim must be a multiple of 16, at most head_dim");
    if (rot_dim && !inv_freq_dev) return set_error(DBA_EINVAL, "dba_cache_append: inv_freq_dev is NULL");
    if (!places_of(cache->k, *cache).nested()) return set_error(DBA_EINVAL, "dba_cache_append: tokens of the cache overlap");
    if (q) {
        const Places to = places_of(*q_out, B, n, q_heads, *cache);
        if (!to.nested()) return set_error(DBA_EINVAL, "dba_cache_append: pieces of q_out overlap");
        if ((!same(*q, *q_out) && meet(to, places_of(*q, B, n, q_heads, *cache))) || meet(to, places_of(*k, B, n, cache->heads, *cache)) ||
            meet(to, places_of(*v, B, n, cache->heads, *cache)))
            return set_error(DBA_EINVAL, "dba_cache_append: q_out overlaps k, v or a part of q");
    }
    AppendParams p;
    p.cache = paged_of(*cache);
    p.k_pages = static_cast<unsigned char *>(cache->k);
    p.v_pages = static_cast<unsigned char *>(cache->v);
    p.q = heads_of(q);
    p.q_out = heads_of(q_out);
    p.k = heads_of(k);
    p.v = heads_of(v);
    p.first = first_dev;
    p.count = count_dev;
    p.position = position_dev;
    p.inv_freq = inv_freq_dev;
    p.n = n;
    p.heads = cache->heads;
    p.q_heads = q ? q_heads : 0;
    p.D = cache->head_dim;
    p.rot = rot_dim;
    p.interleaved = interleaved != 0;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const dim3 grid((unsigned)n, (unsigned)B);
    const int pairs = (p.q_heads + 2 * p.heads) * (((p.D * (int)elem_bytes(cache->format) + 15) / 16 + 1) / 2);
    const unsigned threads = (unsigned)std::min(kAppendThreads, (pairs + 63) / 64 * 64);       // a thread for every two chunks of a token
    const auto kernel = cache->format == DBA_LOGP_F32 ? dba_append_kernel<0> : cache->format == DBA_LOGP_F16 ? dba_append_kernel<1> : dba_append_kernel<2>;
    return launched("dba_cache_append", launch(kernel, grid, dim3(threads), 0, stream, p));
}

DBA_API size_t dba_tree_attend_workspace_bytes(int B, int n, int q_heads, const dba_cache *cache, int max_len)
{
    if (attend_fault(B, n, q_heads, cache, max_len)) return 0;
    const AttendPlan a = attend_plan(B, n, q_heads, *cache, max_len);
    if (a.splits == 1) return 0;
    const size_t rows = attend_rows_of(B, n, q_heads, a);
    return align256(rows * cache->head_dim * 4) + align256(rows * 8);
}

DBA_API int dba_tree_attend(int B, int n, int q_heads, const dba_heads *q, const dba_cache *cache, const int32_t *prefix_dev,
                            const int32_t *tree_dev, const uint64_t *mask_dev, int mask_words, int max_len, float scale,
                            const dba_heads *out, float *out_lse_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    const char *fault = attend_fault(B, n, q_heads, cache, max_len);
    if (fault) return set_error(DBA_EINVAL, "dba_tree_attend: %s", fault);
    if ((fault = heads_fault(q, cache->format)) || (fault = heads_fault(out, cache->format)))
        return set_error(DBA_EINVAL, "dba_tree_attend: %s", fault);
    if (!prefix_dev) return set_error(DBA_EINVAL, "dba_tree_attend: prefix_dev is NULL");
    if (mask_words < 0 || (mask_dev && !tree_dev)) return set_error(DBA_EINVAL, "dba_tree_attend: a mask needs tree_dev and mask_words >= 0");
    if (!(fabsf(scale) <= 1e30f)) return set_error(DBA_EINVAL, "dba_tree_attend: scale is not a number between -1e30 and 1e30");
    const AttendPlan plan = attend_plan(B, n, q_heads, *cache, max_len);
    const size_t need = dba_tree_attend_workspace_bytes(B, n, q_heads, cache, max_len);
    if (need) {
        if (!workspace_dev || misaligned(workspace_dev, 256)) return set_error(DBA_EINVAL, "dba_tree_attend: workspace_dev must be 256-byte aligned");
        if (workspace_bytes < need) return set_error(DBA_ENOMEM, "dba_tree_attend: workspace has %zu bytes, %zu needed", workspace_bytes, need);
    }
    const Places to = places_of(*out, B, n, q_heads, *cache), from = places_of(*q, B, n, q_heads, *cache);
    const Places lse(out_lse_dev, out_lse_dev ? (int64_t)B * n * q_heads * 4 : 0), room(workspace_dev, (int64_t)need);
    if (!to.nested()) return set_error(DBA_EINVAL, "dba_tree_attend: pieces of out overlap");
    if (!same(*q, *out) && meet(to, from)) return set_error(DBA_EINVAL, "dba_tree_attend: out overlaps a part of q");
    if (meet(lse, to) || meet(lse, from)) return set_error(DBA_EINVAL, "dba_tree_attend: out_lse_dev lies in out or q");
    if (meet(room, to) || meet(room, from) || meet(room, lse)) return set_error(DBA_EINVAL, "dba_tree_attend: q, out or out_lse_dev lies in the workspace");
    AttendParams p;
    p.cache = paged_of(*cache);
    p.k_pages = static_cast<const unsigned char *>(cache->k);
    p.v_pages = static_cast<const unsigned char *>(cache->v);
    p.q = heads_of(q);
    p.out = heads_of(out);
    p.prefix = prefix_dev;
    p.tree = tree_dev;
    p.mask = reinterpret_cast<const unsigned long long *>(mask_dev);
    p.lse = out_lse_dev;
    p.n = n;
    p.q_heads = q_heads;
    p.heads = cache->heads;
    p.D = cache->head_dim;
    p.mask_words = mask_words;
    p.max_len = max_len;
    p.scale = scale;
    p.row_tiles = plan.row_tiles;
    p.tile_rows = plan.tile_rows;
    p.splits = plan.splits;
    p.chunk = plan.chunk;
    p.pairs = B * (cache->heads / plan.side);
    p.groups = p.pairs * plan.splits;
    p.part_o = static_cast<float *>(workspace_dev);
    p.part_ml = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace_dev) + align256(attend_rows_of(B, n, q_heads, plan) * cache->head_dim * 4));
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = cache->format == DBA_LOGP_F32 ? attend_launch<0>(p, plan, B, stream)
                       : cache->format == DBA_LOGP_F16 ? attend_launch<1>(p, plan, B, stream) : attend_launch<2>(p, plan, B, stream);
    return launched("dba_tree_attend", e);
}

}  // extern "C"
