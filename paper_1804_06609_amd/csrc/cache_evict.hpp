// Which tokens of a paged cache stay, and their move to other pages: kernels.
#pragma once
#include "paged.hpp"
#include "wave_topk.hpp"

namespace dba {

struct EvictParams {
    Paged from, to;                    // one pool, two tables
    unsigned char *k_pages, *v_pages;
    const float *score;                // [B, heads_s, ..]
    float *new_score;                  // [B, heads_s, width]; nullptr: not wanted
    int64_t score_sent, score_head, new_sent, new_head;
    const int32_t *prefix, *tree, *budget;
    int32_t *new_prefix;
    int32_t *list;                     // [B, heads_s, cap]: places of the tokens that stay, first to last
    int cap, keep, sinks, recent, max_len, width;
    int heads, heads_s, chunks, elem;  // chunks: of 16 bytes, of a head
};

constexpr int kChooseThreads = 1024, kChooseWaves = kChooseThreads / 64;
constexpr int kDigits = 2048, kCopies = 2;

// Inclusive sum over the lanes up to this one.
__device__ __forceinline__ uint32_t wave_sum_up_to(uint32_t v)
{
    const int lane = lane_id();
#pragma unroll
    for (int i = 0; i < 6; ++i) {
        const uint32_t o = (uint32_t)__shfl_up((int)v, 1 << i);
        if (lane >= 1 << i) v += o;
    }
    return v;
}

// One workgroup per sentence and row of scores.  Scores are ranked as 32-bit images in their order (a NaN behind all others); the `need`-th greatest is found
// digit by digit, 11, 11 and 10 bits, from a histogram in LDS, and what lies above it, with as many of its equals as there is room for, first ones
// first, is listed in the order of the places.  A wave has a stretch of its own, so that places come from counts of waves and ballots.
//
// Up to kChooseThreads * NK tokens the images stay in registers; beyond, each pass reads them again.
// Bound: latency; scores are a small part of what the move behind it takes.
template <int NK>
__global__ __launch_bounds__(kChooseThreads) void dba_evict_choose_kernel(EvictParams p)
{
    __shared__ uint32_t s_hist[kCopies][kDigits];
    __shared__ uint32_t s_wave[2][kChooseWaves];
    __shared__ uint32_t s_found[3];
    const int lane = lane_id(), t = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int b = (int)blockIdx.y, head = (int)blockIdx.x;
    const int P = span_of(p.prefix[b], 0, p.max_len).prefix;
    const float *const score = p.score + ((int64_t)b * p.score_sent + (int64_t)head * p.score_head);
    auto sum_of_all = [&](uint32_t v, int slot) -> uint32_t {      // the same in every thread; a barrier on both sides
        v = wave_sum_up_to(v);
        if (lane == 63) s_wave[slot][wave] = v;
        __syncthreads();
        uint32_t all = 0;
        for (int w = 0; w < kChooseWaves; ++w) all += s_wave[slot][w];
        __syncthreads();
        return all;
    };
    auto present = [&](int x) { return token_offset(p.from, b, x) >= 0; };
    auto is_safe = [&](int x) { return x < p.sinks || x >= P - p.recent; };

    // tokens that are there
    const int pages = P > 0 ? ((P - 1) >> p.from.page_shift) + 1 : 0;
    uint32_t mine = 0;
    for (int g = t; g < pages; g += kChooseThreads) {
        const int first = g << p.from.page_shift;
        if (present(first)) mine += (uint32_t)min(1 << p.from.page_shift, P - first);
    }
    const int there = (int)sum_of_all(mine, 0);
    const bool all = there == P;
    const int budget = p.budget ? min(p.keep, max(p.budget[b], 0)) : p.keep;
    const int stay = min(budget, there);
    if (head == 0 && t == 0) p.new_prefix[b] = stay;
    if (stay == 0) return;
    // the first and the last ones go before all others
    int safe = (int)min((int64_t)P, (int64_t)min(p.sinks, P) + min(p.recent, P));
    if (!all) {
        mine = 0;
        for (int x = t; x < P; x += kChooseThreads) mine += is_safe(x) && present(x);
        safe = (int)sum_of_all(mine, 1);
    }
    const bool among_safe = safe >= stay;              // there is no room for all of them
    uint32_t need = (uint32_t)(among_safe ? stay : stay - safe);

    constexpr int kMost = kChooseThreads * NK;         // tokens of a turn
    const int turns = (P + kMost - 1) / kMost;
    uint32_t key[NK];
    int base = 0, reach = 0;                           // of this turn: the wave's first token, 64s of tokens a wave
    auto load = [&](int turn) {
        const int first = turn * kMost, n = min(kMost, P - first);
        reach = (n + kChooseThreads - 1) / kChooseThreads;
        base = first + wave * reach * 64;
#pragma unroll
        for (int x = 0; x < NK; ++x) {
            key[x] = 0;                                // not asked about
            if (x < reach) {
                const int at = base + x * 64 + lane;
                if (at < first + n && is_safe(at) == among_safe && (all || present(at))) {
                    const float s = score[at];
                    key[x] = s != s ? 1u : ord_from_float(s);
                }
            }
        }
    };
    if (turns == 1) load(0);
    uint32_t known = 0, bar = 0, equals = 0;           // the bits found; the least that stays; how many of its equals
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int x = t; x < kDigits; x += kChooseThreads)
            for (int k = 0; k < kCopies; ++k) s_hist[k][x] = 0;
        __syncthreads();
        for (int turn = 0; turn < turns; ++turn) {
            if (turns > 1) load(turn);
#pragma unroll
            for (int x = 0; x < NK; ++x) {
                if (x >= reach) continue;
                const bool in = key[x] != 0 && (pass == 0 || (key[x] >> (shift + bits)) == known);
                const uint32_t digit = (key[x] >> shift) & ((1u << bits) - 1);
                const unsigned long long who = __ballot(in);
                if (who == 0) continue;
                const uint32_t one = (uint32_t)__builtin_amdgcn_readlane((int)digit, __builtin_ctzll(who));
                if (__ballot(in && digit == one) == who) {     // a wave of equals is one addition
                    if (lane == 0) atomicAdd(&s_hist[wave % kCopies][one], (uint32_t)__popcll(who));
                } else if (in) {
                    atomicAdd(&s_hist[wave % kCopies][digit], 1u);
                }
            }
        }
        __syncthreads();
        // from the greatest digit down: thread t has two of them
        const int hi = kDigits - 1 - 2 * t, lo = hi - 1;
        uint32_t n_hi = 0, n_lo = 0;
#pragma unroll
        for (int k = 0; k < kCopies; ++k) {
            n_hi += s_hist[k][hi];
            n_lo += s_hist[k][lo];
        }
        const uint32_t up = wave_sum_up_to(n_hi + n_lo);
        if (lane == 63) s_wave[0][wave] = up;
        __syncthreads();
        uint32_t before = up - n_hi - n_lo;
        for (int w = 0; w < wave; ++w) before += s_wave[0][w];
        if (before < need && before + n_hi + n_lo >= need) {
            const bool in_hi = before + n_hi >= need;
            s_found[0] = (uint32_t)(in_hi ? hi : lo);
            s_found[1] = need - before - (in_hi ? 0 : n_hi);
            s_found[2] = in_hi ? n_hi : n_lo;
        }
        __syncthreads();
        known = known << bits | s_found[0];
        need = s_found[1];
        bar = max(known << shift, 1u);             // (images start at 1)
        equals = need;
        if (s_found[2] == need) {                  // all that are alike so far stay
            equals = 0xFFFFFFFFu;
            break;
        }
    }

    // the list
    int32_t *const list = p.list + ((int64_t)b * p.heads_s + head) * p.cap;
    uint32_t listed = 0, tied = 0;                     // by the turns before
    for (int turn = 0; turn < turns; ++turn) {
        if (turns > 1) load(turn);
        const int last = min(P, (turn + 1) * kMost);
        // sure to stay, and equal to the bar
        auto sure = [&](int x) {
            const int at = base + x * 64 + lane;
            return key[x] > bar || (key[x] == 0 && !among_safe && at < last && is_safe(at) && (all || present(at)));
        };
        uint32_t n_sure = 0, n_tied = 0;
#pragma unroll
        for (int x = 0; x < NK; ++x) {
            if (x >= reach) continue;
            n_sure += (uint32_t)__popcll(__ballot(sure(x)));
            n_tied += (uint32_t)__popcll(__ballot(key[x] == bar));
        }
        __syncthreads();
        if (lane == 0) {
            s_wave[0][wave] = n_sure;
            s_wave[1][wave] = n_tied;
        }
        __syncthreads();
        uint32_t s0 = listed, e0 = tied;
        for (int w = 0; w < kChooseWaves; ++w) {
            const uint32_t a = s_wave[0][w], c = s_wave[1][w];
            if (w < wave) {
                s0 += a;
                e0 += c;
            }
            listed += a;
            tied += c;
        }
        const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
        for (int x = 0; x < NK; ++x) {
            if (x >= reach) continue;
            const bool is_sure = sure(x), is_tied = key[x] == bar;
            const unsigned long long who = __ballot(is_sure), same = __ballot(is_tied);
            const uint32_t e = e0 + (uint32_t)__popcll(same & below), place = s0 + (uint32_t)__popcll(who & below) + min(e, equals);
            if ((is_sure || (is_tied && e < equals)) && place < (uint32_t)p.cap) list[place] = base + x * 64 + lane;
            s0 += (uint32_t)__popcll(who);
            e0 += (uint32_t)__popcll(same);
        }
    }
}

constexpr int kMoveThreads = 256, kMoveItems = 4;      // chunks of keys, and of values, that a thread has under way

// Token j of the new pages is the list's j-th, or behind those the tree's (j - stay)-th.  Bound: memory; each thread moves 16 bytes of keys and of values at
// a time, which of a token lie side by side.
__global__ __launch_bounds__(kMoveThreads) void dba_evict_move_kernel(EvictParams p)
{
    typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
    const int b = (int)blockIdx.y, t = (int)threadIdx.x;
    const Span span = span_of(p.prefix[b], p.tree ? p.tree[b] : 0, p.max_len);
    const int stay = p.new_prefix[b], total = stay + (span.end - span.prefix);
    const int32_t *const list = p.list + (int64_t)b * p.heads_s * p.cap;
    const uint32_t per_token = (uint32_t)(p.heads * p.chunks);
    const uint64_t items = (uint64_t)total * per_token, step = (uint64_t)gridDim.x * kMoveThreads * kMoveItems;
    for (uint64_t x0 = (uint64_t)blockIdx.x * kMoveThreads * kMoveItems; x0 < items; x0 += step) {
        const int j0 = (int)(x0 / per_token);
        const uint32_t in0 = (uint32_t)(x0 - (uint64_t)j0 * per_token), left = (uint32_t)min((uint64_t)kMoveThreads * kMoveItems, items - x0);
        u32x4_t k[kMoveItems], v[kMoveItems];
        int64_t to[kMoveItems];
#pragma unroll
        for (int u = 0; u < kMoveItems; ++u) {
            const uint32_t x = (uint32_t)(u * kMoveThreads + t), tokens = (in0 + x) / per_token;
            to[u] = -1;
            if (x >= left) continue;
            const int j = j0 + (int)tokens;
            const uint32_t in = in0 + x - tokens * per_token, h = in / (uint32_t)p.chunks, c = in - h * (uint32_t)p.chunks;
            const int src = j < stay ? list[(p.heads_s > 1 ? (int64_t)h * p.cap : 0) + j] : span.prefix + (j - stay);
            const int64_t from = token_offset(p.from, b, src), at = token_offset(p.to, b, j);
            if (from < 0 || at < 0) continue;
            const int64_t inside = ((int64_t)h * p.from.head_stride) * p.elem + (int64_t)c * 16;
            k[u] = *reinterpret_cast<const u32x4_t *>(p.k_pages + from * p.elem + inside);
            v[u] = *reinterpret_cast<const u32x4_t *>(p.v_pages + from * p.elem + inside);
            to[u] = at * p.elem + inside;
        }
#pragma unroll
        for (int u = 0; u < kMoveItems; ++u) {
            if (to[u] < 0) continue;
            *reinterpret_cast<u32x4_t *>(p.k_pages + to[u]) = k[u];
            *reinterpret_cast<u32x4_t *>(p.v_pages + to[u]) = v[u];
        }
    }
    if (!p.new_score) return;
    const uint64_t scores = (uint64_t)p.heads_s * (uint32_t)p.width;
    for (uint64_t x = (uint64_t)blockIdx.x * kMoveThreads + t; x < scores; x += (uint64_t)gridDim.x * kMoveThreads) {
        const int h = (int)(x / (uint32_t)p.width), j = (int)(x - (uint64_t)h * (uint32_t)p.width);
        const float *const score = p.score + ((int64_t)b * p.score_sent + (int64_t)h * p.score_head);
        float s = 0.0f;
        if (j < total) s = score[j < stay ? list[(int64_t)h * p.cap + j] : span.prefix + (j - stay)];
        p.new_score[(int64_t)b * p.new_sent + (int64_t)h * p.new_head + j] = s;
    }
}

}  // namespace dba
