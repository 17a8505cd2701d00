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

// The same in every thread: the sum over a workgroup of W waves, which all wait.
template <int W>
__device__ __forceinline__ uint32_t sum_of_all(uint32_t v, uint32_t (&s_wave)[W])
{
    v = wave_sum_up_to(v);
    if (lane_id() == 63) s_wave[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t all = 0;
    for (int w = 0; w < W; ++w) all += s_wave[w];
    __syncthreads();
    return all;
}

// What a choice goes by.
struct Choice {
    int P;                             // tokens to choose from, some of which may not be there
    int stay;                          // so many stay
    uint32_t need;                     // of the kind that the choice is among
    bool all, among_safe;              // all are there; the choice is among the first and last ones, since there is no room for all of those
};

// Scores are ranked as 32-bit images in their order, from 1 on (a NaN, behind all others); 0 is a token that is not asked about.
__device__ __forceinline__ bool evict_present(const EvictParams &p, int b, int x) { return token_offset(p.from, b, x) >= 0; }
__device__ __forceinline__ bool evict_safe(const EvictParams &p, const Choice &c, int x) { return x < p.sinks || x >= c.P - p.recent; }
__device__ __forceinline__ uint32_t evict_key(const EvictParams &p, const Choice &c, int b, int x, float s)
{
    if (evict_safe(p, c, x) != c.among_safe || !(c.all || evict_present(p, b, x))) return 0;
    return s != s ? 1u : ord_from_float(s);
}

// there: of the P tokens, so many are; safe: of the first and last ones, which go before all others, so many.
__device__ __forceinline__ Choice choice_of(const EvictParams &p, int b, int P, int there, int safe)
{
    Choice c;
    c.P = P;
    c.all = there == P;
    c.stay = min(p.budget ? min(p.keep, max(p.budget[b], 0)) : p.keep, there);
    c.among_safe = safe >= c.stay;
    c.need = (uint32_t)(c.among_safe ? c.stay : c.stay - safe);
    return c;
}

// Counts those, by a whole workgroup of W waves, every thread with the same result.  A page is there with all of its tokens, so pages are what is gone through.
template <int W>
__device__ __forceinline__ int2 evict_counts(const EvictParams &p, int b, int P, uint32_t (&s_wave)[W])
{
    const int t = (int)threadIdx.x, pages = P > 0 ? ((P - 1) >> p.from.page_shift) + 1 : 0;
    const int sinks = min(p.sinks, P), rest = max(P - p.recent, sinks);        // places before the one and from the other on are safe
    uint32_t mine = 0, mine_safe = 0;
    for (int g = t; g < pages; g += 64 * W) {
        const int first = g << p.from.page_shift, last = first + min(1 << p.from.page_shift, P - first);
        if (!evict_present(p, b, first)) continue;
        mine += (uint32_t)(last - first);
        mine_safe += (uint32_t)(max(min(last, sinks) - first, 0) + max(last - max(first, rest), 0));
    }
    const int there = (int)sum_of_all<W>(mine, s_wave);
    return make_int2(there, there == P ? sinks + P - rest : (int)sum_of_all<W>(mine_safe, s_wave));
}

// The images are found digit by digit: 11, 11 and 10 bits.
constexpr int kDigits = 2048;
struct Digit {
    int shift, bits;
};
__device__ __forceinline__ Digit digit_of(int pass) { return pass == 0 ? Digit{21, 11} : pass == 1 ? Digit{10, 11} : Digit{0, 10}; }

// Adds a wave's keys to the counts of their digits; a wave of equals is one addition.
__device__ __forceinline__ void count_digit(uint32_t *hist, bool in, uint32_t digit)
{
    const unsigned long long who = __ballot(in);
    if (who == 0) return;
    const uint32_t one = (uint32_t)__builtin_amdgcn_readlane((int)digit, __builtin_ctzll(who));
    if (__ballot(in && digit == one) == who) {
        if (lane_id() == 0) atomicAdd(&hist[one], (uint32_t)__popcll(who));
    } else if (in) {
        atomicAdd(&hist[digit], 1u);
    }
}

// The digit that holds the `need`-th greatest, how many of it are needed, and how many there are.  Thread t has the counts of some digits next to each other,
// thread 0 the greatest ones: n[0] is of digit kDigits - 1 - PER t, the next of one less.
template <int W, int PER>
__device__ __forceinline__ void find_digit(const uint32_t (&n)[PER], uint32_t need, uint32_t (&s_wave)[W], uint32_t (&s_found)[3])
{
    uint32_t sum = 0;
#pragma unroll
    for (int x = 0; x < PER; ++x) sum += n[x];
    const uint32_t up = wave_sum_up_to(sum);
    if (lane_id() == 63) s_wave[threadIdx.x >> 6] = up;
    __syncthreads();
    uint32_t before = up - sum;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) before += s_wave[w];
    if (before < need && before + sum >= need) {
        uint32_t digit = 0, left = 0, count = 0;
        bool found = false;
#pragma unroll
        for (int x = 0; x < PER; ++x) {
            if (!found && before + n[x] >= need) {
                digit = (uint32_t)(kDigits - 1 - PER * (int)threadIdx.x - x);
                left = need - before;
                count = n[x];
                found = true;
            }
            before += n[x];
        }
        s_found[0] = digit;
        s_found[1] = left;
        s_found[2] = count;
    }
    __syncthreads();
}

// The least image that stays, and how many of its equals do, the first ones.
struct Bar {
    uint32_t least, equals;
};

// Writes the places of those of a wave's 64 tokens from x0 on that stay; s0 and e0: tokens sure to stay, and equal to the bar, before them.
__device__ __forceinline__ void list_wave(const EvictParams &p, const Choice &c, const Bar &bar, int b, int32_t *list, int x, bool in, uint32_t key, uint32_t &s0, uint32_t &e0)
{
    const bool sure = in && (key > bar.least || (key == 0 && !c.among_safe && evict_safe(p, c, x) && (c.all || evict_present(p, b, x)))), tied = in && key == bar.least;
    const unsigned long long who = __ballot(sure), same = __ballot(tied), below = (1ull << lane_id()) - 1;
    const uint32_t e = e0 + (uint32_t)__popcll(same & below), place = s0 + (uint32_t)__popcll(who & below) + min(e, bar.equals);
    if ((sure || (tied && e < bar.equals)) && place < (uint32_t)p.cap) list[place] = x;
    s0 += (uint32_t)__popcll(who);
    e0 += (uint32_t)__popcll(same);
}
// How many are sure to stay, and equal to the bar: the same for tokens that are not listed here.
__device__ __forceinline__ uint2 count_of(const EvictParams &p, const Choice &c, const Bar &bar, int b, int x, uint32_t key)
{
    return make_uint2(key > bar.least || (key == 0 && !c.among_safe && evict_safe(p, c, x) && (c.all || evict_present(p, b, x))), key == bar.least);
}

// One workgroup of W waves per sentence and row of scores of up to 64 W NK tokens, whose images stay in registers.  A wave has a stretch of its own, so that
// places come from counts of waves and ballots.
// Bound: latency, a chain of seven to seventeen barriers (two, or four where a page is missing, four a digit, one); scores are a small part of what the move behind it takes.
template <int W, int NK>
__global__ __launch_bounds__(64 * W) void dba_evict_choose_kernel(EvictParams p)
{
    __shared__ uint32_t s_hist[kDigits];
    __shared__ uint32_t s_wave[2][W];
    __shared__ uint32_t s_found[3];
    const int lane = lane_id(), t = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int b = (int)blockIdx.y, head = (int)blockIdx.x;
    const float *const score = p.score + ((int64_t)b * p.score_sent + (int64_t)head * p.score_head);
    const int P = span_of(p.prefix[b], 0, p.max_len).prefix;
    const int reach = (P + 64 * W - 1) / (64 * W), base = wave * reach * 64 + lane;        // 64s of tokens a wave; this lane's first
    float s[NK];
#pragma unroll
    for (int x = 0; x < NK; ++x) s[x] = x < reach && base + x * 64 < P ? score[base + x * 64] : 0.0f;      // (asked for before all else)
    const int2 counts = evict_counts<W>(p, b, P, s_wave[0]);
    const Choice c = choice_of(p, b, P, counts.x, counts.y);
    if (head == 0 && t == 0) p.new_prefix[b] = c.stay;
    if (c.stay == 0) return;
    uint32_t key[NK];
#pragma unroll
    for (int x = 0; x < NK; ++x) key[x] = x < reach && base + x * 64 < P ? evict_key(p, c, b, base + x * 64, s[x]) : 0;
    uint32_t known = 0, need = c.need;
    Bar bar = {0, 0};
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const Digit d = digit_of(pass);
        for (int x = t; x < kDigits; x += 64 * W) s_hist[x] = 0;
        __syncthreads();
#pragma unroll
        for (int x = 0; x < NK; ++x)
            if (x < reach) count_digit(s_hist, key[x] != 0 && (pass == 0 || key[x] >> (d.shift + d.bits) == known), key[x] >> d.shift & ((1u << d.bits) - 1));
        __syncthreads();
        constexpr int PER = kDigits / (64 * W);
        uint32_t n[PER];
#pragma unroll
        for (int x = 0; x < PER; ++x) n[x] = s_hist[kDigits - 1 - PER * t - x];
        find_digit<W, PER>(n, need, s_wave[0], s_found);
        known = known << d.bits | s_found[0];
        need = s_found[1];
        bar = {max(known << d.shift, 1u), need};
        if (s_found[2] == need) {                      // all that are alike so far stay
            bar.equals = 0xFFFFFFFFu;
            break;
        }
    }
    uint32_t n_sure = 0, n_tied = 0;
#pragma unroll
    for (int x = 0; x < NK; ++x) {
        if (x >= reach) continue;
        const uint2 n = base + x * 64 < P ? count_of(p, c, bar, b, base + x * 64, key[x]) : make_uint2(0, 0);
        n_sure += (uint32_t)__popcll(__ballot(n.x));
        n_tied += (uint32_t)__popcll(__ballot(n.y));
    }
    if (lane == 0) {
        s_wave[0][wave] = n_sure;
        s_wave[1][wave] = n_tied;
    }
    __syncthreads();
    uint32_t s0 = 0, e0 = 0;
    for (int w = 0; w < wave; ++w) {
        s0 += s_wave[0][w];
        e0 += s_wave[1][w];
    }
    int32_t *const list = p.list + ((int64_t)b * p.heads_s + head) * p.cap;
#pragma unroll
    for (int x = 0; x < NK; ++x)
        if (x < reach) list_wave(p, c, bar, b, list, base + x * 64, base + x * 64 < P, key[x], s0, e0);
}

// Longer rows in launches with a workgroup for each kEvictPart tokens: what is there of a sentence; counts of the first digit; the bar, from those counts and the tokens of that digit, by one
// workgroup a row; how many stay of each part; the list.  Scores are read five times at most and a sentence's pages once; a part of the list adds up the numbers of those before it.
// (One choice of 16384 of 65000 tokens, 4 sentences: 4.6 + 4.8 + 24 + 4.6 + 6.2 us; one workgroup took 103.  8 choices of 64 of a million tokens 0.37 ms, of four million 1.36; where each
// part counted all scores before it 1.33 and 14.4, and with an absent page among 16 tokens each, which each part looked for, 3.1 and 43.7 instead of 0.42 and 1.51.)
constexpr int kEvictWaves = 16, kEvictPart = 4096, kEvictPer = kEvictPart / (64 * kEvictWaves);

constexpr int kEvictFew = 4096;        // tokens of the first digit that are kept rather than looked for once more

struct EvictLong {
    uint32_t *hist;                    // [B, heads_s, parts, kDigits]
    uint32_t *found;                   // [B, heads_s, 2]: the bar
    int2 *counts;                      // [B]
    uint2 *tally;                      // [B, heads_s, parts]: sure to stay, and equal to the bar
    int parts;
};

__global__ __launch_bounds__(64 * kEvictWaves) void dba_evict_there_kernel(EvictParams p, EvictLong l)
{
    __shared__ uint32_t s_wave[kEvictWaves];
    const int b = (int)blockIdx.x, P = span_of(p.prefix[b], 0, p.max_len).prefix;
    const int2 counts = evict_counts<kEvictWaves>(p, b, P, s_wave);
    if (threadIdx.x == 0) {
        p.new_prefix[b] = choice_of(p, b, P, counts.x, counts.y).stay;
        l.counts[b] = counts;
    }
}

// The choice of a long row, once its sentence's tokens have been counted.
__device__ __forceinline__ Choice choice_of(const EvictParams &p, const EvictLong &l, int b)
{
    return choice_of(p, b, span_of(p.prefix[b], 0, p.max_len).prefix, l.counts[b].x, l.counts[b].y);
}

__global__ __launch_bounds__(64 * kEvictWaves) void dba_evict_count_kernel(EvictParams p, EvictLong l)
{
    __shared__ uint32_t s_hist[kDigits];
    const int t = (int)threadIdx.x, b = (int)blockIdx.z, head = (int)blockIdx.y, first = (int)blockIdx.x * kEvictPart;
    const float *const score = p.score + ((int64_t)b * p.score_sent + (int64_t)head * p.score_head);
    const Choice c = choice_of(p, l, b);
    if (first >= c.P) return;                          // (nobody asks for it)
    for (int x = t; x < kDigits; x += 64 * kEvictWaves) s_hist[x] = 0;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kEvictPer; ++x) {
        const int at = first + x * 64 * kEvictWaves + t;
        const uint32_t key = at < c.P ? evict_key(p, c, b, at, score[at]) : 0;
        count_digit(s_hist, key != 0, key >> digit_of(0).shift);
    }
    __syncthreads();
    uint32_t *const out = l.hist + (((int64_t)b * p.heads_s + head) * l.parts + blockIdx.x) * kDigits;
    for (int x = t; x < kDigits; x += 64 * kEvictWaves) out[x] = s_hist[x];
}

__global__ __launch_bounds__(64 * kEvictWaves) void dba_evict_bar_kernel(EvictParams p, EvictLong l)
{
    __shared__ uint32_t s_hist[kDigits], s_key[kEvictFew], s_wave[kEvictWaves], s_found[3], s_few;
    const int t = (int)threadIdx.x, b = (int)blockIdx.y, head = (int)blockIdx.x;
    const float *const score = p.score + ((int64_t)b * p.score_sent + (int64_t)head * p.score_head);
    const Choice c = choice_of(p, l, b);
    if (c.stay == 0) return;
    constexpr int PER = kDigits / (64 * kEvictWaves);
    uint32_t n[PER] = {}, known = 0, need = c.need, few = 0;      // few: of the first digit, so many in s_key
    const uint32_t *const hist = l.hist + ((int64_t)b * p.heads_s + head) * l.parts * kDigits;
    const int parts = (c.P + kEvictPart - 1) / kEvictPart;
    constexpr int PARTS = 8;                           // whose loads are under way
    for (int part = 0; part < parts; part += PARTS) {
        uint32_t y[PARTS][PER];
#pragma unroll
        for (int z = 0; z < PARTS; ++z)
#pragma unroll
            for (int x = 0; x < PER; ++x) y[z][x] = hist[(int64_t)min(part + z, parts - 1) * kDigits + kDigits - 1 - PER * t - x];
#pragma unroll
        for (int z = 0; z < PARTS; ++z)
#pragma unroll
            for (int x = 0; x < PER; ++x) n[x] += part + z < parts ? y[z][x] : 0;
    }
    Bar bar = {0, 0};
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const Digit d = digit_of(pass);
        if (pass > 0) {
            for (int x = t; x < kDigits; x += 64 * kEvictWaves) s_hist[x] = 0;
            if (t == 0) s_few = 0;
            __syncthreads();
            // (the images of what is looked for are those of the scores between these two; a NaN's is alone in the digit 0)
            const uint32_t lowest = known << (d.shift + d.bits);
            const float least = float_from_ord(max(lowest, ord_from_float(-INFINITY))), most = float_from_ord(min(lowest | ((1u << (d.shift + d.bits)) - 1), ord_from_float(INFINITY)));
            const bool gather = pass == 1 && s_found[2] <= kEvictFew;
            constexpr int U = 16;                      // loads under way
            for (int x0 = 0; x0 < (few ? 0 : c.P); x0 += U * 64 * kEvictWaves) {
                float s[U];
#pragma unroll
                for (int x = 0; x < U; ++x) s[x] = score[min(x0 + x * 64 * kEvictWaves + t, c.P - 1)];
                uint32_t hits = 0, key[U];
#pragma unroll
                for (int x = 0; x < U; ++x) {
                    const bool in = known == 0 ? s[x] != s[x] : (s[x] >= least) & (s[x] <= most);
                    const int at = x0 + x * 64 * kEvictWaves + t;
                    // (evict_key without a branch; zeros of either sign are one image)
                    const bool safe = (at < p.sinks) | (at >= c.P - p.recent);
                    const uint32_t image = known == 0 ? 1u : ord_from_float(s[x]);
                    key[x] = (in & (at < c.P) & (safe == c.among_safe) & (image >> (d.shift + d.bits) == known)) ? image : 0;
                    if (!c.all && key[x] && !evict_present(p, b, at)) key[x] = 0;
                    hits += key[x] != 0;
                }
                if (gather) {                          // a place for each, with one atomic a wave
                    const uint32_t up = wave_sum_up_to(hits);
                    uint32_t place = 0;
                    if (lane_id() == 63 && up) place = atomicAdd(&s_few, up);
                    place = (uint32_t)__builtin_amdgcn_readlane((int)place, 63) + up - hits;
#pragma unroll
                    for (int x = 0; x < U; ++x)
                        if (key[x]) s_key[place++] = key[x];
                } else {
#pragma unroll
                    for (int x = 0; x < U; ++x) count_digit(s_hist, key[x] != 0, key[x] >> d.shift & ((1u << d.bits) - 1));
                }
            }
            if (gather) {
                __syncthreads();
                few = s_few;
            }
            if (few)
                for (uint32_t x = t; x < ((few + 63) & ~63u); x += 64 * kEvictWaves) {
                    const uint32_t key = s_key[min(x, few - 1)];
                    count_digit(s_hist, x < few && key >> (d.shift + d.bits) == known, key >> d.shift & ((1u << d.bits) - 1));
                }
            __syncthreads();
#pragma unroll
            for (int x = 0; x < PER; ++x) n[x] = s_hist[kDigits - 1 - PER * t - x];
        }
        find_digit<kEvictWaves, PER>(n, need, s_wave, s_found);
        known = known << d.bits | s_found[0];
        need = s_found[1];
        bar = {max(known << d.shift, 1u), need};
        if (s_found[2] == need) {
            bar.equals = 0xFFFFFFFFu;
            break;
        }
    }
    if (t == 0) {
        l.found[((int64_t)b * p.heads_s + head) * 2] = bar.least;
        l.found[((int64_t)b * p.heads_s + head) * 2 + 1] = bar.equals;
    }
}

// How many of a wave's stretch of this part are sure to stay, and equal to the bar: each a whole wave's number.  key: their images.
__device__ __forceinline__ uint2 evict_stretch(const EvictParams &p, const Choice &c, const Bar &bar, int b, const float *score, int base, uint32_t (&key)[kEvictPer])
{
    uint2 n = make_uint2(0, 0);
#pragma unroll
    for (int x = 0; x < kEvictPer; ++x) {
        const int at = base + x * 64;
        key[x] = at < c.P ? evict_key(p, c, b, at, score[at]) : 0;
        const uint2 one = at < c.P ? count_of(p, c, bar, b, at, key[x]) : make_uint2(0, 0);
        n.x += (uint32_t)__popcll(__ballot(one.x));
        n.y += (uint32_t)__popcll(__ballot(one.y));
    }
    return n;
}

__global__ __launch_bounds__(64 * kEvictWaves) void dba_evict_tally_kernel(EvictParams p, EvictLong l)
{
    __shared__ uint32_t s_wave[2][kEvictWaves];
    const int lane = lane_id(), t = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), b = (int)blockIdx.z, head = (int)blockIdx.y, first = (int)blockIdx.x * kEvictPart;
    const float *const score = p.score + ((int64_t)b * p.score_sent + (int64_t)head * p.score_head);
    const Choice c = choice_of(p, l, b);
    if (c.stay == 0 || first >= c.P) return;
    const int64_t row = (int64_t)b * p.heads_s + head;
    const Bar bar = {l.found[row * 2], l.found[row * 2 + 1]};
    uint32_t key[kEvictPer];
    const uint2 n = evict_stretch(p, c, bar, b, score, first + wave * kEvictPer * 64 + lane, key);
    if (lane == 0) {
        s_wave[0][wave] = n.x;
        s_wave[1][wave] = n.y;
    }
    __syncthreads();
    if (t) return;
    uint2 all = make_uint2(0, 0);
    for (int w = 0; w < kEvictWaves; ++w) {
        all.x += s_wave[0][w];
        all.y += s_wave[1][w];
    }
    l.tally[row * l.parts + blockIdx.x] = all;
}

__global__ __launch_bounds__(64 * kEvictWaves) void dba_evict_list_kernel(EvictParams p, EvictLong l)
{
    __shared__ uint32_t s_wave[2][kEvictWaves];
    const int lane = lane_id(), t = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), b = (int)blockIdx.z, head = (int)blockIdx.y, first = (int)blockIdx.x * kEvictPart;
    const float *const score = p.score + ((int64_t)b * p.score_sent + (int64_t)head * p.score_head);
    const Choice c = choice_of(p, l, b);
    if (c.stay == 0 || first >= c.P) return;
    const int64_t row = (int64_t)b * p.heads_s + head;
    const Bar bar = {l.found[row * 2], l.found[row * 2 + 1]};
    uint32_t before_sure = 0, before_tied = 0;
    for (int x = t; x < (int)blockIdx.x; x += 64 * kEvictWaves) {
        const uint2 n = l.tally[row * l.parts + x];
        before_sure += n.x;
        before_tied += n.y;
    }
    const int base = first + wave * kEvictPer * 64 + lane;
    uint32_t key[kEvictPer];
    const uint2 n = evict_stretch(p, c, bar, b, score, base, key);
    before_sure = sum_of_all<kEvictWaves>(before_sure, s_wave[0]);
    before_tied = sum_of_all<kEvictWaves>(before_tied, s_wave[1]);
    if (lane == 0) {
        s_wave[0][wave] = n.x;
        s_wave[1][wave] = n.y;
    }
    __syncthreads();
    uint32_t s0 = before_sure, e0 = before_tied;
    for (int w = 0; w < wave; ++w) {
        s0 += s_wave[0][w];
        e0 += s_wave[1][w];
    }
    int32_t *const list = p.list + ((int64_t)b * p.heads_s + head) * p.cap;
#pragma unroll
    for (int x = 0; x < kEvictPer; ++x) list_wave(p, c, bar, b, list, base + x * 64, base + x * 64 < c.P, key[x], s0, e0);
}

constexpr int kMoveThreads = 256, kMoveItems = 4;      // chunks of keys, and of values, that a thread has under way
constexpr int kMoveScores = 8;                         // scores of a thread, where a row is much wider than what is moved

// Token j of the new pages is the list's j-th, or behind those the tree's (j - stay)-th.  Bound: memory; each thread moves 16 bytes of keys and of values at
// a time, which of a token lie side by side.  Nothing that is moved is asked for again, so it goes past the caches (64 x 1200 tokens of 8 heads of 128 in bf16, a choice for
// each head: 134 us, 4.7 TB/s read and written; kept in the caches 140; without the next turn's places under way 158).
__global__ __launch_bounds__(kMoveThreads) void dba_evict_move_kernel(EvictParams p)
{
    typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
    const int b = (int)blockIdx.y, t = (int)threadIdx.x;
    const Span span = span_of(p.prefix[b], p.tree ? p.tree[b] : 0, p.max_len);
    const int stay = p.new_prefix[b], total = stay + (span.end - span.prefix);
    const int32_t *const list = p.list + (int64_t)b * p.heads_s * p.cap;
    const uint32_t per_token = (uint32_t)(p.heads * p.chunks);
    const uint64_t items = (uint64_t)total * per_token, turn = kMoveThreads * kMoveItems, step = (uint64_t)gridDim.x * turn;
    // what a turn needs is asked for ahead: where its tokens come from two turns, their pages one
    int src[kMoveItems];
    int64_t from[kMoveItems], to[kMoveItems];          // bytes; to: -1: nothing to move
    auto item = [&](uint64_t x0, int u, int &j, uint32_t &h, uint32_t &c) -> bool {
        const uint64_t j0 = x0 / per_token;             // (the same for all)
        const uint32_t x = (uint32_t)(x0 - j0 * per_token) + (uint32_t)(u * kMoveThreads + t), tokens = x / per_token, in = x - tokens * per_token;
        j = (int)j0 + (int)tokens;
        h = in / (uint32_t)p.chunks;
        c = in - h * (uint32_t)p.chunks;
        return x0 + (uint64_t)(u * kMoveThreads + t) < items;
    };
    auto ask_source = [&](uint64_t x0) {
#pragma unroll
        for (int u = 0; u < kMoveItems; ++u) {
            int j;
            uint32_t h, c;
            src[u] = -1;
            if (item(x0, u, j, h, c)) src[u] = j < stay ? list[(p.heads_s > 1 ? (int64_t)h * p.cap : 0) + j] : span.prefix + (j - stay);
        }
    };
    auto ask_pages = [&](uint64_t x0) {
#pragma unroll
        for (int u = 0; u < kMoveItems; ++u) {
            int j;
            uint32_t h, c;
            item(x0, u, j, h, c);
            const int64_t old = token_offset(p.from, b, src[u]), at = src[u] < 0 ? -1 : token_offset(p.to, b, j), inside = (int64_t)h * p.from.head_stride * p.elem + (int64_t)c * 16;
            from[u] = old * p.elem + inside;
            to[u] = old < 0 || at < 0 ? -1 : at * p.elem + inside;
        }
    };
    const uint64_t first = (uint64_t)blockIdx.x * turn;
    if (first < items) {
        ask_source(first);
        ask_pages(first);
        ask_source(first + step);
    }
    for (uint64_t x0 = first; x0 < items; x0 += step) {
        u32x4_t k[kMoveItems], v[kMoveItems];
        int64_t at[kMoveItems];
#pragma unroll
        for (int u = 0; u < kMoveItems; ++u) {
            at[u] = to[u];
            if (to[u] < 0) continue;
            k[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p.k_pages + from[u]));
            v[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p.v_pages + from[u]));
        }
        if (x0 + step < items) {
            ask_pages(x0 + step);
            ask_source(x0 + 2 * step);
        }
#pragma unroll
        for (int u = 0; u < kMoveItems; ++u) {
            if (at[u] < 0) continue;
            __builtin_nontemporal_store(k[u], reinterpret_cast<u32x4_t *>(p.k_pages + at[u]));
            __builtin_nontemporal_store(v[u], reinterpret_cast<u32x4_t *>(p.v_pages + at[u]));
        }
    }
    if (!p.new_score) return;
    // (h, j) of heads_s rows of `width`, one behind the other: no division a score
    const uint32_t width = (uint32_t)p.width, start = blockIdx.x * kMoveThreads + (uint32_t)t, stride = gridDim.x * kMoveThreads;
    uint32_t h = start / width, j0 = start - h * width;
    const uint32_t rows_on = stride / width, on = stride - rows_on * width;
    for (; h < (uint32_t)p.heads_s; h += rows_on + (j0 + on >= width), j0 = j0 + on >= width ? j0 + on - width : j0 + on) {
        const int j = (int)j0;
        const float *const score = p.score + ((int64_t)b * p.score_sent + (int64_t)h * p.score_head);
        float s = 0.0f;
        if (j < total) s = score[j < stay ? list[(int64_t)h * p.cap + j] : span.prefix + (j - stay)];
        p.new_score[(int64_t)b * p.new_sent + (int64_t)h * p.new_head + j] = s;
    }
}

}  // namespace dba
