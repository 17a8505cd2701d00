// Selection over beams and vocabulary from logits: kernels.
//
// The score of an extension, score[h] + x - lse[h], falls with the logit x inside a row, so a row's best are known
// before its normaliser is.  One pass over the logits therefore does both: a workgroup takes a part of a row
// into registers, sums the exponentials, and hands on the part's k_out greatest logits (and a few more).
// A second launch, one workgroup per sentence, puts the normalisers together and ranks what has been handed on.
#pragma once
#include <type_traits>

#include "wave_topk.hpp"

namespace dba {

// What a part of a row leaves behind: its greatest logit, log sum exp(x - top) and how many keys it has handed on.
struct SelectPart {
    double log_sum;                    // -inf: nothing; not a number: the row offers nothing
    float top;
    int count;
};

struct SelectParams {
    const float *score;
    const uint8_t *flags;              // null: all rows live
    int32_t *out_token, *out_backptr;
    float *out_score;
    uint8_t *out_flags;
    SelectPart *parts;                 // [B, k_in, nparts]
    u64 *keys;                         // [B, k_in, nparts, cap]
    int64_t sent_stride, row_stride;   // elements
    int k_in, k_out, V, nparts, cap, part_chunks, eos, pad;
};

constexpr int kSelectThreads = 256;    // of the first launch
// 16-byte chunks a thread keeps in registers: as many as 64 registers have room for, since a workgroup's chain of barriers takes 9 us however much it has read
// (when this was chosen, rows of 50000 in 16 bits in three parts instead of four: 158 -> 135 us; with ten registers spill)
constexpr int kSelectChunks = 9;
constexpr int kSelectQueue = 256;      // chunks it looks through for keys
constexpr int kSelectKeys = 1024;      // keys it chooses from
// Extensions the second launch has room for: more than that take looks again.  (20 sentences of 20 rows, 40 slots: 26.8 us, with room for 1024 32.)
constexpr int kSelectFinal = 2048;
constexpr int kSelectLists = 1024;     // parts with such extensions it has room for
constexpr double kLn2 = 0.693147180559945309417232121458;
// log2 e in two parts: a one-part product is off by 1.3e-8 of itself in the same direction for every x, which shows in the sum
constexpr float kLog2eHi = 1.44269502162933349609375f;
constexpr float kLog2eLo = (float)(1.442695040888963407359924681 - 1.44269502162933349609375);

// 2^(x log2 e - m2)
__device__ __forceinline__ float exp2_above(float x, float m2)
{
    return __builtin_amdgcn_exp2f(fmaf(x, kLog2eLo, fmaf(x, kLog2eHi, -m2)));
}

template <int FMT> struct Chunk;       // 16 bytes of logits; loose_t: at any element's address
template <> struct Chunk<0> {
    static __device__ __forceinline__ float most(const uint4 &c)
    {
        return fmaxf(fmaxf(__uint_as_float(c.x), __uint_as_float(c.y)), fmaxf(__uint_as_float(c.z), __uint_as_float(c.w)));
    }
    static constexpr int N = 4;
    typedef float elem_t;
    typedef uint32_t loose_t __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ float get(const uint4 &c, int e) { return __uint_as_float(((const uint32_t *)&c)[e]); }
    static __device__ __forceinline__ float value(float x) { return x; }
    static constexpr uint32_t kNone = 0xFF800000u;
};
template <> struct Chunk<1> {
    static __device__ __forceinline__ float most(const uint4 &c)
    {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        const h2 m = __builtin_elementwise_max(__builtin_elementwise_max(__builtin_bit_cast(h2, c.x), __builtin_bit_cast(h2, c.y)),
                                               __builtin_elementwise_max(__builtin_bit_cast(h2, c.z), __builtin_bit_cast(h2, c.w)));
        return fmaxf((float)m[0], (float)m[1]);
    }
    static constexpr int N = 8;
    typedef uint16_t elem_t;
    typedef uint32_t loose_t __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ float get(const uint4 &c, int e)
    {
        const uint32_t w = ((const uint32_t *)&c)[e >> 1];
        const uint16_t h = (uint16_t)((e & 1) ? w >> 16 : w);
        return (float)__builtin_bit_cast(_Float16, h);
    }
    static __device__ __forceinline__ float value(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
    static constexpr uint32_t kNone = 0xFC00u;
};
template <> struct Chunk<2> {
    // The greatest pair of halves, read as a float, has the greatest upper half: the lower one only decides between equals.  (An
    // infinity over a lower half that is not 0 reads as NaN and is passed over: -inf is no extension, +inf shows in the sum.)
    static __device__ __forceinline__ float most(const uint4 &c)
    {
        const float up = fmaxf(fmaxf(__uint_as_float(c.x), __uint_as_float(c.y)), fmaxf(__uint_as_float(c.z), __uint_as_float(c.w)));
        const float low = fmaxf(fmaxf(__uint_as_float(c.x << 16), __uint_as_float(c.y << 16)), fmaxf(__uint_as_float(c.z << 16), __uint_as_float(c.w << 16)));
        return fmaxf(__uint_as_float(__float_as_uint(up) & 0xFFFF0000u), low);
    }
    static constexpr int N = 8;
    typedef uint16_t elem_t;
    typedef uint32_t loose_t __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ float get(const uint4 &c, int e)
    {
        const uint32_t w = ((const uint32_t *)&c)[e >> 1];
        return __uint_as_float((e & 1) ? w & 0xFFFF0000u : w << 16);
    }
    static __device__ __forceinline__ float value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    static constexpr uint32_t kNone = 0xFF80u;
};

// Sums and maxima over a wave without a trip through LDS.
template <int J>
__device__ __forceinline__ double add_lane_xor(double v)
{
    return v + __longlong_as_double((long long)xor_lane_t<u64, J, true>((u64)__double_as_longlong(v)));
}
__device__ __forceinline__ double wave_sum_double(double v)
{
    return add_lane_xor<32>(add_lane_xor<16>(add_lane_xor<8>(add_lane_xor<4>(add_lane_xor<2>(add_lane_xor<1>(v))))));
}

// A place in a list for every lane of the wave that asks for one: one atomic a wave (lanes' own would be taken one after the other).
__device__ __forceinline__ int place_of_lane(u64 asking, int first)
{
    return first + __builtin_amdgcn_mbcnt_hi((uint32_t)(asking >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)asking, 0));
}
__device__ __forceinline__ int places_for_wave(int n, int *count)
{
    int first = 0;
    if (lane_id() == 0) first = atomicAdd(count, n);
    return __builtin_amdgcn_readfirstlane(first);
}

// Sum of `v` over the workgroup, in every thread.  `room`: one int per wave; ends with a barrier.
template <int THREADS>
__device__ __forceinline__ int block_sum(int v, int *room)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    if (lane_id() == 0) room[threadIdx.x / kWave] = v;
    __syncthreads();
    int s = 0;
    for (int w = 0; w < THREADS / kWave; ++w) s += room[w];
    __syncthreads();
    return s;
}

// A bound that at least k of the wave's J * 64 keys reach (0 = no key), and rarely more than k + k/4 + 4: bisection that stops there.  0 if there
// are fewer than k.  `most`: the greatest key.
template <int J>
__device__ __forceinline__ uint32_t bound_of_kth(const uint32_t (&r)[J], int k, uint32_t most)
{
    auto reached = [&](uint32_t x) {
        int c = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) c += (int)__popcll(__ballot(r[j] >= x));
        return c;
    };
    int count = reached(1u);
    if (count < k) return 0;
    uint32_t least = 0;                                // of the keys there are
#pragma unroll
    for (int j = 0; j < J; ++j) least = max(least, r[j] ? ~r[j] : 0u);
    uint32_t lo = ~wave_max_uniform(least), hi = most;
    while (count > k + (k >> 2) + 4 && lo < hi) {
        const uint32_t mid = lo + ((hi - lo + 1) >> 1);
        const int c = reached(mid);
        if (c >= k) {
            lo = mid;
            count = c;
        } else {
            hi = mid - 1;
        }
    }
    return lo;
}

// One part of one row.  Bound: HBM (the logits are read once), and with 16 bits the VALU nearly: an element takes five
// instructions, one of them the exponential.  So nothing else is done element by element: addresses are the same for a whole wave
// but for its lanes' 16 bytes, the end of a row that does not fill a chunk are single elements of the first wave, and of the chunks only those that
// reach the bar are looked through (128 x 64 rows of 50000 in bf16, 86 % of which are read: 138 to 155 us from run to run, 5.1 to 4.6 TB/s;
// all of them: 148 to 168, 5.5 to 4.9; 64 x 20 of 32000 in fp32, 87 %: 25.4 us, 5.6 TB/s, all: 27.8, 5.9 TB/s).
template <int FMT>
__global__ __launch_bounds__(kSelectThreads, 8) void dba_select_part_kernel(const void *logits, SelectParams p)
{
    typedef Chunk<FMT> C;
    typedef typename C::elem_t elem_t;
    constexpr int T = kSelectThreads, R = kSelectChunks, N = C::N, NW = T / kWave;
    __shared__ uint32_t s_max[T];
    __shared__ double s_sum[NW];
    __shared__ int s_int[NW];
    __shared__ int s_count, s_queued;
    __shared__ uint32_t s_bar;
    __shared__ uint4 s_queue[kSelectQueue];
    __shared__ int s_queue_chunk[kSelectQueue];
    __shared__ u64 s_keys[kSelectKeys];
    const int t = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(t / kWave);
    const int part = (int)blockIdx.x, h = (int)blockIdx.y, b = (int)blockIdx.z;
    const int row = b * p.k_in + h;
    const size_t list = (size_t)row * p.nparts + part;
    SelectPart *out = p.parts + list;
    u64 *out_keys = p.keys + list * p.cap;
    const float score = p.score[row];
    const int flags = p.flags ? p.flags[row] : 0;
    if ((flags & (DBA_FLAG_FINISHED | DBA_FLAG_DEAD)) || !(fabsf(score) < INFINITY)) {
        // a completed hypothesis goes on with pad_id at its own score; the others offer nothing
        const bool goes_on = part == 0 && (flags & DBA_FLAG_FINISHED) && !(flags & DBA_FLAG_DEAD) && fabsf(score) < INFINITY;
        if (t == 0) {
            if (goes_on) out_keys[0] = make_key(0.0f, (uint32_t)p.pad);
            *out = SelectPart{0.0, 0.0f, goes_on ? 1 : 0};
        }
        return;
    }
    const elem_t *src = static_cast<const elem_t *>(logits) + ((int64_t)b * p.sent_stride + (int64_t)h * p.row_stride);
    // Chunks are counted from the row's start, wherever it lies in memory, so that rows that are alike are summed alike and their extensions are equal.
    // (Of 16-byte loads only those at odd multiples of two bytes cost more: 128 x 64 rows of 50001 in bf16 171 us, by a 16-byte grid of memory, which
    // sums rows of other offsets in other groups, 152; 64 x 20 of 32001 in fp32 35 either way.)  The elements behind the last whole chunk are taken one by one, by the
    // first N threads of the part they lie in.
    typedef typename C::loose_t loose_t;
    const loose_t *chunks = reinterpret_cast<const loose_t *>(src);
    auto chunk_at = [](const loose_t *at) { const loose_t v = *at; return make_uint4(v.x, v.y, v.z, v.w); };
    const int whole = p.V / N;
    const int c0 = part * p.part_chunks, c1 = min(c0 + p.part_chunks, whole);
    auto wave_chunk = [&](int r) { return c0 + wave * kWave + r * T; };
    auto has_round = [&](int r) { return wave_chunk(r) < c1; };       // the same for the whole wave
    auto none = [] { const uint32_t w = N == 4 ? C::kNone : C::kNone | (C::kNone << 16); return make_uint4(w, w, w, w); };
    auto load_round = [&](int r) {                     // what is not a whole chunk of this part is -inf
        const int cw = wave_chunk(r);
        const loose_t *from = chunks + cw;
        if (cw + kWave <= c1) return chunk_at(from + (uint32_t)lane);
        uint4 v = none();
        if (cw + lane < c1) v = chunk_at(from + (uint32_t)lane);
        return v;
    };
    uint4 raw[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (has_round(r)) raw[r] = load_round(r);
    float edge = -INFINITY;                            // a single element
    const int edge_at = whole * N + t;
    if (t < N && c0 <= whole && whole - c0 < p.part_chunks && edge_at < p.V) edge = C::value(src[edge_at]);
    float top = edge, most_of[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        most_of[r] = has_round(r) ? C::most(raw[r]) : -INFINITY;
        top = fmaxf(top, most_of[r]);
    }
    s_max[t] = top > -INFINITY ? ord_from_float(top) : 0u;
    if (t == 0) s_count = s_queued = 0;
    __syncthreads();
    // k_out threads hold something that reaches the k_out-th greatest of the threads' maxima, or a bound a little below it: so does
    // everything that can be among the part's k_out greatest.  One wave finds the bound while the others go on with the sum.
    uint32_t r4[NW];
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
        r4[j] = s_max[j * kWave + lane];
        most = most > r4[j] ? most : r4[j];
    }
    most = wave_max_uniform(most);
    if (wave == ((part + h) & (NW - 1))) {
        const uint32_t at_least = bound_of_kth<NW>(r4, p.k_out, most);
        if (lane == 0) s_bar = at_least;
    }
    const float most_x = most ? float_from_ord(most) : 0.0f;
    // The sum: a few dozen terms a thread in fp32 (each is off by 1e-7 of itself, either way), the threads' in 64 bits.  The reference is
    // the rounded product itself, so that no error of its own comes in.  What that rounding leaves, though, grows with the logits: at a mask's -1e10 every
    // term is 2^247.  So from 2^20 on, where it is still 0.1, logits are subtracted first, which is exact wherever a term is not 0.
    const float m2 = most_x * kLog2eHi;
    const bool huge = !(fabsf(most_x) < 0x1p20f);
    float part_sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (!huge) {
        part_sum[0] = exp2_above(edge, m2);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (has_round(r)) {
#pragma unroll
                for (int e = 0; e < N; ++e) part_sum[e & 3] += exp2_above(C::get(raw[r], e), m2);
            }
    } else {
        auto term = [&](float x) { return exp2_above(x - most_x, 0.0f); };
        part_sum[0] = term(edge);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (has_round(r)) {
#pragma unroll
                for (int e = 0; e < N; ++e) part_sum[e & 3] += term(C::get(raw[r], e));
            }
    }
    const float sum = (part_sum[0] + part_sum[1]) + (part_sum[2] + part_sum[3]);
    const double total = wave_sum_double((double)sum);
    if (lane == 0) s_sum[wave] = total;
    __syncthreads();
    // the few chunks that reach the bar go through LDS, where all threads share their elements out
    const float bar = s_bar ? float_from_ord(s_bar) : -3.402823466e38f;     // (-inf and NaN reach no bar)
    int hits = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) hits += (int)__popcll(__ballot(most_of[r] >= bar));
    if (hits) {
        int at = places_for_wave(hits, &s_queued);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const u64 in = __ballot(most_of[r] >= bar);
            const int mine = place_of_lane(in, at);
            if (most_of[r] >= bar && mine < kSelectQueue) {
                s_queue[mine] = raw[r];
                s_queue_chunk[mine] = wave_chunk(r) + lane;
            }
            at += (int)__popcll(in);
        }
    }
    auto put = [&](bool wanted, float x, int at) {
        const u64 in = __ballot(wanted);
        if (!in) return;
        const int mine = place_of_lane(in, places_for_wave((int)__popcll(in), &s_count));
        if (wanted && mine < kSelectKeys) s_keys[mine] = make_key(x, (uint32_t)at);
    };
    if (wave == 0) put(edge >= bar, edge, edge_at);
    __syncthreads();
    const int queued = s_queued;
    if (queued <= kSelectQueue) {
        typedef elem_t __attribute__((may_alias)) elem_of_chunk;
        const elem_of_chunk *elems = reinterpret_cast<const elem_of_chunk *>(s_queue);
        for (int i0 = wave * kWave; i0 < queued * N; i0 += T) {
            const int i = i0 + lane;
            const bool is = i < queued * N;
            const float x = is ? C::value(elems[i]) : -INFINITY;
            put(x >= bar, x, is ? s_queue_chunk[i / N] * N + i % N : 0);
        }
    }
    __syncthreads();
    int count = s_count;
    if (queued <= kSelectQueue && count > p.cap && count <= kSelectKeys) {
        // short rows, or the best next to each other: the first wave hands on those from a bound that at least k_out and at most
        // cap of the keys reach (they all differ)
        if (wave == 0) {
            constexpr int J = kSelectKeys / kWave;
            u64 key[J];
#pragma unroll
            for (int j = 0; j < J; ++j) key[j] = j * kWave + lane < count ? s_keys[j * kWave + lane] : 0;
            u64 lo = 1, hi = ~0ull;
            int n = count;
            while (n > p.cap && lo < hi) {
                const u64 mid = lo + ((hi - lo) >> 1) + 1;
                int c = 0;
#pragma unroll
                for (int j = 0; j < J; ++j) c += (int)__popcll(__ballot(key[j] >= mid));
                if (c >= p.k_out) {
                    lo = mid;
                    n = c;
                } else {
                    hi = mid - 1;
                }
            }
            int at = 0;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const u64 in = __ballot(key[j] >= lo && key[j]);
                if ((in >> lane) & 1) out_keys[place_of_lane(in, at)] = key[j];
                at += (int)__popcll(in);
            }
            if (lane == 0) s_int[0] = at;              // (not s_count: other waves may not have read it yet)
        }
        __syncthreads();
        count = s_int[0];
    } else if (count > p.cap || queued > kSelectQueue) {
        // a great many equal logits: exactly k_out, by bisection on the keys
        auto each = [&](auto f) {
            if (edge >= bar) f(make_key(edge, (uint32_t)edge_at));
#pragma unroll 1
            for (int r = 0; r < R && has_round(r); ++r) {
                const uint4 again = load_round(r);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float x = C::get(again, e);
                    if (x >= bar) f(make_key(x, (uint32_t)((wave_chunk(r) + lane) * N + e)));
                }
            }
        };
        u64 lo = 1, hi = ~0ull;
        while (lo < hi) {
            const u64 mid = lo + ((hi - lo) >> 1) + 1;
            int n = 0;
            each([&](u64 key) { n += key >= mid; });
            n = block_sum<T>(n, s_int);
            if (n >= p.k_out) lo = mid;
            else hi = mid - 1;
            if (n == p.k_out) break;
        }
        if (t == 0) s_count = 0;
        __syncthreads();
        each([&](u64 key) {
            if (key >= lo) {
                const int at = atomicAdd(&s_count, 1);
                if (at < p.cap) s_keys[at] = key;
            }
        });
        __syncthreads();
        count = min(s_count, p.cap);
        for (int i = t; i < count; i += T) out_keys[i] = s_keys[i];
    } else {
        for (int i = t; i < count; i += T) out_keys[i] = s_keys[i];
    }
    if (t == 0) {
        double s = 0.0;
        for (int w = 0; w < NW; ++w) s += s_sum[w];
        // relative to the part's greatest logit, not to its rounded product
        *out = SelectPart{huge ? log(s) : log(s) + ((double)m2 * kLn2 - (double)most_x), most_x, count};
    }
}

__device__ __forceinline__ u64 ord_from_double(double s)
{
    const u64 u = (u64)__double_as_longlong(s + 0.0);
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

__device__ __forceinline__ double double_from_ord(u64 o)
{
    return __longlong_as_double((long long)((o >> 63) ? (o & 0x7FFFFFFFFFFFFFFFull) : ~o));
}

// One sentence: normalisers, then the k_out best of what its rows' parts have handed on.  Bound: latency, a chain of loads and barriers through
// code that no other launch has left in the instruction cache (4.7 us for 5 lists, 9.1 for 80, 18.5 for 192 with k_out = 64).
template <int T>
__global__ __launch_bounds__(T) void dba_select_sentence_kernel(SelectParams p)
{
    constexpr int NW = T / kWave;
    __shared__ double s_base[DBA_MAX_BEAM];       // score - log sum exp(x - top); NaN where the row offers nothing
    __shared__ float s_top[DBA_MAX_BEAM];
    __shared__ int s_done[DBA_MAX_BEAM];
    __shared__ uint32_t s_max[T];
    __shared__ int s_int[NW];
    __shared__ int s_count, s_lists;
    __shared__ SelectPart s_part[T];
    __shared__ double s_term[T];
    __shared__ uint32_t s_list[kSelectLists];
    __shared__ u64 s_ord[2 * kSelectFinal];
    __shared__ uint32_t s_flat[2 * kSelectFinal];
    const int t = (int)threadIdx.x, b = (int)blockIdx.x, wave = t / kWave;
    const int lists = p.k_in * p.nparts;
    const SelectPart *parts = p.parts + (size_t)b * lists;
    const u64 *keys = p.keys + (size_t)b * lists * p.cap;
    // what the parts have left behind: in LDS where a thread can take one part, which saves two trips to memory
    const bool held = lists <= T;
    if (held && t < lists) s_part[t] = parts[t];
    const int row_flags = t < p.k_in && p.flags ? p.flags[b * p.k_in + t] : 0;
    const float row_score = t < p.k_in ? p.score[b * p.k_in + t] : 0.0f;
    __syncthreads();
    auto part_of = [&](int i) { return held ? s_part[i] : parts[i]; };
    // of a row's parts, the exponential of each relative to the row's greatest logit: a part a thread where they are held
    auto top_of_row = [&](int h) {
        float most = -INFINITY;
        for (int i = 0; i < p.nparts; ++i) {
            const SelectPart q = part_of(h * p.nparts + i);
            if (q.log_sum != -INFINITY) most = fmaxf(most, q.top);
        }
        return most;
    };
    auto term_of = [&](int i, float most) {
        const SelectPart q = part_of(i);
        return q.log_sum != -INFINITY ? exp(q.log_sum + ((double)q.top - (double)most)) : 0.0;
    };
    if (held && p.nparts > 1) {
        if (t < lists) s_term[t] = term_of(t, top_of_row(t / p.nparts));
        __syncthreads();
    }
    if (t < p.k_in) {
        double base = (double)row_score;
        float most = 0.0f;
        if (!(row_flags & DBA_FLAG_FINISHED)) {
            double log_sum = part_of(t * p.nparts).log_sum;
            most = part_of(t * p.nparts).top;
            if (p.nparts > 1) {
                most = top_of_row(t);
                double sum = 0.0;
                for (int i = t * p.nparts; i < (t + 1) * p.nparts; ++i) sum += held ? s_term[i] : term_of(i, most);
                log_sum = log(sum);
            }
            base -= log_sum;
        }
        s_top[t] = most;
        s_done[t] = row_flags & DBA_FLAG_FINISHED;
        s_base[t] = fabs(base) < INFINITY ? base : __longlong_as_double(0x7FF8000000000000ll);
    }
    if (t == 0) s_count = s_lists = 0;
    __syncthreads();
    auto score_of = [&](int h, float x) { return s_base[h] + ((double)x - (double)s_top[h]); };
    auto best_of = [&](int list) -> uint32_t {    // of a list: the image of its greatest score, 0 if it has none
        const SelectPart q = part_of(list);
        if (!q.count) return 0;
        const double s = score_of(list / p.nparts, q.top);
        return s == s ? ord_from_float((float)s) : 0u;
    };
    // The k_out-th greatest of the lists' best scores is reached by k_out extensions: lists whose best does not reach it are not looked at.
    auto kth = [&](uint32_t mine, int n) {         // n: threads from there on have nothing
        s_max[t] = mine;
        __syncthreads();
        auto of = [&](auto &r) {
            uint32_t most = 0;
            constexpr int J = sizeof(r) / sizeof(r[0]);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                r[j] = s_max[j * kWave + lane_id()];
                most = max(most, r[j]);
            }
            return bound_of_kth<J>(r, p.k_out, wave_max_uniform(most));
        };
        uint32_t r4[4], r[NW];
        return NW == 4 || n <= 4 * kWave ? of(r4) : of(r);
    };
    uint32_t top = 0;
    for (int i = t; i < lists; i += T) top = max(top, best_of(i));
    uint32_t bar = kth(top, lists);
    for (int i = t; i < lists; i += T) {
        const uint32_t best = best_of(i);
        if (best && best >= bar) {
            const int at = atomicAdd(&s_lists, 1);
            if (at < kSelectLists) s_list[at] = (uint32_t)i;
        }
    }
    __syncthreads();
    const int active = s_lists;
    // every extension of the lists that count: f(score, coordinate); 64 keys a wave at a time, U such loads under way (the first time
    // eight; where a sentence needs more looks, one, as the code of this kernel comes through the instruction cache in every launch)
    auto each_by = [&](auto under_way, auto f) {
        constexpr int U = decltype(under_way)::value;
        const int pieces = (p.cap + kWave - 1) / kWave, n = (active <= kSelectLists ? active : lists) * pieces;
        for (int i0 = wave; i0 < n; i0 += U * NW) {
            u64 key[U];
            int row[U];
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int i = i0 + x * NW, piece = pieces == 2 ? i & 1 : 0;
                key[x] = 0;
                row[x] = 0;
                if (i >= n) continue;                  // (the same for the whole wave)
                const int at = pieces == 2 ? i >> 1 : i, list = active <= kSelectLists ? (int)s_list[at] : at;
                const int j = piece * kWave + lane_id();
                row[x] = list / p.nparts;
                if (j < part_of(list).count) key[x] = keys[(size_t)list * p.cap + j];
            }
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const double s = score_of(row[x], float_from_ord((uint32_t)(key[x] >> 32)));
                if (key[x] && s == s) f(s, (uint32_t)row[x] * (uint32_t)p.V + key_flat(key[x]));
            }
        }
    };
    auto each = [&](auto f) { each_by(std::integral_constant<int, 1>{}, f); };
    auto put = [&](u64 ord, uint32_t flat, int from) {
        const int at = atomicAdd(&s_count, 1);
        if (at < kSelectFinal) {
            s_ord[from + at] = ord;
            s_flat[from + at] = flat;
        }
    };
    each_by(std::integral_constant<int, 8>{}, [&](double s, uint32_t flat) {
        if (ord_from_float((float)s) >= bar) put(ord_from_double(s), flat, 0);
    });
    __syncthreads();
    int count = s_count, from = 0;
    if (count > kSelectFinal) {
        // hardly more lists than slots: a better bound, from the threads' greatest
        top = 0;
        each([&](double s, uint32_t) { top = max(top, ord_from_float((float)s)); });
        bar = max(bar, kth(top, T));
        if (t == 0) s_count = 0;
        __syncthreads();
        each([&](double s, uint32_t flat) {
            if (ord_from_float((float)s) >= bar) put(ord_from_double(s), flat, 0);
        });
        __syncthreads();
        count = s_count;
        __syncthreads();                           // (read by all before it is set again)
    }
    if (count > kSelectFinal) {
        // the k_out-th greatest score by bisection, then of its equals the first coordinates
        u64 lo = 0, hi = ~0ull;
        while (lo < hi) {
            const u64 mid = lo + ((hi - lo) >> 1) + 1;
            int n = 0;
            each([&](double s, uint32_t) { n += ord_from_double(s) >= mid; });
            n = block_sum<T>(n, s_int);
            if (n >= p.k_out) lo = mid;
            else hi = mid - 1;
        }
        int more = 0;
        each([&](double s, uint32_t) { more += ord_from_double(s) > lo; });
        more = block_sum<T>(more, s_int);
        uint32_t first = 0, last = ~0u;            // the least coordinate up to which enough of the equals lie
        while (first < last) {
            const uint32_t mid = first + ((last - first) >> 1);
            int n = 0;
            each([&](double s, uint32_t flat) { n += ord_from_double(s) == lo && flat <= mid; });
            n = block_sum<T>(n, s_int);
            if (n >= p.k_out - more) last = mid;
            else first = mid + 1;
        }
        if (t == 0) s_count = 0;
        __syncthreads();
        each([&](double s, uint32_t flat) {
            const u64 o = ord_from_double(s);
            if (o > lo || (o == lo && flat <= last)) put(o, flat, 0);
        });
        __syncthreads();
        count = min(s_count, kSelectFinal);
    } else if (count > p.k_out + 16) {
        // fewer to rank: those that reach the k_out-th greatest of the threads' maxima
        top = 0;
        for (int i = t; i < count; i += T) top = max(top, (uint32_t)(s_ord[i] >> 32));
        bar = kth(top, count);
        if (t == 0) s_count = 0;
        __syncthreads();
        for (int i = t; i < count; i += T)
            if ((uint32_t)(s_ord[i] >> 32) >= bar) put(s_ord[i], s_flat[i], kSelectFinal);
        __syncthreads();
        count = s_count;
        from = kSelectFinal;
    }
    int32_t *token = p.out_token + (size_t)b * p.k_out, *back = p.out_backptr + (size_t)b * p.k_out;
    float *score = p.out_score + (size_t)b * p.k_out;
    uint8_t *flags = p.out_flags + (size_t)b * p.k_out;
    // sixteen threads count what goes before an extension
    for (int i = t / 16; i < (count + 3) / 4 * 4; i += T / 16) {       // (whole waves: the lanes of one exchange below)
        const bool is = i < count;
        const u64 o = is ? s_ord[from + i] : 0;
        const uint32_t f = is ? s_flat[from + i] : 0;
        int rank = 0;
        for (int j = t & 15; j < count; j += 16) rank += s_ord[from + j] > o || (s_ord[from + j] == o && s_flat[from + j] < f);
#pragma unroll
        for (int d = 8; d; d >>= 1) rank += __shfl_xor(rank, d);
        if (!is || (t & 15) || rank >= p.k_out) continue;
        const int h = (int)(f / (uint32_t)p.V), w = (int)(f - (uint32_t)h * (uint32_t)p.V);
        token[rank] = w;
        back[rank] = h;
        score[rank] = (float)double_from_ord(o);
        flags[rank] = w == p.eos || s_done[h] ? DBA_FLAG_FINISHED : 0;
    }
    for (int i = count + t; i < p.k_out; i += T) {
        token[i] = p.pad;
        back[i] = -1;
        score[i] = -INFINITY;
        flags[i] = DBA_FLAG_DEAD;
    }
}

}  // namespace dba
