// Decoder states follow the back-pointers: kernel.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dba {

constexpr int kReorderStates = 24;     // in one launch (their descriptions travel as a kernel argument)
constexpr int kReorderThreads = 256;

struct ReorderState {
    unsigned char *dst;
    const unsigned char *src;
    int64_t dst_sent, dst_row, dst_seg, src_sent, src_row, src_seg;
    uint32_t segs, per_seg;            // pieces, columns of a piece
    uint32_t col_bytes;                // 1, 2, 4, 8 or 16
    uint32_t first_block;              // of this state, in a sentence's blocks
};

struct ReorderParams {
    const int32_t *back;
    int k, n_states;
    ReorderState s[kReorderStates];
};

// A thread owns one column of a sentence's rows: it reads what every new row needs of it before it writes any, so dst may be
// src.  KB: the greatest k it has registers for.  Bound: HBM; a parent of several rows comes from the cache after its first read (12 tensors of
// 64 x 20 rows, 1.47 GB in and out: 294 us, 5.0 TB/s; torch's copy of as much reaches 5.2).
template <int KB, typename W>
__device__ __forceinline__ void reorder_column(const ReorderParams &p, const ReorderState &s, int b, uint32_t column)
{
    if (column >= s.segs * s.per_seg) return;
    const uint32_t seg = column / s.per_seg, in = column - seg * s.per_seg;
    const unsigned char *src = s.src + (b * s.src_sent + seg * s.src_seg + (int64_t)in * (int64_t)sizeof(W));
    unsigned char *dst = s.dst + (b * s.dst_sent + seg * s.dst_seg + (int64_t)in * (int64_t)sizeof(W));
    const int32_t *back = p.back + (int64_t)b * p.k;
    const bool in_place = s.src == s.dst;
    W v[KB];
#pragma unroll
    for (int h = 0; h < KB; ++h) {
        v[h] = W{};
        if (h < p.k) {
            const int from = back[h];
            if ((uint32_t)from < (uint32_t)p.k && !(in_place && from == h))
                v[h] = *reinterpret_cast<const W *>(src + from * s.src_row);
        }
    }
#pragma unroll
    for (int h = 0; h < KB; ++h)
        if (h < p.k && !(in_place && back[h] == h)) *reinterpret_cast<W *>(dst + h * s.dst_row) = v[h];
}

template <int KB>
__global__ __launch_bounds__(kReorderThreads) void dba_reorder_kernel(ReorderParams p)
{
    const int b = (int)blockIdx.y;
    const uint32_t block = blockIdx.x;
    int i = 0;
    while (i + 1 < p.n_states && block >= p.s[i + 1].first_block) ++i;
    const ReorderState &s = p.s[i];
    const uint32_t column = (block - s.first_block) * kReorderThreads + threadIdx.x;
    switch (s.col_bytes) {
        case 16: reorder_column<KB, uint4>(p, s, b, column); break;
        case 8: reorder_column<KB, uint2>(p, s, b, column); break;
        case 4: reorder_column<KB, uint32_t>(p, s, b, column); break;
        case 2: reorder_column<KB, uint16_t>(p, s, b, column); break;
        default: reorder_column<KB, uint8_t>(p, s, b, column); break;
    }
}

}  // namespace dba
