// Launches of the attention kernels of one format; each format is a source file of its own, which compile side by side.
#pragma once
#include "entry.hpp"
#include "tree_attend.hpp"

namespace dba {

template <int FMT, int DP, int QT, bool ROWS, int SIDE>
hipError_t attend_one(const AttendParams &p, hipStream_t stream)
{
    constexpr int lds = AttendShape<FMT, DP, QT, ROWS>::LDS;
    static_assert(lds + 4 * 16 * QT * 8 + 256 <= 160 * 1024, "LDS of a compute unit");
    if constexpr (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&dba_attend_kernel<FMT, DP, QT, ROWS, SIDE>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    const unsigned blocks = ((unsigned)p.groups + 7) / 8 * 8 * (unsigned)p.row_tiles, wide = blocks < 65536 ? blocks : 65536;
    return launch(dba_attend_kernel<FMT, DP, QT, ROWS, SIDE>, dim3(wide, (blocks + wide - 1) / wide), dim3(256), lds, stream, p);
}

template <int FMT, int DP, int QT>
hipError_t attend_tiles(const AttendParams &p, const AttendPlan &plan, hipStream_t stream)
{
    return plan.side == 2 ? attend_one<FMT, DP, QT, false, 2>(p, stream) : attend_one<FMT, DP, QT, false, 1>(p, stream);
}

template <int FMT, int DP>
hipError_t attend_rows(const AttendParams &p, const AttendPlan &plan, hipStream_t stream)
{
    if (plan.shared) return attend_one<FMT, DP, (DP <= 128 ? 2 : 1), true, 1>(p, stream);
    if constexpr (kAttendWidest<FMT, DP> >= 4)
        if (plan.QT == 4) return attend_tiles<FMT, DP, 4>(p, plan, stream);
    if constexpr (kAttendWidest<FMT, DP> >= 2)
        if (plan.QT == 2) return attend_tiles<FMT, DP, 2>(p, plan, stream);
    return attend_tiles<FMT, DP, 1>(p, plan, stream);
}

template <int FMT>
hipError_t attend_launch(const AttendParams &p, const AttendPlan &plan, int B, hipStream_t stream)
{
    const hipError_t e = plan.DP == 64 ? attend_rows<FMT, 64>(p, plan, stream)
                 : plan.DP == 128 ? attend_rows<FMT, 128>(p, plan, stream) : attend_rows<FMT, 256>(p, plan, stream);
    if (e != hipSuccess || p.splits == 1) return e;
    const int rows = p.n * (p.q_heads / p.heads), Q = (int64_t)B * p.heads * rows >= 16384 ? 4 : 1;
    return launch(Q == 4 ? dba_attend_join_kernel<FMT, 4> : dba_attend_join_kernel<FMT, 1>, dim3((unsigned)((rows + 4 * Q - 1) / (4 * Q)), (unsigned)p.heads, (unsigned)B),
                  dim3(256), 0, stream, p, plan.tile, __builtin_ctz((unsigned)plan.tile_rows));
}

}  // namespace dba
