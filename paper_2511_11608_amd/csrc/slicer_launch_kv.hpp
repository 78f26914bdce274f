// Launchers of the cache's kernels, instantiated by element type (a translation unit each) and by head size rounded up to 32.
#pragma once

#include <algorithm>

#include "slicer_kv_attend.hpp"
#include "slicer_kv_cache.hpp"

namespace slicer {

// Workgroups of an append or a read: blocks of a sequence, and the (sequence, head) pairs over the other two dimensions.
inline dim3 kv_grid(int64_t blocks, int64_t pairs)
{
    const int64_t y = std::min<int64_t>(pairs, 32768);
    return dim3((unsigned)blocks, (unsigned)y, (unsigned)((pairs + y - 1) / y));
}

// Head sizes up to this one have registers for 32 rows at a time; larger ones (fp32 queries) would spill.
constexpr int kWideTile = 160;

struct KvAttendLaunch {
    int tile_rows;            // rows of a tile of the sequences that are split: 16 or 32
    int split_tiles;          // their tiles
    int row_blocks, page_blocks;
    int prompt_tiles;         // row tiles of the other sequences; 0: no sequence can have that many rows
    int prompt_slots;         // workgroups that keep weights on the way
    int mass_blocks;          // workgroups a head that add up weights; 0: no weights
};

template <int DT> hipError_t launch_kv_append(const KvAppendArgs& a, int64_t blocks, hipStream_t st);
template <int DT> hipError_t launch_kv_read(const KvReadArgs& a, int64_t blocks, hipStream_t st);
template <int DT> hipError_t launch_kv_attend(const KvAttendArgs& a, const KvAttendLaunch& p, hipStream_t st);

#ifdef SLICER_KV_INSTANTIATE

template <typename F>
inline void kv_by_size(int dp, F f)
{
    switch (dp) {
        case 32: f(std::integral_constant<int, 32>()); break;
        case 64: f(std::integral_constant<int, 64>()); break;
        case 96: f(std::integral_constant<int, 96>()); break;
        case 128: f(std::integral_constant<int, 128>()); break;
        case 160: f(std::integral_constant<int, 160>()); break;
        case 192: f(std::integral_constant<int, 192>()); break;
        case 224: f(std::integral_constant<int, 224>()); break;
        default: f(std::integral_constant<int, 256>()); break;
    }
}

template <int DT>
hipError_t launch_kv_append(const KvAppendArgs& a, int64_t blocks, hipStream_t st)
{
    kv_by_size(a.kv.dp, [&](auto dp) {
        hipLaunchKernelGGL((kv_append_kernel<DT, decltype(dp)::value>), kv_grid(blocks, (int64_t)a.kv.seqs * a.kv.G), dim3(256), 0, st, a);
    });
    return hipGetLastError();
}

template <int DT>
hipError_t launch_kv_read(const KvReadArgs& a, int64_t blocks, hipStream_t st)
{
    kv_by_size(a.kv.dp, [&](auto dp) {
        hipLaunchKernelGGL((kv_read_kernel<DT, decltype(dp)::value>), kv_grid(2 * blocks, (int64_t)a.kv.seqs * a.kv.G), dim3(256), 0, st, a);
    });
    return hipGetLastError();
}

template <int DT>
hipError_t launch_kv_attend(const KvAttendArgs& a, const KvAttendLaunch& p, hipStream_t st)
{
    const unsigned pairs = (unsigned)(a.kv.seqs * a.kv.G);
    kv_by_size(a.kv.dp, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        if (p.split_tiles) {
            const dim3 grid(pairs * (unsigned)(p.split_tiles * a.splits));
            if (p.tile_rows == 16) hipLaunchKernelGGL((kv_split_kernel<DT, DP, 1>), grid, dim3(256), 0, st, a);
            else if constexpr (DP <= kWideTile) hipLaunchKernelGGL((kv_split_kernel<DT, DP, 2>), grid, dim3(256), 0, st, a);
            if (p.row_blocks + p.page_blocks)
                hipLaunchKernelGGL((kv_join_kernel<DT, DP>), dim3(pairs * (unsigned)(p.row_blocks + p.page_blocks)), dim3(256), 0, st, a, p.row_blocks, p.page_blocks, p.tile_rows);
        }
        if (p.prompt_tiles) {
            const unsigned tiles = pairs * (unsigned)(p.prompt_tiles * a.prompt_splits);
            hipLaunchKernelGGL((kv_prompt_kernel<DT, DP>), dim3(p.mass_blocks ? std::min(tiles, (unsigned)p.prompt_slots) : tiles), dim3(256), 0, st, a, p.prompt_tiles);
            if (a.prompt_splits > 1)
                hipLaunchKernelGGL((kv_prompt_join_kernel<DT, DP>), dim3(pairs * (unsigned)(p.prompt_tiles * kTileRows / 4)), dim3(256), 0, st, a, p.prompt_tiles);
            if (p.mass_blocks) hipLaunchKernelGGL((kv_mass_kernel<DT>), dim3(pairs * (unsigned)p.mass_blocks), dim3(256), 0, st, a, p.prompt_tiles, p.mass_blocks);
        }
    });
    return hipGetLastError();
}

#endif

}  // namespace slicer
