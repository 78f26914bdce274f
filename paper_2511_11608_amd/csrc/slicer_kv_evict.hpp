// Shrinking the attention cache: the pages with the least accumulated weight leave it (gfx950, wave64).
#pragma once

#include "slicer_kv.hpp"

namespace slicer {

struct KvEvictArgs {
    const int32_t* table;
    const int32_t* lens;
    const float* mass;            // [seqs][heads][max_pages]
    int seqs, G, max_pages;
    int keep, sink, recent;
    int32_t* out_table;
    int32_t* out_lens;
    float* out_mass;
    int32_t* freed;
    int32_t* n_freed;
    u64* keys;                    // workspace: [seqs][max_pages]
};

// Order-preserving key of a sum of weights; NaN above everything.
__device__ inline u64 weight_key(double w)
{
    const u64 u = (u64)__double_as_longlong(w);
    if (w != w) return ~0ull;
    return u >> 63 ? ~u : u | 1ull << 63;
}

// Which complete pages of a sequence stay: the first `sink`, the last `recent`, and the heaviest of the others up to `keep` in all, equal
// weights by the lower place.  A page's weight is the sum over the heads in fp64, in their order, so that its rank is that of the exact sum
// (fp32 sums would rank near-equal pages by their rounding).  One workgroup a sequence: the keys once, then a most-significant-digit-first
// selection of the last key that stays, and one ordered pass that closes the gaps.  Source and destination may be the same arrays: a chunk of pages is
// read before it is written, and nothing moves up.
__global__ __launch_bounds__(1024) void kv_evict_kernel(KvEvictArgs a)
{
    constexpr int BLOCK = 1024, RB = 8;
    __shared__ u32 hist[1 << RB];
    __shared__ u32 scan[BLOCK / kWave + 1];
    __shared__ u32 sel[3];
    const int b = blockIdx.x, tid = threadIdx.x;
    const int64_t row = (int64_t)b * a.max_pages;
    const float* mass = a.mass + row * a.G;
    float* out_mass = a.out_mass + row * a.G;
    int len = a.lens[b];
    len = len < 0 ? 0 : len > (int64_t)a.max_pages * kPage ? a.max_pages * kPage : len;
    const int full = len / kPage, P = a.max_pages;
    const int lo = full > a.keep ? a.sink : 0, hi = full > a.keep ? full - a.recent : 0;       // candidates
    u32 need = full > a.keep ? (u32)(a.keep - a.sink - a.recent) : 0;
    u64* keys = a.keys + row;
    for (int p = lo + tid; p < hi; p += BLOCK) {
        double w = 0.0;
        for (int g = 0; g < a.G; ++g) w += (double)mass[(int64_t)g * P + p];
        keys[p] = weight_key(w);
    }
    __syncthreads();
    // the smallest key that stays, and how many of the keys equal to it
    u64 prefix = 0, mask = 0;
    u32 left = need;
    if (need) {
        for (int shift = 64 - RB; shift >= 0; shift -= RB) {
            for (int i = tid; i < 1 << RB; i += BLOCK) hist[i] = 0;
            __syncthreads();
            for (int p = lo + tid; p < hi; p += BLOCK) {
                const u64 k = keys[p];
                if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << RB) - 1)], 1u);
            }
            __syncthreads();
            if (tid < kWave) {                                                  // from the top: 4 bins a lane
                const int top = (1 << RB) - 1 - tid * 4;
                u32 h[4], sum = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) { h[j] = hist[top - j]; sum += h[j]; }
                u32 before = wave_scan_dpp(sum) - sum;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (before < left && left <= before + h[j]) { sel[0] = (u32)(top - j); sel[1] = left - before; sel[2] = h[j]; }
                    before += h[j];
                }
            }
            __syncthreads();
            prefix |= (u64)sel[0] << shift;
            mask |= ((u64)((1u << RB) - 1)) << shift;
            left = sel[1];
            const bool done = sel[2] == left;                                   // the whole bin stays
            __syncthreads();
            if (done) break;
        }
    }
    // pages in their order: gone, or moved up by the number of those gone before them
    u32 gone_before = 0, equal_before = 0;
    for (int base = 0; base < P; base += BLOCK) {
        const int p = base + tid;
        const bool candidate = p >= lo && p < hi;
        u64 k = 0;
        if (candidate) k = keys[p] & mask;
        const bool equal = candidate && need && k == prefix;
        u32 n_equal, n_gone;
        const u32 e = block_excl_scan<BLOCK>(equal, scan, &n_equal) + equal_before;
        const bool stays = p < P && (!candidate || (need && (k > prefix || (equal && e < left))));
        const bool gone = p < P && !stays;
        const u32 before = block_excl_scan<BLOCK>(gone, scan, &n_gone) + gone_before;
        const int id = p < P ? a.table[row + p] : 0;
        __syncthreads();
        if (stays) a.out_table[row + p - before] = id;
        if (gone) a.freed[row + before] = id;
        for (int g = 0; g < a.G; ++g) {
            const float m = p < P ? mass[(int64_t)g * P + p] : 0.0f;
            __syncthreads();
            if (stays) out_mass[(int64_t)g * P + p - before] = m;
        }
        equal_before += n_equal;
        gone_before += n_gone;
        __syncthreads();
    }
    for (int p = tid; p < P; p += BLOCK) {
        if (p >= P - (int)gone_before) {
            a.out_table[row + p] = -1;
            for (int g = 0; g < a.G; ++g) out_mass[(int64_t)g * P + p] = 0.0f;
        }
        if (p >= (int)gone_before) a.freed[row + p] = -1;
    }
    if (tid == 0) {
        a.out_lens[b] = len - kPage * (int)gone_before;
        a.n_freed[b] = (int)gone_before;
    }
}

}  // namespace slicer
