// Shrinking the attention cache: the pages with the least accumulated weight leave it (gfx950, wave64).
//
// Complete pages of a sequence that stay: the first `sink`, the last `recent`, and the heaviest of the others up to `keep` in all, equal weights by the
// lower place.  A page's weight is the sum over the heads in fp64, in their order, so that its rank is that of the exact sum (fp32 sums would
// rank near-equal pages by their rounding).  The last key that stays is found digit by digit from the highest bit in which keys differ; one ordered pass then
// closes the gaps.  Source and destination may be the same arrays: whatever is written was read before, and nothing moves up.
// Bound by latency: tables of up to 1024 pages take one launch, a page a thread; longer ones four, of which only the cut has one workgroup a sequence (1 x 16384 pages of 8
// heads: keys 2.6, cut 19, places 5, moves 6.6 us).  The places in the cut's workgroup too: 40 us a call against 34, 1 x 40000 pages 93 against 71, but 256 x 1100 35 against
// 37; in every head's move: 46; all in one workgroup 110.
#pragma once

#include "slicer_kv.hpp"

namespace slicer {

constexpr int kEvictSmall = 1024;         // pages
constexpr int kEvictRun = 16;             // pages a thread at a time

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
    u64* keys;                    // workspace, longer tables: [seqs][max_pages], then
    struct EvictCut* cuts;        // [seqs]
    uint2* counts;                // [seqs][chunks] keys above the cut and equal to it among kEvictSmall pages from `lo`
    int32_t* from;                // [seqs][max_pages] the place that a place's entry comes from, -1: none
    int chunks;
};

// Order-preserving key of a sum of weights; NaN above everything.
__device__ inline u64 weight_key(double w)
{
    const u64 u = (u64)__double_as_longlong(w);
    if (w != w) return ~0ull;
    return u >> 63 ? ~u : u | 1ull << 63;
}

struct KvEvictRange { int len, full, lo, hi; u32 need; };      // lo .. hi - 1: pages that may go, of which `need` stay

__device__ inline KvEvictRange evict_range(const KvEvictArgs& a, int b)
{
    KvEvictRange r;
    const int64_t l = a.lens[b];
    r.len = (int)(l < 0 ? 0 : l > (int64_t)a.max_pages * kPage ? (int64_t)a.max_pages * kPage : l);
    r.full = r.len / kPage;
    const bool over = r.full > a.keep;
    r.lo = over ? a.sink : 0;
    r.hi = over ? r.full - a.recent : 0;
    r.need = over ? (u32)(a.keep - a.sink - a.recent) : 0;
    return r;
}

__device__ inline u64 evict_key(const KvEvictArgs& a, int b, int p)
{
    const float* m = a.mass + (int64_t)b * a.G * a.max_pages + p;
    double w = 0.0;
#pragma unroll 8
    for (int g = 0; g < a.G; ++g) w += (double)m[(int64_t)g * a.max_pages];
    return weight_key(w);
}

struct EvictCut { u64 prefix, mask; u32 left; };               // keys above prefix under the mask stay, and the first `left` equal to it

// The cut among the keys that `each` hands to its argument.  LDS: hist 2048 words, ext 2 x BLOCK / 64 of u64, scan BLOCK / 64 + 1, sel 3.
template <int BLOCK, typename F>
__device__ inline EvictCut evict_cut(u32 need, F each, u32* hist, u64* ext, u32* scan, u32* sel)
{
    constexpr int RB = 11, NW = BLOCK / kWave;
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    EvictCut cut = {0, 0, need};
    u64 some = 0, all = ~0ull;                                 // bits set in any key, in every key
    each([&](u64 k) { some |= k; all &= k; });
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        some |= __shfl_xor(some, o);
        all &= __shfl_xor(all, o);
    }
    if (lane == 0) { ext[wid] = some; ext[NW + wid] = all; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) { some |= ext[w]; all &= ext[NW + w]; }
    const u64 differ = some & ~all;
    int top = differ ? 64 - __clzll((long long)differ) : 0;                     // bits from `top` on are the same in all keys,
    const int low = differ ? __ffsll((long long)differ) - 1 : 0;               // and so are those below `low`
    cut.mask = top >= 64 ? 0 : ~0ull << top;
    cut.prefix = all & cut.mask;
    while (top > low) {
        const int shift = top > RB ? top - RB : 0, bits = top - shift;
        for (int i = tid; i < 1 << RB; i += BLOCK) hist[i] = 0;
        __syncthreads();
        each([&](u64 k) {
            if ((k & cut.mask) != cut.prefix) return;
            // one addition for all lanes whose key falls where the first one's does: equal weights are many
            const u32 bin = (u32)(k >> shift) & ((1u << bits) - 1), first = (u32)__builtin_amdgcn_readfirstlane((int)bin);
            const u64 with = __ballot(bin == first);
            if (bin != first) atomicAdd(&hist[bin], 1u);
            else if (mask_rank(with) == 0) atomicAdd(&hist[bin], (u32)__popcll(with));
        });
        __syncthreads();
        constexpr int PB = (1 << RB) / BLOCK;                  // bins a thread, from the top
        u32 h[PB], sum = 0, total;
#pragma unroll
        for (int j = 0; j < PB; ++j) {
            h[j] = hist[(1 << RB) - 1 - tid * PB - j];
            sum += h[j];
        }
        u32 before = block_excl_scan<BLOCK>(sum, scan, &total);
#pragma unroll
        for (int j = 0; j < PB; ++j) {
            if (before < cut.left && cut.left <= before + h[j]) { sel[0] = (u32)((1 << RB) - 1 - tid * PB - j); sel[1] = cut.left - before; sel[2] = h[j]; }
            before += h[j];
        }
        __syncthreads();
        cut.prefix |= (u64)sel[0] << shift;
        cut.mask = shift ? ~0ull << shift : ~0ull;
        cut.left = sel[1];
        const bool done = sel[2] == cut.left;                  // the whole bin stays
        __syncthreads();
        if (done) break;
        top = shift;
    }
    return cut;
}

__device__ inline bool evict_stays(const EvictCut& cut, u32 need, u64 k, u32 equals_before)
{
    k &= cut.mask;
    return need && (k > cut.prefix || (k == cut.prefix && equals_before < cut.left));
}

// Up to 1024 pages: a page a thread.  Up to 256 a thread counts the keys that come before its own (256 x 66 pages: 8 us, 11 with the cut).
template <int BLOCK>
__global__ __launch_bounds__(BLOCK) void kv_evict_small_kernel(KvEvictArgs a)
{
    constexpr bool COUNT = BLOCK <= 256;
    __shared__ u64 keys[COUNT ? BLOCK : 1];
    __shared__ u32 hist[COUNT ? 1 : 2048];
    __shared__ u64 ext[2 * BLOCK / kWave];
    __shared__ u32 scan[BLOCK / kWave + 1];
    __shared__ u32 sel[3];
    const int b = blockIdx.x, p = threadIdx.x, P = a.max_pages;
    const int64_t row = (int64_t)b * P;
    const KvEvictRange r = evict_range(a, b);
    const bool candidate = p >= r.lo && p < r.hi;
    const u64 key = candidate && r.need ? evict_key(a, b, p) : 0;
    const int id = p < P ? a.table[row + p] : -1;
    bool stays = p < P && !candidate;
    u32 n;
    if constexpr (COUNT) {
        keys[p] = key;
        __syncthreads();
        u32 rank = 0;
        for (int i = r.lo; i < r.hi; ++i) rank += keys[i] > key || (keys[i] == key && i < p);
        if (candidate) stays = rank < r.need;
    } else {
        EvictCut cut = {0, 0, 0};
        if (r.need) cut = evict_cut<BLOCK>(r.need, [&](auto use) { if (candidate) use(key); }, hist, ext, scan, sel);
        const u32 equals = block_excl_scan<BLOCK>(candidate && (key & cut.mask) == cut.prefix, scan, &n);
        if (candidate) stays = evict_stays(cut, r.need, key, equals);
    }
    const u32 before = block_excl_scan<BLOCK>(p < P && !stays, scan, &n);
    const int to = p - (int)before;
    if (stays) a.out_table[row + to] = id;
    else if (p < P) a.freed[row + before] = id;
    if (p < P && p >= P - (int)n) a.out_table[row + p] = -1;
    if (p < P && p >= (int)n) a.freed[row + p] = -1;
    if (p == 0) {
        a.out_lens[b] = r.len - kPage * (int)n;
        a.n_freed[b] = (int)n;
    }
    for (int g = 0; g < a.G; g += 4) {                         // four heads at a time
        float m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = p < P && g + i < a.G ? a.mass[(row * a.G) + (int64_t)(g + i) * P + p] : 0.0f;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (g + i >= a.G || p >= P) continue;
            float* out = a.out_mass + row * a.G + (int64_t)(g + i) * P;
            if (stays) out[to] = m[i];
            if (p >= P - (int)n) out[p] = 0.0f;
        }
    }
}

static __global__ __launch_bounds__(256) void kv_evict_keys_kernel(KvEvictArgs a, int blocks)
{
    const int b = blockIdx.x / blocks, p = blockIdx.x % blocks * 256 + threadIdx.x;
    const KvEvictRange r = evict_range(a, b);
    if (r.need && p >= r.lo && p < r.hi) a.keys[(int64_t)b * a.max_pages + p] = evict_key(a, b, p);
}

// The cut of one sequence, and how many keys are above and equal in each kEvictSmall pages of the range.
static __global__ __launch_bounds__(1024) void kv_evict_cut_kernel(KvEvictArgs a)
{
    constexpr int BLOCK = kEvictSmall, E = kEvictRun;
    __shared__ u32 hist[2048];
    __shared__ u64 ext[2 * BLOCK / kWave];
    __shared__ u32 scan[BLOCK / kWave + 1];
    __shared__ u32 sel[3];
    __shared__ u32 count[2 * E];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const KvEvictRange r = evict_range(a, b);
    const u64* keys = a.keys + (int64_t)b * a.max_pages;
    EvictCut cut = {0, 0, 0};
    if (r.need) {
        // sixteen keys a thread; they stay in registers where that is all of them
        u64 k[E];
        auto load = [&](int base) {
#pragma unroll
            for (int e = 0; e < E; ++e) k[e] = base + e * BLOCK + tid < r.hi ? keys[base + e * BLOCK + tid] : 0;
        };
        const bool once = r.hi - r.lo <= BLOCK * E;
        if (once) load(r.lo);
        cut = evict_cut<BLOCK>(r.need, [&](auto use) {
            for (int base = r.lo; base < r.hi; base += BLOCK * E) {
                if (!once) load(base);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (base + e * BLOCK + tid < r.hi) use(k[e]);
            }
        }, hist, ext, scan, sel);
        uint2* counts = a.counts + (int64_t)b * a.chunks;
        for (int base = r.lo; base < r.hi; base += BLOCK * E) {
            if (!once) load(base);
            if (tid < 2 * E) count[tid] = 0;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool in = base + e * BLOCK + tid < r.hi;
                const u64 above = __ballot(in && (k[e] & cut.mask) > cut.prefix), equal = __ballot(in && (k[e] & cut.mask) == cut.prefix);
                if (lane == 0 && above) atomicAdd(&count[2 * e], (u32)__popcll(above));
                if (lane == 0 && equal) atomicAdd(&count[2 * e + 1], (u32)__popcll(equal));
            }
            __syncthreads();
            if (tid < E && base + tid * BLOCK < r.hi) counts[(base - r.lo) / BLOCK + tid] = make_uint2(count[2 * tid], count[2 * tid + 1]);
            __syncthreads();
        }
    }
    if (tid == 0) a.cuts[b] = cut;
}

// Where a sequence's entries come from and which pages go, kEvictSmall pages of the range a workgroup, which counts what stays before them; the entries outside
// the range are shared out.
static __global__ __launch_bounds__(1024) void kv_evict_places_kernel(KvEvictArgs a)
{
    constexpr int BLOCK = kEvictSmall;
    __shared__ u32 scan[BLOCK / kWave + 1];
    const int b = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x, P = a.max_pages;
    const int64_t row = (int64_t)b * P;
    const KvEvictRange r = evict_range(a, b);
    const EvictCut cut = a.cuts[b];
    const int gone = r.hi - r.lo - (int)r.need;
    const int first = r.lo + c * BLOCK, p = first + tid;
    if (first < r.hi) {                                         // (the same for all threads)
        u32 above = 0, equal = 0, n;
        if (r.need) {
            const uint2* counts = a.counts + (int64_t)b * a.chunks;
            u32 mine = 0, equals = 0;
            for (int i = tid; i < c; i += BLOCK) {
                mine += counts[i].x;
                equals += counts[i].y;
            }
            block_excl_scan<BLOCK>(mine, scan, &above);
            block_excl_scan<BLOCK>(equals, scan, &equal);
        }
        const u32 before = above + (equal < cut.left ? equal : cut.left);       // that stay
        const bool in = p < r.hi;
        const u64 key = r.need && in ? a.keys[row + p] : 0;
        const u32 equals = equal + block_excl_scan<BLOCK>(in && (key & cut.mask) == cut.prefix, scan, &n);
        const bool stays = in && evict_stays(cut, r.need, key, equals);
        const u32 rank = before + block_excl_scan<BLOCK>(stays, scan, &n);
        if (stays) a.from[row + r.lo + rank] = p;
        else if (in) a.freed[row + p - r.lo - rank] = a.table[row + p];
    }
    for (int q = c * BLOCK + tid; q < P; q += a.chunks * BLOCK) {
        if (q < r.lo) a.from[row + q] = q;
        else if (q >= r.hi) a.from[row + q - gone] = q;
        if (q >= P - gone) a.from[row + q] = -1;
        if (q >= gone) a.freed[row + q] = -1;
    }
    if (c == 0 && tid == 0) a.n_freed[b] = gone;
}

// Of one sequence the weights of a head, or the table: 16384 places at a time are read before they are written, since source and destination may be the same.
static __global__ __launch_bounds__(1024) void kv_evict_move_kernel(KvEvictArgs a)
{
    constexpr int BLOCK = 1024, E = kEvictRun;
    const int b = blockIdx.x / (a.G + 1), g = blockIdx.x % (a.G + 1), P = a.max_pages;
    const int64_t row = (int64_t)b * P;
    const bool table = g == a.G;
    const int32_t* from = a.from + row;
    const u32* in = table ? (const u32*)a.table + row : (const u32*)a.mass + row * a.G + (int64_t)g * P;
    u32* out = table ? (u32*)a.out_table + row : (u32*)a.out_mass + row * a.G + (int64_t)g * P;
    const u32 none = table ? (u32)-1 : 0;                       // the bits of -1 and of 0.0f
    for (int base = 0; base < P; base += BLOCK * E) {
        u32 m[E];
        int at[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int p = base + e * BLOCK + threadIdx.x;
            at[e] = p < P ? from[p] : -1;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) m[e] = at[e] >= 0 ? in[at[e]] : none;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int p = base + e * BLOCK + threadIdx.x;
            if (p < P) out[p] = m[e];
        }
        __syncthreads();
    }
    if (table && threadIdx.x == 0) {
        const KvEvictRange r = evict_range(a, b);
        a.out_lens[b] = r.len - kPage * (r.hi - r.lo - (int)r.need);
    }
}

}  // namespace slicer
