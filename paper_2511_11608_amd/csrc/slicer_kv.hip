// C ABI of the attention cache in 8 bits (see include/slicer.h): argument checks, workspace carving and launches.
#include "../../include/slicer.h"

#include <hip/hip_runtime.h>
#include <algorithm>
#include <cmath>

#include "slicer_launch.hpp"
#include "slicer_launch_kv.hpp"
#include "slicer_kv_evict.hpp"

using namespace slicer;

namespace {

int round32(int d) { return (d + 31) / 32 * 32; }

int check_kv(const slicer_kv* kv)
{
    if (!kv || kv->seqs < 1 || kv->kv_heads < 1 || kv->max_pages < 1 || kv->max_pages > 1 << 24) return SLICER_EINVAL;
    if (kv->n_pages < 1 || kv->n_pages >= (int64_t)1 << 31) return SLICER_EINVAL;
    if ((int64_t)kv->seqs * kv->kv_heads >= (int64_t)1 << 22) return SLICER_EINVAL;
    if (kv->head_dim < 8 || kv->head_dim > 256 || kv->head_dim % 8) return SLICER_EINVAL;
    if (kv->n_pages > ((int64_t)1 << 62) / ((int64_t)kv->kv_heads * (2 * kPage * round32(kv->head_dim)))) return SLICER_EINVAL;       // bytes of the pages
    return SLICER_OK;
}

int check_call(const slicer_kv* kv, int dt, int64_t tokens, const int32_t* starts, int max_new)
{
    int rc = check_kv(kv);
    if (rc) return rc;
    if (dt != SLICER_F32 && dt != SLICER_BF16) return SLICER_EUNSUPPORTED;
    if (!kv->pages || !kv->scales || !kv->tails || !kv->page_table || !kv->lens) return SLICER_EINVAL;
    if (((uintptr_t)kv->pages | (uintptr_t)kv->scales | (uintptr_t)kv->tails) & 15) return SLICER_EINVAL;      // read 16 bytes at a time
    if (tokens < 0 || tokens >= (int64_t)1 << 31 || (tokens > 0 && (!starts || max_new < 1))) return SLICER_EINVAL;
    return SLICER_OK;
}

KvView view_of(const slicer_kv* kv)
{
    KvView v;
    v.pages = (uint8_t*)kv->pages;
    v.scales = kv->scales;
    v.tails = (uint16_t*)kv->tails;
    v.table = kv->page_table;
    v.lens = kv->lens;
    v.seqs = kv->seqs;
    v.G = kv->kv_heads;
    v.D = kv->head_dim;
    v.dp = round32(kv->head_dim);
    v.max_pages = kv->max_pages;
    v.n_pages = kv->n_pages;
    return v;
}

// whether every row of a strided tensor may be read 16 bytes at a time
bool wide_rows(const void* p, int dt, int64_t token, int64_t head)
{
    const int64_t e = dt == SLICER_F32 ? 4 : 8;
    return ((uintptr_t)p & 15) == 0 && token % e == 0 && head % e == 0;
}

// Blocks of 64 token places that a sequence's new tokens can touch; the kernels go round where a launch cannot have as many.
int64_t blocks_of(int64_t tokens, int max_new) { return std::min<int64_t>((std::min<int64_t>(tokens, max_new) + kPage - 2) / kPage + 1, 65536); }

// Workgroups of 256 threads in one dimension of a launch (which counts threads in 32 bits).
constexpr int64_t kMaxGroups = (int64_t)1 << 24;

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

struct AttendPlan {
    int splits, rows_pad, few_rows, prompt_splits, slot_pages;
    KvAttendLaunch launch;
    size_t off_part_ml, off_part_o, off_page_w, off_prompt_ml, off_prompt_o, off_row_total, off_row_w, off_tile_mass, total;
};

AttendPlan plan_attend(const slicer_kv* kv, int heads, int64_t tokens, int max_new, int64_t max_len, bool mass)
{
    AttendPlan p;
    const int64_t pairs = (int64_t)kv->seqs * kv->kv_heads, R = heads / kv->kv_heads;
    const int64_t rows = std::min<int64_t>(std::min<int64_t>(tokens, max_new) * R, (int64_t)1 << 31);
    const int64_t pages = std::min<int64_t>(kv->max_pages, (std::max<int64_t>(max_len, 1) + kPage - 1) / kPage);
    const int64_t dp = round32(kv->head_dim);
    // Where all sequences bring as many tokens, and more rows than are split, nothing is left to the kernels of the split rows (and should a sequence
    // have fewer after all, the others take it).
    const bool even = rows > kSplitRows && tokens == (int64_t)kv->seqs * max_new;
    p.few_rows = even ? 0 : kSplitRows;
    p.rows_pad = even ? 0 : (int)std::min<int64_t>(rows, kSplitRows);
    p.launch.tile_rows = p.rows_pad > 16 && dp <= kWideTile ? 32 : 16;
    p.launch.split_tiles = (p.rows_pad + p.launch.tile_rows - 1) / p.launch.tile_rows;
    const int64_t tiles = pairs * std::max(p.launch.split_tiles, 1);
    // The cache is shared out while that gives no more than a workgroup a CU, and no further than a page for each of its four wavefronts.  Up to two a CU balance no better and
    // leave more starts and more parts to join.  us for the append and the attention of a step, at most 256 workgroups and at least 512: 20 x 2000..2100 tokens, 8 heads of 256,
    // fp32 74 and 105; 40 x 2000..2100, 8 of 160 70 and 81; 24 x 3000..5000, 8 of 64 29 and 32; 1 x 30000, 8 of 128 24 and 27; 2 x 262016 195 and 195.  At most 128: 2 x 262016 230.
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(256 / tiles, (pages + 3) / 4));
    // Unsplit sequences that leave at least three eighths of the CUs of their one or two rounds empty (129 to 160 and 257 to 320 tiles; from three rounds on the last one's empty CUs are too
    // small a part for the rule, and nothing was measured there) are split in three where a wavefront still has eight pages of each share: 17 x 9000..12000 tokens, 8 heads of 128
    // 90 us, unsplit 101, 33 x 9000..12000 160 and 181, fp32 33 x 4600..6200, 8 of 256 193 and 240; shorter ones lose (33 x 2250..3000 63 and 60), and so do fuller rounds
    // (24 x 9000..12000 127 and 115).
    if (tiles > 128 && tiles * 8 <= (tiles + 255) / 256 * 256 * 5 && pages >= 96) p.splits = 3;
    p.launch.row_blocks = p.splits > 1 ? p.rows_pad : 0;
    p.launch.page_blocks = p.rows_pad && mass && (p.splits > 1 || p.rows_pad > 16 || kv->max_pages > kMassPages) ? (int)((pages + 255) / 256) : 0;
    p.launch.prompt_tiles = rows > kSplitRows ? (int)((rows + kTileRows - 1) / kTileRows) : 0;
    // Row tiles that do not fill the chip share their pages out, four at least to a workgroup (4 x 256..513 queries of 8 heads of 64 behind 3000 to 6000 tokens 103 -> 58 us a
    // step; 1 x 1700 queries with no cache before them, where half of the tiles are short, 41 -> 46).
    const int64_t ptiles = pairs * std::max(p.launch.prompt_tiles, 1);
    p.prompt_splits = ptiles < 256 ? (int)std::max<int64_t>(1, std::min<int64_t>(512 / ptiles, pages / 4)) : 1;
    p.launch.mass_blocks = mass && p.launch.prompt_tiles ? (int)((pages + (p.prompt_splits > 1 ? 3 : 255)) / (p.prompt_splits > 1 ? 4 : 256)) : 0;
    // Workgroups that have 1 KB a page each to keep a tile's weights in: all of them where pages are shared out; else at most 512, and 256 where 512 took
    // more than 2 GB.
    p.slot_pages = (kv->max_pages + p.prompt_splits - 1) / p.prompt_splits;
    const size_t slot = (size_t)p.slot_pages * kTileRows * sizeof(float2);
    const int64_t groups = ptiles * p.prompt_splits;
    p.launch.prompt_slots = !p.launch.mass_blocks ? 0 : (int)(p.prompt_splits > 1 ? groups : std::min<int64_t>(groups, slot * 512 <= (size_t)2 << 30 ? 512 : 256));
    size_t o = 0;
    const size_t slots = (size_t)pairs * p.rows_pad * p.splits, rows_all = p.launch.prompt_tiles && p.prompt_splits > 1 ? (size_t)ptiles * kTileRows : 0;
    p.off_part_ml = o; o += align256(slots * sizeof(float2));
    p.off_part_o = o; o += align256(p.splits > 1 ? slots * dp * sizeof(float) : 0);
    p.off_page_w = o; o += align256(mass ? (size_t)pairs * kv->max_pages * p.rows_pad * sizeof(float2) : 0);
    p.off_prompt_ml = o; o += align256(rows_all * p.prompt_splits * sizeof(float2));
    p.off_prompt_o = o; o += align256(rows_all * p.prompt_splits * dp * sizeof(float));
    p.off_row_total = o; o += align256(mass ? rows_all * sizeof(float2) : 0);
    p.off_row_w = o; o += align256(slot * p.launch.prompt_slots);
    p.off_tile_mass = o; o += align256(p.launch.mass_blocks && p.prompt_splits == 1 ? (size_t)ptiles * kv->max_pages * sizeof(float) : 0);
    p.total = o;
    return p;
}

int fail(hipError_t e) { return e == hipSuccess ? SLICER_OK : note_hip_error(e); }

}  // namespace

extern "C" {

int slicer_kv_sizes(const slicer_kv* kv, size_t* pages_bytes, size_t* scales_bytes, size_t* tails_bytes)
{
    int rc = check_kv(kv);
    if (rc) return rc;
    const size_t dp = (size_t)round32(kv->head_dim), heads = (size_t)kv->kv_heads;
    if (pages_bytes) *pages_bytes = (size_t)kv->n_pages * heads * 2 * kPage * dp;
    if (scales_bytes) *scales_bytes = (size_t)kv->n_pages * heads * 2 * sizeof(float);
    if (tails_bytes) *tails_bytes = (size_t)kv->seqs * heads * 2 * kPage * dp * sizeof(uint16_t);
    return SLICER_OK;
}

int slicer_kv_append(const slicer_kv* kv, const void* k, const void* v, slicer_dtype dt, int64_t tokens, const int32_t* starts, int max_new,
                     int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, void* hip_stream)
{
    int rc = check_call(kv, (int)dt, tokens, starts, max_new);
    if (rc) return rc;
    if (tokens == 0) return SLICER_OK;
    if (!k || !v) return SLICER_EINVAL;
    KvAppendArgs a;
    a.kv = view_of(kv);
    a.k = k;
    a.v = v;
    a.k_token = k_token;
    a.k_head = k_head;
    a.v_token = v_token;
    a.v_head = v_head;
    a.starts = starts;
    a.tokens = tokens;
    a.wide = wide_rows(k, (int)dt, k_token, k_head) && wide_rows(v, (int)dt, v_token, v_head);
    const int64_t blocks = blocks_of(tokens, max_new);
    return fail(dt == SLICER_F32 ? launch_kv_append<0>(a, blocks, (hipStream_t)hip_stream) : launch_kv_append<1>(a, blocks, (hipStream_t)hip_stream));
}

int slicer_kv_attend_sizes(const slicer_kv* kv, int heads, int64_t tokens, int max_new, int64_t max_len, int with_mass, size_t* workspace_bytes)
{
    int rc = check_kv(kv);
    if (rc) return rc;
    if (heads < 1 || heads % kv->kv_heads || tokens < 0 || tokens >= (int64_t)1 << 31 || (tokens > 0 && max_new < 1) || max_len < 0) return SLICER_EINVAL;
    if (workspace_bytes) *workspace_bytes = tokens ? plan_attend(kv, heads, tokens, max_new, max_len, with_mass != 0).total : 0;
    return SLICER_OK;
}

int slicer_kv_attend(const slicer_kv* kv, const void* q, slicer_dtype dt, int heads, int64_t tokens, const int32_t* starts, int max_new,
                     int64_t max_len, int64_t q_token, int64_t q_head, double scale, int causal, void* out, float* lse, float* mass, double mass_decay,
                     void* workspace, void* hip_stream)
{
    int rc = check_call(kv, (int)dt, tokens, starts, max_new);
    if (rc) return rc;
    const float scale2 = (float)(std::fabs(scale) * 1.44269504088896340736);           // of scores that are exponents of 2
    if (heads < 1 || heads % kv->kv_heads || !std::isfinite(scale2) || !(mass_decay >= 0.0 && mass_decay <= 1.0) || max_len < 0) return SLICER_EINVAL;
    if (tokens == 0) return SLICER_OK;
    if (!q || !out || (((uintptr_t)out | (uintptr_t)workspace) & 15)) return SLICER_EINVAL;
    const AttendPlan p = plan_attend(kv, heads, tokens, max_new, max_len, mass != nullptr);
    if (p.total && !workspace) return SLICER_EINVAL;
    const int64_t pairs = (int64_t)kv->seqs * kv->kv_heads;
    for (int64_t n : {(int64_t)p.launch.split_tiles * p.splits, (int64_t)p.launch.row_blocks + p.launch.page_blocks, (int64_t)p.launch.prompt_tiles * (p.prompt_splits > 1 ? kTileRows : 1), (int64_t)p.launch.mass_blocks})
        if (pairs * n >= kMaxGroups) return SLICER_EINVAL;        // more workgroups than a launch can have
    KvAttendArgs a;
    a.kv = view_of(kv);
    a.q = q;
    a.q_token = q_token;
    a.q_head = q_head;
    a.starts = starts;
    a.tokens = tokens;
    a.R = heads / kv->kv_heads;
    a.H = heads;
    a.max_new = max_new;
    a.causal = causal != 0;
    a.scale = scale2;
    a.flip = scale < 0.0;
    a.out = out;
    a.lse = lse;
    a.mass = mass;
    a.decay = (float)mass_decay;
    a.wide_q = wide_rows(q, (int)dt, q_token, q_head);
    a.splits = p.splits;
    a.rows_pad = p.rows_pad;
    uint8_t* ws = (uint8_t*)workspace;
    a.part_ml = (float2*)(ws + p.off_part_ml);
    a.part_o = (float*)(ws + p.off_part_o);
    a.page_w = (float2*)(ws + p.off_page_w);
    a.few_rows = p.few_rows;
    a.prompt_splits = p.prompt_splits;
    a.slot_pages = p.slot_pages;
    a.prompt_ml = (float2*)(ws + p.off_prompt_ml);
    a.prompt_o = (float*)(ws + p.off_prompt_o);
    a.row_total = (float2*)(ws + p.off_row_total);
    a.row_w = (float2*)(ws + p.off_row_w);
    a.tile_mass = (float*)(ws + p.off_tile_mass);
    return fail(dt == SLICER_F32 ? launch_kv_attend<0>(a, p.launch, (hipStream_t)hip_stream) : launch_kv_attend<1>(a, p.launch, (hipStream_t)hip_stream));
}

int slicer_kv_read(const slicer_kv* kv, void* k, void* v, slicer_dtype dt, int64_t tokens, const int32_t* starts, int max_new, void* hip_stream)
{
    int rc = check_call(kv, (int)dt, tokens, starts, max_new);
    if (rc) return rc;
    if (tokens == 0) return SLICER_OK;
    if (!k || !v) return SLICER_EINVAL;
    KvReadArgs a;
    a.kv = view_of(kv);
    a.k = k;
    a.v = v;
    a.starts = starts;
    a.tokens = tokens;
    a.wide = (((uintptr_t)k | (uintptr_t)v) & 15) == 0;
    const int64_t blocks = blocks_of(tokens, max_new);
    return fail(dt == SLICER_F32 ? launch_kv_read<0>(a, blocks, (hipStream_t)hip_stream) : launch_kv_read<1>(a, blocks, (hipStream_t)hip_stream));
}

int slicer_kv_evict(const slicer_kv* kv, const float* mass, int keep_pages, int sink_pages, int recent_pages, int32_t* page_table_out, int32_t* lens_out,
                    float* mass_out, int32_t* freed, int32_t* n_freed, void* workspace, void* hip_stream)
{
    int rc = check_kv(kv);
    if (rc) return rc;
    if (!kv->page_table || !kv->lens || !mass || !page_table_out || !lens_out || !mass_out || !freed || !n_freed || !workspace || ((uintptr_t)workspace & 15)) return SLICER_EINVAL;
    if (keep_pages < 0 || sink_pages < 0 || recent_pages < 0 || (int64_t)sink_pages + recent_pages > keep_pages) return SLICER_EINVAL;
    KvEvictArgs a;
    a.table = kv->page_table;
    a.lens = kv->lens;
    a.mass = mass;
    a.seqs = kv->seqs;
    a.G = kv->kv_heads;
    a.max_pages = kv->max_pages;
    a.keep = keep_pages;
    a.sink = sink_pages;
    a.recent = recent_pages;
    a.out_table = page_table_out;
    a.out_lens = lens_out;
    a.out_mass = mass_out;
    a.freed = freed;
    a.n_freed = n_freed;
    a.keys = (u64*)workspace;
    a.chunks = (kv->max_pages + kEvictSmall - 1) / kEvictSmall;
    a.cuts = (EvictCut*)(a.keys + (size_t)kv->seqs * kv->max_pages);
    a.counts = (uint2*)(a.cuts + kv->seqs);
    a.from = (int32_t*)(a.counts + (size_t)kv->seqs * a.chunks);
    hipStream_t st = (hipStream_t)hip_stream;
    const dim3 seqs((unsigned)kv->seqs);
    if (kv->max_pages <= 256) {
        hipLaunchKernelGGL(kv_evict_small_kernel<256>, seqs, dim3(256), 0, st, a);
    } else if (kv->max_pages <= kEvictSmall) {
        hipLaunchKernelGGL(kv_evict_small_kernel<kEvictSmall>, seqs, dim3(kEvictSmall), 0, st, a);
    } else {
        const int64_t blocks = (kv->max_pages + 255) / 256;
        if (std::max<int64_t>(a.chunks, kv->kv_heads + 1) * kv->seqs >= kMaxGroups / 4) return SLICER_EINVAL;      // workgroups of 1024 threads; blocks <= 4 * chunks
        hipLaunchKernelGGL(kv_evict_keys_kernel, dim3((unsigned)(blocks * kv->seqs)), dim3(256), 0, st, a, (int)blocks);
        hipLaunchKernelGGL(kv_evict_cut_kernel, seqs, dim3(1024), 0, st, a);
        hipLaunchKernelGGL(kv_evict_places_kernel, dim3((unsigned)(a.chunks * kv->seqs)), dim3(kEvictSmall), 0, st, a);
        hipLaunchKernelGGL(kv_evict_move_kernel, dim3((unsigned)(kv->seqs * (kv->kv_heads + 1))), dim3(1024), 0, st, a);
    }
    return fail(hipGetLastError());
}

}  // extern "C"
