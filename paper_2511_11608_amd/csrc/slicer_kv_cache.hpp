// Writing and reading back the attention cache (gfx950, wave64).
#pragma once

#include "slicer_kv.hpp"

namespace slicer {

struct KvAppendArgs {
    KvView kv;
    const void *k, *v;
    int64_t k_token, k_head, v_token, v_head;     // strides in elements
    const int32_t* starts;
    int64_t tokens;
    int wide;                                     // rows may be read 16 bytes at a time
};

// New tokens into the cache.  Blocks of 64 token places, counted from the page that is open: a block that gets full becomes a
// page of codes (amax over the 64 x D values of a head, scale = amax / 127, code = rint(x * (127 / amax)), three single fp32
// operations), the last one that does not goes to the tail.  Where the first block reads the tail and the last one writes it, one workgroup makes
// both; a head's other blocks are made of new tokens alone.  Memory bound: 2 bytes read and 1 written an element; all of a thread's loads
// are under way before the first is used (14 200 tokens of 8 x 128, bf16, 87 MB: 21 us; one load after the other 37).
// A token with a value that is not finite in its key or value is held as a NaN key and a zero value in the tail, and takes part in its page as
// zeros under a NaN key scale: every query that sees the page (in the tail, the token) gets NaN, no other does.

// four bf16 values (two words) times `inv`, rounded to whole numbers (1.5 * 2^23 added: nearest, ties to even), their low bytes; |x| <= amax, so that
// the product stays within 127 of zero and no bound need be applied
__device__ inline u32 codes_of(u32 a, u32 b, float inv)
{
    const float y0 = __uint_as_float(a << 16) * inv + 12582912.0f, y1 = __uint_as_float(a & 0xFFFF0000u) * inv + 12582912.0f;
    const float y2 = __uint_as_float(b << 16) * inv + 12582912.0f, y3 = __uint_as_float(b & 0xFFFF0000u) * inv + 12582912.0f;
    const u32 lo = __builtin_amdgcn_perm(__float_as_uint(y1), __float_as_uint(y0), 0x0C0C0400u), hi = __builtin_amdgcn_perm(__float_as_uint(y3), __float_as_uint(y2), 0x04000C0Cu);
    return lo | hi;
}

__device__ inline u32 max_magnitude(u32 m, uint4 w)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const u32 e = (&w.x)[j] & 0x7FFF7FFFu;
        m = max(m, max(e & 0xFFFFu, e >> 16));
    }
    return m;
}

template <int DT, int DP>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a)
{
    constexpr int LD = DP + 8;                    // elements of a staged row: rows start 4 banks apart
    constexpr int CPT = DP / 8, NCH = DP / 32;    // chunks of eight elements: of a token, of a thread
    __shared__ __align__(16) uint16_t x[2][kPage * LD];
    __shared__ u32 bad[kPage];
    __shared__ uint2 wave_max[4];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    const int bg = blockIdx.y + gridDim.y * blockIdx.z;
    if (bg >= a.kv.seqs * a.kv.G) return;
    const int b = bg / a.kv.G, g = bg % a.kv.G;
    const KvSeq s = kv_seq(a.kv, a.starts, a.tokens, b);
    const int n = s.n < s.len ? s.n : s.len;      // (a length below the number of new tokens holds the last of them)
    const int64_t first = s.first + (s.n - n);
    if (n == 0) return;
    const int D = a.kv.D, old = s.len - n, held = old & (kPage - 1), page0 = old / kPage;
    const int blocks = (held + n + kPage - 1) / kPage, whole = (held + n) / kPage;      // the last is blocks - 1: whole unless blocks > whole
    uint16_t* const tail_k = a.kv.tails + kv_tail(a.kv, b, g);
    uint16_t* const tail_v = tail_k + kPage * DP;

    // full blocks are dealt to the workgroups
    for (int p = blockIdx.x; p < whole; p += gridDim.x) {
        const int from_tail = p == 0 ? held : 0;
        const int64_t page = a.kv.table[(int64_t)b * a.kv.max_pages + page0 + p];        // (page0 + p < len / 64 <= max_pages)
        uint4 kk[NCH], vv[NCH], tv[NCH];
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int t = (i * 256 + tid) / CPT, d = (i * 256 + tid) % CPT * 8;
            kk[i] = vv[i] = tv[i] = uint4{0, 0, 0, 0};
            if (t >= from_tail) {
                if (d < D) {
                    const int64_t tok = first + (int64_t)p * kPage + t - held;
                    kk[i] = Row8<DT>::bf16(a.k, tok * a.k_token + g * a.k_head + d, a.wide);
                    vv[i] = Row8<DT>::bf16(a.v, tok * a.v_token + g * a.v_head + d, a.wide);
                }
            } else {
                kk[i] = *(const uint4*)(tail_k + t * DP + d);
            }
            if (from_tail) tv[i] = *(const uint4*)(tail_v + (i * 256 + tid) * 8);        // two elements of four tokens
        }
        u32 mk = 0, mv = 0;
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int t = (i * 256 + tid) / CPT, d = (i * 256 + tid) % CPT * 8;
            *(uint4*)&x[0][t * LD + d] = kk[i];
            mk = max_magnitude(mk, kk[i]);
            if (t >= from_tail) *(uint4*)&x[1][t * LD + d] = vv[i];
            mv = max_magnitude(mv, vv[i]);
            if (from_tail) {
                const int at = (i * 256 + tid) * 2, t0 = at / DP * 4, e0 = at % DP;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const u32 e = (&tv[i].x)[j >> 1] >> ((j & 1) * 16) & 0xFFFFu;
                    if (t0 + (j & 3) < from_tail) {
                        x[1][(t0 + (j & 3)) * LD + e0 + (j >> 2)] = (uint16_t)e;
                        mv = max(mv, e & 0x7FFFu);
                    }
                }
            }
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            mk = max(mk, (u32)__shfl_xor((int)mk, o));
            mv = max(mv, (u32)__shfl_xor((int)mv, o));
        }
        if (lane == 0) wave_max[wid] = uint2{mk, mv};
        __syncthreads();
        auto maxima = [&]() {
            mk = max(max(wave_max[0].x, wave_max[1].x), max(wave_max[2].x, wave_max[3].x));
            mv = max(max(wave_max[0].y, wave_max[1].y), max(wave_max[2].y, wave_max[3].y));
        };
        maxima();
        const bool any_bad = mk >= 0x7F80u || mv >= 0x7F80u;
        if (any_bad) {                            // rare: which tokens, zeros in their place, and the others' maxima
            __syncthreads();
            if (tid < kPage) bad[tid] = 0;
            __syncthreads();
            for (int i = tid; i < kPage * CPT; i += 256)
                if (max_magnitude(max_magnitude(0, *(const uint4*)&x[0][i / CPT * LD + i % CPT * 8]), *(const uint4*)&x[1][i / CPT * LD + i % CPT * 8]) >= 0x7F80u) bad[i / CPT] = 1;
            __syncthreads();
            mk = mv = 0;
            for (int i = tid; i < kPage * CPT; i += 256) {
                uint4 *const k8 = (uint4*)&x[0][i / CPT * LD + i % CPT * 8], *const v8 = (uint4*)&x[1][i / CPT * LD + i % CPT * 8];
                if (bad[i / CPT]) *k8 = *v8 = uint4{0, 0, 0, 0};
                mk = max_magnitude(mk, *k8);
                mv = max_magnitude(mv, *v8);
            }
#pragma unroll
            for (int o = 32; o; o >>= 1) {
                mk = max(mk, (u32)__shfl_xor((int)mk, o));
                mv = max(mv, (u32)__shfl_xor((int)mv, o));
            }
            if (lane == 0) wave_max[wid] = uint2{mk, mv};
            __syncthreads();
            maxima();
        }
        const float ak = __uint_as_float(mk << 16), av = __uint_as_float(mv << 16);
        const float ik = ak >= kKvTiny ? 127.0f / ak : 0.0f, iv = av >= kKvTiny ? 127.0f / av : 0.0f;
        if (page >= 0 && page < a.kv.n_pages) {
            uint8_t* const rec = a.kv.pages + kv_record(a.kv, page, g);
            if (tid == 0)
                *(float2*)(a.kv.scales + (page * a.kv.G + g) * 2) = float2{any_bad ? __uint_as_float(0x7FC00000u) : ak >= kKvTiny ? ak / 127.0f : 0.0f,
                                                                          av >= kKvTiny ? av / 127.0f : 0.0f};
#pragma unroll
            for (int q = 0; q < (4 * DP + 255) / 256; ++q) {                    // 16 bytes of keys: two tokens' eight elements
                const int i = q * 256 + tid, l = i & 63, st = i >> 6, T2 = st / (DP / 32), sl = st % (DP / 32);
                if (i >= 4 * DP) break;
                const uint16_t* from = &x[0][(T2 * 32 + (l & 15)) * LD + sl * 32 + (l >> 4) * 8];
                const uint4 w0 = *(const uint4*)from, w1 = *(const uint4*)(from + 16 * LD);
                *(uint4*)(rec + (size_t)i * 16) = uint4{codes_of(w0.x, w0.y, ik), codes_of(w0.z, w0.w, ik), codes_of(w1.x, w1.y, ik), codes_of(w1.z, w1.w, ik)};
            }
#pragma unroll
            for (int q = 0; q < (4 * DP + 255) / 256; ++q) {                    // 16 bytes of values: one element of sixteen tokens
                const int i = q * 256 + tid, l = i & 63;
                if (i >= 4 * DP) break;
                const uint16_t* from = &x[1][(l >> 4) * 4 * LD + (i >> 6) * 16 + (l & 15)];
                u32 r[4];
#pragma unroll
                for (int T = 0; T < 4; ++T) {
                    const uint16_t* f = from + T * 16 * LD;
                    r[T] = codes_of(f[0] | (u32)f[LD] << 16, f[2 * LD] | (u32)f[3 * LD] << 16, iv) ^ 0x80808080u;
                }
                *(uint4*)(rec + (size_t)kPage * DP + (size_t)i * 16) = uint4{r[0], r[1], r[2], r[3]};
            }
        }
        __syncthreads();
    }
    // what is left goes to the tail: behind the first block, by its workgroup, where that was made of it
    if (blocks == whole || blockIdx.x != (held && whole ? 0u : (unsigned)whole % gridDim.x)) return;
    const int from = whole == 0 ? held : 0, end = held + n - whole * kPage;
    if (tid < kPage) bad[tid] = 0;
    __syncthreads();
    for (int i = tid; i < (end - from) * CPT; i += 256) {
        const int t = from + i / CPT, d = i % CPT * 8;
        uint4 k8 = {0, 0, 0, 0}, v8 = {0, 0, 0, 0};
        if (d < D) {
            const int64_t tok = first + (int64_t)whole * kPage + t - held;
            k8 = Row8<DT>::bf16(a.k, tok * a.k_token + g * a.k_head + d, a.wide);
            v8 = Row8<DT>::bf16(a.v, tok * a.v_token + g * a.v_head + d, a.wide);
        }
        if (max_magnitude(max_magnitude(0, k8), v8) >= 0x7F80u) bad[t] = 1;
        *(uint4*)(tail_k + t * DP + d) = k8;
#pragma unroll
        for (int j = 0; j < 8; ++j) tail_v[((t >> 2) * DP + d + j) * 4 + (t & 3)] = (uint16_t)((&v8.x)[j >> 1] >> ((j & 1) * 16));
    }
    __syncthreads();
    for (int i = tid; i < (end - from) * CPT; i += 256) {        // (the same chunks: a thread overwrites what it wrote)
        const int t = from + i / CPT, d = i % CPT * 8;
        if (!bad[t]) continue;
        *(uint4*)(tail_k + t * DP + d) = uint4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) tail_v[((t >> 2) * DP + d + j) * 4 + (t & 3)] = 0;
    }
}

struct KvReadArgs {
    KvView kv;
    void *k, *v;                                  // [tokens][heads][D], contiguous
    const int32_t* starts;
    int64_t tokens;
    int wide;
};

// What the cache stands for, a sequence's first tokens: code * scale in fp32 and the tail's bf16, rounded to the output's type once.
// A record is read once, in its own order, and turned into rows through LDS; memory bound (14 200 tokens of 8 x 128, bf16, 87 MB: 17 us).
template <int DT, int DP>
__global__ __launch_bounds__(256) void kv_read_kernel(KvReadArgs a)
{
    typedef typename Elem<DT>::raw_t raw_t;
    constexpr int LD = DP + (DT == 0 ? 4 : 8), NR = (4 * DP + 255) / 256;
    __shared__ __align__(16) raw_t x[kPage * LD];
    const int tid = threadIdx.x, values = blockIdx.x & 1;       // keys and values by workgroups of their own
    const int bg = blockIdx.y + gridDim.y * blockIdx.z;
    if (bg >= a.kv.seqs * a.kv.G) return;
    const int b = bg / a.kv.G, g = bg % a.kv.G, D = a.kv.D;
    const KvSeq s = kv_seq(a.kv, a.starts, a.tokens, b);
    const int n = s.n < s.len ? s.n : s.len, full = s.len / kPage;
    auto raw = [](float f) -> raw_t {
        if constexpr (DT == 0) return __float_as_uint(f);
        else return (raw_t)Row8<0>::f32_to_bf16_any(f);
    };
    raw_t* const out = (raw_t*)(values ? a.v : a.k);
    for (int p = blockIdx.x >> 1; p * kPage < n; p += gridDim.x >> 1) {
        const int end = min(n - p * kPage, kPage);
        if (p < full) {
            int64_t page = a.kv.table[(int64_t)b * a.kv.max_pages + p];
            const bool there = page >= 0 && page < a.kv.n_pages;
            if (!there) page = 0;
            const uint8_t* rec = a.kv.pages + kv_record(a.kv, page, g) + (size_t)values * kPage * DP;
            uint4 r[NR];
#pragma unroll
            for (int q = 0; q < NR; ++q)
                if (q * 256 + tid < 4 * DP) r[q] = *(const uint4*)(rec + (size_t)(q * 256 + tid) * 16);
            const float sc = there ? a.kv.scales[(page * a.kv.G + g) * 2 + values] : __uint_as_float(0x7FC00000u);
#pragma unroll
            for (int q = 0; q < NR; ++q) {
                const int i = q * 256 + tid, l = i & 63, st = i >> 6;
                if (i >= 4 * DP) break;
                if (!values) {
                    raw_t* to = &x[(st / (DP / 32) * 32 + (l & 15)) * LD + st % (DP / 32) * 32 + (l >> 4) * 8];
#pragma unroll
                    for (int j = 0; j < 16; ++j) to[(j >> 3) * 16 * LD + (j & 7)] = raw((float)(int)(int8_t)((&r[q].x)[j >> 2] >> ((j & 3) * 8)) * sc);
                } else {
                    raw_t* to = &x[(l >> 4) * 4 * LD + st * 16 + (l & 15)];
#pragma unroll
                    for (int j = 0; j < 16; ++j) to[((j >> 2) * 16 + (j & 3)) * LD] = raw((float)((int)((&r[q].x)[j >> 2] >> ((j & 3) * 8) & 255u) - 128) * sc);
                }
            }
        } else {
            const uint16_t* tail = a.kv.tails + kv_tail(a.kv, b, g) + values * kPage * DP;
            for (int i = tid; i < end * DP; i += 256) {
                const int t = i / DP, d = i % DP;
                const u32 e = values ? tail[((t >> 2) * DP + d) * 4 + (t & 3)] : tail[i];
                x[t * LD + d] = DT == 0 ? (raw_t)(e << 16) : (raw_t)e;
            }
        }
        __syncthreads();
        constexpr int E = 16 / sizeof(raw_t);
        for (int i = tid; i < end * (DP / E); i += 256) {
            const int t = i / (DP / E), d = (i % (DP / E)) * E;
            if (d >= D) continue;
            raw_t* to = out + ((s.first + p * kPage + t) * a.kv.G + g) * D + d;
            if (a.wide) {
                *(uint4*)to = *(const uint4*)&x[t * LD + d];
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) to[j] = x[t * LD + d + j];      // (D is a multiple of 8)
            }
        }
        __syncthreads();
    }
}

}  // namespace slicer
