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
// operations), the last one that does not goes to the tail.  One workgroup makes both the first block, which reads the tail, and the last one, which
// writes it; a head's other blocks are made of new tokens alone.  Memory bound: 2 bytes read and 1 written an element.
// A token with a value that is not finite in its key or value is held as a NaN key and a zero value in the tail, and takes part in its page as
// zeros under a NaN key scale: every query that sees the page (in the tail, the token) gets NaN, no other does.
template <int DT, int DP>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a)
{
    constexpr int LD = DP + 8;                    // elements of a staged row: rows start 4 banks apart
    __shared__ __align__(16) uint16_t x[2][kPage * LD];
    __shared__ u32 bad[kPage];
    __shared__ u32 wave_max[2][4];
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

    // full blocks are dealt to the workgroups; the open one comes behind the first workgroup's
    for (int p = blockIdx.x;; p += gridDim.x) {
        const bool full = p < whole;
        if (!full) {
            if (blockIdx.x != 0 || blocks == whole) break;
            p = whole;
        }
        // places of this block that are taken from the tail and from the new tokens
        const int from_tail = p == 0 ? held : 0, end = full ? kPage : held + n - p * kPage;
        if (tid < kPage) bad[tid] = 0;
        __syncthreads();
        for (int i = tid; i < kPage * (DP / 8); i += 256) {
            const int t = i / (DP / 8), d = (i % (DP / 8)) * 8;
            uint4 kk = {0, 0, 0, 0}, vv = {0, 0, 0, 0};
            if (t >= from_tail && t < end && d < D) {
                const int64_t tok = first + (int64_t)p * kPage + t - held;
                kk = Row8<DT>::bf16(a.k, tok * a.k_token + g * a.k_head + d, a.wide);
                vv = Row8<DT>::bf16(a.v, tok * a.v_token + g * a.v_head + d, a.wide);
            } else if (full && t < from_tail) {
                kk = *(const uint4*)(tail_k + t * DP + d);
                uint16_t e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = tail_v[((t >> 2) * DP + d + j) * 4 + (t & 3)];
                __builtin_memcpy(&vv, e, 16);
            }
            *(uint4*)&x[0][t * LD + d] = kk;
            *(uint4*)&x[1][t * LD + d] = vv;
            u32 odd = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u32 wk = (&kk.x)[j], wv = (&vv.x)[j];
                odd |= (wk & 0x7F80u) == 0x7F80u || (wk & 0x7F800000u) == 0x7F800000u ||
                       (wv & 0x7F80u) == 0x7F80u || (wv & 0x7F800000u) == 0x7F800000u;
            }
            if (odd) bad[t] = 1;
        }
        __syncthreads();
        if (full) {
            const int64_t page = page0 + p < a.kv.max_pages ? a.kv.table[(int64_t)b * a.kv.max_pages + page0 + p] : -1;
            u32 mk = 0, mv = 0;
            for (int i = tid; i < kPage * (DP / 8); i += 256) {
                const int t = i / (DP / 8), d = (i % (DP / 8)) * 8;
                if (bad[t]) continue;
                const uint4 kk = *(const uint4*)&x[0][t * LD + d], vv = *(const uint4*)&x[1][t * LD + d];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const u32 wk = (&kk.x)[j] & 0x7FFF7FFFu, wv = (&vv.x)[j] & 0x7FFF7FFFu;
                    mk = max(mk, max(wk & 0xFFFFu, wk >> 16));
                    mv = max(mv, max(wv & 0xFFFFu, wv >> 16));
                }
            }
#pragma unroll
            for (int o = 32; o; o >>= 1) {
                mk = max(mk, (u32)__shfl_xor((int)mk, o));
                mv = max(mv, (u32)__shfl_xor((int)mv, o));
            }
            if (lane == 0) { wave_max[0][wid] = mk; wave_max[1][wid] = mv; }
            const bool any_bad = __syncthreads_or(tid < kPage && bad[tid]);
            mk = max(max(wave_max[0][0], wave_max[0][1]), max(wave_max[0][2], wave_max[0][3]));
            mv = max(max(wave_max[1][0], wave_max[1][1]), max(wave_max[1][2], wave_max[1][3]));
            const float ak = __uint_as_float(mk << 16), av = __uint_as_float(mv << 16);
            const float ik = ak >= kKvTiny ? 127.0f / ak : 0.0f, iv = av >= kKvTiny ? 127.0f / av : 0.0f;
            if (page >= 0 && page < a.kv.n_pages) {
                uint8_t* const rec = a.kv.pages + kv_record(a.kv, page, g);
                if (tid == 0) {
                    float* sc = a.kv.scales + (page * a.kv.G + g) * 2;
                    sc[0] = any_bad ? __uint_as_float(0x7FC00000u) : ak >= kKvTiny ? ak / 127.0f : 0.0f;
                    sc[1] = av >= kKvTiny ? av / 127.0f : 0.0f;
                }
                for (int i = tid; i < 4 * DP; i += 256) {                   // 16 bytes of keys: two tokens' eight elements
                    const int l = i & 63, st = i >> 6, T2 = st / (DP / 32), sl = st % (DP / 32);
                    uint4 r;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int t = (2 * T2 + h) * 16 + (l & 15), d = sl * 32 + (l >> 4) * 8;
                        const uint4 w = *(const uint4*)&x[0][t * LD + d];
                        const float m = bad[t] ? 0.0f : ik;
                        u32 c[2] = {0, 0};
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const u32 e = j & 1 ? (&w.x)[j >> 1] & 0xFFFF0000u : (&w.x)[j >> 1] << 16;
                            const float y = bad[t] ? 0.0f : fminf(fmaxf(rintf(__uint_as_float(e) * m), -127.0f), 127.0f);
                            c[j >> 2] |= ((u32)(int)y & 255u) << ((j & 3) * 8);
                        }
                        (&r.x)[2 * h] = c[0];
                        (&r.x)[2 * h + 1] = c[1];
                    }
                    *(uint4*)(rec + (size_t)i * 16) = r;
                }
                for (int i = tid; i < 4 * DP; i += 256) {                   // 16 bytes of values: one element of sixteen tokens
                    const int l = i & 63, d = (i >> 6) * 16 + (l & 15);
                    uint4 r;
#pragma unroll
                    for (int T = 0; T < 4; ++T) {
                        u32 c = 0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int t = T * 16 + (l >> 4) * 4 + j;
                            const float e = __uint_as_float((u32)x[1][t * LD + d] << 16);
                            const float y = bad[t] ? 0.0f : fminf(fmaxf(rintf(e * iv), -127.0f), 127.0f);
                            c |= ((u32)((int)y + 128) & 255u) << (j * 8);
                        }
                        (&r.x)[T] = c;
                    }
                    *(uint4*)(rec + (size_t)kPage * DP + (size_t)i * 16) = r;
                }
            }
        } else {
            for (int i = tid; i < kPage * (DP / 8); i += 256) {
                const int t = i / (DP / 8), d = (i % (DP / 8)) * 8;
                if (t < from_tail || t >= end) continue;
                uint4 kk = *(const uint4*)&x[0][t * LD + d], vv = *(const uint4*)&x[1][t * LD + d];
                if (bad[t]) {
                    kk = uint4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
                    vv = uint4{0, 0, 0, 0};
                }
                *(uint4*)(tail_k + t * DP + d) = kk;
#pragma unroll
                for (int j = 0; j < 8; ++j) tail_v[((t >> 2) * DP + d + j) * 4 + (t & 3)] = (uint16_t)((&vv.x)[j >> 1] >> ((j & 1) * 16));
            }
        }
        __syncthreads();
        if (!full) break;
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
// A record is read once, in its own order, and turned into rows through LDS; memory bound.
template <int DT, int DP>
__global__ __launch_bounds__(256) void kv_read_kernel(KvReadArgs a)
{
    typedef typename Elem<DT>::raw_t raw_t;
    constexpr int LD = DP + (DT == 0 ? 4 : 8);
    __shared__ __align__(16) raw_t x[kPage * LD];
    const int tid = threadIdx.x;
    const int bg = blockIdx.y + gridDim.y * blockIdx.z;
    if (bg >= a.kv.seqs * a.kv.G) return;
    const int b = bg / a.kv.G, g = bg % a.kv.G, D = a.kv.D;
    const KvSeq s = kv_seq(a.kv, a.starts, a.tokens, b);
    const int n = s.n < s.len ? s.n : s.len, full = s.len / kPage;
    auto raw = [](float f) -> raw_t {
        if constexpr (DT == 0) return __float_as_uint(f);
        else return (raw_t)Row8<0>::f32_to_bf16_any(f);
    };
    for (int p = blockIdx.x; p * kPage < n; p += gridDim.x) {
        const int end = min(n - p * kPage, kPage);
        int64_t page = p < full ? a.kv.table[(int64_t)b * a.kv.max_pages + p] : 0;
        const bool there = page >= 0 && page < a.kv.n_pages;
        if (!there) page = 0;
        const float nan = __uint_as_float(0x7FC00000u);
        for (int kv = 0; kv < 2; ++kv) {
            if (p < full) {
                const uint8_t* rec = a.kv.pages + kv_record(a.kv, page, g) + (size_t)kv * kPage * DP;
                const float sc = there ? a.kv.scales[(page * a.kv.G + g) * 2 + kv] : nan;
                for (int i = tid; i < 4 * DP; i += 256) {
                    const uint4 r = *(const uint4*)(rec + (size_t)i * 16);
                    const int l = i & 63, st = i >> 6;
                    if (kv == 0) {
                        const int T2 = st / (DP / 32), d = st % (DP / 32) * 32 + (l >> 4) * 8;
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const int t = (2 * T2 + (j >> 3)) * 16 + (l & 15);
                            x[t * LD + d + (j & 7)] = raw((float)(int)(int8_t)((&r.x)[j >> 2] >> ((j & 3) * 8)) * sc);
                        }
                    } else {
                        const int d = st * 16 + (l & 15);
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const int t = (j >> 2) * 16 + (l >> 4) * 4 + (j & 3);
                            x[t * LD + d] = raw((float)((int)((&r.x)[j >> 2] >> ((j & 3) * 8) & 255u) - 128) * sc);
                        }
                    }
                }
            } else {
                const uint16_t* tail = a.kv.tails + kv_tail(a.kv, b, g) + kv * kPage * DP;
                for (int i = tid; i < end * DP; i += 256) {
                    const int t = i / DP, d = i % DP;
                    const u32 e = kv == 0 ? tail[i] : tail[((t >> 2) * DP + d) * 4 + (t & 3)];
                    x[t * LD + d] = DT == 0 ? (raw_t)(e << 16) : (raw_t)e;
                }
            }
            __syncthreads();
            constexpr int E = 16 / sizeof(raw_t);
            raw_t* out = (raw_t*)(kv == 0 ? a.k : a.v);
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
}

}  // namespace slicer
