// The attention cache in 8 bits: formats and helpers shared by its kernels (gfx950, wave64).
//
// A page holds 64 tokens of one sequence.  The record of (page, head) is 64 * dp bytes of key codes and 64 * dp bytes of value
// codes (dp = head size rounded up to 32, the rest zero), in the order in which the lanes of a 16 x 16 x 32 matrix product want
// them, so that a wavefront reads a record with 16-byte loads of consecutive lanes and never moves a code between lanes:
//   keys    byte ((T/2 * dp/32 + s) * 64 + lane) * 16 + (T%2) * 8 + j   token 16 T + lane%16, element 32 s + lane/16 * 8 + j
//   values  byte (t * 64 + lane) * 16 + T * 4 + j                       token 16 T + lane/16 * 4 + j, element 16 t + lane%16
// Key codes are signed; value codes have 128 added (what turns them into fp16 wants them so, see codes_f16).
// The product of keys and queries leaves a lane with the probabilities of the very tokens whose values it holds: the sums over tokens
// of the second product run in the order of the value record, and probabilities stay in their lanes too.
//
// Tokens of a page that is not full are kept as bf16 in the sequence's tail: keys [64][dp], values [16][dp][4] (token 4 i + j of
// element d at (i * dp + d) * 4 + j: one new token touches dp/16 lines instead of dp, and four tokens of an element are one load).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "slicer_common.hpp"

namespace slicer {

constexpr int kPage = 64;                 // SLICER_KV_PAGE
constexpr float kKvTiny = 0x1p-119f;      // below it 127 / amax would leave the range of fp32: the page holds zeros

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct KvView {
    uint8_t* pages;
    float* scales;            // [n_pages][heads][2]
    uint16_t* tails;          // [seqs][heads][2][64 * dp]
    const int32_t* table;     // [seqs][max_pages]
    const int32_t* lens;      // [seqs]
    int seqs, G, D, dp, max_pages;
    int64_t n_pages;
};

// New tokens of a sequence among the packed ones, and its length.  Whatever the arrays hold, the token range lies in [0, tokens)
// and the length in the table's reach.
struct KvSeq { int64_t first; int n, len; };

__device__ inline KvSeq kv_seq(const KvView& kv, const int32_t* starts, int64_t tokens, int b)
{
    KvSeq s;
    int64_t i0 = starts[b], i1 = starts[b + 1];
    i0 = i0 < 0 ? 0 : i0 > tokens ? tokens : i0;
    i1 = i1 < i0 ? i0 : i1 > tokens ? tokens : i1;
    s.first = i0;
    s.n = (int)(i1 - i0);
    const int64_t cap = (int64_t)kv.max_pages * kPage;
    const int64_t l = kv.lens[b];
    s.len = (int)(l < 0 ? 0 : l > cap ? cap : l);
    return s;
}

__device__ inline size_t kv_record(const KvView& kv, int64_t page, int g) { return ((size_t)page * kv.G + g) * (size_t)(2 * kPage * kv.dp); }
__device__ inline size_t kv_tail(const KvView& kv, int b, int g) { return ((size_t)b * kv.G + g) * (size_t)(2 * kPage * kv.dp); }

// eight signed codes -> bf16, exact: the upper half of an fp32 holds any whole number up to 256
__device__ inline bf16x8 codes_bf16(u32 w0, u32 w1)
{
    u32 r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u32 w = i < 2 ? w0 : w1;
        const int sh = (i & 1) * 16;
        const float a = (float)(int)(int8_t)(w >> sh), b = (float)(int)(int8_t)(w >> (sh + 8));
        r[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
    bf16x8 v;
    __builtin_memcpy(&v, r, 16);
    return v;
}

// four codes with 128 added -> fp16, exact: 0x6400 + u is the fp16 number 1024 + u, from which 1152 is taken
__device__ inline uint2 codes_f16(u32 w)
{
    const u32 lo = __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u), hi = __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u);
    const f16x2 c = {(_Float16)1152.0f, (_Float16)1152.0f};
    f16x2 a, b;
    __builtin_memcpy(&a, &lo, 4);
    __builtin_memcpy(&b, &hi, 4);
    a = a - c;
    b = b - c;
    uint2 r;
    __builtin_memcpy(&r.x, &a, 4);
    __builtin_memcpy(&r.y, &b, 4);
    return r;
}

__device__ inline f16x8 f16_of(uint2 a, uint2 b)
{
    const uint4 r = {a.x, a.y, b.x, b.y};
    f16x8 v;
    __builtin_memcpy(&v, &r, 16);
    return v;
}

__device__ inline bf16x8 bf16_of(uint4 r)
{
    bf16x8 v;
    __builtin_memcpy(&v, &r, 16);
    return v;
}

// Eight consecutive elements of a query, key or value row, wherever it starts: 16-byte loads where `wide` says that the address allows them.
template <int DT>
struct Row8;

template <>
struct Row8<1> {
    __device__ static inline uint4 bf16(const void* p, int64_t at, bool wide)
    {
        const uint16_t* x = (const uint16_t*)p + at;
        if (wide) return *(const uint4*)x;
        uint4 r;
        r.x = x[0] | (u32)x[1] << 16;
        r.y = x[2] | (u32)x[3] << 16;
        r.z = x[4] | (u32)x[5] << 16;
        r.w = x[6] | (u32)x[7] << 16;
        return r;
    }
};

template <>
struct Row8<0> {
    __device__ static inline void f32(const void* p, int64_t at, bool wide, float* f)
    {
        const float* x = (const float*)p + at;
        if (wide) {
            const float4 a = *(const float4*)x, b = *(const float4*)(x + 4);
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
            f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = x[j];
        }
    }
    __device__ static inline uint4 bf16(const void* p, int64_t at, bool wide)
    {
        float f[8];
        f32(p, at, wide, f);
        uint4 r;
        r.x = f32_to_bf16_any(f[0]) | f32_to_bf16_any(f[1]) << 16;
        r.y = f32_to_bf16_any(f[2]) | f32_to_bf16_any(f[3]) << 16;
        r.z = f32_to_bf16_any(f[4]) | f32_to_bf16_any(f[5]) << 16;
        r.w = f32_to_bf16_any(f[6]) | f32_to_bf16_any(f[7]) << 16;
        return r;
    }
    // nearest even, NaN stays NaN
    __device__ static inline u32 f32_to_bf16_any(float f)
    {
        const u32 u = __float_as_uint(f);
        return (u & 0x7FFFFFFFu) > 0x7F800000u ? 0x7FC0u : f32_to_bf16_rne(f);
    }
};

}  // namespace slicer
