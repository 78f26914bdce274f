// Attention over the cache in 8 bits (gfx950, wave64): o = softmax(scale q k^T) v with a running maximum and sum, in one pass over the pages.
//
// Codes enter the matrix products as they are, exact in bf16 (keys) and fp16 (values); a page's two scales are factors of its scores and of its
// probabilities.  What a product rounds is therefore the queries (bf16 queries are exact, fp32 ones are split into three bf16 numbers) and the probabilities:
// times 2^13 they are held in fp16 (11 bits, down to 2^-27 of the largest; fp32 outputs take a second fp16 number for the rest), in prompts times 2^8 and the ratio of two
// value scales, 2^-6 to 2 (where the ratio is smallest: 11 bits down to 2^-16 of the largest, steps of 2^-26 below).  bf16 probabilities would have added as much error as the
// output's own rounding.  Scores, maxima, sums (of the probabilities before that rounding) and outputs are fp32 throughout.
// The tail's values are bf16 as they came and would not fit fp16: there the probabilities are split into bf16 numbers.
#pragma once

#include <type_traits>

#include "slicer_kv.hpp"

namespace slicer {

// Sequences with at most this many query rows a cache head (new tokens times query heads a head) split the cache over workgroups; others take a
// workgroup per 128 rows.
constexpr int kSplitRows = 64;
// Tables of at most this many pages: weights of rows that one workgroup has all of are made where they arise.
constexpr int kMassPages = 64;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kPBias = 13.0f;

struct KvAttendArgs {
    KvView kv;
    const void* q;
    int64_t q_token, q_head;
    const int32_t* starts;
    int64_t tokens;
    int R, H, max_new, causal;
    float scale;                  // of the scores, times log2(e); not negative
    int flip;                     // queries are negated instead
    void* out;                    // [tokens][H][D]
    float* lse;                   // [tokens][H] or null
    float* mass;                  // [seqs][G][max_pages] or null
    float decay;
    int wide_q;
    // split rows: [row][splits] (maximum, sum), [row][splits][dp] sums of values; row = (sequence, head, row) with rows_pad rows a head
    int splits, rows_pad;
    float2* part_ml;
    float* part_o;
    float2* page_w;               // [sequence, head][max_pages][rows_pad] a page's sum of weights under a maximum
    // other rows: sequences of at most few_rows rows a head are not looked at; with prompt_splits > 1 a row tile's pages are shared out, and [row][splits]
    // (maximum, sum), [row][splits][dp] sums of values, [row] totals are kept; with weights [workgroup][slot_pages][128] a page's sum of a tile's
    // rows, and [sequence, head][tiles][max_pages] of the tile
    int few_rows, prompt_splits, slot_pages;
    float2* prompt_ml;
    float* prompt_o;
    float2* row_total;
    float2* row_w;
    float* tile_mass;
};

// queries -> bf16 operands: element j of part i
template <int DT>
struct QParts;
template <>
struct QParts<1> {
    static constexpr int N = 1;
    static constexpr int NP = 1;          // fp16 numbers a probability is held in
    static constexpr int NB = 2;          // bf16 numbers
    __device__ static inline void load(const KvAttendArgs& a, int64_t at, bf16x8* p)
    {
        uint4 w = Row8<1>::bf16(a.q, at, a.wide_q);
        const u32 sign = a.flip ? 0x80008000u : 0u;
        w.x ^= sign;
        w.y ^= sign;
        w.z ^= sign;
        w.w ^= sign;
        p[0] = bf16_of(w);
    }
};
template <>
struct QParts<0> {
    static constexpr int N = 3;
    static constexpr int NP = 2;
    static constexpr int NB = 3;
    __device__ static inline void load(const KvAttendArgs& a, int64_t at, bf16x8* p)
    {
        float f[8];
        Row8<0>::f32(a.q, at, a.wide_q, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (a.flip) f[j] = -f[j];
            const __bf16 h = (__bf16)f[j];
            const float r = f[j] - (float)h;
            const __bf16 m = (__bf16)r;
            p[0][j] = h;
            p[1][j] = m;
            p[2][j] = (__bf16)(r - (float)m);
        }
    }
};

__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

template <int DT>
__device__ inline void store4(void* out, int64_t at, f32x4 v)
{
    if constexpr (DT == 0) {
        *(f32x4*)((float*)out + at) = v;
    } else {
        uint2 r;
        const bf16x2 a = {(__bf16)v[0], (__bf16)v[1]}, b = {(__bf16)v[2], (__bf16)v[3]};
        __builtin_memcpy(&r.x, &a, 4);
        __builtin_memcpy(&r.y, &b, 4);
        *(uint2*)((uint16_t*)out + at) = r;
    }
}

// ---- few rows: the cache is split over workgroups -------------------------------------------------------------------------
//
// A workgroup has one cache head of one sequence, 16 QT query rows and a share of the pages; its four wavefronts take pages in turn, each with
// sums of its own, which meet in LDS at the end.  S^T = K Q^T and O^T = V^T P^T, so that a lane holds one row's scores and probabilities.  Codes go from memory to
// registers to the matrix units; a page's values are on their way while its scores are made, the next page's keys while its values are used.
// Memory bound: 2 * D bytes a token and head.  Measured, 8 cache heads of 128, bf16: 2 x 262016 tokens before 32 heads 182 us (1.07 GB, 5.9 TB/s; a large copy moves
// 4.95), 256 x 500..2047 tokens before 64 heads 151 us (0.67 GB, 4.4 TB/s: four rounds of workgroups that start with dependent loads).
// Of the second shape: loads without a page's lead and four wavefronts a SIMD 183 us, three wavefronts 155.
template <int DT, int DP, int QT>
__global__ __launch_bounds__(256, (QT == 1 && DP <= 160) || (QT == 1 && DP == 192 && DT == 1) || (QT == 2 && DP * (DT == 1 ? 1 : 2) <= 128) ? 2 : 1) void kv_split_kernel(KvAttendArgs a)
{
    constexpr int KS = DP / 32, DTL = DP / 16, NQ = QParts<DT>::N, NP = QParts<DT>::NP, NB = QParts<DT>::NB;
    constexpr int LDO = DP + 4;
    __shared__ __align__(16) float xo[4][16][LDO];
    __shared__ float2 xml[4][16 * QT];
    __shared__ float2 xw[QT == 1 ? kMassPages * 16 : 1];               // a page's sums of weights under a maximum, where all of them are here
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, c = lane & 15, gq = lane >> 4;
    constexpr int TR = 16 * QT;                          // rows of the tile
    const int row_tiles = (a.rows_pad + TR - 1) / TR;
    const int split = blockIdx.x % a.splits, rt = (blockIdx.x / a.splits) % row_tiles, bg = blockIdx.x / a.splits / row_tiles;
    const int b = bg / a.kv.G, g = bg % a.kv.G, D = a.kv.D;
    const bool own_mass = QT == 1 && a.mass && a.splits == 1 && row_tiles == 1 && a.kv.max_pages <= kMassPages;
    // places of this wavefront's pages: those of the next 64 lie in the lanes.  Where the first is known before the length, they are asked for at once
    // (a workgroup starts with a chain of dependent loads, 1 us each under load: length, place, codes)
    const int32_t* const table = a.kv.table + (int64_t)b * a.kv.max_pages;
    int early = -1;
    if (a.splits == 1 && wid + 4 * lane < a.kv.max_pages) early = table[wid + 4 * lane];
    KvSeq s = kv_seq(a.kv, a.starts, a.tokens, b);
    const int n_all = s.n;
    s.n = s.n < a.max_new ? s.n : a.max_new;
    const int rows = (int)min((int64_t)s.n * a.R, (int64_t)kSplitRows + 1);
    if (rt * TR >= rows || rows > kSplitRows) return;
    int lim[QT];                                         // tokens that the lane's rows see
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        const int rr = rt * TR + x * 16 + c;
        lim[x] = rr >= rows ? 0 : a.causal ? s.len - n_all + rr / a.R + 1 : s.len;
    }
    const int last_row = min(rows, rt * TR + TR) - 1;
    const int most = a.causal ? max(0, s.len - n_all + last_row / a.R + 1) : s.len;
    const int least = a.causal ? s.len - n_all + (rt * TR) / a.R + 1 : s.len;          // every row of the tile sees as many
    const int full = s.len / kPage, units = (most + kPage - 1) / kPage;
    const int per = (units + a.splits - 1) / a.splits, u0 = split * per, u1 = min(units, u0 + per);
    const int64_t slot0 = ((int64_t)bg * a.rows_pad + rt * TR) * a.splits + split;      // of the tile's first row
    if (u0 >= u1 && a.splits > 1) {
        if (tid < TR && rt * TR + tid < rows) a.part_ml[slot0 + (int64_t)tid * a.splits] = float2{-__builtin_inff(), 0.0f};
        return;
    }

    bf16x8 q[QT][NQ][KS];
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        const int rr = rt * TR + x * 16 + c;
        const bool live = rr < rows;
        const int64_t at = (s.first + (live ? rr / a.R : 0)) * a.q_token + (g * a.R + rr % a.R) * a.q_head;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            bf16x8 p[NQ];
            const int d = k * 32 + gq * 8;
            if (live && d < D) QParts<DT>::load(a, at + d, p);
#pragma unroll
            for (int i = 0; i < NQ; ++i) q[x][i][k] = live && d < D ? p[i] : bf16x8{};
        }
    }

    float m[QT], l[QT];                                  // of the lane's rows; l: of the lane's own tokens
    f32x4 o[QT][DTL];
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        m[x] = -__builtin_inff();
        l[x] = 0.0f;
#pragma unroll
        for (int t = 0; t < DTL; ++t) o[x][t] = f32x4{0, 0, 0, 0};
    }
    float2* const page_w = a.page_w + (int64_t)bg * a.kv.max_pages * a.rows_pad;

    // scores of a page -> probabilities (times 2^13), the running maximum and sum; returns what the sums so far are to be multiplied by
    auto softmax = [&](int x, f32x4* sc, float factor, int u) {
        const int left = lim[x] - u * kPage - gq * 4;    // tokens that the row sees from the lane's first on
        float mx = -__builtin_inff();
        if (u * kPage + kPage <= least) {
#pragma unroll
            for (int T = 0; T < 4; ++T)
#pragma unroll
                for (int r = 0; r < 4; ++r) { sc[T][r] *= factor; mx = fmaxf(mx, sc[T][r]); }
        } else {
#pragma unroll
            for (int T = 0; T < 4; ++T)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    sc[T][r] = T * 16 + r < left ? sc[T][r] * factor : -__builtin_inff();
                    mx = fmaxf(mx, sc[T][r]);
                }
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float mn = fmaxf(m[x], mx), ms = mn == -__builtin_inff() ? 0.0f : mn;
        const float alpha = exp2_of(m[x] - ms);
        float sum = 0.0f;
        // (the maximum first: under it every difference is right to half a step of its own, whereas bias - maximum is rounded to the maximum's, from 2^26 on
        // to more than fp16's room above 2^13)
#pragma unroll
        for (int T = 0; T < 4; ++T)
#pragma unroll
            for (int r = 0; r < 4; ++r) { sc[T][r] = exp2_of((sc[T][r] - ms) + kPBias); sum += sc[T][r]; }
        m[x] = mn;
        l[x] = __builtin_fmaf(l[x], alpha, sum);
        if (a.mass) {
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            const int rr = rt * TR + x * 16 + c;
            if (gq == 0 && rr < rows) {
                if (QT == 1 && own_mass) xw[u * 16 + c] = float2{ms, sum};
                else page_w[(int64_t)u * a.rows_pad + rr] = float2{ms, sum};
            }
        }
        return alpha;
    };

    // this wavefront's pages: u0 + wid, u0 + wid + 4, ...
    const int ufull = min(u1, full);
    int64_t my_page = 0;
    float my_ks = 0.0f, my_vs = 0.0f;
    auto fetch = [&](int u, bool known) {                // lane i: page u + 4 i
        const int up = u + 4 * lane;
        my_page = 0;
        my_ks = my_vs = 0.0f;
        if (up < ufull) {
            const int64_t id = known ? early : table[up];
            const bool there = id >= 0 && id < a.kv.n_pages;
            my_page = there ? id : 0;
            const float2 sc = *(const float2*)(a.kv.scales + (my_page * a.kv.G + g) * 2);
            my_ks = there ? sc.x : __uint_as_float(0x7FC00000u);       // a page that is not there: NaN for who sees it, zeros for the other rows
            my_vs = there ? sc.y : 0.0f;
        }
    };
    auto record = [&](int i) {
        const u32 id = bcast((u32)my_page, i);
        return (const uint4*)(a.kv.pages + kv_record(a.kv, id, g)) + lane;
    };
    int u = u0 + wid;
    uint4 kb[2 * KS], vb[DTL];
    const uint4* rec = nullptr;
    if (u < ufull) {
        fetch(u, a.splits == 1);
        rec = record(0);
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) kb[i] = rec[i * 64];
    }
    for (int it = 0; u < ufull; u += 4, ++it) {
        const float ks = __uint_as_float(bcast(__float_as_uint(my_ks), it & 63)) * a.scale, vs = __uint_as_float(bcast(__float_as_uint(my_vs), it & 63));
#pragma unroll
        for (int i = 0; i < DTL; ++i) vb[i] = rec[(2 * KS + i) * 64];
        f32x4 sc[QT][4];
#pragma unroll
        for (int x = 0; x < QT; ++x)
#pragma unroll
            for (int T = 0; T < 4; ++T) sc[x][T] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int T2 = 0; T2 < 2; ++T2)
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const uint4 w = kb[T2 * KS + k];
                const bf16x8 k0 = codes_bf16(w.x, w.y), k1 = codes_bf16(w.z, w.w);
#pragma unroll
                for (int x = 0; x < QT; ++x)
#pragma unroll
                    for (int i = 0; i < NQ; ++i) {
                        sc[x][2 * T2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[x][i][k], sc[x][2 * T2], 0, 0, 0);
                        sc[x][2 * T2 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[x][i][k], sc[x][2 * T2 + 1], 0, 0, 0);
                    }
            }
        if (u + 4 < ufull) {
            if ((it & 63) == 63) fetch(u + 4, false);
            rec = record((it + 1) & 63);
#pragma unroll
            for (int i = 0; i < 2 * KS; ++i) kb[i] = rec[i * 64];
        }
        float alpha[QT];
        f16x8 p[QT][NP][2];
#pragma unroll
        for (int x = 0; x < QT; ++x) {
            alpha[x] = softmax(x, sc[x], ks, u);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float f = sc[x][2 * h + (j >> 2)][j & 3];
                    const _Float16 hi = (_Float16)f;
                    p[x][0][h][j] = hi;
                    if constexpr (NP > 1) p[x][1][h][j] = (_Float16)(f - (float)hi);
                }
        }
#pragma unroll
        for (int t = 0; t < DTL; ++t) {
            const f16x8 v0 = f16_of(codes_f16(vb[t].x), codes_f16(vb[t].y)), v1 = f16_of(codes_f16(vb[t].z), codes_f16(vb[t].w));
#pragma unroll
            for (int x = 0; x < QT; ++x) {
                f32x4 acc = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[x][i][0], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[x][i][1], acc, 0, 0, 0);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) o[x][t][r] = __builtin_fmaf(acc[r], vs, o[x][t][r] * alpha[x]);
            }
        }
    }
    if (u < u1 && u == full) {                           // the tail, as the last page
        const int count = s.len - full * kPage;
        const uint16_t* tk = a.kv.tails + kv_tail(a.kv, b, g);
        const uint16_t* tv = tk + kPage * DP;
#pragma unroll
        for (int x = 0; x < QT; ++x) {
            f32x4 sc[4];
#pragma unroll
            for (int T = 0; T < 4; ++T) {
                sc[T] = f32x4{0, 0, 0, 0};
                if (T * 16 < count) {
#pragma unroll
                    for (int k = 0; k < KS; ++k) {
                        const bf16x8 w = bf16_of(*(const uint4*)(tk + (T * 16 + c) * DP + k * 32 + gq * 8));
#pragma unroll
                        for (int i = 0; i < NQ; ++i) sc[T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, q[x][i][k], sc[T], 0, 0, 0);
                    }
                }
            }
            const float alpha = softmax(x, sc, a.scale, u);
            bf16x8 p[NB][2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float f = sc[2 * h + (j >> 2)][j & 3];
#pragma unroll
                    for (int i = 0; i < NB; ++i) {
                        p[i][h][j] = (__bf16)f;
                        f -= (float)p[i][h][j];
                    }
                }
#pragma unroll
            for (int t = 0; t < DTL; ++t) {
#pragma unroll
                for (int r = 0; r < 4; ++r) o[x][t][r] *= alpha;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32 w[4];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {        // four tokens of an element; those behind the last are whatever the memory held
                        const int t0 = (2 * h + e) * 16 + gq * 4;
                        uint2 r = {0, 0};
                        if (t0 < count) r = *(const uint2*)(tv + ((t0 >> 2) * DP + t * 16 + c) * 4);
                        const int left = count - t0;
                        w[2 * e] = left >= 2 ? r.x : left == 1 ? r.x & 0xFFFFu : 0u;
                        w[2 * e + 1] = left >= 4 ? r.y : left == 3 ? r.y & 0xFFFFu : 0u;
                    }
                    const bf16x8 v = bf16_of(uint4{w[0], w[1], w[2], w[3]});
#pragma unroll
                    for (int i = 0; i < NB; ++i) o[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[i][h], o[x][t], 0, 0, 0);
                }
            }
        }
    }

    // the four wavefronts' sums under one maximum
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        l[x] += __shfl_xor(l[x], 16);
        l[x] += __shfl_xor(l[x], 32);
        if (gq == 0) xml[wid][x * 16 + c] = float2{m[x], l[x]};
    }
    __syncthreads();
    auto total = [&](int r) {                            // (maximum, sum) of a row of the tile
        const float M = fmaxf(fmaxf(xml[0][r].x, xml[1][r].x), fmaxf(xml[2][r].x, xml[3][r].x)), Ms = M == -__builtin_inff() ? 0.0f : M;
        float L = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) L += xml[w][r].y * exp2_of(xml[w][r].x - Ms);
        return float2{M, L};
    };
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        const float M = total(x * 16 + c).x, f = exp2_of(m[x] - (M == -__builtin_inff() ? 0.0f : M));
        if (x) __syncthreads();
#pragma unroll
        for (int t = 0; t < DTL; ++t) *(f32x4*)&xo[wid][c][t * 16 + gq * 4] = o[x][t] * f;
        __syncthreads();
        for (int i = tid; i < 16 * (DP / 4); i += 256) {
            const int r = i / (DP / 4), d = i % (DP / 4) * 4, rw = rt * TR + x * 16 + r;
            if (rw >= rows || d >= D) continue;
            f32x4 v = *(const f32x4*)&xo[0][r][d];
#pragma unroll
            for (int w = 1; w < 4; ++w) v += *(const f32x4*)&xo[w][r][d];
            if (a.splits > 1) {
                *(f32x4*)(a.part_o + (slot0 + (int64_t)(x * 16 + r) * a.splits) * DP + d) = v;
            } else {
                const float L = total(x * 16 + r).y;
                store4<DT>(a.out, ((s.first + rw / a.R) * a.H + g * a.R + rw % a.R) * (int64_t)D + d, v * (L == 0.0f ? 0.0f : 1.0f / L));
            }
        }
    }
    if (tid < TR && rt * TR + tid < rows) {
        const float2 ml = total(tid);
        const int rw = rt * TR + tid;
        if (a.splits > 1 || (a.mass && !own_mass)) a.part_ml[slot0 + (int64_t)tid * a.splits] = ml;
        if (a.splits == 1 && a.lse) a.lse[(s.first + rw / a.R) * a.H + g * a.R + rw % a.R] = ml.y == 0.0f ? -__builtin_inff() : (ml.x - kPBias + __log2f(ml.y)) * kLn2;
    }
    if (QT == 1 && own_mass) {                           // sixteen lanes a page
        const float2 ml = total(c);
        const int pages = (s.len + kPage - 1) / kPage;
        for (int p = tid >> 4; p < pages; p += 16) {
            float sum = 0.0f;
            if (p < units && c < rows) {
                const float2 w = xw[p * 16 + c];
                if (w.y != 0.0f) sum = w.y * exp2_of(w.x - ml.x) / ml.y;
            }
#pragma unroll
            for (int o = 8; o; o >>= 1) sum += __shfl_xor(sum, o);
            if (c == 0) {
                float* to = a.mass + (int64_t)bg * a.kv.max_pages + p;
                *to = a.decay == 0.0f ? sum : __builtin_fmaf(*to, a.decay, sum);
            }
        }
    }
}

// (maximum, sum) of a split row from its parts, by one wavefront; every lane gets them.
__device__ inline float2 kv_row_total(const float2* ml, int splits, int lane)
{
    float M = -__builtin_inff(), L = 0.0f;
    for (int i = lane; i < splits; i += kWave) M = fmaxf(M, ml[i].x);
#pragma unroll
    for (int o = 32; o; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    if (M == -__builtin_inff()) M = 0.0f;
    for (int i = lane; i < splits; i += kWave) L += ml[i].y * exp2_of(ml[i].x - M);
#pragma unroll
    for (int o = 32; o; o >>= 1) L += __shfl_xor(L, o);
    return float2{M, L};
}

// A row's output from its parts, by a workgroup: all four wavefronts read parts at once, several a load (with one wavefront a row, part after part, 64 parts took
// 64 us instead of 5).
template <int DT, int DP>
__device__ inline void kv_join_row(const KvAttendArgs& a, const float2* ml, const float* parts, int splits, float2 total, int64_t at, float (*xo)[DP])
{
    constexpr int LPP = DP / 4, PPW = kWave / LPP;       // lanes a part, parts a load (one where a part takes more than half of the lanes)
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, D = a.kv.D;
    const int part = PPW > 1 ? lane / LPP : 0, d = (PPW > 1 ? lane % LPP : lane) * 4;
    f32x4 v = {0, 0, 0, 0};
    if (part < PPW && d < D) {
#pragma unroll 4
        for (int i = wid * PPW + part; i < splits; i += 4 * PPW) {
            const float2 p = ml[i];
            const f32x4 x = *(const f32x4*)(parts + (int64_t)i * DP + d) * exp2_of(p.x - total.x);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += p.y != 0.0f ? x[e] : 0.0f;           // (a part without a sum was not written)
        }
    }
    if constexpr (PPW > 1) {
#pragma unroll
        for (int q = 1; q < PPW; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float f = __shfl(v[e], (lane + q * LPP) & 63);
                if (part == 0) v[e] += f;
            }
    }
    if (part == 0 && d < DP) *(f32x4*)&xo[wid][d] = v;
    __syncthreads();
    if (tid * 4 < D) {
        v = *(const f32x4*)&xo[0][tid * 4];
#pragma unroll
        for (int w = 1; w < 4; ++w) v += *(const f32x4*)&xo[w][tid * 4];
        store4<DT>(a.out, at * D + tid * 4, v * (total.y == 0.0f ? 0.0f : 1.0f / total.y));
    }
    if (tid == 0 && a.lse) a.lse[at] = total.y == 0.0f ? -__builtin_inff() : (total.x - kPBias + __log2f(total.y)) * kLn2;
}

// A row's share of a page's weight: its sum there under a maximum, the row's maximum and one over its sum.
__device__ inline float kv_weight(float2 w, float2 row) { return w.y == 0.0f || row.y == 0.0f ? 0.0f : w.y * exp2_of(w.x - row.x) * row.y; }

// What the workgroups of a split sequence left is put together: outputs, a workgroup per row, and the pages' weights, which can only be told now that
// the rows' sums are known, a workgroup per 256 pages.
template <int DT, int DP>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttendArgs a, int row_blocks, int page_blocks, int tile_rows)
{
    __shared__ float2 xml[kSplitRows];
    __shared__ __align__(16) float xo[4][DP];
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
    const int blk = blockIdx.x % (row_blocks + page_blocks), bg = blockIdx.x / (row_blocks + page_blocks);
    const int b = bg / a.kv.G, g = bg % a.kv.G;
    KvSeq s = kv_seq(a.kv, a.starts, a.tokens, b);
    const int n_all = s.n;
    s.n = s.n < a.max_new ? s.n : a.max_new;
    const int rows = (int)min((int64_t)s.n * a.R, (int64_t)kSplitRows + 1);
    if (rows == 0 || rows > kSplitRows) return;
    if (blk < row_blocks) {
        if (blk >= rows) return;
        const int64_t slot = ((int64_t)bg * a.rows_pad + blk) * a.splits;
        const float2 ml = kv_row_total(a.part_ml + slot, a.splits, lane);
        kv_join_row<DT, DP>(a, a.part_ml + slot, a.part_o + slot * DP, a.splits, ml, (s.first + blk / a.R) * a.H + g * a.R + blk % a.R, xo);
        return;
    }
    for (int r = wid; r < rows; r += 4) {
        const float2 ml = kv_row_total(a.part_ml + ((int64_t)bg * a.rows_pad + r) * a.splits, a.splits, lane);
        if (lane == 0) xml[r] = float2{ml.x, 1.0f / ml.y};
    }
    __syncthreads();
    for (int p = (blk - row_blocks) * 256 + tid; p < (s.len + kPage - 1) / kPage; p += page_blocks * 256) {
        const float2* w = a.page_w + ((int64_t)bg * a.kv.max_pages + p) * a.rows_pad;
        float sum = 0.0f;
        for (int r = 0; r < rows; ++r) {
            // a row's tile came to the pages that the tile's last row sees some token of
            const int top = a.causal ? s.len - n_all + min(rows - 1, r | (tile_rows - 1)) / a.R + 1 : s.len;
            if (p * kPage < top) sum += kv_weight(w[r], xml[r]);
        }
        float* to = a.mass + (int64_t)bg * a.kv.max_pages + p;
        *to = a.decay == 0.0f ? sum : __builtin_fmaf(*to, a.decay, sum);
    }
}

// ---- many rows: a workgroup per 128 of them --------------------------------------------------------------------------------
//
// Four wavefronts of 32 rows (token after token, a token's query heads of the cache head next to each other) share the pages: a page's codes are loaded one
// page ahead, turned into bf16 and fp16 operands once for all four and read from LDS as the lanes want them.  S^T = K Q^T and O^T = V^T P^T in 32 x 32 x 16
// products, a lane has the scores of one row.  Bound by the matrix units, the exponentials and LDS reads, in about equal parts.
// What was measured on 8 x 2048 queries, 32 heads over 8 of 128 (275 GFLOP), with the append: the pipeline of one wavefront, product by product with the vector
// instructions that run beside it, 371 us (the kernel alone 354 at best, 780 TFLOP/s, where a large matrix product reaches 1390); when it came in, 390 against 444 for a page after the other
// and 568 with 64 rows a wavefront (half of the LDS reads, one wavefront a SIMD): two wavefronts hide each other's waits better than one hides its own.  A page takes a wavefront 1.33 us
// alone on its SIMD, two of them 2.2; in the whole kernel vector instructions are issued 57 % of the time, the matrix units work 36 %, LDS 32 %.
// Scores and value scales that no model has (kSteep, page_scales) are outside what the pipeline can hold; a tile that meets them is done again, page after page.  With every tile
// done so, the same shape takes 697 us.

constexpr int kTileRows = 128;

// Share `i` of `n` of a row tile's pages.
struct KvShare { int first, end; };
__host__ __device__ inline KvShare kv_share(int units, int n, int i)
{
    const int per = (units + n - 1) / n, first = i * per < units ? i * per : units;
    return KvShare{first, first + per < units ? first + per : units};
}

template <int DP>
struct PromptTile {
    static constexpr int KK = DP / 16, DL = DP / 32;
    // elements of a page as operands: keys [2][KK][64 lanes][8], values [DL][4][64][8]
    static constexpr int kKeys = 2 * KK * 64 * 8, kAll = 2 * kKeys;
};

// record i of 16 bytes -> operands of 32 x 32 x 16 products in LDS: half `part` of a record of keys, word `part` of a record of values
template <int DP>
__device__ inline void stage_keys(uint16_t* to, int i, uint4 w, int part)
{
    constexpr int KK = DP / 16;
    const int l = i & 63, st = i >> 6, T2 = st / (DP / 32), sl = st % (DP / 32), gq = l >> 4, cc = l & 15;
    *(bf16x8*)(to + (((T2 * KK + sl * 2 + (gq >> 1)) * 64) + (gq & 1) * 32 + part * 16 + cc) * 8) = part ? codes_bf16(w.z, w.w) : codes_bf16(w.x, w.y);
}

template <int DP>
__device__ inline void stage_values(uint16_t* to, int i, uint4 w, int part)
{
    const int l = i & 63, dt = i >> 6, gq = l >> 4, cc = l & 15;
    *(uint2*)(to + (((dt >> 1) * 4 + part) * 64 + (gq & 1) * 32 + (dt & 1) * 16 + cc) * 8 + (gq >> 1) * 4) = codes_f16((&w.x)[part]);
}

// the tail: bf16 operands, nothing behind its last token
template <int DP>
__device__ inline void stage_tail(uint16_t* keys, uint16_t* values, const uint16_t* tk, int count, int tid)
{
    constexpr int KK = DP / 16;
    const uint16_t* tv = tk + kPage * DP;
    for (int i = tid; i < 2 * KK * 64; i += 256) {
        const int l = i & 63, kk = (i >> 6) % KK, tt = (i >> 6) / KK, t = tt * 32 + (l & 31);
        uint4 w = {0, 0, 0, 0};
        if (t < count) w = *(const uint4*)(tk + t * DP + kk * 16 + (l >> 5) * 8);
        *(uint4*)(keys + (size_t)i * 8) = w;
    }
    for (int i = tid; i < (DP / 32) * 4 * 64; i += 256) {
        const int l = i & 63, kk = (i >> 6) & 3, dl = i >> 8, d = dl * 32 + (l & 31);
        u32 w[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {                    // tokens (kk/2) 32 + 8 (2 (kk%2) + e) + 4 (lane/32) + 0..3
            const int t0 = (kk >> 1) * 32 + 8 * (2 * (kk & 1) + e) + 4 * (l >> 5), left = count - t0;
            uint2 r = {0, 0};
            if (left > 0) r = *(const uint2*)(tv + ((t0 >> 2) * DP + d) * 4);
            w[2 * e] = left >= 2 ? r.x : left == 1 ? r.x & 0xFFFFu : 0u;
            w[2 * e + 1] = left >= 4 ? r.y : left == 3 ? r.y & 0xFFFFu : 0u;
        }
        *(uint4*)(values + (size_t)i * 8) = uint4{w[0], w[1], w[2], w[3]};
    }
}

// Probabilities are held times 2^8 here: a row's maximum may grow by 2^6 before its sums are scaled down to it (nearly every page raises the
// maximum of some row, hardly any by that much), and a page's value scale may be twice the one that outputs are held in: 2^15 at most in fp16.
constexpr float kPromptBias = 8.0f, kSlack = 6.0f;
// Maxima beyond this (times log2(e); no model's) are not for the pipeline: its exponent, score * factor + (bias - maximum) in one instruction, takes a product that was
// not rounded from a maximum that was, and is off by half a step of it: 2^-13 here, as much as the score itself, but more than fp16's room from 2^24 on.
constexpr float kSteep = 4096.0f;

__device__ inline float other_half(float x, float* mine)             // the values of lanes l and l + 32 of a pair, in both of them
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    *mine = __uint_as_float(r[0]);
    return __uint_as_float(r[1]);
}

// `row_tiles` of 128 rows a head; workgroups that keep weights of a tile's rows by page on the way (a.mass) have a part of row_w each.
template <int DT, int DP>
__global__ __launch_bounds__(256, DP * (DT == 1 ? 1 : 2) <= 128 ? 2 : 1) void kv_prompt_kernel(KvAttendArgs a, int row_tiles)
{
    constexpr int KK = DP / 16, DL = DP / 32, NQ = QParts<DT>::N, NP = QParts<DT>::NP, NB = QParts<DT>::NB;
    constexpr int NR = (4 * DP + 255) / 256;             // records of keys (and of values) a thread
    constexpr int WR = 32, TR = kTileRows;               // rows of a wavefront, of the tile
    __shared__ __align__(16) uint16_t buf[2][PromptTile<DP>::kAll];
    __shared__ float2 xrow[TR];
    __shared__ int xcareful;
    const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, c = lane & 31, h = lane >> 5;
    const int heads = a.kv.seqs * a.kv.G, D = a.kv.D;
    float2* const my_w = a.row_w + (size_t)blockIdx.x * a.slot_pages * TR;
    // (fewer than 2^24 tiles, so that rows and tiles are numbers of 32 bits: divisions of 64 bits took a good part of a short tile's start)
    const u32 R = (u32)a.R, n_tiles = (u32)heads * (u32)row_tiles * (u32)a.prompt_splits;
    for (u32 tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
        // the longest tiles first; a head's tiles on one XCD (workgroup i runs on XCD i % 8), whose L2 its pages then are in
        const u32 turn = tile / (u32)heads;
        const int bg = (int)(tile - turn * (u32)heads), split = (int)(turn % (u32)a.prompt_splits), rt = row_tiles - 1 - (int)(turn / (u32)a.prompt_splits);
        const int b = (int)((u32)bg / (u32)a.kv.G), g = bg - b * a.kv.G;
        KvSeq s = kv_seq(a.kv, a.starts, a.tokens, b);
        const int n_all = s.n;
        s.n = s.n < a.max_new ? s.n : a.max_new;
        const u32 rows = (u32)s.n * R, row0 = (u32)rt * TR;
        if (rows <= (u32)a.few_rows || row0 >= rows) continue;
        const u32 last_row = min(rows, row0 + TR) - 1;
        const int most = a.causal ? max(0, s.len - n_all + (int)(last_row / R) + 1) : s.len;
        const int least = a.causal ? s.len - n_all + (int)(row0 / R) + 1 : s.len;
        // this workgroup's share of the pages; from here on pages are counted from its first
        const KvShare share = kv_share((most + kPage - 1) / kPage, a.prompt_splits, split);
        const int full = s.len / kPage - share.first, units = share.end - share.first, ufull = max(min(units, full), 0);
        const int32_t* table = a.kv.table + (int64_t)b * a.kv.max_pages + share.first;

        bf16x8 q[NQ][KK];
        const u32 rr = row0 + wid * WR + c;
        const bool live = rr < rows;
        const int qi = live ? (int)(rr / R) : 0, qh = g * a.R + (live ? (int)(rr - (u32)qi * R) : 0);
        const int lim = (!live ? 0 : a.causal ? s.len - n_all + qi + 1 : s.len) - share.first * kPage;
        const int64_t q_at = (s.first + qi) * a.q_token + qh * a.q_head + h * 8;
#pragma unroll
        for (int k = 0; k < KK; ++k) {
            bf16x8 p[NQ];
            const bool there = live && k * 16 < D - h * 8;
            if (there) QParts<DT>::load(a, q_at + k * 16, p);
#pragma unroll
            for (int i = 0; i < NQ; ++i) q[i][k] = there ? p[i] : bf16x8{};
        }

        // outputs are held in units of vref, the scale of some page; the same in all wavefronts
        float m = -__builtin_inff(), l = 0.0f, vref = 0.0f, vfirst = 0.0f;
        bool careful = false;                            // the pages have to be gone through again, see below
        f32x16 o[DL];
#pragma unroll
        for (int t = 0; t < DL; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;
        auto rescale = [&](float f) {
#pragma unroll
            for (int t = 0; t < DL; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[t][r] *= f;
        };
        auto finite_max = [&]() { return m == -__builtin_inff() ? 0.0f : m; };
        auto scores = [&](const uint16_t* keys, f32x16* sc) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) sc[t][r] = 0.0f;
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bf16x8 w = *(const bf16x8*)(keys + ((t * KK + k) * 64 + lane) * 8);
#pragma unroll
                    for (int i = 0; i < NQ; ++i) sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, q[i][k], sc[t], 0, 0, 0);
                }
        };

        uint4 kb[NR], vb[NR];
        auto mine = [&](int i) { return DP % 64 == 0 || i * 256 + tid < 4 * DP; };      // whether the thread's i-th record is one
        // places and scales of 64 pages lie in the lanes
        u32 my_page = 0;
        float my_ks = 0.0f, my_vs = 0.0f;
        auto fetch = [&](int u) {
            my_page = 0;
            my_ks = my_vs = 0.0f;
            if (u + lane < ufull) {
                const int64_t id = table[u + lane];
                const bool there = id >= 0 && id < a.kv.n_pages;
                my_page = there ? (u32)id : 0u;
                const float2 sc = *(const float2*)(a.kv.scales + ((int64_t)my_page * a.kv.G + g) * 2);
                my_ks = there ? sc.x : __uint_as_float(0x7FC00000u);
                my_vs = there ? sc.y : 0.0f;
            }
        };
        auto load_keys = [&](int lane_of) {
            const uint4* rec = (const uint4*)(a.kv.pages + kv_record(a.kv, bcast(my_page, lane_of), g));
#pragma unroll
            for (int i = 0; i < NR; ++i)
                if (mine(i)) kb[i] = rec[i * 256 + tid];
        };
        auto load_values = [&](int lane_of) {
            const uint4* rec = (const uint4*)(a.kv.pages + kv_record(a.kv, bcast(my_page, lane_of), g)) + 4 * DP;
#pragma unroll
            for (int i = 0; i < NR; ++i)
                if (mine(i)) vb[i] = rec[i * 256 + tid];
        };
        auto stage_k = [&](int which) {
#pragma unroll
            for (int i = 0; i < 2 * NR; ++i)
                if (mine(i >> 1)) stage_keys<DP>(buf[which], (i >> 1) * 256 + tid, kb[i >> 1], i & 1);
        };
        auto stage_v = [&](int which) {
#pragma unroll
            for (int i = 0; i < 4 * NR; ++i)
                if (mine(i >> 2)) stage_values<DP>(buf[which] + PromptTile<DP>::kKeys, (i >> 2) * 256 + tid, vb[i >> 2], i & 3);
        };
        // what a page's scores are multiplied by, and its value scale over vref: its logarithm and inverse.  vref follows the scales: a page's is within
        // 2^-6 .. 2 of it, so that probabilities keep their bits (a page of zeros: any).  Scales more than 2^30 from the first are not for the pipeline: a row's sums
        // in units of a page that it has no weight on would leave fp32's range
        float factor = 0.0f, lr = 0.0f, back = 1.0f;
        auto page_scales = [&](int lane_of) {
            const float ks = __uint_as_float(bcast(__float_as_uint(my_ks), lane_of)), vs = __uint_as_float(bcast(__float_as_uint(my_vs), lane_of));
            factor = ks * a.scale;
            if (vs > 2.0f * vref || (vs > 0.0f && vs < vref * 0.015625f)) {
                if (vref > 0.0f) {
                    rescale(vref / vs);
                    careful |= vs > vfirst * 0x1p30f || vs < vfirst * 0x1p-30f;
                } else {
                    vfirst = vs;
                }
                vref = vs;
            }
            const float ratio = vs > 0.0f ? vs * __builtin_amdgcn_rcpf(vref) : 1.0f;
            lr = __log2f(ratio);
            back = __builtin_amdgcn_rcpf(ratio);
        };
        // a new maximum of the lane's scores: the sums so far are scaled down to it where it is far above the old one
        auto new_maximum = [&](float mx) {
            float here;
            mx = other_half(mx, &here);
            mx = fmaxf(mx, here) * factor;               // (the factor is not negative)
            if (__any(mx > m + kSlack)) {
                const float mn = fmaxf(m, mx), alpha = exp2_of(m - (mn == -__builtin_inff() ? 0.0f : mn));
                rescale(alpha);
                l *= alpha;
                m = mn;
                careful |= fabsf(m) > kSteep && m != -__builtin_inff();
            }
        };
        auto page_weight = [&](int u, float sum) {
            if (a.mass) {
                float here;
                sum = other_half(sum, &here);
                if (h == 0) my_w[(size_t)u * TR + wid * WR + c] = float2{finite_max(), (sum + here) * back};
            }
        };
        // the lane's largest score; `mask`: rows may not see the whole page
        auto lane_max = [&](auto mask, const f32x16* sc, int u) {
            const int left = lim - u * kPage - h * 4;
            float mx = -__builtin_inff();
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) mx = fmaxf(mx, !decltype(mask)::value || t * 32 + (r >> 2) * 8 + (r & 3) < left ? sc[t][r] : -__builtin_inff());
            return mx;
        };
        // a score -> the probability times 2^8 and the page's scale over vref
        auto exponential = [&](auto mask, f32x16* sc, int e, int left, float off) {
            float f = exp2_of(__builtin_fmaf(sc[e >> 4][e & 15], factor, off));
            if constexpr (decltype(mask)::value) f = (e >> 4) * 32 + ((e & 15) >> 2) * 8 + (e & 3) < left ? f : 0.0f;
            sc[e >> 4][e & 15] = f;
            return f;
        };
        auto products = [&](const uint16_t* values, const f32x16* sc) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f16x8 p[NP];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float f = sc[k >> 1][(k & 1) * 8 + j];
                    const _Float16 hi = (_Float16)f;
                    p[0][j] = hi;
                    if constexpr (NP > 1) p[1][j] = (_Float16)(f - (float)hi);
                }
#pragma unroll
                for (int t = 0; t < DL; ++t) {
                    const f16x8 v = *(const f16x8*)(values + ((t * 4 + k) * 64 + lane) * 8);
#pragma unroll
                    for (int i = 0; i < NP; ++i) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[i], o[t], 0, 0, 0);
                }
            }
        };

        // outside the pipeline: scores -> probabilities times 2^8 under their exact maximum; returns what the sums so far are to be multiplied by
        auto weigh = [&](f32x16* sc, int u) {
            const int left = lim - u * kPage - h * 4;
            float mx = -__builtin_inff(), here, sum = 0.0f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    sc[t][r] = t * 32 + (r >> 2) * 8 + (r & 3) < left ? sc[t][r] * factor : -__builtin_inff();
                    mx = fmaxf(mx, sc[t][r]);
                }
            mx = other_half(mx, &here);
            const float mn = fmaxf(m, fmaxf(mx, here)), ms = mn == -__builtin_inff() ? 0.0f : mn, alpha = exp2_of(m - ms);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    sc[t][r] = exp2_of((sc[t][r] - ms) + kPromptBias);
                    sum += sc[t][r];
                }
            m = mn;
            l = __builtin_fmaf(l, alpha, sum);
            page_weight(u, sum);
            return alpha;
        };

        __syncthreads();                                 // (the tile before may still be read)
        if (tid == 0) xcareful = 0;
        // The pages in a pipeline: while a page's probabilities are made and multiplied by its values, the next page's scores are
        // made, and the operands of the keys behind those and of the next values go to LDS: matrix and vector instructions of one wavefront
        // run at the same time.  Page u has its keys in buf[u % 2] one step before its values.
        const int whole = min(ufull, max(least - share.first * kPage, 0) / kPage);         // pages that every row sees all of
        if (ufull > 0) {
            int base = 0;                                // page of the lanes' first place
            fetch(0);
            load_keys(0);
            load_values(0);
            stage_k(0);
            stage_v(0);
            load_keys(min(1, ufull - 1));
            stage_k(1);
            __syncthreads();
            load_keys(min(2, ufull - 1));
            load_values(min(1, ufull - 1));
            f32x16 sa[2], sb[2];
            scores(buf[0], sa);
            __syncthreads();                             // (the first step writes the keys of page 2 there)
            page_scales(0);
            new_maximum(lane_max(std::true_type(), sa, 0));
            auto step = [&](auto mask, int u, f32x16* sc, f32x16* next) {
                constexpr int NS = 4 * DL, kAhead = 3;       // operands of a page's keys, and of its values; read that far ahead
                const uint16_t *keys = buf[(u + 1) & 1], *values = buf[u & 1] + PromptTile<DP>::kKeys;
                uint4 op[2 * NS];
                auto ask = [&](int i) {
                    if (i < NS) op[i] = *(const uint4*)(keys + (((i & 1) * KK + (i >> 1)) * 64 + lane) * 8);
                    else if (i < 2 * NS) op[i] = *(const uint4*)(values + (((i - NS) % DL * 4 + (i - NS) / DL) * 64 + lane) * 8);
                };
                float part[4] = {0.0f, 0.0f, 0.0f, 0.0f}, mx = -__builtin_inff();
                const float off = kPromptBias + lr - finite_max();
                const int left = lim - u * kPage - h * 4;
                f16x8 p[2][NP];
                auto narrow = [&](int k) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float f = sc[k >> 1][(k & 1) * 8 + j];
                        const _Float16 hi = (_Float16)f;
                        p[k & 1][0][j] = hi;
                        if constexpr (NP > 1) p[k & 1][1][j] = (_Float16)(f - (float)hi);
                    }
                };
#pragma unroll
                for (int i = 0; i < kAhead; ++i) ask(i);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) next[t][r] = 0.0f;
                // every product is followed by the vector instructions that run beside it, in an order that the compiler may not change (left to it, products
                // came in a row, each behind a wait for its operand)
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    ask(i + kAhead);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) next[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf16_of(op[i]), q[n][i >> 1], next[i & 1], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int e = i * 32 / NS; e < (i + 1) * 32 / NS; ++e) part[e & 3] += exponential(mask, sc, e, left, off);
                    __builtin_amdgcn_sched_barrier(0);
                }
                narrow(0);
                const float sum = (part[0] + part[1]) + (part[2] + part[3]);
                l = __builtin_fmaf(sum, back, l);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    const int k = i / DL, t = i % DL;
                    ask(NS + i + kAhead);
#pragma unroll
                    for (int n = 0; n < NP; ++n) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, op[NS + i]), p[k & 1][n], o[t], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if (t == DL - 1 && k < 3) narrow(k + 1);
#pragma unroll
                    for (int e = 0; e < 6 * NR; ++e) {       // what goes to LDS, in pieces: four of a record of values, two of a record of keys
                        if (e * NS / (6 * NR) != i) continue;
                        const int rec = e / 6, piece = e % 6;
                        if (!mine(rec)) continue;
                        if (piece < 2) stage_keys<DP>(buf[u & 1], rec * 256 + tid, kb[rec], piece);
                        else stage_values<DP>(buf[(u + 1) & 1] + PromptTile<DP>::kKeys, rec * 256 + tid, vb[rec], piece - 2);
                    }
#pragma unroll
                    for (int e = i * 32 / NS; e < (i + 1) * 32 / NS; ++e) {
                        const int t = e / 16, r = e % 16;
                        mx = fmaxf(mx, !decltype(mask)::value || t * 32 + (r >> 2) * 8 + (r & 3) + kPage < left ? next[t][r] : -__builtin_inff());
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                page_weight(u, sum);
                if (u + 4 - base > 64) {                 // (places up to u + 3 are asked for below)
                    base = u;
                    fetch(u);
                }
                load_keys(min(u + 3, ufull - 1) - base);
                load_values(min(u + 2, ufull - 1) - base);
                page_scales(u + 1 - base);
                new_maximum(mx);
                __syncthreads();
            };
            int u = 0;
            // (a choice between the two for every page had the compiler put 744 bytes a lane into scratch memory: 1860 us instead of 400)
            for (; u + 2 < whole; u += 2) {
                step(std::false_type(), u, sa, sb);
                step(std::false_type(), u + 1, sb, sa);
            }
            for (; u + 2 < ufull; u += 2) {
                step(std::true_type(), u, sa, sb);
                step(std::true_type(), u + 1, sb, sa);
            }
            if (u + 1 < ufull) {
                step(std::true_type(), u, sa, sb);
                ++u;
#pragma unroll
                for (int t = 0; t < 2; ++t) sa[t] = sb[t];
            }
            // the last page
            const float off = kPromptBias + lr - finite_max();
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 32; ++e) sum += exponential(std::true_type(), sa, e, lim - u * kPage - h * 4, off);
            l = __builtin_fmaf(sum, back, l);
            page_weight(u, sum);
            products(buf[u & 1] + PromptTile<DP>::kKeys, sa);
            if (careful) xcareful = 1;
            __syncthreads();
            if (xcareful) {
                // what the pipeline cannot hold: page after page, the products of each on their own, outputs in units of 1
                vref = back = 1.0f;
                m = -__builtin_inff();
                l = 0.0f;
#pragma unroll
                for (int t = 0; t < DL; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;
                for (u = 0; u < ufull; ++u) {
                    if ((u & 63) == 0) fetch(u);
                    load_keys(u & 63);
                    load_values(u & 63);
                    __syncthreads();
                    stage_k(0);
                    stage_v(0);
                    __syncthreads();
                    factor = __uint_as_float(bcast(__float_as_uint(my_ks), u & 63)) * a.scale;
                    const float vs = __uint_as_float(bcast(__float_as_uint(my_vs), u & 63));
                    scores(buf[0], sa);
                    const float alpha = weigh(sa, u);
                    f16x8 p[4][NP];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const float f = sa[e >> 4][e & 15];
                        const _Float16 hi = (_Float16)f;
                        p[e >> 3][0][e & 7] = hi;
                        if constexpr (NP > 1) p[e >> 3][1][e & 7] = (_Float16)(f - (float)hi);
                    }
#pragma unroll
                    for (int t = 0; t < DL; ++t) {
                        f32x16 acc;
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const f16x8 v = *(const f16x8*)(buf[0] + PromptTile<DP>::kKeys + ((t * 4 + k) * 64 + lane) * 8);
#pragma unroll
                            for (int i = 0; i < NP; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[k][i], acc, 0, 0, 0);
                        }
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[t][r] = __builtin_fmaf(acc[r], vs, o[t][r] * alpha);
                    }
                }
            }
        }
        if (units > max(full, 0)) {                      // the tail is in this share
            const int count = s.len % kPage;
            __syncthreads();
            stage_tail<DP>(buf[0], buf[0] + PromptTile<DP>::kKeys, a.kv.tails + kv_tail(a.kv, b, g), count, tid);
            __syncthreads();
            f32x16 sc[2];
            scores(buf[0], sc);
            factor = a.scale;
            back = 1.0f;
            const uint16_t* values = buf[0] + PromptTile<DP>::kKeys;
            rescale(weigh(sc, full) * vref);
            vref = 1.0f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                bf16x8 p[NB];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float f = sc[k >> 1][(k & 1) * 8 + j];
#pragma unroll
                    for (int i = 0; i < NB; ++i) {
                        p[i][j] = (__bf16)f;
                        f -= (float)p[i][j];
                    }
                }
#pragma unroll
                for (int t = 0; t < DL; ++t) {
                    const bf16x8 v = *(const bf16x8*)(values + ((t * 4 + k) * 64 + lane) * 8);
#pragma unroll
                    for (int i = 0; i < NB; ++i) o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[i], o[t], 0, 0, 0);
                }
            }
        }
        float here;
        l = other_half(l, &here);
        l += here;
        if (live) {
            const int64_t at = (s.first + qi) * a.H + qh, slot = (((int64_t)bg * row_tiles + rt) * TR + wid * WR + c) * a.prompt_splits + split;
            const float f = a.prompt_splits > 1 ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;      // (not times vref at once: that may leave fp32's normal range)
#pragma unroll
            for (int t = 0; t < DL; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int d = t * 32 + k * 8;
                    const f32x4 v = f32x4{o[t][k * 4], o[t][k * 4 + 1], o[t][k * 4 + 2], o[t][k * 4 + 3]} * f * vref;
                    if (a.prompt_splits > 1) *(f32x4*)(a.prompt_o + slot * DP + h * 4 + d) = v;
                    else if (d < D - h * 4) store4<DT>(a.out, at * D + h * 4 + d, v);
                }
            if (h == 0) {
                if (a.prompt_splits > 1) a.prompt_ml[slot] = float2{m, l};
                else if (a.lse) a.lse[at] = l == 0.0f ? -__builtin_inff() : (finite_max() - kPromptBias + __log2f(l)) * kLn2;
            }
        }
        if (a.mass && a.prompt_splits == 1) {
            // a page's sums of the tile's rows, now that the rows' own are known
            if (h == 0) xrow[wid * WR + c] = float2{finite_max(), live ? 1.0f / l : 0.0f};
            __syncthreads();                             // (also for the stores to my_w)
            const float2 r0 = xrow[lane], r1 = xrow[lane + 64];
            float* to = a.tile_mass + ((int64_t)bg * row_tiles + rt) * a.kv.max_pages;
            const int pages = (s.len + kPage - 1) / kPage;
            for (int p0 = wid * 4; p0 < pages; p0 += 16) {       // four pages' loads at a time
                float2 w[4][2];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const size_t from = (size_t)min(p0 + e, max(units - 1, 0)) * TR + lane;
                    w[e][0] = my_w[from];
                    w[e][1] = my_w[from + 64];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float sum = kv_weight(w[e][0], r0) + kv_weight(w[e][1], r1);
#pragma unroll
                    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
                    if (lane == 0 && p0 + e < pages) to[p0 + e] = p0 + e < units ? sum : 0.0f;
                }
            }
        }
    }
}

// Rows of prompts whose pages were shared out (few row tiles before a long cache): a wavefront per row, several parts a load.  (A workgroup per row, as for the split
// rows, whose parts are many: 35 us for 29000 rows of two parts.)  With weights, the rows' totals are kept for the pages' sums.
template <int DT, int DP>
__global__ __launch_bounds__(256) void kv_prompt_join_kernel(KvAttendArgs a, int row_tiles)
{
    constexpr int LPP = DP / 4, PPW = kWave / LPP;       // lanes a part, parts a load
    const int lane = threadIdx.x & 63, D = a.kv.D, splits = a.prompt_splits;
    const u32 row = blockIdx.x * 4 + (threadIdx.x >> 6), per_head = (u32)row_tiles * kTileRows;
    const int bg = (int)(row / per_head), b = bg / a.kv.G, g = bg - b * a.kv.G;
    const u32 r = row - (u32)bg * per_head;
    const KvSeq s = kv_seq(a.kv, a.starts, a.tokens, b);
    const u32 rows = (u32)min(s.n, a.max_new) * (u32)a.R;
    if (rows <= (u32)a.few_rows || r >= rows) return;
    const u32 token = r / (u32)a.R;
    const int64_t at = (s.first + token) * a.H + g * a.R + (r - token * (u32)a.R);
    const float2* ml = a.prompt_ml + (size_t)row * splits;
    const float* parts = a.prompt_o + (size_t)row * splits * DP;
    const float2 total = kv_row_total(ml, splits, lane);
    const int part = PPW > 1 ? lane / LPP : 0, d = (PPW > 1 ? lane % LPP : lane) * 4;
    f32x4 v = {0, 0, 0, 0};
    if (part < PPW && d < D) {
#pragma unroll 4
        for (int i = part; i < splits; i += PPW) v += *(const f32x4*)(parts + (size_t)i * DP + d) * exp2_of(ml[i].x - total.x);
    }
    if constexpr (PPW > 1) {
#pragma unroll
        for (int q = 1; q < PPW; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float f = __shfl(v[e], (lane + q * LPP) & 63);
                if (part == 0) v[e] += f;
            }
    }
    if (part == 0 && d < D) store4<DT>(a.out, at * D + d, v * (total.y == 0.0f ? 0.0f : 1.0f / total.y));
    if (lane == 0 && a.lse) a.lse[at] = total.y == 0.0f ? -__builtin_inff() : (total.x - kPromptBias + __log2f(total.y)) * kLn2;
    if (lane == 0 && a.mass) a.row_total[row] = float2{total.x, 1.0f / total.y};
}

// The pages' weights over the row tiles, in their order: of tiles that have summed their rows' up, or (pages shared out) over the rows, a wavefront a page.
template <int DT>
__global__ __launch_bounds__(256) void kv_mass_kernel(KvAttendArgs a, int row_tiles, int page_blocks)
{
    const int bg = blockIdx.x / page_blocks, b = bg / a.kv.G;
    const KvSeq s = kv_seq(a.kv, a.starts, a.tokens, b);
    const int n = min(s.n, a.max_new);
    const int64_t rows = (int64_t)n * a.R;
    if (rows <= a.few_rows) return;
    const int tiles = (int)((rows + kTileRows - 1) / kTileRows), pages = (s.len + kPage - 1) / kPage;
    float* const mass = a.mass + (int64_t)bg * a.kv.max_pages;
    if (a.prompt_splits == 1) {
        for (int p = blockIdx.x % page_blocks * 256 + threadIdx.x; p < pages; p += page_blocks * 256) {
            const float* from = a.tile_mass + (int64_t)bg * row_tiles * a.kv.max_pages + p;
            float sum = 0.0f;
#pragma unroll 8
            for (int t = 0; t < tiles; ++t) sum += from[(int64_t)t * a.kv.max_pages];
            mass[p] = a.decay == 0.0f ? sum : __builtin_fmaf(mass[p], a.decay, sum);
        }
        return;
    }
    const int heads = a.kv.seqs * a.kv.G, lane = threadIdx.x & 63;
    for (int p = blockIdx.x % page_blocks * 4 + (threadIdx.x >> 6); p < pages; p += page_blocks * 4) {
        float sum = 0.0f;
        for (int t = 0; t < tiles; ++t) {
            const int64_t last_row = min(rows, (int64_t)(t + 1) * kTileRows) - 1;
            const int most = a.causal ? max(0, s.len - s.n + (int)(last_row / a.R) + 1) : s.len, units = (most + kPage - 1) / kPage;
            if (p >= units) continue;
            const int split = p / kv_share(units, a.prompt_splits, 0).end;
            const size_t slot = ((size_t)(row_tiles - 1 - t) * a.prompt_splits + split) * heads + bg;
            const float2* w = a.row_w + (slot * a.slot_pages + (p - kv_share(units, a.prompt_splits, split).first)) * kTileRows;
            const float2* total = a.row_total + ((int64_t)bg * row_tiles + t) * kTileRows;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if ((int64_t)t * kTileRows + i * 64 + lane < rows) sum += kv_weight(w[i * 64 + lane], total[i * 64 + lane]);
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        if (lane == 0) mass[p] = a.decay == 0.0f ? sum : __builtin_fmaf(mass[p], a.decay, sum);
    }
}

}  // namespace slicer
