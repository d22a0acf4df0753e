// Causal attention of a flattened batch's rows over a paged cache of 8-bit keys and values.
//
//   x_s = scale q . k_s (or cap tanh(x_s / cap)),   out = sum_s 2^(l x_s - m) v_s / sum_s 2^(l x_s - m),   l = log2(e), m the row's largest l x_s
//
// computed in one pass over the tokens: m, the sum and the unnormalised output are kept in fp32 and scaled when m grows.
//
// Scores: v_mfma_scale_f32_*_f8f6f4 takes the keys' bytes as they lie and their page's E8M0 scale beside them, so no key is widened.  A bf16 query has eight significant bits,
// two E4M3 terms: q = (hi + lo / 16) 2^e exactly for elements from 2^-13 of the row's largest on (others to 2^-21 of it), one product each, which at twice
// bf16's rate is what a bf16 product would cost.  Inside one instruction the matrix unit drops what lies more than about 2^-15 below its largest product: measured
// relative errors of 1e-5 to 5e-5 of a sum, not growing with the number of instructions (the accumulator is full fp32).
// Outputs: weights as bf16 (2^-9 of each; their sum is taken before they are rounded), values widened to bf16, exactly, scale included (v_cvt_scalef32_pk_bf16_fp8: two
// elements in 4 clocks).  The weights as two E4M3 terms would spare that, but v_cvt_pk_fp8_f32 takes 16 clocks for two elements: 22 clocks a weight against 2,
// and the widening is done once for many rows.
//
// The scores are formed as K Q^T, tokens down the rows of the result: a lane then holds tokens of ONE query row, in the order in which the
// instruction wants them as the right operand of V^T P^T.  No score crosses lanes but for the row's maximum and sum, and none goes through shared memory.
//
// Measured: a prompt of 8192 tokens, 32 query on 16 key heads of 128, 533 to 540 us or 1.0 PFLOP/s where a large bf16 product reaches 1.3: matrix unit busy 45 % of the cycles, vector
// instructions (softmax, and values on their way to shared memory) 48 %, and two wavefronts of a SIMD overlap the two only in part.  Decode steps are bound by memory: 48 clients with up to
// 4096 tokens in the window, 538 MB, 98 us or 5.5 TB/s.  With 48 query heads on one key head (16 clients, contexts to 131072, 196 MB and 18.7 GFLOP) 53 us, 3.7 TB/s: one wavefront a SIMD.
#pragma once
#include <type_traits>

#include "block_device.hpp"

namespace symb {

// ---- up to 48 rows ----------------------------------------------------------------------------------------------------------------
// In a chunk of 64 tokens, lane (n = lane % 16, g = lane / 16) gives
//   left operand, keys    tile s (0..3): token kv_token(s, n), elements 16g .. 16g+15 and (head of 128) 64+16g .., its page's scale
//   right operand         query row n, the same elements
//   result                tokens kv_token(s, 4g + r), r = 0..3, of row n: all four tiles' are the tokens 16g .. 16g+15
//   left operand, values  channel 16j + n, step q (0, 1): tokens 16g + 8q .. +7, half of 16 bytes as they lie in the cache
constexpr int kKvChunk = 64;              // tokens
// A row's weights are 2^(x - m) with an m that its largest x may exceed by up to this: the outputs need not be scaled whenever a larger score comes.  bf16 and fp32 hold the
// weights just as well.
constexpr float kKvSlack = 8.f;

// A run of tokens for some of the query rows of one key head.  Row r of a segment's key head is query head r % group of token r / group.
struct KvItem {
    int32_t table;                        // the segment's first entry in the page table
    int32_t row0, rows;                   // its first row in the batch; its rows times the query heads of a key head
    int32_t past;
    int32_t r0;                           // the item's first row
    int32_t begin, end;                   // tokens: a multiple of the chunk; one past the last that any of the rows sees
    int32_t part;                         // partial result's first row, -1: the item is all there is
};

struct KvAttentionParams {
    const KvItem* items;
    int32_t tiles;                        // how many of them are tiles of 128 rows: the first ones
    const int32_t* page_table;
    const unsigned char* k;
    const unsigned char* v;
    const unsigned char* k_scale;
    const unsigned char* v_scale;
    const bf16* q;
    bf16* out;
    float* part_o;                        // [part rows][D], unnormalised
    float* part_ml;                       // [part rows][2]: maximum (log2 units, never NaN), sum (NaN in a row that is)
    int64_t q_stride, out_stride;
    int32_t num_pages, kv_heads, group, page_shift, window;
    int32_t part_rows;                    // of one key head
    float scale;                          // log2(e) times it
    float cap, to_cap;                    // cap / scale, and kKvRoot scale / cap: the scores are capped before they are scaled
};

__device__ __forceinline__ int kv_token(int s, int m) { return 16 * (m >> 2) + 4 * s + (m & 3); }

// Four values as two E4M3 terms each, hi + lo / 16.
__device__ __forceinline__ void kv_two_terms(float a, float b, float c, float d, int& hi, int& lo) {
    hi = pack4_e4m3(a, b, c, d);
    const floatx2 u = e4m3_lo(hi), w = e4m3_hi(hi);
    typedef __attribute__((__vector_size__(2 * sizeof(short)))) short shortx2;
    shortx2 v = {0, 0};                                            // (converts what it is given over 1/16)
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, a - u[0], b - u[1], 0.0625f, false);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, c - w[0], d - w[1], 0.0625f, true);
    lo = __builtin_bit_cast(int, v);
}
// amax / 2^e in [128, 256): infinities and NaN in a query become NaN.
__device__ __forceinline__ int kv_query_exponent(float amax) { return max((as_int(amax) >> 23) - 127 - 7, -100); }

// A query row as right operand, in two E4M3 terms, and its scales.  Head of 128: hi and lo are operands of their own.  Head of 64: hi holds both, the elements
// with lo's in the upper half of the 128.
template <int D>
struct KvQuery {
    intx8 hi, lo;
    int hi_scale, lo_scale;
};
template <int D>
__device__ __forceinline__ void kv_query(KvQuery<D>& o, const bf16* q, bool valid, int g) {
    float x[D / 4];
    float amax = 0.f;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {                             // chunks of eight: elements 16g + 8(c % 2) + 64(c / 2)
        intx4 w = intx4{0, 0, 0, 0};
        if (valid) w = *(const intx4*)(q + 16 * g + 8 * (c & 1) + 64 * (c >> 1));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[8 * c + 2 * i] = bf16_lo((unsigned)w[i]);
            x[8 * c + 2 * i + 1] = bf16_hi((unsigned)w[i]);
            amax = fmaxf(amax, fmaxf(finite_abs(x[8 * c + 2 * i]), finite_abs(x[8 * c + 2 * i + 1])));
        }
    }
    amax = across_rows(amax, Max());
    const int e = kv_query_exponent(amax);
    const float inv = pow2(-e);
    int hi[D / 16], lo[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) kv_two_terms(x[4 * i] * inv, x[4 * i + 1] * inv, x[4 * i + 2] * inv, x[4 * i + 3] * inv, hi[i], lo[i]);
    if constexpr (D == 128) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o.hi[i] = hi[i], o.lo[i] = lo[i];
        o.hi_scale = e + 127;
        o.lo_scale = e + 123;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) o.hi[i] = hi[i], o.hi[4 + i] = lo[i];
        o.hi_scale = g < 2 ? e + 127 : e + 123;
    }
}

__device__ __forceinline__ floatx4 kv_mfma(const intx8& a, const intx8& b, const floatx4& c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}

// Behind the last matrix instruction of a loop, before its results are read in other code: the 19 wait states that the longest of them needs.
__device__ __forceinline__ void kv_settle() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 3");
    __builtin_amdgcn_sched_barrier(0);
}

// Scores s, not yet scaled, to cap tanh(s / cap).  With y = s / cap, cap (1 - 2 / (e^2y + 1)) is good to 2^-21 of the cap or so, which far below the cap may be more than the score itself: there it is the
// series s (1 - y^2 / 3 + 2 y^4 / 15 - 17 y^6 / 315), whose next term is 2^-21 of s at y = 1/4.  Either way a score is off by 2^-19 of itself at most, whatever the cap.  Where no score of a
// wavefront's chunk has come up to a quarter of the cap, which models choose well above their scores, the series is all there is, and no instruction of it is a transcendental one.
// The series is formed in z = (r y)^2, r the 6th root of 17 / 315, as s + s z (z (2 / (15 r^4) - z) - 1 / (3 r^2)): two instructions with a literal each, and no constant in a register.
// Measured: a prompt of 8192 tokens, 16 heads of 64, capped, 285 us (260 with the first formula alone, 171 without a cap); 32 on 16 heads of 128, 4 prompts of 8192 tokens in all, 253 (244); decode steps, bound
// by memory, as before.
constexpr float kKvSeries = 0.25f, kKvRoot = 0.6147375f;
template <class V, int N>
__device__ __forceinline__ void kv_cap(const KvAttentionParams& p, V (&s)[N]) {
    constexpr int kEach = sizeof(V) / sizeof(float);
    auto series = [&](float x) {
        const float u = x * p.to_cap, z = u * u;
        return __builtin_fmaf(x * z, __builtin_fmaf(z, 0.9336408f - z, -0.8820624f), x);
    };
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < kEach; ++e) top = fmaxf(top, fabsf(s[i][e]));
    if (__any(top * p.to_cap > kKvSeries * kKvRoot)) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                float x = s[i][e];
                asm volatile("" : "+v"(x));                        // (its series is formed here, not ahead of the branch: registers)
                const float u = x * p.to_cap;
                float far = p.cap * (1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(u * (2.885390082f / kKvRoot)) + 1.f)), near = series(x);
                asm volatile("" : "+v"(far), "+v"(near));          // (both: the compiler would branch for every score)
                s[i][e] = fabsf(u) > kKvSeries * kKvRoot ? far : near;
                if (e & 1) __builtin_amdgcn_sched_barrier(0);      // (two at a time: registers)
            }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < kEach; ++e) s[i][e] = series(s[i][e]);
    }
}

// The page of a token, the same in all lanes, so through the scalar cache: page numbers then arrive beside the keys and values under way, not behind them.  Only pages of the tokens
// lo .. hi-1 are looked up (others are hidden: any page will do); for a number outside the pool page 0 is read, with a key scale of 0xff: its tokens' scores
// are NaN, so the rows that see them are, and the others are none the wiser.
__device__ __forceinline__ int kv_look_up(const KvAttentionParams& p, int table, int token, int lo, int hi) {
    typedef const __attribute__((address_space(4))) int32_t* Table;
    return ((Table)(uintptr_t)p.page_table)[table + (max(min(token, hi - 1), lo) >> p.page_shift)];
}
__device__ __forceinline__ int kv_outside(const KvAttentionParams& p, int page) { return (unsigned)page < (unsigned)p.num_pages ? 0 : 0xff; }      // (to be or'd with the scale)
__device__ __forceinline__ int kv_in_pool(int page, int outside) { return outside ? 0 : page; }

__device__ __forceinline__ float kv_scale(int byte) { return as_float(byte << 23); }
// Eight E4M3 values times a power of two as bf16.
__device__ __forceinline__ bf16x8 kv_widen(int a, int b, float scale) {
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    const bf16x2 w[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true)};
    return bf16x8{w[0][0], w[0][1], w[1][0], w[1][1], w[2][0], w[2][1], w[3][0], w[3][1]};
}
__device__ __forceinline__ bf16x8 kv_pack8(float a, float b, float c, float d, float e, float f, float g, float h) {
    return __builtin_bit_cast(bf16x8, intx4{(int)pack2_bf16(a, b), (int)pack2_bf16(c, d), (int)pack2_bf16(e, f), (int)pack2_bf16(g, h)});
}

// What a hidden token holds must not meet a weight, 0 x NaN being NaN.  Where not every row sees every token, values of tokens that no row sees (outside lo .. hi-1) are cleared, and so
// are NaN, infinities with them, among the others; if there are any, the rows that see them get them in a pass of its own: ones in their places times ones where a row sees the token.
__device__ __forceinline__ int kv_keep_bytes(int t, int lo, int hi) {      // of four tokens' bytes, t .. t+3: ones where a token is in lo .. hi-1
    const int a = lo - t, b = hi - t;
    const unsigned below = b >= 4 ? ~0u : b > 0 ? (1u << (8 * b)) - 1 : 0u;
    const unsigned above = a <= 0 ? ~0u : a < 4 ? ~0u << (8 * a) : 0u;
    return (int)(below & above);
}
// 0xff in the place of each E4M3 byte that is NaN or, at its page's scale of 2^(byte - 127), 2^128 or more: as bf16 those widen to infinity.  From byte 247 on that begins at code (262 - byte) << 3;
// byte 255 makes NaN of every code.  `step` takes the first of them to the sign bit.
__device__ __forceinline__ unsigned kv_nan_step(int byte) { return 0x01010101u * (unsigned)(byte < 247 ? 1 : byte < 255 ? 8 * (byte - 246) : 128); }
__device__ __forceinline__ int kv_nan_bytes(int w, unsigned step) { return (int)((((((unsigned)w & 0x7f7f7f7fu) + step) & 0x80808080u) >> 7) * 255u); }
// The scale of what is left: a zero at scale 255 would be NaN again.
__device__ __forceinline__ int kv_clean_scale(int byte) { return min(byte, 254); }
// Four wavefronts share an item's tokens, chunk by chunk, each for all of its R x 16 rows, and join through shared memory.  Keys and values go straight from memory into
// registers, the next chunk's keys and this one's values while this one's scores are formed: up to 16 KB on their way in every wavefront, and two wavefronts a SIMD for up to
// 16 rows, one for more.
template <int D, int R>
struct KvRowsShared {
    float join[4][16][D + 4];
    float stat[R][4][16][2];
};
template <int D, int R, bool CAP>
__device__ __forceinline__ void kv_rows(const KvAttentionParams& p, const KvItem& it, int h, KvRowsShared<D, R>& shared) {
    constexpr int kTiles = D / 16, kWords = D / 64;
    auto& join = shared.join;
    auto& stat = shared.stat;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    // tokens that this lane's rows see (from the window's on: see_lo); those that every row of the item sees, and those that some row does
    int see_hi[R];
    auto see_lo = [&](int hi) { return p.window ? max(hi - p.window, 0) : 0; };
    const int last = min(it.r0 + 16 * R - 1, it.rows - 1);
    const int all_hi = it.past + it.r0 / p.group + 1, all_lo = p.window ? max(it.past + last / p.group + 1 - p.window, 0) : 0;
    const int any_hi = it.past + last / p.group + 1, any_lo = p.window ? max(all_hi - p.window, 0) : 0;
    KvQuery<D> q[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = it.r0 + 16 * r + n, pos = it.past + row / p.group;
        const bool valid = row < it.rows;
        see_hi[r] = valid ? pos + 1 : 0;
        kv_query<D>(q[r], p.q + (int64_t)(it.row0 + row / p.group) * p.q_stride + (h * p.group + row % p.group) * D, valid, g);
    }
    floatx4 o[R][kTiles];
    float m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int j = 0; j < kTiles; ++j) o[r][j] = floatx4{0, 0, 0, 0};
    }
    struct Keys {
        intx4 k[4][kWords];
        int scale, outside0, outside1;
    };
    const int in_page = (1 << p.page_shift) - 1;
    int page0, page1, next0, next1;                                // of a chunk's first and last 32 tokens, in the pool; numbers of the chunk whose keys are asked for next
    auto look_up = [&](int t) {
        next0 = kv_look_up(p, it.table, t, any_lo, it.end);
        next1 = kv_look_up(p, it.table, t + 32, any_lo, it.end);
    };
    auto ask_keys = [&](Keys& c, int t0) {
        c.outside0 = kv_outside(p, next0);
        c.outside1 = kv_outside(p, next1);
        page0 = kv_in_pool(next0, c.outside0);
        page1 = kv_in_pool(next1, c.outside1);
        look_up(t0 + 4 * kKvChunk);
        const int64_t block = (int64_t)(n & 8 ? page1 : page0) * p.kv_heads + h;
        const unsigned char* k = p.k + ((block << p.page_shift) + ((t0 + kv_token(0, n)) & in_page)) * D + 16 * g;
        c.scale = p.k_scale[block];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int w = 0; w < kWords; ++w) c.k[s][w] = *(const intx4*)(k + 4 * s * D + 64 * w);
    };
    intx4 v[kTiles];
    int vscale;
    auto ask_values = [&](int t0) {
        const int64_t block = (int64_t)(g & 2 ? page1 : page0) * p.kv_heads + h;
        const unsigned char* at = p.v + ((block * D + n) << p.page_shift) + ((t0 + 16 * g) & in_page);
        vscale = p.v_scale[block];
#pragma unroll
        for (int j = 0; j < kTiles; ++j) v[j] = *(const intx4*)(at + ((16 * j) << p.page_shift));
    };
    auto work = [&](const Keys& c, int t0) {
        const bool whole = t0 >= all_lo && t0 + kKvChunk <= all_hi;                    // every row sees all of it
        const int kscale = c.scale | (n & 8 ? c.outside1 : c.outside0);
        bf16x8 w[R][2];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            floatx4 s[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const intx8 a = __builtin_shufflevector(c.k[i][0], c.k[i][kWords - 1], 0, 1, 2, 3, 4, 5, 6, 7);
                s[i] = kv_mfma(a, q[r].hi, floatx4{0, 0, 0, 0}, kscale, q[r].hi_scale);
                if constexpr (D == 128) s[i] = kv_mfma(a, q[r].lo, s[i], kscale, q[r].lo_scale);
            }
            kv_settle();
            if constexpr (CAP) kv_cap(p, s);
            if (!whole) {
                int end = see_hi[r];
                asm volatile("" : "+v"(end));                      // (a branch: as a selection it would cost every chunk three instructions a score, and the window's end a register)
                const int hi = end - t0 - 16 * g, lo = see_lo(end) - t0 - 16 * g;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[i][e] = 4 * i + e < hi && 4 * i + e >= lo ? s[i][e] : -INFINITY;
            }
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, s[i][e]);
            top = across_rows(top, Max()) * p.scale;               // (the scores stay as they are: their factor goes into the exponent)
            // m follows the row's maximum once that has outgrown it 2^kKvSlack-fold
            if (__any(top > m[r] + kKvSlack)) {
                top = fmaxf(m[r], top);
                const float shrink = __builtin_amdgcn_exp2f(m[r] - (top == -INFINITY ? 0.f : top));
                m[r] = top;
                l[r] *= shrink;
#pragma unroll
                for (int j = 0; j < kTiles; ++j) o[r][j] *= shrink;
            }
            const float base = m[r] == -INFINITY ? 0.f : -m[r];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[i][e] = __builtin_amdgcn_exp2f(s[i][e] * p.scale + base);
                    l[r] += s[i][e];
                }
#pragma unroll
            for (int i = 0; i < 2; ++i) w[r][i] = kv_pack8(s[2 * i][0], s[2 * i][1], s[2 * i][2], s[2 * i][3], s[2 * i + 1][0], s[2 * i + 1][1], s[2 * i + 1][2], s[2 * i + 1][3]);
        }
        if (!whole) {
            int keep[4], found = 0;
            unsigned step = kv_nan_step(vscale);
#pragma unroll
            for (int i = 0; i < 4; ++i) keep[i] = kv_keep_bytes(t0 + 16 * g + 4 * i, any_lo, any_hi);
#pragma unroll
            for (int j = 0; j < kTiles; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[j][i] &= keep[i];
                    found |= kv_nan_bytes(v[j][i], step);
                }
            if (__any(found != 0)) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    intx8 seen, is;
                    asm volatile("" : "+v"(step));                 // (found again where they are needed, not kept: registers)
                    int end = see_hi[r];
                    asm volatile("" : "+v"(end));
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        seen[i] = 0x38383838 & kv_keep_bytes(t0 + 16 * g + 4 * i, see_lo(end), end);               // (1)
                        seen[4 + i] = is[4 + i] = 0;
                    }
#pragma unroll
                    for (int j = 0; j < kTiles; ++j) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) is[i] = kv_nan_bytes(v[j][i], step) & 0x38383838;
                        const floatx4 cnt = kv_mfma(is, seen, floatx4{0, 0, 0, 0}, 127, 127);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[r][j][e] += cnt[e] != 0.f ? NAN : 0.f;
                        __builtin_amdgcn_sched_barrier(0);         // (one at a time: registers)
                    }
                }
                asm volatile("" : "+v"(step));
#pragma unroll
                for (int j = 0; j < kTiles; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[j][i] &= ~kv_nan_bytes(v[j][i], step);
            }
            vscale = kv_clean_scale(vscale);
        }
        const float scale = kv_scale(vscale);
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bf16x8 b = kv_widen(v[j][2 * i], v[j][2 * i + 1], scale);
#pragma unroll
                for (int r = 0; r < R; ++r) o[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, w[r][i], o[r][j], 0, 0, 0);
            }
            if (j & 1) __builtin_amdgcn_sched_barrier(0);
        }
        kv_settle();                                               // (the next chunk may scale the outputs at once)
    };
    Keys even, odd;
    int t0 = it.begin + wave * kKvChunk;
    if (t0 < it.end) {
        look_up(t0);
        ask_keys(even, t0);
    }
    while (t0 < it.end) {
        const int t1 = t0 + 4 * kKvChunk, t2 = t1 + 4 * kKvChunk;
        ask_values(t0);
        if (t1 < it.end) ask_keys(odd, t1);
        work(even, t0);
        if (t1 >= it.end) break;
        ask_values(t1);
        if (t2 < it.end) ask_keys(even, t2);
        work(odd, t1);
        t0 = t2;
    }
    // the four wavefronts' results: o 2^(m - M) added up, and so the sums
#pragma unroll
    for (int r = 0; r < R; ++r) {
        l[r] = across_rows(l[r], Add());
        if (g == 0) {
            stat[r][wave][n][0] = m[r];
            stat[r][wave][n][1] = l[r];
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        __syncthreads();
        float M = -INFINITY, sum = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) M = fmaxf(M, stat[r][k][n][0]);
        const float base = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += stat[r][k][n][1] * __builtin_amdgcn_exp2f(stat[r][k][n][0] - base);
        // without parts the outputs leave here as they are: the division goes into the factor
        const float mine = __builtin_amdgcn_exp2f(m[r] - base) * (it.part >= 0 ? 1.f : 1.f / sum);
#pragma unroll
        for (int j = 0; j < kTiles; ++j) *(floatx4*)&join[wave][n][16 * j + 4 * g] = o[r][j] * mine;
        if (it.part >= 0 && wave == 0 && g == 0 && it.r0 + 16 * r + n < it.rows) {
            float* ml = p.part_ml + ((int64_t)h * p.part_rows + it.part + 16 * r + n) * 2;
            ml[0] = M;
            ml[1] = sum;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 16 * D / 4; i += 256) {
            const int row = i / (D / 4), d = i % (D / 4) * 4, rr = it.r0 + 16 * r + row;
            if (rr >= it.rows) continue;
            floatx4 v = *(const floatx4*)&join[0][row][d];
#pragma unroll
            for (int k = 1; k < 4; ++k) v += *(const floatx4*)&join[k][row][d];
            if (it.part >= 0)
                *(floatx4*)(p.part_o + ((int64_t)h * p.part_rows + it.part + 16 * r + row) * D + d) = v;
            else
                *(intx2*)(p.out + (int64_t)(it.row0 + rr / p.group) * p.out_stride + (h * p.group + rr % p.group) * D + d) = intx2{(int)pack2_bf16(v[0], v[1]), (int)pack2_bf16(v[2], v[3])};
        }
    }
}

// ---- tiles of 128 rows ------------------------------------------------------------------------------------------------------------
// Prompts: four wavefronts with 32 rows each on the same tokens, 64 at a time through shared memory, keys as they are, values widened on the way.  In a chunk of 64
// tokens, lane (n = lane % 32, g = lane / 32) gives
//   left operand, keys    tile u (0, 1): token kv_tile_token(u, n), elements 64w + 16g .. and 64w + 32 + 16g .. (w: half of a head of 128)
//   right operand         query row n, the same elements
//   result                element e: token 32u + 16(e / 8) + 8g + e % 8 of row n
//   left operand, values  channel 32j + n, step q (0..3): tokens 16q + 8g .. +7
constexpr int kKvTileRows = 128, kKvTileChunk = 64;

__device__ __forceinline__ int kv_tile_token(int u, int m) { return 32 * u + 16 * (m >> 4) + 8 * ((m >> 2) & 1) + 4 * ((m >> 3) & 1) + (m & 3); }

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float kv_floatx16;
__device__ __forceinline__ kv_floatx16 kv_mfma32(const intx8& a, const intx8& b, const kv_floatx16& c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}
// f over the two halves of the wavefront.
template <class F>
__device__ __forceinline__ float across_halves(float v, F f) {
    auto b = __builtin_amdgcn_permlane32_swap(as_int(v), as_int(v), false, false);
    return f(as_float((int)b[0]), as_float((int)b[1]));
}

// Where vector c (16 bytes) of a row lies in shared memory: of a token's key (`bytes` long) or a channel's 64 values (128 bytes).  A wavefront's reads take the same vector of 32
// rows: any 16 lanes meet all 64 banks once.
__device__ __forceinline__ int kv_lds(int bytes, int row, int c) { return row * bytes + 16 * (c ^ (bytes == 128 ? (row >> 1) & 7 : (row >> 2) & 3)); }

// Where vector c of row `row` (0..31) of a wavefront's queries or outputs lies: 16 lanes that take the same vector of 16 rows, or a row's vectors, meet all banks once.
template <int D>
__device__ __forceinline__ int kv_strip(int row, int c) { return row * 2 * D + 16 * (c ^ (row & (D / 8 - 1))); }
__device__ __forceinline__ void wave_sync() {                     // what a wavefront's lanes have written to shared memory, to its other lanes
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int D>
struct KvTileShared {
    unsigned char keys[2][64 * D], values[2][128 * D];
    int noted[2];
};
template <int D, bool CAP>
__device__ __forceinline__ void kv_tile(const KvAttentionParams& p, const KvItem& it, int h, KvTileShared<D>& shared) {
    constexpr int kHalves = D / 64, kTiles = D / 32, kVecs = D / 64;       // kVecs: vectors of keys (and of values) a thread moves a chunk
    auto& keys = shared.keys;
    auto& values = shared.values;
    auto& noted = shared.noted;
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 31, g = lane >> 5;
    const int w0 = it.r0 + 32 * wave, r = w0 + n, pos = it.past + r / p.group;
    const int see_hi = pos + 1 - 8 * g, see_lo = (p.window ? max(pos + 1 - p.window, 0) : 0) - 8 * g;      // (as the lane counts a chunk's tokens: from 8g on)
    // The wavefront's rows come and go in vectors of 16 bytes, whole rows side by side, and through its own part of the shared memory (before the first chunk, behind the last).  As each lane
    // holds them, a row's pieces of 16 bytes would go one by one: 32 prompts of 256 tokens of 32 heads 73 us, so 65.
    constexpr int kMoveRows = 512 / D, kMoves = 32 / kMoveRows;
    const int move_row = lane / (D / 8), move_vec = lane % (D / 8), own_token = pos - it.past;
    unsigned char* strip = (unsigned char*)&shared + wave * 64 * D;
    // of the wavefront's rows: the tokens that all see, and those that any sees (none at all: a wavefront behind the last row)
    const int last = min(w0 + 31, it.rows - 1);
    const bool some = w0 < it.rows;
    const int all_hi = it.past + w0 / p.group + 1, any_hi = some ? min(it.past + last / p.group + 1, it.end) : 0;
    const int any_lo = p.window ? max(all_hi - p.window, 0) : 0, all_lo = p.window ? max(it.past + last / p.group + 1 - p.window, 0) : 0;
    // of all the tile's rows: the tokens that all see, and the first that any sees
    const int tile_all_hi = it.past + it.r0 / p.group + 1, tile_all_lo = p.window ? max(it.past + min(it.r0 + kKvTileRows - 1, it.rows - 1) / p.group + 1 - p.window, 0) : 0;
    const int tile_lo = p.window ? max(it.past + it.r0 / p.group + 1 - p.window, 0) : 0;

    // Keys and values of a chunk, from memory to registers and from there to shared memory: pass i of the workgroup (head of 128), or half i of it (head of 64), moves
    // the tokens 32i .. 32i+31, so that a page's address is the same in a wavefront's lanes.
    const int in_page = (1 << p.page_shift) - 1, kt = tid / (D / 16), kc = tid % (D / 16), vd = D == 128 ? tid >> 1 : (tid & 127) >> 1, vc = tid & 1;
    const int k_off = (kt & in_page & 31) * D + 16 * kc, v_off = (vd << p.page_shift) + 16 * vc;
    const int k_lds = kv_lds(D, kt, kc);                       // (32 tokens on: a fixed distance)
    intx4 kv[kVecs], vv[kVecs];
    int kscale[2], next_kscale[2], next_vscale[2], outside[2];
    auto ask = [&](int t0) {
        int64_t block[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int page = kv_look_up(p, it.table, t0 + 32 * u, tile_lo, it.end);
            outside[u] = kv_outside(p, page);
            block[u] = (int64_t)kv_in_pool(page, outside[u]) * p.kv_heads + h;
            next_kscale[u] = p.k_scale[block[u]];
            next_vscale[u] = p.v_scale[block[u]];
        }
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int u = D == 128 ? i : wave >> 1, slot = (t0 + 32 * u) & in_page;
            kv[i] = *(const intx4*)(p.k + ((block[u] << p.page_shift) + slot) * D + k_off);
            vv[i] = *(const intx4*)(p.v + ((block[u] * D) << p.page_shift) + slot + v_off);
        }
    };
    ask(it.begin);                                                 // (on their way while the queries are split)
    __builtin_amdgcn_sched_barrier(0);
    intx8 qh[kHalves], ql[kHalves];
    int q_scale;
    {
        intx4 w[kMoves];
#pragma unroll
        for (int i = 0; i < kMoves; ++i) {
            const int row = kMoveRows * i + move_row, token = __shfl(own_token, row);
            w[i] = intx4{0, 0, 0, 0};
            if (w0 + row < it.rows) w[i] = *(const intx4*)(p.q + (int64_t)(it.row0 + token) * p.q_stride + (h * p.group + w0 + row - token * p.group) * D + 8 * move_vec);
        }
#pragma unroll
        for (int i = 0; i < kMoves; ++i) *(intx4*)(strip + kv_strip<D>(kMoveRows * i + move_row, move_vec)) = w[i];
        wave_sync();
        float x[D / 2], amax = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {                         // chunks of eight: elements 16g + 8(c % 2) + 32(c / 2)
            const intx4 w = *(const intx4*)(strip + kv_strip<D>(n, 2 * g + (c & 1) + 4 * (c >> 1)));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[8 * c + 2 * i] = bf16_lo((unsigned)w[i]);
                x[8 * c + 2 * i + 1] = bf16_hi((unsigned)w[i]);
                amax = fmaxf(amax, fmaxf(finite_abs(x[8 * c + 2 * i]), finite_abs(x[8 * c + 2 * i + 1])));
            }
        }
        amax = across_halves(amax, Max());
        const int e = kv_query_exponent(amax);
        const float inv = pow2(-e);
        q_scale = e + 127;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            int hi, lo;
            kv_two_terms(x[4 * i] * inv, x[4 * i + 1] * inv, x[4 * i + 2] * inv, x[4 * i + 3] * inv, hi, lo);
            qh[i >> 3][i & 7] = hi;
            ql[i >> 3][i & 7] = lo;
        }
    }
    kv_floatx16 o[kTiles];
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[j][e] = 0.f;

    float m = -INFINITY, l = 0.f;

    // Where not every row of the tile sees the whole chunk, its values are cleaned on the way: tokens that no row sees are cleared, and so is NaN among the
    // others, which is noted (by the chunk's first token: a note of an earlier chunk means nothing).
    auto put = [&](int buf, int t0) {
        const bool edge = t0 < tile_all_lo || t0 + kKvTileChunk > tile_all_hi;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int u = D == 128 ? i : wave >> 1;
            *(intx4*)(keys[buf] + k_lds + 32 * D * i) = kv[i];
            if (edge) {
                int found = 0;
                const unsigned step = kv_nan_step(next_vscale[u]);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int v = vv[i][w] & kv_keep_bytes(t0 + 32 * u + 16 * vc + 4 * w, tile_lo, it.end), nan = kv_nan_bytes(v, step);
                    found |= nan;
                    vv[i][w] = v & ~nan;
                }
                if (found) noted[buf] = t0;
            }
            const float scale = kv_scale(edge ? kv_clean_scale(next_vscale[u]) : next_vscale[u]);
#pragma unroll
            for (int c = 0; c < 2; ++c) *(bf16x8*)(values[buf] + kv_lds(128, vd, 4 * u + 2 * vc + c)) = kv_widen(vv[i][2 * c], vv[i][2 * c + 1], scale);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) kscale[u] = next_kscale[u] | outside[u];
    };
    // NaN that `put` has cleared, to the rows that see it: ones in its places times ones where a row sees the token.
    auto give_nan = [&](int t0) {
        for (int q = 0; q < 4; ++q) {
            const int from = t0 + 16 * q, t = from + 8 * g;
            const int page = kv_look_up(p, it.table, from, tile_lo, it.end);
            const int64_t block = (int64_t)kv_in_pool(page, kv_outside(p, page)) * p.kv_heads + h;
            const unsigned step = kv_nan_step(p.v_scale[block]);
            intx4 seen;
#pragma unroll
            for (int i = 0; i < 4; ++i) seen[i] = (from + 2 * i >= see_lo && from + 2 * i < see_hi ? 0x3f80 : 0) | (from + 2 * i + 1 >= see_lo && from + 2 * i + 1 < see_hi ? 0x3f800000 : 0);
#pragma unroll
            for (int j = 0; j < kTiles; ++j) {
                const intx2 v = *(const intx2*)(p.v + ((block * D + 32 * j + n) << p.page_shift) + (t & in_page));
                intx4 is;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int nan = kv_nan_bytes(v[i >> 1] & kv_keep_bytes(t + 4 * (i >> 1), tile_lo, it.end), step) >> (16 * (i & 1));
                    is[i] = (nan & 1 ? 0x3f80 : 0) | (nan & 0x100 ? 0x3f800000 : 0);
                }
                kv_floatx16 cnt;
#pragma unroll
                for (int e = 0; e < 16; ++e) cnt[e] = 0.f;
                cnt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, is), __builtin_bit_cast(bf16x8, seen), cnt, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[j][e] += cnt[e] != 0.f ? NAN : 0.f;
            }
        }
    };
    const int t_lane = kv_tile_token(0, n);
    if (tid < 2) noted[tid] = -1;
    __syncthreads();
    put(0, it.begin);
    __syncthreads();
    int buf = 0;
    for (int t0 = it.begin; t0 < it.end; t0 += kKvTileChunk, buf ^= 1) {
        const bool more = t0 + kKvTileChunk < it.end;
        if (more) ask(t0 + kKvTileChunk);
        if (t0 < any_hi && t0 + kKvTileChunk > any_lo) {           // (the same in all lanes)
            kv_floatx16 s[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[u][e] = 0.f;
#pragma unroll
                for (int w = 0; w < kHalves; ++w) {
                    const unsigned char* at = keys[buf] + 32 * D * u;
                    const intx4 a = *(const intx4*)(at + kv_lds(D, t_lane, 4 * w + g)), b = *(const intx4*)(at + kv_lds(D, t_lane, 4 * w + 2 + g));
                    const intx8 k = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
                    s[u] = kv_mfma32(k, qh[w], s[u], kscale[u], q_scale);
                    s[u] = kv_mfma32(k, ql[w], s[u], kscale[u], q_scale - 4);
                }
            }
            kv_settle();
            if constexpr (CAP) kv_cap(p, s);
            if (t0 < all_lo || t0 + kKvTileChunk > all_hi) {       // not every row sees all of it
                asm volatile("");                                  // (a branch: as a selection it would cost every chunk)
                const int hi = see_hi - t0, lo = see_lo - t0;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int t = 32 * u + 16 * (e >> 3) + (e & 7);
                        s[u][e] = t < hi && t >= lo ? s[u][e] : -INFINITY;
                    }
            }
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, s[u][e]);
            top = across_halves(top, Max()) * p.scale;             // (the scores stay as they are: their factor goes into the exponent)
            if (__any(top > m + kKvSlack)) {
                top = fmaxf(m, top);
                const float shrink = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
                m = top;
                l *= shrink;
#pragma unroll
                for (int j = 0; j < kTiles; ++j) o[j] *= shrink;
            }
            const float base = m == -INFINITY ? 0.f : -m;
            bf16x8 w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[e] = __builtin_amdgcn_exp2f(s[q >> 1][8 * (q & 1) + e] * p.scale + base);
                    l += y[e];
                }
                w[q] = kv_pack8(y[0], y[1], y[2], y[3], y[4], y[5], y[6], y[7]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int j = 0; j < kTiles; ++j) {
                    const bf16x8 v = *(const bf16x8*)(values[buf] + 32 * 128 * j + kv_lds(128, n, 2 * q + g));
                    o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[q], o[j], 0, 0, 0);
                }
            if (noted[buf] == t0) {
                kv_settle();
                give_nan(t0);
            }
        }
        if (more) put(buf ^ 1, t0 + kKvTileChunk);
        __syncthreads();
    }
    kv_settle();
    l = across_halves(l, Add());
    int at = tid;
    asm volatile("" : "+v"(at));                                   // (the lane's place is formed again here, not kept over the loop: registers)
    strip = (unsigned char*)&shared + (at >> 6) * 64 * D;
    at &= 63;
    const int own = at & 31, half = at >> 5;
    if (it.part >= 0) {
        if (w0 + own >= it.rows) return;
        const int64_t to = (int64_t)h * p.part_rows + it.part + w0 + own - it.r0;
        if (half == 0) {
            p.part_ml[to * 2] = m;
            p.part_ml[to * 2 + 1] = l;
        }
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *(floatx4*)(p.part_o + to * D + 32 * j + 8 * a + 4 * half) = floatx4{o[j][4 * a], o[j][4 * a + 1], o[j][4 * a + 2], o[j][4 * a + 3]};
        return;
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int a = 0; a < 4; ++a)
            *(intx2*)(strip + kv_strip<D>(own, 4 * j + a) + 8 * half) = intx2{(int)pack2_bf16(o[j][4 * a] * inv, o[j][4 * a + 1] * inv), (int)pack2_bf16(o[j][4 * a + 2] * inv, o[j][4 * a + 3] * inv)};
    wave_sync();
    const int token_of = (w0 + own) / p.group;
#pragma unroll
    for (int i = 0; i < kMoves; ++i) {
        const int row = kMoveRows * i + at / (D / 8), token = __shfl(token_of, row);
        if (w0 + row < it.rows)
            *(intx4*)(p.out + (int64_t)(it.row0 + token) * p.out_stride + (h * p.group + w0 + row - token * p.group) * D + 8 * (at % (D / 8))) =
                *(const intx4*)(strip + kv_strip<D>(row, at % (D / 8)));
    }
}

// Tiles, and items of up to 16 rows behind them, in one launch: both have two wavefronts a SIMD (head of 64: three; 16 heads of 8192 tokens 171 us, 196 with two), and a batch of prompts and decode steps is done when the longer of the two is.
template <int D, bool CAP>
SYMB_KERNEL __launch_bounds__(256, D == 64 ? 3 : 2) void symb_kv_attention_kernel(KvAttentionParams p) {
    __shared__ union __attribute__((aligned(16))) {
        KvTileShared<D> tile;
        KvRowsShared<D, 1> rows;
    } shared;
    const int i = blockIdx.x / p.kv_heads, h = blockIdx.x % p.kv_heads;
    const KvItem it = p.items[i];
    if (i < p.tiles) kv_tile<D, CAP>(p, it, h, shared.tile);
    else kv_rows<D, 1, CAP>(p, it, h, shared.rows);
}
// Items of 17 to 48 rows: one wavefront a SIMD.
template <int D, int R, bool CAP>
SYMB_KERNEL __launch_bounds__(256, 1) void symb_kv_rows_kernel(KvAttentionParams p) {
    __shared__ KvRowsShared<D, R> shared;
    const KvItem it = p.items[blockIdx.x / p.kv_heads];
    kv_rows<D, R, CAP>(p, it, blockIdx.x % p.kv_heads, shared);
}

// The parts of up to 16 rows' results: part i of row r at partial row part0 + stride i + r.
struct KvJoinItem {
    int32_t row0, rows, r0, part0, parts, stride;
};
struct KvJoinParams {
    const KvJoinItem* items;
    const float* part_o;
    const float* part_ml;
    bf16* out;
    int64_t out_stride;
    int32_t kv_heads, group, part_rows;
};
// A workgroup a row: a long context has dozens of parts, 1024 / D of which are read at once; joined in a fixed order.
template <int D>
SYMB_KERNEL __launch_bounds__(256) void symb_kv_join_kernel(KvJoinParams p) {
    constexpr int kLanes = D / 4, kSets = 256 / kLanes;
    __shared__ float top[4];
    __shared__ floatx4 part[kSets][kLanes];
    __shared__ float sums[kSets];
    const KvJoinItem it = p.items[blockIdx.x / p.kv_heads];
    const int h = blockIdx.x % p.kv_heads, row = it.r0 + blockIdx.y, tid = threadIdx.x;
    if (row >= it.rows) return;
    const int64_t at = (int64_t)h * p.part_rows + it.part0 + blockIdx.y;
    float M = -INFINITY;
    for (int k = tid; k < it.parts; k += 256) M = fmaxf(M, p.part_ml[(at + (int64_t)it.stride * k) * 2]);
    M = across_wave(M, Max());
    if ((tid & 63) == 0) top[tid >> 6] = M;
    __syncthreads();
    M = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    const float base = M == -INFINITY ? 0.f : M;
    const int set = tid / kLanes, d = tid % kLanes * 4;
    float sum = 0.f;
    floatx4 v = floatx4{0, 0, 0, 0};
#pragma unroll 4
    for (int k = set; k < it.parts; k += kSets) {
        const int64_t a = at + (int64_t)it.stride * k;
        const float f = __builtin_amdgcn_exp2f(p.part_ml[a * 2] - base);
        sum += p.part_ml[a * 2 + 1] * f;
        v += *(const floatx4*)(p.part_o + a * D + d) * f;
    }
    part[set][tid % kLanes] = v;
    if (d == 0) sums[set] = sum;
    __syncthreads();
    if (tid >= kLanes) return;
    sum = sums[0];
    v = part[0][tid];
#pragma unroll
    for (int k = 1; k < kSets; ++k) {
        sum += sums[k];
        v += part[k][tid];
    }
    *(intx2*)(p.out + (int64_t)(it.row0 + row / p.group) * p.out_stride + (h * p.group + row % p.group) * D + d) =
        intx2{(int)pack2_bf16(v[0] / sum, v[1] / sum), (int)pack2_bf16(v[2] / sum, v[3] / sum)};
}
// A workgroup for all of an item's rows, D / 4 lanes a row.
template <int D>
SYMB_KERNEL __launch_bounds__(256) void symb_kv_join_rows_kernel(KvJoinParams p) {
    constexpr int kLanes = D / 4, kSets = 256 / kLanes;
    const KvJoinItem it = p.items[blockIdx.x / p.kv_heads];
    const int h = blockIdx.x % p.kv_heads, d = threadIdx.x % kLanes * 4;
    for (int r = threadIdx.x / kLanes; r < min(16, it.rows - it.r0); r += kSets) {
        const int row = it.r0 + r;
        const int64_t at = (int64_t)h * p.part_rows + it.part0 + r;
        float M = -INFINITY;
        for (int k = 0; k < it.parts; ++k) M = fmaxf(M, p.part_ml[(at + (int64_t)it.stride * k) * 2]);
        const float base = M == -INFINITY ? 0.f : M;
        float sum = 0.f;
        floatx4 v = floatx4{0, 0, 0, 0};
#pragma unroll 4
        for (int k = 0; k < it.parts; ++k) {
            const int64_t a = at + (int64_t)it.stride * k;
            const float f = __builtin_amdgcn_exp2f(p.part_ml[a * 2] - base);
            sum += p.part_ml[a * 2 + 1] * f;
            v += *(const floatx4*)(p.part_o + a * D + d) * f;
        }
        *(intx2*)(p.out + (int64_t)(it.row0 + row / p.group) * p.out_stride + (h * p.group + row % p.group) * D + d) =
            intx2{(int)pack2_bf16(v[0] / sum, v[1] / sum), (int)pack2_bf16(v[2] / sum, v[3] / sum)};
    }
}

}  // namespace symb
