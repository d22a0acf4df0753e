// Causal attention of a flattened batch's rows over a paged cache of 8-bit keys and values.
//
//   x_s = scale q . k_s (or cap tanh(x_s / cap)),   out = sum_s 2^(l x_s - m) v_s / sum_s 2^(l x_s - m),   l = log2(e), m the row's largest l x_s
//
// computed in one pass over the tokens: m, the sum and the unnormalised output are kept in fp32 and scaled when m grows.
//
// Both products run on v_mfma_scale_f32_16x16x128_f8f6f4 with the cache's bytes as they lie, E8M0 scales included: nothing is widened, and a page's scale
// costs no instruction.  A bf16 query has eight significant bits, two E4M3 terms: q = (hi + lo / 16) 2^e exactly for elements within 2^-14 of the row's largest
// (others to 2^-18 of it), one product each.  The weights 2^(l x - m) enter the second product the same way, with nine significant bits, one more than a
// bf16 weight has.  Two products at twice bf16's rate cost what one bf16 product would, and the widening of keys and values (two instructions for
// every four bytes and 16 rows) falls away.  Inside one instruction, the matrix unit drops what lies more than about 2^-15 below its largest product: measured
// relative errors of 1e-5 to 5e-5 of a sum, not growing with the number of instructions (the accumulator is full fp32), a hundredth of the output's rounding.
//
// The scores are formed as K Q^T, tokens down the rows of the result: a lane then holds 32 tokens of ONE query row, in the order in which the
// instruction wants them as the right operand of V^T P^T.  No score crosses lanes but for the row's maximum and sum, and none goes through shared memory.
// In a chunk of 128 tokens, lane (n = lane % 16, g = lane / 16) gives
//   left operand, keys    tile s (0..7): token kv_token(s, n), elements 16g .. 16g+15 and (head of 128) 64+16g ..
//   right operand         query row n, the same elements
//   result                tokens kv_token(s, 4g + r), r = 0..3, of row n: with s = 0..3 the tokens 16g .. 16g+15, with s = 4..7 64+16g ..
//   left operand, values  channel 16j + n, tokens 16g .. 16g+15 and 64+16g .., 16 bytes each as they lie in the cache
//   scales                of the 32 elements (tokens) 32g .. 32g+31 of row (channel) n
#pragma once
#include <type_traits>

#include "block_device.hpp"

namespace symb {

constexpr int kKvChunk = 128;             // tokens

// A run of tokens for up to 16 query rows of one key head.  Row r of a segment's key head is query head r % group of token r / group.
struct KvRowsItem {
    int32_t table;                        // the segment's first entry in the page table
    int32_t row0, rows;                   // its first row in the batch; its rows times the query heads of a key head
    int32_t past;
    int32_t r0;                           // the item's first row
    int32_t begin, end;                   // tokens: a multiple of 128; one past the last that any of the rows sees
    int32_t part;                         // partial result's first row, -1: the item is all there is
};

struct KvAttentionParams {
    const void* items;                    // KvRowsItem or KvTileItem
    const int32_t* page_table;
    const unsigned char* k;
    const unsigned char* v;
    const unsigned char* k_scale;
    const unsigned char* v_scale;
    const bf16* q;
    bf16* out;
    float* part_o;                        // [part rows][D], unnormalised
    float* part_ml;                       // [part rows][2]: maximum (log2 units), sum
    int64_t q_stride, out_stride;
    int32_t num_pages, kv_heads, group, page_shift, window;
    int32_t part_rows;                    // of one key head
    float scale, cap;                     // cap > 0: its value in log2 units, and scale / cap in `scale`; else scale in log2 units
};

__device__ __forceinline__ int kv_token(int s, int m) { return 16 * (m >> 2) + 4 * (s & 3) + (m & 3) + 64 * (s >> 2); }

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

// A score in log2 units.
template <bool CAP>
__device__ __forceinline__ float kv_score(const KvAttentionParams& p, float s) {
    if (!CAP) return s * p.scale;
    // cap tanh(y) = cap (1 - 2 / (e^2y + 1)): at most cap 2^-23 off, which is what a score of that size is held to
    const float y = s * p.scale;
    return p.cap * (1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * 2.885390082f) + 1.f));
}

// The pages of a chunk as one lane needs them.  Only pages of the tokens lo .. hi-1 are looked up (others are hidden: any page will do); a number outside
// the pool is reported, and page 0 read in its place.
struct KvChunk {
    int kpage[2], vpage[2];               // of tile s: kpage[s / 4]; of the value tokens 16g and 64+16g
    int kscale[2], vscale;
};
__device__ __forceinline__ int kv_page(const KvAttentionParams& p, int table, int token, int lo, int hi, bool& bad) {
    const int page = p.page_table[table + (max(min(token, hi - 1), lo) >> p.page_shift)];
    const bool in = (unsigned)page < (unsigned)p.num_pages;
    bad |= !in;
    return in ? page : 0;
}
__device__ __forceinline__ void kv_pages(KvChunk& c, const KvAttentionParams& p, int table, int t0, int lo, int hi, int n, int g, bool& bad) {
    int pg[4];                                                     // the same in all lanes
#pragma unroll
    for (int i = 0; i < 4; ++i) pg[i] = kv_page(p, table, t0 + 32 * i, lo, hi, bad);
    c.kpage[0] = n & 8 ? pg[1] : pg[0];
    c.kpage[1] = n & 8 ? pg[3] : pg[2];
    c.vpage[0] = g & 2 ? pg[1] : pg[0];
    c.vpage[1] = g & 2 ? pg[3] : pg[2];
    c.vscale = g & 2 ? (g & 1 ? pg[3] : pg[2]) : (g & 1 ? pg[1] : pg[0]);
}

// The value operand of one channel with the bytes outside [lo, hi) cleared: what a hidden token holds must not meet a weight, 0 x NaN being NaN.
__device__ __forceinline__ int kv_keep(int w, int t, int lo, int hi) {     // bytes t .. t+3
    const int a = lo - t, b = hi - t;
    const unsigned below = b >= 4 ? ~0u : b > 0 ? (1u << (8 * b)) - 1 : 0u;
    const unsigned above = a <= 0 ? ~0u : a < 4 ? ~0u << (8 * a) : 0u;
    return (int)((unsigned)w & below & above);
}

// 0x80 in the place of each byte that is NaN.
__device__ __forceinline__ unsigned kv_nan_bytes(int w) { return (((unsigned)w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// Four wavefronts share an item's tokens, chunk by chunk, and join through shared memory.  Keys and values go straight from memory into the operands' registers: a
// wavefront has up to 32 KB on their way, keys of the next chunk asked for as soon as the scores of this one are formed.
template <int D, bool CAP>
SYMB_KERNEL __launch_bounds__(256, D == 64 ? 2 : 1) void symb_kv_rows_kernel(KvAttentionParams p) {
    constexpr int kTiles = D / 16, kWords = D / 64;
    __shared__ float join[4][16][D + 4];
    __shared__ float stat[4][16][2];
    const KvRowsItem it = ((const KvRowsItem*)p.items)[blockIdx.x / p.kv_heads];
    const int h = blockIdx.x % p.kv_heads;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int r = it.r0 + n, pos = it.past + r / p.group;
    const bool valid = r < it.rows;
    const int see_hi = valid ? pos + 1 : 0, see_lo = p.window ? max(pos + 1 - p.window, 0) : 0;       // tokens this lane's row sees
    // tokens that every row of the item sees, and those that some row does
    const int last = min(it.r0 + 15, it.rows - 1);
    const int all_hi = it.past + it.r0 / p.group + 1, all_lo = p.window ? max(it.past + last / p.group + 1 - p.window, 0) : 0;
    const int any_hi = it.past + last / p.group + 1, any_lo = p.window ? max(all_hi - p.window, 0) : 0;
    KvQuery<D> q;
    kv_query<D>(q, p.q + (int64_t)(it.row0 + r / p.group) * p.q_stride + (h * p.group + r % p.group) * D, valid, g);
    bool bad = false;
    floatx4 o[kTiles];
#pragma unroll
    for (int j = 0; j < kTiles; ++j) o[j] = floatx4{0, 0, 0, 0};
    float m = -INFINITY, l = 0.f;
    intx4 kb[8][kWords];
    const int P = 1 << p.page_shift;
    KvChunk c;
    auto ask_keys = [&](int t0) {
        kv_pages(c, p, it.table, t0, any_lo, it.end, n, g, bad);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t block = (int64_t)c.kpage[u] * p.kv_heads + h;
            const unsigned char* at = p.k + (block << p.page_shift) * D + 16 * g;
            c.kscale[u] = p.k_scale[block];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const unsigned char* row = at + ((t0 + kv_token(4 * u + s, n)) & (P - 1)) * D;
#pragma unroll
                for (int w = 0; w < kWords; ++w) kb[4 * u + s][w] = *(const intx4*)(row + 64 * w);
            }
        }
        c.vscale = p.v_scale[(int64_t)c.vscale * p.kv_heads + h];
    };
    int t0 = it.begin + wave * kKvChunk;
    if (t0 < it.end) ask_keys(t0);
    for (; t0 < it.end; t0 += 4 * kKvChunk) {
        intx4 vb[kTiles][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const unsigned char* at = p.v + ((((int64_t)c.vpage[u] * p.kv_heads + h) * D + n) << p.page_shift) + ((t0 + 64 * u + 16 * g) & (P - 1));
#pragma unroll
            for (int j = 0; j < kTiles; ++j) vb[j][u] = *(const intx4*)(at + ((int64_t)(16 * j) << p.page_shift));
        }
        const int vscale = c.vscale;
        floatx4 s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int ks = c.kscale[i >> 2];
            if constexpr (D == 128) {
                const intx8 a = __builtin_shufflevector(kb[i][0], kb[i][1], 0, 1, 2, 3, 4, 5, 6, 7);
                s[i] = kv_mfma(a, q.hi, floatx4{0, 0, 0, 0}, ks, q.hi_scale);
                s[i] = kv_mfma(a, q.lo, s[i], ks, q.lo_scale);
            } else {
                const intx8 a = __builtin_shufflevector(kb[i][0], kb[i][0], 0, 1, 2, 3, 4, 5, 6, 7);
                s[i] = kv_mfma(a, q.hi, floatx4{0, 0, 0, 0}, ks, q.hi_scale);
            }
        }
        if (t0 + 4 * kKvChunk < it.end) ask_keys(t0 + 4 * kKvChunk);
        const bool whole = t0 >= all_lo && t0 + kKvChunk <= all_hi;
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = kv_score<CAP>(p, s[i][e]);
                if (!whole) {
                    const int t = t0 + kv_token(i, 4 * g + e);
                    x = t < see_hi && t >= see_lo ? x : -INFINITY;
                }
                s[i][e] = x;
                top = fmaxf(top, x);
            }
        top = fmaxf(m, across_rows(top, Max()));
        const float base = top == -INFINITY ? 0.f : top;           // (a row that has seen nothing yet)
        const float shrink = __builtin_amdgcn_exp2f(m - base);
        m = top;
        l *= shrink;
        // weights times 256, so that their lower term stays within E4M3 down to 2^-21 of the largest
        intx8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[e] = __builtin_amdgcn_exp2f(s[i][e] - base + 8.f);
                l += y[e];
            }
            int a, b;
            kv_two_terms(y[0], y[1], y[2], y[3], a, b);
            hi[i] = a;
            lo[i] = b;
        }
#pragma unroll
        for (int j = 0; j < kTiles; ++j) o[j] *= shrink;
        if (!whole) {
            // a NaN among the values of a token that only some rows see: cleared, and given to the rows that see it
            bool nan = false;
#pragma unroll
            for (int j = 0; j < kTiles; ++j)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int v = kv_keep(vb[j][u][w], t0 + 64 * u + 16 * g + 4 * w, any_lo, any_hi);
                        vb[j][u][w] = v;
                        nan |= kv_nan_bytes(v) != 0;
                    }
            if (__any(nan)) {
                intx8 seen;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    int v = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int t = t0 + kv_token(i, 4 * g + e);
                        if (t < see_hi && t >= see_lo) v |= 0x38 << (8 * e);                   // 1
                    }
                    seen[i] = v;
                }
#pragma unroll
                for (int j = 0; j < kTiles; ++j) {
                    intx8 is;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int v = vb[j][i >> 2][i & 3];
                        const unsigned mask = (kv_nan_bytes(v) >> 7) * 255u;
                        is[i] = (int)(mask & 0x38383838u);
                        vb[j][i >> 2][i & 3] = (int)((unsigned)v & ~mask);
                    }
                    const floatx4 cnt = kv_mfma(is, seen, floatx4{0, 0, 0, 0}, 127, 127);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (cnt[e] != 0.f) o[j][e] = NAN;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
            const intx8 a = __builtin_shufflevector(vb[j][0], vb[j][1], 0, 1, 2, 3, 4, 5, 6, 7);
            o[j] = kv_mfma(a, hi, o[j], vscale, 127);
            o[j] = kv_mfma(a, lo, o[j], vscale, 123);
        }
    }
    l = across_rows(l, Add());
    if (__any(bad)) m = NAN;
    // the four wavefronts' results: o 2^(m - M) added up, and so the sums
    if (g == 0) {
        stat[wave][n][0] = m;
        stat[wave][n][1] = l;
    }
    __syncthreads();
    float M = -INFINITY, sum = 0.f;
    bool nan = false;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        M = fmaxf(M, stat[w][n][0]);
        nan |= stat[w][n][0] != stat[w][n][0];
    }
    const float base = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < 4; ++w) sum += stat[w][n][1] * __builtin_amdgcn_exp2f(stat[w][n][0] - base);
    const float mine = nan ? NAN : __builtin_amdgcn_exp2f(m - base);
#pragma unroll
    for (int j = 0; j < kTiles; ++j) *(floatx4*)&join[wave][n][16 * j + 4 * g] = o[j] * mine;
    if (wave == 0 && g == 0) {
        // (stat's first row is read by the lanes of this column alone from here on)
        if (it.part >= 0 && valid) {
            float* ml = p.part_ml + ((int64_t)h * p.part_rows + it.part + n) * 2;
            ml[0] = nan ? NAN : M;
            ml[1] = sum;
        }
    }
    __syncthreads();
    if (wave == 0 && g == 0) stat[0][n][1] = sum;
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * D / 4; i += 256) {
        const int row = i / (D / 4), d = i % (D / 4) * 4, rr = it.r0 + row;
        if (rr >= it.rows) continue;
        floatx4 v = *(const floatx4*)&join[0][row][d];
#pragma unroll
        for (int w = 1; w < 4; ++w) v += *(const floatx4*)&join[w][row][d];
        if (it.part >= 0) {
            *(floatx4*)(p.part_o + ((int64_t)h * p.part_rows + it.part + row) * D + d) = v;
        } else {
            const float s = stat[0][row][1];
            *(intx2*)(p.out + (int64_t)(it.row0 + rr / p.group) * p.out_stride + (h * p.group + rr % p.group) * D + d) =
                intx2{(int)pack2_bf16(v[0] / s, v[1] / s), (int)pack2_bf16(v[2] / s, v[3] / s)};
        }
    }
}

// ---- tiles of 128 rows ------------------------------------------------------------------------------------------------------------
// Prompts: four wavefronts with 32 rows each on the same tokens, 64 at a time through shared memory.  The products are v_mfma_scale_f32_32x32x64_f8f6f4, scores
// again as K Q^T: in a chunk of 64 tokens, lane (n = lane % 32, g = lane / 32) gives
//   left operand, keys    tile u (0, 1): token kv_tile_token(u, n), elements 64w + 16g .. and 64w + 32 + 16g .. (w: half of a head of 128)
//   right operand         query row n, the same elements
//   result                element 4a + b: token 32u + 16g + 4a + b of row n
//   left operand, values  channel 32j + n, tokens 16g .. 16g+15 and 32 + 16g ..
//   scales                of the 32 tokens (elements) 32g .. 32g+31
constexpr int kKvTileRows = 128, kKvTileChunk = 64;

struct KvTileItem {
    int32_t table, row0, rows, past;      // as in KvRowsItem
    int32_t r0;
    int32_t begin, end;                   // begin: a multiple of 64
    int32_t part;
};

__device__ __forceinline__ int kv_tile_token(int u, int m) { return 32 * u + 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }

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

// Where vector c (16 bytes) of a row lies in shared memory.  A wavefront's reads take the same vector of 32 rows: any 16 lanes in a row's order meet all 64 banks once.
__device__ __forceinline__ int kv_lds_key(int D, int t, int c) {          // D: bytes of a token
    return D == 128 ? t * 128 + 16 * (c ^ (((t >> 1) & 3) | ((t >> 4) & 1) << 2)) : t * 64 + 16 * (c ^ (((t >> 2) & 1) | ((t >> 4) & 1) << 1));
}
__device__ __forceinline__ int kv_lds_value(int d, int c) { return d * 64 + 16 * (c ^ ((d >> 2) & 3)); }

template <int D, bool CAP>
SYMB_KERNEL __launch_bounds__(256, 2) void symb_kv_tile_kernel(KvAttentionParams p) {
    constexpr int kHalves = D / 64, kTiles = D / 32, kVecs = D / 64;       // kVecs: vectors of keys (and of values) a thread moves a chunk
    __shared__ __attribute__((aligned(16))) unsigned char keys[2][64 * D], values[2][64 * D];
    const KvTileItem it = ((const KvTileItem*)p.items)[blockIdx.x / p.kv_heads];
    const int h = blockIdx.x % p.kv_heads, tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 31, g = lane >> 5;
    const int w0 = it.r0 + 32 * wave, r = w0 + n, pos = it.past + r / p.group;
    const bool valid = r < it.rows;
    const int see_hi = pos + 1, see_lo = p.window ? max(pos + 1 - p.window, 0) : 0;
    // of the wavefront's rows: the tokens that all see, and those that any sees (none at all: a wavefront behind the last row)
    const int last = min(w0 + 31, it.rows - 1);
    const bool some = w0 < it.rows;
    const int all_hi = it.past + w0 / p.group + 1, any_hi = some ? min(it.past + last / p.group + 1, it.end) : 0;
    const int any_lo = p.window ? max(all_hi - p.window, 0) : 0, all_lo = p.window ? max(it.past + last / p.group + 1 - p.window, 0) : 0;
    const int tile_lo = p.window ? max(it.past + it.r0 / p.group + 1 - p.window, 0) : 0;

    intx8 qh[kHalves], ql[kHalves];
    int q_scale;
    {
        const bf16* q = p.q + (int64_t)(it.row0 + r / p.group) * p.q_stride + (h * p.group + r % p.group) * D;
        float x[D / 2], amax = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {                         // chunks of eight: elements 16g + 8(c % 2) + 32(c / 2)
            intx4 w = intx4{0, 0, 0, 0};
            if (valid) w = *(const intx4*)(q + 16 * g + 8 * (c & 1) + 32 * (c >> 1));
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
    bool bad = false;

    // Keys and values of a chunk, from memory to registers and from there to shared memory: pass i of the workgroup (head of 128), or half i of it (head of 64), moves
    // the tokens 32i .. 32i+31, so that a page's address is the same in a wavefront's lanes.
    const int in_page = (1 << p.page_shift) - 1, kt = tid / (D / 16), kc = tid % (D / 16), vd = D == 128 ? tid >> 1 : (tid & 127) >> 1, vc = tid & 1;
    const int k_off = (kt & in_page & 31) * D + 16 * kc, v_off = (vd << p.page_shift) + 16 * vc;
    const int k_lds = kv_lds_key(D, kt, kc);                       // (32 tokens on: a fixed distance)
    intx4 kv[kVecs], vv[kVecs];
    int kscale[2], vscale, next_kscale[2], next_vscale;
    auto ask = [&](int t0) {
        int64_t block[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            block[u] = (int64_t)kv_page(p, it.table, t0 + 32 * u, tile_lo, it.end, bad) * p.kv_heads + h;
            next_kscale[u] = p.k_scale[block[u]];
        }
        next_vscale = p.v_scale[g ? block[1] : block[0]];
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int u = D == 128 ? i : wave >> 1, slot = (t0 + 32 * u) & in_page;
            kv[i] = *(const intx4*)(p.k + ((block[u] << p.page_shift) + slot) * D + k_off);
            vv[i] = *(const intx4*)(p.v + ((block[u] * D) << p.page_shift) + slot + v_off);
        }
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            *(intx4*)(keys[buf] + k_lds + 32 * D * i) = kv[i];
            *(intx4*)(values[buf] + kv_lds_value(vd, vc + 2 * (D == 128 ? i : wave >> 1))) = vv[i];
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) kscale[u] = next_kscale[u];
        vscale = next_vscale;
    };
    // One chunk; WHOLE: all of the wavefront's rows see all of it.
    auto chunk = [&](auto WHOLE, int t0, int buf) {
        constexpr bool whole = decltype(WHOLE)::value;
        kv_floatx16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int t = kv_tile_token(0, n);
#pragma unroll
            for (int e = 0; e < 16; ++e) s[u][e] = 0.f;
#pragma unroll
            for (int w = 0; w < kHalves; ++w) {
                const unsigned char* at = keys[buf] + 32 * D * u;
                const intx4 a = *(const intx4*)(at + kv_lds_key(D, t, 4 * w + g)), b = *(const intx4*)(at + kv_lds_key(D, t, 4 * w + 2 + g));
                const intx8 k = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
                s[u] = kv_mfma32(k, qh[w], s[u], kscale[u], q_scale);
                s[u] = kv_mfma32(k, ql[w], s[u], kscale[u], q_scale - 4);
            }
        }
        // without a cap the scores stay as they are: their factor goes into the exponent
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                if (CAP) s[u][e] = kv_score<true>(p, s[u][e]);
                if (!whole) {
                    const int t = t0 + 32 * u + 16 * g + e;
                    s[u][e] = t < see_hi && t >= see_lo ? s[u][e] : -INFINITY;
                }
                top = fmaxf(top, s[u][e]);
            }
        const float factor = CAP ? 1.f : p.scale;
        top = across_halves(top, Max()) * factor;
        // m follows the row's maximum once that has outgrown it 16-fold: weights up to 2^(4 + 4)
        if (__any(top > m + 4.f)) {
            top = fmaxf(m, top);
            const float shrink = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
            m = top;
            l *= shrink;
#pragma unroll
            for (int j = 0; j < kTiles; ++j) o[j] *= shrink;
        }
        const float base = 4.f - (m == -INFINITY ? 0.f : m);
        intx8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[e] = __builtin_amdgcn_exp2f(s[i >> 2][4 * (i & 3) + e] * factor + base);
                l += y[e];
            }
            int a, b;
            kv_two_terms(y[0], y[1], y[2], y[3], a, b);
            hi[i] = a;
            lo[i] = b;
        }
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
            const unsigned char* at = values[buf] + 32 * 64 * j;
            intx4 a = *(const intx4*)(at + kv_lds_value(n, g)), b = *(const intx4*)(at + kv_lds_value(n, 2 + g));
            if constexpr (!whole) {
                bool nan = false;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    a[w] = kv_keep(a[w], t0 + 16 * g + 4 * w, any_lo, any_hi);
                    b[w] = kv_keep(b[w], t0 + 32 + 16 * g + 4 * w, any_lo, any_hi);
                    nan |= (kv_nan_bytes(a[w]) | kv_nan_bytes(b[w])) != 0;
                }
                if (__any(nan)) {
                    // a NaN among the values of a token that only some rows see: cleared, and given to the rows that see it
                    intx8 seen, is;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        int v = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int t = t0 + 32 * (i >> 2) + 16 * g + 4 * (i & 3) + e;
                            if (t < see_hi && t >= see_lo) v |= 0x38 << (8 * e);           // 1
                        }
                        seen[i] = v;
                        const int w = i < 4 ? a[i & 3] : b[i & 3];
                        const unsigned mask = (kv_nan_bytes(w) >> 7) * 255u;
                        is[i] = (int)(mask & 0x38383838u);
                        if (i < 4) a[i & 3] = (int)((unsigned)w & ~mask);
                        else b[i & 3] = (int)((unsigned)w & ~mask);
                    }
                    kv_floatx16 cnt;
#pragma unroll
                    for (int e = 0; e < 16; ++e) cnt[e] = 0.f;
                    cnt = kv_mfma32(is, seen, cnt, 127, 127);
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[j][e] += cnt[e] != 0.f ? NAN : 0.f;
                }
            }
            const intx8 v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
            o[j] = kv_mfma32(v, hi, o[j], vscale, 127);
            o[j] = kv_mfma32(v, lo, o[j], vscale, 123);
        }
    };
    ask(it.begin);
    put(0);
    __syncthreads();
    int buf = 0;
    for (int t0 = it.begin; t0 < it.end; t0 += kKvTileChunk, buf ^= 1) {
        const bool more = t0 + kKvTileChunk < it.end;
        if (more) ask(t0 + kKvTileChunk);
        if (t0 >= all_lo && t0 + kKvTileChunk <= all_hi) chunk(std::true_type(), t0, buf);             // (the same in all lanes)
        else if (t0 < any_hi && t0 + kKvTileChunk > any_lo) chunk(std::false_type(), t0, buf);
        if (more) put(buf ^ 1);
        __syncthreads();
    }
    l = across_halves(l, Add());
    if (__any(bad)) m = NAN;
    if (!valid) return;
    if (it.part >= 0) {
        const int64_t at = (int64_t)h * p.part_rows + it.part + r - it.r0;
        if (g == 0) {
            p.part_ml[at * 2] = m;
            p.part_ml[at * 2 + 1] = l;
        }
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *(floatx4*)(p.part_o + at * D + 32 * j + 8 * a + 4 * g) = floatx4{o[j][4 * a], o[j][4 * a + 1], o[j][4 * a + 2], o[j][4 * a + 3]};
        return;
    }
    const float inv = (m != m ? m : 1.f) / l;
    bf16* out = p.out + (int64_t)(it.row0 + r / p.group) * p.out_stride + (h * p.group + r % p.group) * D;
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int a = 0; a < 4; ++a)
            *(intx2*)(out + 32 * j + 8 * a + 4 * g) = intx2{(int)pack2_bf16(o[j][4 * a] * inv, o[j][4 * a + 1] * inv), (int)pack2_bf16(o[j][4 * a + 2] * inv, o[j][4 * a + 3] * inv)};
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
template <int D>
SYMB_KERNEL __launch_bounds__(256) void symb_kv_join_kernel(KvJoinParams p) {
    const KvJoinItem it = p.items[blockIdx.x / p.kv_heads];
    const int h = blockIdx.x % p.kv_heads;
    for (int i = threadIdx.x; i < 16 * D / 4; i += 256) {
        const int row = i / (D / 4), d = i % (D / 4) * 4, rr = it.r0 + row;
        if (rr >= it.rows) continue;
        const int64_t at = (int64_t)h * p.part_rows + it.part0 + row;
        float M = -INFINITY, sum = 0.f;
        bool nan = false;
        for (int k = 0; k < it.parts; ++k) {
            const float m = p.part_ml[(at + (int64_t)it.stride * k) * 2];
            nan |= m != m;
            M = fmaxf(M, m);
        }
        const float base = M == -INFINITY ? 0.f : M;
        floatx4 v = floatx4{0, 0, 0, 0};
        for (int k = 0; k < it.parts; ++k) {
            const float f = __builtin_amdgcn_exp2f(p.part_ml[(at + (int64_t)it.stride * k) * 2] - base);
            sum += p.part_ml[(at + (int64_t)it.stride * k) * 2 + 1] * f;
            v += *(const floatx4*)(p.part_o + (at + (int64_t)it.stride * k) * D + d) * f;
        }
        if (nan) sum = NAN;
        *(intx2*)(p.out + (int64_t)(it.row0 + rr / p.group) * p.out_stride + (h * p.group + rr % p.group) * D + d) =
            intx2{(int)pack2_bf16(v[0] / sum, v[1] / sum), (int)pack2_bf16(v[2] / sum, v[3] / sum)};
    }
}

}  // namespace symb
