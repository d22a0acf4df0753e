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
    const KvRowsItem* items;
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
    const int e = max((as_int(amax) >> 23) - 127 - 7, -100);       // amax / 2^e in [128, 256); infinities and NaN become NaN
    const float inv = pow2(-e);
    int hi[D / 16], lo[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = x[4 * i + j] * inv;
        hi[i] = pack4_e4m3(y[0], y[1], y[2], y[3]);
        const floatx2 a = e4m3_lo(hi[i]), b = e4m3_hi(hi[i]);
        lo[i] = pack4_e4m3((y[0] - a[0]) * 16.f, (y[1] - a[1]) * 16.f, (y[2] - b[0]) * 16.f, (y[3] - b[1]) * 16.f);
    }
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
    const KvRowsItem it = p.items[blockIdx.x / p.kv_heads];
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
            hi[i] = pack4_e4m3(y[0], y[1], y[2], y[3]);
            const floatx2 a = e4m3_lo(hi[i]), b = e4m3_hi(hi[i]);
            lo[i] = pack4_e4m3((y[0] - a[0]) * 16.f, (y[1] - a[1]) * 16.f, (y[2] - b[0]) * 16.f, (y[3] - b[1]) * 16.f);
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

// The parts of up to 16 rows' results: part i of row r at partial row part0 + 16 i + r.
struct KvJoinItem {
    int32_t row0, rows, r0, part0, parts;
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
            const float m = p.part_ml[(at + 16 * k) * 2];
            nan |= m != m;
            M = fmaxf(M, m);
        }
        const float base = M == -INFINITY ? 0.f : M;
        floatx4 v = floatx4{0, 0, 0, 0};
        for (int k = 0; k < it.parts; ++k) {
            const float f = __builtin_amdgcn_exp2f(p.part_ml[(at + 16 * k) * 2] - base);
            sum += p.part_ml[(at + 16 * k) * 2 + 1] * f;
            v += *(const floatx4*)(p.part_o + (at + 16 * k) * D + d) * f;
        }
        if (nan) sum = NAN;
        *(intx2*)(p.out + (int64_t)(it.row0 + rr / p.group) * p.out_stride + (h * p.group + rr % p.group) * D + d) =
            intx2{(int)pack2_bf16(v[0] / sum, v[1] / sum), (int)pack2_bf16(v[2] / sum, v[3] / sum)};
    }
}

}  // namespace symb
