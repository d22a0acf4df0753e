// New keys and values into the paged 8-bit cache, keys and queries turned by their positions.
//
// One workgroup takes one page's share of a segment for one head: of the keys or of the values; or the queries of the same rows, of one head (64 threads) or eight.  It holds the new
// values in registers (fp32, turned), forms their largest magnitude, from it the page's scale 2^e with max / 2^e in (224, 448], and rounds once.  If the
// page holds earlier tokens and its scale grows, those are read, scaled by the power of two that the scale grew by and held again.  Bound by memory: a new
// key or value costs 2 bytes in and 1 out, a query 2 and 2, and the angles 4 for each element of a row unless several heads share what was loaded.
// Measured: 8000 rows of 32 query and 32 key heads of 128 without turning (328 MB) in 69 us, 4.75 TB/s of the 4.93 that a large copy reaches; 6009 rows of 32 query and 16 key heads (175 MB) in 42 us where eight query
// heads share the angles, 45 with one and 48 with sixteen (too few workgroups); 48 us also where the queries come behind the keys in the grid.  A decode step's call
// is a launch, 10 to 11 us with the host's part.
#pragma once
#include "block_device.hpp"

namespace symb {

struct KvPage {                           // the rows of one segment that go to one page
    int32_t table;                        // its entry in the page table
    int32_t row0, rows;                   // rows of the flattened batch
    int32_t pos0;                         // the first one's position; its slot is pos0 % page_tokens
};

struct KvAppendParams {
    const KvPage* pages;
    const int32_t* page_table;
    unsigned char* k;
    unsigned char* v;
    unsigned char* k_scale;
    unsigned char* v_scale;
    const float* rotation;                // [positions][dim]: cosines, sines
    const bf16* q_in;
    bf16* q_out;
    const bf16* k_in;
    const bf16* v_in;
    int64_t q_stride, q_out_stride, k_stride, v_stride;
    int32_t num_pages, kv_heads, q_heads, page_shift;
    int32_t turned, adjacent;             // elements of a head that are turned; pairs side by side instead of half of them apart
    int32_t heads_q, q_groups;            // query heads a workgroup, workgroups for them
};

// Sixteen elements of a head's row, `slot` 0 .. D/16-1, in two chunks of eight that hold whole pairs.
__device__ __forceinline__ bool kv_slot_halves(const KvAppendParams& p, int slot, bool turn) { return turn && slot * 16 < p.turned && !p.adjacent; }
__device__ __forceinline__ int kv_chunk0(const KvAppendParams& p, int slot, bool turn) { return kv_slot_halves(p, slot, turn) ? slot : 2 * slot; }
__device__ __forceinline__ int kv_chunk1(const KvAppendParams& p, int slot, bool turn) { return kv_slot_halves(p, slot, turn) ? slot + (p.turned >> 4) : 2 * slot + 1; }
struct KvAngles {                         // of a slot's eight pairs
    float c[8], s[8];
};
__device__ __forceinline__ bool kv_turned(const KvAppendParams& p, int slot, bool turn) { return turn && slot * 16 < p.turned; }
__device__ __forceinline__ void kv_angles(const KvAppendParams& p, int slot, int pos, KvAngles& a) {
    const float* cs = p.rotation + (int64_t)pos * p.turned + slot * 8;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const floatx4 u = *(const floatx4*)(cs + 4 * h), w = *(const floatx4*)(cs + (p.turned >> 1) + 4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) a.c[4 * h + i] = u[i], a.s[4 * h + i] = w[i];
    }
}
__device__ __forceinline__ void kv_turn(const KvAppendParams& p, const intx4 a, const intx4 b, int slot, bool turn, const KvAngles& t, float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo((unsigned)a[i]);
        x[2 * i + 1] = bf16_hi((unsigned)a[i]);
        x[8 + 2 * i] = bf16_lo((unsigned)b[i]);
        x[8 + 2 * i + 1] = bf16_hi((unsigned)b[i]);
    }
    if (!kv_turned(p, slot, turn)) return;
    float u[8], w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float first = p.adjacent ? x[2 * i] : x[i], second = p.adjacent ? x[2 * i + 1] : x[8 + i];
        u[i] = first * t.c[i] - second * t.s[i];
        w[i] = second * t.c[i] + first * t.s[i];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = p.adjacent ? (i & 1 ? w[i >> 1] : u[i >> 1]) : (i < 8 ? u[i] : w[i - 8]);
}

// The smallest e with amax <= 448 * 2^e, within E8M0 and fp32's normal powers of two.
__device__ __forceinline__ int kv_exponent(float amax) {
    const int u = as_int(amax);
    return max((u >> 23) - 127 - 8 + ((u & 0x7fffff) > 0x600000), -126);
}

// THREADS 256: pages with many new rows, up to 128.  THREADS 64: at most kKvFewRows of them, as in decode steps: 16 times the workgroups that 256
// threads would leave with almost nothing to do.
constexpr int kKvFewRows = 8;
template <int D, int THREADS>
SYMB_KERNEL __launch_bounds__(THREADS) void symb_kv_append_kernel(KvAppendParams p) {
    constexpr int kSlots = D / 16, kPasses = THREADS == 64 ? kKvFewRows * kSlots / 64 + (kKvFewRows * kSlots < 64) : 128 * kSlots / 256;
    __shared__ float red[4];
    __shared__ __attribute__((aligned(16))) unsigned char tile[THREADS == 64 ? 16 : D * 128];
    const KvPage pg = p.pages[blockIdx.x];
    const int tid = threadIdx.x, P = 1 << p.page_shift;
    int y = blockIdx.y;
    constexpr int kHeads = THREADS == 64 ? 1 : 4;
    if (y < p.q_groups) {                                          // queries of the same rows, and of several heads: the angles of a row are the same for all
        const int h0 = y * p.heads_q, nh = min(p.heads_q, p.q_heads - h0);
        for (int i = tid; i < pg.rows * kSlots; i += THREADS) {
            const int slot = i % kSlots, r = i / kSlots;
            KvAngles t;
            if (kv_turned(p, slot, true)) kv_angles(p, slot, pg.pos0 + r, t);
            const bf16* in = p.q_in + (int64_t)(pg.row0 + r) * p.q_stride + h0 * D;
            bf16* out = p.q_out + (int64_t)(pg.row0 + r) * p.q_out_stride + h0 * D;
            const int c0 = kv_chunk0(p, slot, true) * 8, c1 = kv_chunk1(p, slot, true) * 8;
            for (int h = 0; h < nh; h += kHeads, in += kHeads * D, out += kHeads * D) {
                intx4 a[kHeads], b[kHeads];                        // (all loads first: q_out may be q, so the compiler may not move them over a store)
#pragma unroll
                for (int k = 0; k < kHeads; ++k)
                    if (h + k < nh) a[k] = *(const intx4*)(in + k * D + c0), b[k] = *(const intx4*)(in + k * D + c1);
#pragma unroll
                for (int k = 0; k < kHeads; ++k) {
                    if (h + k >= nh) break;
                    float x[16];
                    kv_turn(p, a[k], b[k], slot, true, t, x);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        a[k][j] = (int)pack2_bf16(x[2 * j], x[2 * j + 1]);
                        b[k][j] = (int)pack2_bf16(x[8 + 2 * j], x[8 + 2 * j + 1]);
                    }
                    *(intx4*)(out + k * D + c0) = a[k];
                    *(intx4*)(out + k * D + c1) = b[k];
                }
            }
        }
        return;
    }
    y -= p.q_groups;
    const int page = p.page_table[pg.table];
    if ((unsigned)page >= (unsigned)p.num_pages) return;           // (no such page: nothing is stored)
    const bool is_v = y >= p.kv_heads;
    const int h = is_v ? y - p.kv_heads : y;
    const int64_t block = (int64_t)page * p.kv_heads + h;
    unsigned char* scale = (is_v ? p.v_scale : p.k_scale) + block;
    unsigned char* codes = (is_v ? p.v : p.k) + ((block * D) << p.page_shift);
    const int first = pg.pos0 & (P - 1);
    const int old_byte = first ? *scale : 0;
    const bf16* rows = (is_v ? p.v_in + (int64_t)pg.row0 * p.v_stride : p.k_in + (int64_t)pg.row0 * p.k_stride) + h * D;
    const int64_t stride = is_v ? p.v_stride : p.k_stride;
    const int ntask = pg.rows * kSlots;
    float x[kPasses][16], amax = 0.f;
#pragma unroll
    for (int q = 0; q < kPasses; ++q) {
        const int i = q * THREADS + tid;
        if (i < ntask) {
            KvAngles t;
            if (kv_turned(p, i % kSlots, !is_v)) kv_angles(p, i % kSlots, pg.pos0 + i / kSlots, t);
            const bf16* row = rows + (i / kSlots) * stride;
            kv_turn(p, *(const intx4*)(row + kv_chunk0(p, i % kSlots, !is_v) * 8), *(const intx4*)(row + kv_chunk1(p, i % kSlots, !is_v) * 8), i % kSlots, !is_v, t, x[q]);
#pragma unroll
            for (int j = 0; j < 16; ++j) amax = fmaxf(amax, finite_abs(x[q][j]));
        }
    }
    amax = across_wave(amax, Max());
    if (THREADS > 64) {
        if ((tid & 63) == 0) red[tid >> 6] = amax;
        __syncthreads();
        amax = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    }
    const int byte = max(kv_exponent(amax) + 127, old_byte);
    const float inv = pow2(127 - byte);
    if (first && byte > old_byte) {                                // the kept tokens at the new scale
        const float f = pow2(old_byte - byte);
        const int vecs = (is_v ? D * ((first + 15) >> 4) : first * (D / 16)), per = is_v ? (first + 15) >> 4 : D / 16;
        for (int i = tid; i < vecs; i += THREADS) {
            // keys: tokens 0 .. first-1 are whole rows; values: the first slots of every channel's row (slots behind `first` keep their bytes or are written below)
            unsigned char* at = codes + (is_v ? (i / per) * P + (i % per) * 16 : i * 16);
            const int keep = is_v ? first - (i % per) * 16 : 16;
            intx4 w = *(const intx4*)at;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const floatx2 lo = e4m3_lo(w[j]), hi = e4m3_hi(w[j]);
                const int n = pack4_e4m3(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
                const int left = keep - 4 * j;
                const unsigned m = left >= 4 ? ~0u : left > 0 ? (1u << (8 * left)) - 1 : 0u;
                w[j] = (int)(((unsigned)n & m) | ((unsigned)w[j] & ~m));
            }
            *(intx4*)at = w;
        }
    }
    if (tid == 0) *scale = (unsigned char)byte;
    if (is_v) __syncthreads();                                     // (the kept tokens' vectors may hold new slots: those are written after them)
#pragma unroll
    for (int q = 0; q < kPasses; ++q) {
        const int i = q * THREADS + tid, r = i / kSlots;
        if (i < ntask) {
            intx4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pack4_e4m3(x[q][4 * j] * inv, x[q][4 * j + 1] * inv, x[q][4 * j + 2] * inv, x[q][4 * j + 3] * inv);
            if (!is_v) {
                *(intx2*)(codes + (first + r) * D + kv_chunk0(p, i % kSlots, true) * 8) = intx2{w[0], w[1]};
                *(intx2*)(codes + (first + r) * D + kv_chunk1(p, i % kSlots, true) * 8) = intx2{w[2], w[3]};
            } else {
                unsigned char* to = (THREADS > 64 ? tile : codes) + (i % kSlots) * 16 * P + first + r;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int b = 0; b < 4; ++b) to[(4 * j + b) * P] = (unsigned char)((unsigned)w[j] >> (8 * b));
            }
        }
    }
    if (!is_v || THREADS == 64) return;
    // the values' tile, a channel's tokens side by side, out in vectors of 16 tokens; single bytes where the new slots begin or end inside one
    __syncthreads();
    const int end = first + pg.rows, g0 = first >> 4, per = ((end + 15) >> 4) - g0;
    for (int i = tid; i < D * per; i += THREADS) {
        const int at = (i / per) * P + (g0 + i % per) * 16, s0 = (g0 + i % per) * 16;
        if (s0 >= first && s0 + 16 <= end) {
            *(intx4*)(codes + at) = *(const intx4*)(tile + at);
        } else {
            for (int s = max(s0, first); s < min(s0 + 16, end); ++s) codes[at + s - s0] = tile[at + s - s0];
        }
    }
}

}  // namespace symb
