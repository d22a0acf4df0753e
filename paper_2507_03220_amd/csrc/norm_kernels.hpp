// LayerNorm / RMSNorm of a flattened batch, every row with its own segment's weight, and the backward pass.
//
//   forward   z = (x - mu) r,  y = z w + b;   RMS: mu = 0
//   backward  g = dy w,  dx = r (g - z mean(g z) - mean(g)),  dw = sum_t dy z,  db = sum_t dy
//
// Both are bound by memory: forward reads and writes a row once (4 bytes an element), backward reads x and dy and writes dx (6 bytes).  So a row is read
// once, into registers as the bf16 pairs it came in, and everything else happens there: the mean first and then the squares about it (one pass with
// sums of x and x^2 cancels where the mean is large beside the deviation), in fp32.  Measured: 16384 rows of 6144 forward in 75 us, 5.4 TB/s; 20480 of 4608 backward 120 us, 4.7 TB/s, its partial
// sums and their reduction (5 us) included.  A single row is a launch: the kernel 2.1 us, 8 with the host's part.
#pragma once
#include "block_device.hpp"

namespace symb {

struct NormDesc {
    const bf16* w;
    const bf16* b;
    float* dw;
    float* db;
};

struct NormFwdParams {
    const bf16* X;
    bf16* Y;
    const int32_t* off;
    const NormDesc* norm;
    int32_t S, T, width;
    float eps, base;
};

struct NormVec {                          // eight consecutive elements
    unsigned v[4];
    __device__ __forceinline__ float get(int i) const { return i & 1 ? bf16_hi(v[i >> 1]) : bf16_lo(v[i >> 1]); }
};
__device__ __forceinline__ NormVec norm_load(const bf16* p) { return __builtin_bit_cast(NormVec, *(const intx4*)p); }
__device__ __forceinline__ void norm_store(bf16* p, const float* y) {
    intx4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (int)pack2_bf16(y[2 * i], y[2 * i + 1]);
    *(intx4*)p = o;
}
// The weight of eight columns (base added; ones without one).
__device__ __forceinline__ void norm_weight(const bf16* w, float base, int col, float (&out)[8]) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = 1.f;
        return;
    }
    const NormVec t = norm_load(w + col);
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = base + t.get(i);
}

// Keeps the pairs packed from one use to the next: the compiler would hold the widened values, at twice the registers.  (Where those fit, holding them is 7 % faster.)
template <int NV>
__device__ __forceinline__ void norm_packed(NormVec (&v)[NV]) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(v[i].v[j]));
}

// N sums over the WAVES wavefronts that share a row, in a fixed order; `slot` tells apart two uses with one barrier between them.
template <int WAVES, int N>
__device__ __forceinline__ void norm_sums(float (&s)[N], float (*lds)[WAVES][N], int wave, int slot) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = across_wave(s[i], Add());
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[slot][wave][i] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i] = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) s[i] += lds[slot][w][i];
        }
    }
}

// WAVES wavefronts on a row, NV vectors of eight elements a lane; workgroups of four wavefronts at least.
template <bool RMS, int WAVES, int NV>
SYMB_KERNEL __launch_bounds__(WAVES < 4 ? 256 : WAVES * 64) void symb_norm_fwd_kernel(NormFwdParams p) {
    constexpr int kRows = WAVES < 4 ? 4 / WAVES : 1, kLanes = WAVES * 64;
    __shared__ float lds[2][WAVES][1];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int t = blockIdx.x * kRows + (kRows > 1 ? wave : 0);
    const int lane = kRows > 1 ? threadIdx.x & 63 : threadIdx.x;
    if (t >= p.T) return;                              // (whole wavefronts; a row that several share has a workgroup of its own)
    const int nvec = p.width >> 3;
    const bf16* x = p.X + (int64_t)t * p.width;
    NormVec v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = i * kLanes + lane;
        v[i] = c < nvec ? norm_load(x + c * 8) : NormVec{{0, 0, 0, 0}};
    }
    const NormDesc nd = p.norm[seg_of_row(p.off, 0, p.S - 1, t)];
    float mu = 0.f, s[1];
    if (!RMS) {
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] += v[i].get(j);
        norm_sums<WAVES, 1>(s, lds, wave, 0);
        mu = s[0] / p.width;
    }
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i * kLanes + lane < nvec)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = v[i].get(j) - mu;
                s[0] += d * d;
            }
    norm_sums<WAVES, 1>(s, lds, wave, 1);
    const float r = 1.f / sqrtf(s[0] / p.width + p.eps);
    bf16* y = p.Y + (int64_t)t * p.width;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = i * kLanes + lane;
        if (c >= nvec) continue;
        float w[8], o[8];
        norm_weight(nd.w, p.base, c * 8, w);
        NormVec b{{0, 0, 0, 0}};
        if (nd.b) b = norm_load(nd.b + c * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = (v[i].get(j) - mu) * r * w[j] + b.get(j);
        norm_store(y + c * 8, o);
    }
}

// A run of rows of one segment; its sums of dy z and dy go to row `part` of the partial sums.
struct NormChunk {
    int32_t seg, row0, rows, part;
};
struct NormBwdParams {
    const bf16* X;
    const bf16* dY;
    bf16* dX;
    const NormDesc* norm;
    const NormChunk* chunks;
    float* part_w;                        // [parts][width]
    float* part_b;
    int32_t width;
    float eps, base;
};

// BIAS: some segment wants dbias.  One workgroup a chunk, the whole width across its lanes: a lane meets the same columns in every row, so the weight gradient's sums stay in its registers.
template <bool RMS, bool BIAS, int WAVES, int NV>
SYMB_KERNEL __launch_bounds__(WAVES * 64) void symb_norm_bwd_kernel(NormBwdParams p) {
    constexpr int kLanes = WAVES * 64;
    constexpr bool kAhead = WAVES * NV < 32;           // (two rows of the widest do not fit the registers)
    __shared__ float lds[2][WAVES][2];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x;
    const NormChunk ch = p.chunks[blockIdx.x];
    const NormDesc nd = p.norm[ch.seg];
    const int nvec = p.width >> 3;
    const float inv = 1.f / p.width;
    float aw[NV][8] = {}, ab[NV][8] = {};
    NormVec w[NV], x[NV], dy[NV];
    auto ask = [&](int64_t at) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = i * kLanes + lane;
            if (c >= nvec) continue;
            x[i] = norm_load(p.X + at + c * 8);
            dy[i] = norm_load(p.dY + at + c * 8);
        }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = i * kLanes + lane;
        x[i] = dy[i] = NormVec{{0, 0, 0, 0}};          // (columns behind the last one count as zeros, weight included)
        w[i] = nd.w && c < nvec ? norm_load(nd.w + c * 8) : NormVec{{0, 0, 0, 0}};
    }
    const float base = nd.w ? p.base : 1.f;
    int64_t at = (int64_t)ch.row0 * p.width;
    if (kAhead) ask(at);
    for (int k = 0; k < ch.rows; ++k, at += p.width) {
        if (!kAhead) {
            ask(at);
            __builtin_amdgcn_sched_barrier(0);
        }
        float mu = 0.f, mg = 0.f, s[2];
        if (!RMS) {
            s[0] = s[1] = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    s[0] += x[i].get(j);
                    s[1] += dy[i].get(j) * (base + w[i].get(j));
                }
            norm_sums<WAVES, 2>(s, lds, wave, 0);
            mu = s[0] * inv;
            mg = s[1] * inv;
            if (!kAhead) norm_packed(x), norm_packed(dy), norm_packed(w);
        }
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * kLanes + lane < nvec)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = x[i].get(j) - mu;
                    s[0] += d * d;
                    s[1] += dy[i].get(j) * (base + w[i].get(j)) * d;
                }
        NormVec x0[NV], dy0[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) x0[i] = x[i], dy0[i] = dy[i];
        if (!kAhead) norm_packed(x0), norm_packed(dy0), norm_packed(w);
        if (kAhead && k + 1 < ch.rows) ask(at + p.width);        // the next row's way, while the sums of this one cross the wavefronts
        norm_sums<WAVES, 2>(s, lds, wave, RMS ? k & 1 : 1);             // (one barrier a row: two rows in turn)
        const float r = 1.f / sqrtf(s[0] * inv + p.eps), mgz = s[1] * r * inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = i * kLanes + lane;
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float z = (x0[i].get(j) - mu) * r, g = dy0[i].get(j);
                o[j] = r * (g * (base + w[i].get(j)) - mg - z * mgz);
                aw[i][j] += g * z;
                if (BIAS) ab[i][j] += g;
            }
            if (c < nvec) norm_store(p.dX + at + c * 8, o);
        }
    }
    if (ch.part < 0) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = i * kLanes + lane;
        if (c >= nvec) continue;
        const int64_t at = (int64_t)ch.part * p.width + c * 8;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (nd.dw) *(floatx4*)(p.part_w + at + 4 * q) = floatx4{aw[i][4 * q], aw[i][4 * q + 1], aw[i][4 * q + 2], aw[i][4 * q + 3]};
            if (BIAS && nd.db) *(floatx4*)(p.part_b + at + 4 * q) = floatx4{ab[i][4 * q], ab[i][4 * q + 1], ab[i][4 * q + 2], ab[i][4 * q + 3]};
        }
    }
}

// Segments that share their gradients: parts part0 .. part0 + parts - 1, added in that order.
struct NormGroup {
    float* dw;
    float* db;
    int32_t part0, parts;
};
struct NormReduceParams {
    const float* part_w;
    const float* part_b;
    const NormGroup* groups;
    int32_t width, accumulate;
};
// 64 columns a workgroup, 16 parts at once; each lane's sum in the order of the parts, the 16 sums one after the other.
SYMB_KERNEL __launch_bounds__(256) void symb_norm_reduce_kernel(NormReduceParams p) {
    __shared__ floatx4 sums[16][16];
    const int lane = threadIdx.x & 15, set = threadIdx.x >> 4, c = blockIdx.x * 64 + lane * 4;
    const NormGroup g = p.groups[blockIdx.y];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float* out = k ? g.db : g.dw;
        if (!out) continue;                            // (the same in all lanes)
        floatx4 s = floatx4{0, 0, 0, 0};
        if (c < p.width) {
            const float* part = (k ? p.part_b : p.part_w) + (int64_t)g.part0 * p.width + c;
#pragma unroll 4
            for (int i = set; i < g.parts; i += 16) s += *(const floatx4*)(part + (int64_t)i * p.width);
        }
        sums[set][lane] = s;
        __syncthreads();
        if (set == 0 && c < p.width) {
#pragma unroll
            for (int i = 1; i < 16; ++i) s += sums[i][lane];
            if (p.accumulate) s += *(const floatx4*)(out + c);
            *(floatx4*)(out + c) = s;
        }
        __syncthreads();
    }
}

}  // namespace symb
