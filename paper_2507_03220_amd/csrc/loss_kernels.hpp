// Losses through the frozen vocabulary matrix W [V][d] without its logits, and their gradient: cross entropy of a label, and divergence from a teacher's top entries.
//
//   s_v = x . W_v,   z_v = cap tanh(s_v / cap) or s_v,   p = softmax(z / T)
//   L = -log p_label (T = 1),  or  T^2 sum_j q_j (log q_j - log p_{id_j}),  q = softmax of the row's entries / T
//   dx = g T sum_v (p_v - q_v) z'_v W_v,   q_v = [v = label] or the sum of the q_j with id_j = v,  z' = 1 - (z / cap)^2
//
// Two products, bound by the matrix cores: X W^T, and the weights with W.  No third one, because what lies between them, the unnormalised weights 2^(t_v) of a chunk of rows, t_v = a z_v - b,
// is held (bf16) until their sums are known: b makes the label's (a teacher's best entry's) weight one, so it is known beforehand from one dot product a row, sums are never zero, and a weight
// grows beyond 2^64 only where another score lies that far above.  Such columns of a row are held 2^shift smaller, and made equal again when the row's sums meet.
// The label's own weight is left out of the sum S of the others: the loss is log(1 + S) and its entry of p - q is -S / (1 + S), neither a difference of two numbers that may be almost equal.
// A row's entries of q go into the held weights in fp32, rounded once with them.
#pragma once
#include "block_device.hpp"
#include "gemm16_kernel.hpp"

namespace symb {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct LossDesc {
    float scale, temperature;
};
struct LossParams {
    const bf16* X;
    const bf16* W;
    bf16* dX;                             // or null: losses alone
    const int32_t* flags;                 // [T] the label of every row, or whether it has a teacher (0); negative: the row takes no part
    int32_t* own_flags;                   // flags, where they are made of `ids`
    const int32_t* ids;                   // [T][K] or null
    const float* teacher;                 // [T][K]
    float* loss;                          // [S] or null
    float* row_loss;                      // [T]
    const int32_t* off;                   // [S + 1]
    const LossDesc* losses;               // [S]
    int32_t* rows;                        // [T] the rows that take part, in order
    int32_t* count;                       // how many they are
    float* gain;                          // [S] scale, over the segment's rows that take part if the loss is a mean
    float* scores;                        // [T][K] a z_j - b of a row's entries
    float* slopes;                        // [T][K] z'
    float* shares;                        // [T][K] q
    float2* row_ab;                       // [T] a and b
    float* row_base;                      // [T] sum_j q_j (log q_j - (a z_j - b) ln 2)
    float2* stats;                        // [column parts][chunk] shift and sum of a row's weights
    float* row_gain;                      // [chunk] what a row's product is multiplied with
    bf16* held;                           // [chunk][pitch] weights
    float* parts;                         // partial tiles of the second product
    int64_t part_tiles;                   // room for that many
    int32_t T, S, V, pitch, width, K;
    int32_t chunk0, chunk;                // the chunk's first row (of those that take part) and its length at most
    int32_t group_m, mean;
    float cap, to_cap;                    // 1 / cap
};

// cap tanh(s / cap) and its slope.  1 - 2 / (e^2|y| + 1) is off by some 2^-24 of the cap, which may be more than a score far below it: there it is the series.
__device__ __forceinline__ float loss_capped(float s, float cap, float to_cap, float& slope) {
    const float y = s * to_cap, y2 = y * y;
    const float r = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(fabsf(y) * (2.f * kLog2e)) + 1.f);
    const float far = copysignf(cap * (1.f - 2.f * r), s);
    const float part = y2 * (1.f / 3 - y2 * (2.f / 15 - y2 * (17.f / 315 - y2 * (62.f / 2835))));
    const float near = s - s * part, u = y - y * part;
    const bool is_near = fabsf(y) < 0.25f;
    slope = is_near ? 1.f - u * u : 4.f * r * (1.f - r);
    return is_near ? near : far;
}

// ---- which rows take part -----------------------------------------------------------------------------------------------------------
// A row with a teacher: flag 0, and the softmax of its entries (absent ones: share 0).  One wavefront a row.
SYMB_KERNEL __launch_bounds__(256) void symb_loss_teacher_kernel(LossParams p) {
    const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (t >= p.T) return;
    const int32_t* ids = p.ids + (int64_t)t * p.K;
    const float* l = p.teacher + (int64_t)t * p.K;
    float* q = p.shares + (int64_t)t * p.K;
    const float to_t = 1.f / p.losses[seg_of_row(p.off, 0, p.S - 1, t)].temperature;
    bool any = false;
    float most = -__builtin_inff();
    for (int j = lane; j < p.K; j += 64)
        if (ids[j] >= 0) {
            any = true;
            most = fmaxf(most, l[j]);
        }
    const bool part = __ballot(any) != 0;
    if (lane == 0) p.own_flags[t] = part ? 0 : -1;
    if (!part) return;
    most = across_wave(most, Max());
    float sum = 0.f;
    for (int j = lane; j < p.K; j += 64) {
        const float e = ids[j] >= 0 ? expf((l[j] - most) * to_t) : 0.f;
        q[j] = e;
        sum += e;
    }
    sum = across_wave(sum, Add());
    for (int j = lane; j < p.K; j += 64) q[j] /= sum;
}

// Sum of `v` over the workgroup's 256 threads.
__device__ __forceinline__ int loss_count(int v, int* lds) {
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0] + lds[1] + lds[2] + lds[3];
    __syncthreads();
    return v;
}
// The first workgroups list the rows of 256 each (every one counts those before its own); one a segment counts its rows.
SYMB_KERNEL __launch_bounds__(256) void symb_loss_rows_kernel(LossParams p) {
    __shared__ int lds[4];
    const int lists = (p.T + 255) / 256, b = blockIdx.x;
    if (b < lists) {
        int before = 0;
        for (int t = threadIdx.x; t < b * 256; t += 256) before += p.flags[t] >= 0;
        before = loss_count(before, lds);
        const int t = b * 256 + threadIdx.x;
        const bool part = t < p.T && p.flags[t] >= 0;
        const unsigned long long mine = __ballot(part);
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if (lane == 0) lds[wave] = __popcll(mine);
        __syncthreads();
        int at = before + __popcll(mine & ((1ull << lane) - 1));
        for (int w = 0; w < wave; ++w) at += lds[w];
        if (part) p.rows[at] = t;
        if (b == lists - 1 && threadIdx.x == 0) *p.count = before + lds[0] + lds[1] + lds[2] + lds[3];
        return;
    }
    const int i = b - lists;
    int n = 0;
    for (int t = p.off[i] + threadIdx.x; t < p.off[i + 1]; t += 256) n += p.flags[t] >= 0;
    n = loss_count(n, lds);
    if (threadIdx.x == 0) p.gain[i] = p.mean ? p.losses[i].scale / (float)max(n, 1) : p.losses[i].scale;
}

// ---- the scores of a row's own entries ----------------------------------------------------------------------------------------------
// One workgroup a row: its entries' dot products, a wavefront each in turn; a and b; rows that take no part get their zeros.
SYMB_KERNEL __launch_bounds__(256) void symb_loss_entries_kernel(LossParams p) {
    __shared__ float best[4];
    const int t = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), nvec = p.width >> 3;
    const int flag = p.flags[t];
    if (flag < 0) {
        if (threadIdx.x == 0) p.row_loss[t] = 0.f;
        if (p.dX)
            for (int c = threadIdx.x; c < nvec; c += 256) *(intx4*)(p.dX + (int64_t)t * p.width + c * 8) = intx4{0, 0, 0, 0};
        return;
    }
    const bf16* x = p.X + (int64_t)t * p.width;
    const float a = p.ids ? kLog2e / p.losses[seg_of_row(p.off, 0, p.S - 1, t)].temperature : kLog2e;
    float most = -__builtin_inff();
    for (int j = wave; j < p.K; j += 4) {
        const int id = p.ids ? p.ids[(int64_t)t * p.K + j] : flag;
        if (id < 0) continue;
        float s = 0.f;
        if (id < p.V) {
            const bf16* w = p.W + (int64_t)id * p.width;
            for (int c = lane; c < nvec; c += 64) {
                const intx4 u = *(const intx4*)(x + c * 8), v = *(const intx4*)(w + c * 8);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s = fmaf(bf16_lo((unsigned)u[i]), bf16_lo((unsigned)v[i]), s);
                    s = fmaf(bf16_hi((unsigned)u[i]), bf16_hi((unsigned)v[i]), s);
                }
            }
            s = across_wave(s, Add());
        } else s = __builtin_nanf("");               // (a number outside the vocabulary is never followed)
        float slope = 1.f;
        if (p.cap > 0.f) s = loss_capped(s, p.cap, p.to_cap, slope);
        const float z = s * a;
        if (lane == 0) {
            p.scores[(int64_t)t * p.K + j] = z;
            p.slopes[(int64_t)t * p.K + j] = slope;
        }
        most = z != z || most != most ? __builtin_nanf("") : fmaxf(most, z);
    }
    if (lane == 0) best[wave] = most;
    __syncthreads();
    float b = best[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) b = b != b || best[w] != best[w] ? __builtin_nanf("") : fmaxf(b, best[w]);
    if (threadIdx.x == 0) p.row_ab[t] = make_float2(a, b);
    if (!p.ids || wave) return;
    float base = 0.f;
    for (int j = lane; j < p.K; j += 64) {
        const int64_t at = (int64_t)t * p.K + j;
        if (p.ids[at] < 0) continue;
        const float z = p.scores[at] - b, q = p.shares[at];
        p.scores[at] = z;
        if (!(q == 0.f)) base += q * (logf(q) - z * kLn2);
    }
    base = across_wave(base, Add());
    if (lane == 0) p.row_base[t] = base;
}

// ---- products -------------------------------------------------------------------------------------------------------------------------
// A tile of Aop [rows][K] times Bop ([columns][K], or [K][columns] if NN) into the accumulation registers, with the loops of gemm16_asm.hpp: stages st0 .. st0 + KF - 1 of 64, and what K leaves
// behind the last whole stage if `tail`.  a_at(row): where a row of the tile starts, in elements from a_tile; b_tile: its first column at k = 0, `ldb` elements from the next (NN: from the next k);
// `columns`: how many there are.  The lane layout is that of symb_gemm16_kernel.
template <int BLK, bool NN, class Row>
__device__ __forceinline__ void loss_tile(unsigned char* smem, const bf16* a_tile, Row a_at, const bf16* b_tile, int ldb, int columns, int st0, int KF, bool tail, int K) {
    using TT = Gemm16Tile<BLK, BLK>;
    constexpr int BM = TT::BM, BN = TT::BN, NT = TT::NT;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm0 = (wave >> 1) * TT::WM, wn0 = (wave & 1) * TT::WN, l15 = lane & 15, lg = lane >> 4;
    const unsigned lds0 = (unsigned)(size_t)smem;
    auto frag_a = [&](int ks, int q) __attribute__((always_inline)) { return (unsigned)(lds_off_kmajor(wm0 + l15, ks * 4 + q * 2 + (lg >> 1)) + ((lg & 1) << 3)); };
    auto frag_b_nt = [&](int ks, int q) __attribute__((always_inline)) { return (unsigned)(lds_off_kmajor(wn0 + l15, ks * 4 + q * 2 + (lg >> 1)) + ((lg & 1) << 3)); };
    auto frag_b_nn = [&](int j) __attribute__((always_inline)) {
        const int k = (lg >> 1) * 8 + (lg & 1) * 4 + (l15 >> 2), n = wn0 + j * 16 + ((l15 & 3) << 2);
        return (unsigned)(lds_off_nmajor16<BN>(k, n >> 3) + ((n & 7) << 1));
    };
    if (KF == 0) {
        if constexpr (BLK == 8) asm volatile(SYMB_GEMM16_ZERO ::: SYMB_GEMM16_ACLOBBERS);
        else asm volatile(SYMB_GEMM16S_ZERO ::: SYMB_GEMM16S_ACLOBBERS);
    } else {
        constexpr int NVB = BLK > 4 ? BLK : 4;
        unsigned vA[4], vB[NVB], ab[BLK], bb[BLK];
#pragma unroll
        for (int j = 0; j < 4; ++j) vA[j] = lds0 + frag_a(j >> 1, j & 1);
#pragma unroll
        for (int j = 0; j < NVB; ++j) vB[j] = lds0 + (NN ? frag_b_nn(j % BLK) : frag_b_nt((j >> 1) & 1, j & 1));
#pragma unroll
        for (int j = 0; j < BLK; ++j) {
            const int row = (wave * BLK + j) * 8 + (lane >> 3), kc = (lane & 7) ^ swz_row(row);
            ab[j] = (a_at(row) + kc * 8) * 2u;
            if constexpr (!NN) bb[j] = ((unsigned)min(row, columns - 1) * (unsigned)ldb + kc * 8) * 2u;
            else {
                constexpr int CPR = BN / 8;
                const int krow = (wave * BLK + j) * (64 / CPR) + lane / CPR, nc = (lane % CPR) ^ swz_nmajor16(krow);
                bb[j] = ((unsigned)krow * (unsigned)ldb + (unsigned)min(nc * 8, columns - 8)) * 2u;
            }
        }
        const unsigned long long ga = (unsigned long long)(a_tile + (size_t)st0 * 64);
        const unsigned long long gb = (unsigned long long)(b_tile + (size_t)st0 * 64 * (NN ? ldb : 1));
        const unsigned stride_b = NN ? 128u * (unsigned)ldb : 128u;
        const unsigned swa = (unsigned)__builtin_amdgcn_readfirstlane((int)lds0 + wave * (1024 * BLK));
        if constexpr (BLK == 8) {
#define SYMB_LOSS_LOOP_OPERANDS                                                                                     \
    :                                                                                                              \
    : "v"(vA[0]), "v"(vA[1]), "v"(vA[2]), "v"(vA[3]), "v"(vB[0]), "v"(vB[1]), "v"(vB[2]), "v"(vB[3]), "v"(vB[4]),  \
      "v"(vB[5]), "v"(vB[6]), "v"(vB[7]), "v"(ab[0]), "v"(ab[1]), "v"(ab[2]), "v"(ab[3]), "v"(ab[4]), "v"(ab[5]), "v"(ab[6]), "v"(ab[7]),  \
      "v"(bb[0]), "v"(bb[1]), "v"(bb[2]), "v"(bb[3]), "v"(bb[4]), "v"(bb[5]), "v"(bb[6]), "v"(bb[7]),              \
      "s"(ga), "s"(gb), "s"(stride_b), "s"(KF), "s"(swa)                                                           \
    : "memory", "scc", SYMB_GEMM16_SCLOBBERS, SYMB_GEMM16_VCLOBBERS, SYMB_GEMM16_ACLOBBERS
            if constexpr (NN) asm volatile(SYMB_GEMM16_LOOP_NN SYMB_LOSS_LOOP_OPERANDS);
            else asm volatile(SYMB_GEMM16_LOOP_NT SYMB_LOSS_LOOP_OPERANDS);
#undef SYMB_LOSS_LOOP_OPERANDS
        } else {
#define SYMB_LOSS_LOOP_OPERANDS                                                                                     \
    :                                                                                                              \
    : "v"(vA[0]), "v"(vA[1]), "v"(vA[2]), "v"(vA[3]), "v"(vB[0]), "v"(vB[1]), "v"(vB[2]), "v"(vB[3]),              \
      "v"(ab[0]), "v"(ab[1]), "v"(ab[2]), "v"(ab[3]), "v"(bb[0]), "v"(bb[1]), "v"(bb[2]), "v"(bb[3]),              \
      "s"(ga), "s"(gb), "s"(stride_b), "s"(KF), "s"(swa)                                                           \
    : "memory", "scc", SYMB_GEMM16_SCLOBBERS, SYMB_GEMM16S_VCLOBBERS, SYMB_GEMM16S_ACLOBBERS
            if constexpr (NN) asm volatile(SYMB_GEMM16S_LOOP_NN SYMB_LOSS_LOOP_OPERANDS);
            else asm volatile(SYMB_GEMM16S_LOOP_NT SYMB_LOSS_LOOP_OPERANDS);
#undef SYMB_LOSS_LOOP_OPERANDS
        }
        __builtin_amdgcn_s_barrier();                // everything landed and read before LDS is reused
    }
    const int k0 = K / 64 * 64;
    if (!tail || k0 == K) return;
    // what is left of K, through registers: chunk i of a thread lies 32 rows (KSTEP k-rows) below chunk 0
    constexpr int CA = BM * 8 / NT, RSTEP = NT / 8, KSTEP = NT / (BN / 8);
    unsigned char *const sA = smem, *const sB = smem + TT::UNIT_A;
    const int lrow = tid >> 3, lkc = (tid & 7) * 8, nn_k = tid / (BN / 8), nn_nc = tid % (BN / 8);
    uint4 ra[CA], rb[CA];
#pragma unroll
    for (int i = 0; i < CA; ++i) {
        ra[i] = ld_global_16(a_tile + a_at(lrow + i * RSTEP) + k0 + lkc, k0 + lkc < K);
        if constexpr (!NN) rb[i] = ld_global_16(b_tile + (size_t)min(lrow + i * RSTEP, columns - 1) * ldb + k0 + lkc, k0 + lkc < K);
        else {
            const int k = k0 + nn_k + i * KSTEP;
            rb[i] = ld_global_16(b_tile + (size_t)min(k, K - 1) * ldb + min(nn_nc * 8, columns - 8), k < K);
        }
    }
    const int a_lds0 = lds_off_kmajor(lrow, tid & 7), b_lds0 = NN ? lds_off_nmajor16<BN>(nn_k, nn_nc) : a_lds0;
#pragma unroll
    for (int i = 0; i < CA; ++i) {
        *reinterpret_cast<uint4*>(sA + a_lds0 + i * RSTEP * 128) = ra[i];
        *reinterpret_cast<uint4*>(sB + b_lds0 + i * (NN ? KSTEP * (BN * 2) : RSTEP * 128)) = rb[i];
    }
    __syncthreads();
    const unsigned all = (1u << BLK) - 1;
    for (int ks = 0; ks < (K - k0 + 31) >> 5; ++ks) {
        const unsigned va0 = lds0 + frag_a(ks, 0), va1 = lds0 + frag_a(ks, 1);
        if constexpr (!NN) {
            const unsigned vb0 = lds0 + TT::UNIT_A + frag_b_nt(ks, 0), vb1 = lds0 + TT::UNIT_A + frag_b_nt(ks, 1);
            if constexpr (BLK == 8)
                asm volatile(SYMB_GEMM16_KSTEP32_NT : : "v"(va0), "v"(va1), "v"(vb0), "v"(vb1), "s"(all) : "memory", "scc", SYMB_GEMM16_VCLOBBERS, SYMB_GEMM16_ACLOBBERS);
            else
                asm volatile(SYMB_GEMM16S_KSTEP32_NT : : "v"(va0), "v"(va1), "v"(vb0), "v"(vb1), "s"(all) : "memory", "scc", SYMB_GEMM16S_VCLOBBERS, SYMB_GEMM16S_ACLOBBERS);
        } else {
            unsigned vb[BLK];
#pragma unroll
            for (int j = 0; j < BLK; ++j) vb[j] = lds0 + TT::UNIT_A + frag_b_nn(j) + ks * 32 * (BN * 2);
            if constexpr (BLK == 8)
                asm volatile(SYMB_GEMM16_KSTEP32_NN : : "v"(va0), "v"(va1), "v"(vb[0]), "v"(vb[1]), "v"(vb[2]), "v"(vb[3]), "v"(vb[4]), "v"(vb[5]), "v"(vb[6]), "v"(vb[7]), "s"(all)
                             : "memory", "scc", SYMB_GEMM16_VCLOBBERS, SYMB_GEMM16_ACLOBBERS);
            else
                asm volatile(SYMB_GEMM16S_KSTEP32_NN : : "v"(va0), "v"(va1), "v"(vb[0]), "v"(vb[1]), "v"(vb[2]), "v"(vb[3]), "s"(all)
                             : "memory", "scc", SYMB_GEMM16S_VCLOBBERS, SYMB_GEMM16S_ACLOBBERS);
        }
    }
    __syncthreads();
}

// Rows of this chunk that take part.
__device__ __forceinline__ int loss_chunk_rows(const LossParams& p) { return min(*p.count - p.chunk0, p.chunk); }

// Tile number `lin` of m_tiles x n_tiles, group_m rows of tiles at a time: tiles that run side by side share their operands in L2.
__device__ __forceinline__ void loss_place(int lin, int m_tiles, int n_tiles, int group_m, int& tm, int& tn) {
    const int width = group_m * n_tiles, first = lin / width * group_m, rows = min(m_tiles - first, group_m);
    tm = first + lin % width % rows;
    tn = lin % width / rows;
}

// X W^T of a chunk, a tile a workgroup: its rows' sums of weights, and the weights themselves where the gradient wants them.
template <int BLK, bool GRAD, bool CAP>
SYMB_KERNEL __launch_bounds__(256) void symb_loss_scores_kernel(const LossParams p) {
    using TT = Gemm16Tile<BLK, BLK>;
    constexpr int BM = TT::BM, BN = TT::BN, CP = TT::C_PITCH;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int rows = loss_chunk_rows(p);
    if (rows <= 0) return;
    const int m_tiles = (rows + BM - 1) / BM, n_tiles = (p.V + BN - 1) / BN, total = m_tiles * n_tiles, per_xcd = (total + 7) >> 3;
    const int lin = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || lin >= total) return;
    int tm, tn;
    loss_place(lin, m_tiles, n_tiles, p.group_m, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN;
    const int32_t* const list = p.rows + p.chunk0;
    const int first = list[m0];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm0 = (wave >> 1) * TT::WM, wn0 = (wave & 1) * TT::WN, l15 = lane & 15, lg = lane >> 4;
    // what the epilogue needs of this lane's rows
    float a[BLK], b[BLK];
    int label[BLK];
#pragma unroll
    for (int i = 0; i < BLK; ++i) {
        const int t = list[min(m0 + wm0 + 16 * i + l15, rows - 1)];
        const float2 ab = p.row_ab[t];
        a[i] = ab.x;
        b[i] = ab.y;
        label[i] = p.ids ? -1 : p.flags[t] - (n0 + wn0 + 4 * lg);              // of block j, element e: 16 j + e
    }
    auto a_at = [&](int row) __attribute__((always_inline)) { return (unsigned)(list[min(m0 + row, rows - 1)] - first) * (unsigned)p.width; };
    loss_tile<BLK, false>(smem, p.X + (size_t)first * p.width, a_at, p.W + (size_t)n0 * p.width, p.width, p.V - n0, 0, p.width / 64, true, p.width);

    const unsigned c_lane = (unsigned)((wm0 + l15) * CP + (wn0 + lg * 4) * 2);
    const int left = p.V - (n0 + wn0 + 4 * lg);                                // columns of this lane: 16 j + e < left
    const bool edge = n0 + BN > p.V;
    float2* const stats = p.stats + (size_t)(2 * tn + (wave & 1)) * p.chunk + m0 + wm0;
    static_for<0, BLK>([&](auto I) __attribute__((always_inline)) {
        constexpr int i = decltype(I)::value;
        float w[BLK][4], slope[CAP ? BLK : 1][4];
        float sum = 0.f, shift = 0.f;
        static_for<0, BLK>([&](auto J) __attribute__((always_inline)) {
            constexpr int j = decltype(J)::value;
            acc16_read4<4 * (BLK * i + j)>(w[j][0], w[j][1], w[j][2], w[j][3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (CAP) w[j][e] = loss_capped(w[j][e], p.cap, p.to_cap, slope[j][e]);
                w[j][e] = fmaf(w[j][e], a[i], -b[i]);
                if (edge && 16 * j + e >= left) w[j][e] = -__builtin_inff();
            }
        });
        auto weights = [&]() __attribute__((always_inline)) {
            sum = 0.f;
#pragma unroll
            for (int j = 0; j < BLK; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = __builtin_amdgcn_exp2f(w[j][e] - shift);
                    sum += 16 * j + e == label[i] ? 0.f : v;
                }
            sum = across_rows(sum, Add());
        };
        weights();
        if (__any(!(sum < 0x1p64f))) {                                         // scores far above the row's own entries (or NaN)
            float most = w[0][0];
#pragma unroll
            for (int j = 0; j < BLK; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, w[j][e]);
            most = across_rows(most, Max());
            shift = sum < 0x1p64f ? 0.f : most;
            weights();
        }
        if (lg == 0) stats[16 * i + l15] = make_float2(shift, sum);            // (rows behind the last one have room)
        if constexpr (GRAD) {
#pragma unroll
            for (int j = 0; j < BLK; ++j) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = __builtin_amdgcn_exp2f(w[j][e] - shift);
                    if constexpr (CAP) v[e] *= slope[j][e];
                }
                *reinterpret_cast<uint2*>(smem + c_lane + i * 16 * CP + j * 32) = make_uint2(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]));
            }
        }
    });
    if constexpr (GRAD) {
        __syncthreads();
        constexpr int LPR = BN / 8, RPP = 256 / LPR;
        const int col = (lane % LPR) * 8, r0 = wave * (64 / LPR) + lane / LPR;
        if (n0 + col < p.pitch) {
            bf16* const out = p.held + (size_t)m0 * p.pitch + n0 + col;
#pragma unroll 8
            for (int r = r0; r < BM; r += RPP)
                if (m0 + r < rows) *reinterpret_cast<uint4*>(out + (size_t)r * p.pitch) = *reinterpret_cast<const uint4*>(smem + r * CP + col * 2);
        }
    }
}

// ---- sums, losses, and the entries of q ---------------------------------------------------------------------------------------------
constexpr int kJoinRows = 16, kJoinSets = 32;
// 16 rows a workgroup of 512: the column parts' sums in a fixed order, the rows' losses, and their entries of p - q into the held weights.  `parts`: column parts of `cols` columns.
SYMB_KERNEL __launch_bounds__(kJoinRows* kJoinSets) void symb_loss_join_kernel(const LossParams p, int parts, int cols) {
    __shared__ float2 lds[kJoinSets][kJoinRows];
    __shared__ float row_most[kJoinRows], row_sum[kJoinRows];
    const int rows = loss_chunk_rows(p), m0 = blockIdx.x * kJoinRows;
    if (m0 >= rows) return;
    const int r = threadIdx.x % kJoinRows, set = threadIdx.x / kJoinRows, m = m0 + r;
    // pairs (most, sum): the sum counts in units of 2^most
    auto join = [](float2 x, float2 y) {
        const float top = fmaxf(x.x, y.x);
        return make_float2(top, (x.x == top ? x.y : x.y * exp2f(x.x - top)) + (y.x == top ? y.y : y.y * exp2f(y.x - top)));
    };
    float2 s = make_float2(0.f, 0.f);
    if (m < rows)
#pragma unroll 4
        for (int c = set; c < parts; c += kJoinSets) s = join(s, p.stats[(size_t)c * p.chunk + m]);
    lds[set][r] = s;
    __syncthreads();
    if (set == 0 && m < rows) {
        for (int k = 1; k < kJoinSets; ++k) s = join(s, lds[k][r]);
        const int t = p.rows[p.chunk0 + m], seg = seg_of_row(p.off, 0, p.S - 1, t);
        float loss, l = s.y;
        if (!p.ids) {
            loss = s.x == 0.f ? log1pf(s.y) : s.x * kLn2 + logf(s.y + exp2f(-s.x));
            l += exp2f(-s.x);
            if (p.dX) p.row_gain[m] = p.gain[seg] / l;
        } else {
            const float T = p.losses[seg].temperature;
            loss = T * T * (p.row_base[t] + s.x * kLn2 + logf(l));
            if (p.dX) p.row_gain[m] = p.gain[seg] * T / l;
        }
        if (!(fabsf(p.row_ab[t].y) < __builtin_inff())) {              // (infinite scores among its entries)
            loss = __builtin_nanf("");
            if (p.dX) p.row_gain[m] = loss;
        }
        p.row_loss[t] = loss;
        row_most[r] = s.x;
        row_sum[r] = s.y;
    }
    if (!p.dX) return;
    __syncthreads();
    // columns that were held in other units than the row's
    for (int k = 0; k < kJoinRows && m0 + k < rows; ++k) {
        const float most = row_most[k];
        if (!(most > 0.f)) continue;
        bf16* const held = p.held + (size_t)(m0 + k) * p.pitch;
        for (int c = threadIdx.x; c < p.pitch; c += kJoinRows * kJoinSets) {
            const float shift = c < p.V ? p.stats[(size_t)(c / cols) * p.chunk + m0 + k].x : most;
            if (shift != most) held[c] = (bf16)((float)held[c] * exp2f(shift - most));
        }
    }
    __syncthreads();
    for (int k = threadIdx.x; k < kJoinRows * p.K; k += kJoinRows * kJoinSets) {
        const int row = k / p.K, j = k - row * p.K;
        if (m0 + row >= rows) continue;
        const int t = p.rows[p.chunk0 + m0 + row];
        const int64_t at = (int64_t)t * p.K;
        const float most = row_most[row], l = row_sum[row];
        bf16* const held = p.held + (size_t)(m0 + row) * p.pitch;
        if (!p.ids) {
            const int id = p.flags[t];
            if (id < p.V) held[id] = (bf16)(-l * p.slopes[at]);
            continue;
        }
        const int id = p.ids[at + j];
        if (id < 0 || id >= p.V) continue;
        float q = 0.f;                                // (a token that the row names twice: both entries write the same)
        for (int o = 0; o < p.K; ++o) q += p.ids[at + o] == id ? p.shares[at + o] : 0.f;
        held[id] = (bf16)((exp2f(p.scores[at + j] - most) - q * l) * p.slopes[at + j]);
    }
}

// ---- the gradient's product -----------------------------------------------------------------------------------------------------------
// Parts that the second product's inner dimension (the vocabulary) is cut into: as few rounds of workgroups as possible, weighed against the partial tiles' way through memory.
// Whole numbers: the kernels that ask for it have to agree.  room: partial tiles that fit the workspace.
template <int BLK>
struct LossGrad {
    static constexpr int kSlots = BLK == 8 ? 256 : 512;                        // workgroups at once
    static constexpr int kStageNs = BLK == 8 ? 1200 : 700, kPartNs = BLK == 8 ? 30000 : 15000;
    static constexpr int kMostParts = 128;
};
__host__ __device__ constexpr int64_t loss_grad_ns(int64_t tiles, int stages, int n, int slots, int stage_ns, int part_ns) {
    return (tiles * n + slots - 1) / slots * ((int64_t)((stages + n - 1) / n) * stage_ns + part_ns);
}
template <int BLK>
__host__ __device__ inline int loss_grad_parts(int rows, int width, int V, int64_t room) {
    using G = LossGrad<BLK>;
    constexpr int BM = 32 * BLK;
    const int64_t tiles = (int64_t)((rows + BM - 1) / BM) * ((width + BM - 1) / BM);
    const int stages = V / 64;
    int best = 1;
    int64_t least = loss_grad_ns(tiles, stages, 1, G::kSlots, G::kStageNs, G::kPartNs);
    for (int n = 2; n <= G::kMostParts && tiles * n <= room && stages / n >= 4; ++n) {
        const int64_t ns = loss_grad_ns(tiles, stages, n, G::kSlots, G::kStageNs, G::kPartNs);
        if (ns * 200 < least * 199) least = ns, best = n;
    }
    return best;
}

template <int BLK>
SYMB_KERNEL __launch_bounds__(256) void symb_loss_grad_kernel(const LossParams p) {
    using TT = Gemm16Tile<BLK, BLK>;
    constexpr int BM = TT::BM, BN = TT::BN;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int rows = loss_chunk_rows(p);
    if (rows <= 0) return;
    const int m_tiles = (rows + BM - 1) / BM, n_tiles = (p.width + BN - 1) / BN, tiles = m_tiles * n_tiles;
    const int n = loss_grad_parts<BLK>(rows, p.width, p.V, p.part_tiles), total = tiles * n, per_xcd = (total + 7) >> 3;
    const int lin = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || lin >= total) return;
    const int part = lin / tiles;
    int tm, tn;
    loss_place(lin % tiles, m_tiles, n_tiles, p.group_m, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN, stages = p.V / 64;
    const int st0 = (int)((int64_t)stages * part / n), st1 = (int)((int64_t)stages * (part + 1) / n);
    auto a_at = [&](int row) __attribute__((always_inline)) { return (unsigned)(min(m0 + row, rows - 1) - m0) * (unsigned)p.pitch; };
    loss_tile<BLK, true>(smem, p.held + (size_t)m0 * p.pitch, a_at, p.W + n0, p.width, p.width - n0, st0, st1 - st0, part == n - 1, p.V);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned lane_off = (unsigned)(wave * (BLK * BLK * 1024) + lane * 16);
    const unsigned long long mine = (unsigned long long)(p.parts + (size_t)(part * tiles + tm * n_tiles + tn) * (BM * BN));
    if constexpr (BLK == 8) asm volatile(SYMB_GEMM16_STORE_PARTIAL : : "v"(lane_off), "s"(mine) : "memory", SYMB_GEMM16_VCLOBBERS);
    else asm volatile(SYMB_GEMM16S_STORE_PARTIAL : : "v"(lane_off), "s"(mine) : "memory", SYMB_GEMM16S_VCLOBBERS);
}

// The parts of a tile added in order, times the row's gain, to the rows they belong to.  A workgroup takes one wavefront's 16 rows of a tile.
template <int BLK>
SYMB_KERNEL __launch_bounds__(256) void symb_loss_reduce_kernel(const LossParams p) {
    constexpr int BM = 32 * BLK;
    const int rows = loss_chunk_rows(p);
    if (rows <= 0) return;
    const int n_tiles = (p.width + BM - 1) / BM, m_tiles = (rows + BM - 1) / BM, tiles = m_tiles * n_tiles;
    const int tile = blockIdx.x / (4 * BLK), wave = blockIdx.x / BLK % 4, i = blockIdx.x % BLK;
    const int m = tile / n_tiles * BM + (wave >> 1) * (BM / 2) + 16 * i + (threadIdx.x & 15);
    if (tile >= tiles || m >= rows) return;
    const int n = loss_grad_parts<BLK>(rows, p.width, p.V, p.part_tiles);
    const float gain = p.row_gain[m];
    bf16* const out = p.dX + (size_t)p.rows[p.chunk0 + m] * p.width;
    for (int j = threadIdx.x >> 6; j < BLK; j += 4) {
        const int col = tile % n_tiles * BM + (wave & 1) * (BM / 2) + 16 * j + 4 * (threadIdx.x >> 4 & 3);
        if (col >= p.width) continue;
        const float* src = p.parts + (size_t)tile * (BM * BM) + (size_t)(wave * BLK * BLK + BLK * i + j) * 256 + (threadIdx.x & 63) * 4;
        floatx4 s = *(const floatx4*)src;
#pragma unroll 4
        for (int k = 1; k < n; ++k) s += *(const floatx4*)(src + (size_t)k * tiles * (BM * BM));
        *(uint2*)(out + col) = make_uint2(pack2_bf16(s[0] * gain, s[1] * gain), pack2_bf16(s[2] * gain, s[3] * gain));
    }
}

// A segment's loss: its rows' in a fixed order.
SYMB_KERNEL __launch_bounds__(256) void symb_loss_segments_kernel(LossParams p) {
    __shared__ float lds[4];
    __shared__ int counts[4];
    const int i = blockIdx.x;
    float s = 0.f;
    int n = 0;
    for (int t = p.off[i] + threadIdx.x; t < p.off[i + 1]; t += 256) {
        s += p.row_loss[t];
        n += p.flags[t] >= 0;
    }
    s = across_wave(s, Add());
    n = loss_count(n, counts);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = lds[0] + lds[1] + lds[2] + lds[3];
        p.loss[i] = p.mean ? s / (float)max(n, 1) : s;
    }
}

}  // namespace symb
