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
// 3584 rows of 4608 over 256000, not capped: 5.7 to 5.9 ms the first product and its sums, 11.4 to 11.8 both, 1.43 to 1.48 PFLOP/s, where a library's bare product of 8192 such rows reaches 1.52; capped 3 to 6 % more
// of the first.  The chip is power-limited: what an epilogue leaves idle comes back as clock.
#pragma once
#include "block_device.hpp"
#include "gemm16_kernel.hpp"

namespace symb {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

constexpr int kTwoRows = 64;

struct LossDesc {
    float scale, temperature;
};
struct LossRow {                          // of a row that takes part: its weights are 2^(a z - b), and its segment
    float a, b;
    int32_t seg, entries;                 // entries: of the teacher, in the order of their ids
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
    LossRow* info;                        // [T]
    float2* label;                        // [T] z' of the label, and its own weight: what rounding b makes of one
    int32_t* sorted;                      // [T][K] a row's ids in their order, absent ones left out,
    float* shares;                        // [T][K] their q,
    float* scores;                        // [T][K] and their s, from the first product
    uint16_t* starts;                     // [T][column tiles + 1] how many of them lie before each of its tiles
    float2* stats;                        // [column parts][chunk] shift and sum of a row's weights
    float* row_gain;                      // [chunk] what a row's product is multiplied with
    bf16* held;                           // [chunk][pitch] weights
    float* parts;                         // partial tiles of the second product
    int32_t* part_count;                  // in how many parts each tile comes
    int64_t part_tiles;                   // room for that many
    int32_t T, S, V, pitch, width, K;
    int32_t chunk0, chunk;                // the chunk's first row (of those that take part) and its length at most
    int32_t tile_shift;                   // columns of a tile of the first product: 2^tile_shift
    int32_t group_m, mean;
    int32_t grad_tile;                    // LossTileKind of the second product
    int32_t two;                          // weights are held in two terms, the second kTwoRows rows below the first
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

// tanh(y) for |y| <= kLossNear: y times a polynomial in y^2, 2^-27 of it at most and what fp32 rounds (the coefficients: least largest relative error, from exchanged extrema).
constexpr float kLossNear = 1.22f;
__device__ __forceinline__ float loss_tanh(float y) {
    const float u = y * y;
    float r = 6.16943486e-05f;
    r = fmaf(r, u, -0.00056751579f);
    r = fmaf(r, u, 0.00256464523f);
    r = fmaf(r, u, -0.00808763789f);
    r = fmaf(r, u, 0.0215047049f);
    r = fmaf(r, u, -0.0538685345f);
    r = fmaf(r, u, 0.133319376f);
    r = fmaf(r, u, -0.333332569f);
    r = fmaf(r, u, 1.f);
    return y * r;
}

// ---- which rows take part, and their own scores -------------------------------------------------------------------------------------
// s = x . W_id over a wavefront, in 64 bits: a sure row's loss hangs on how far this one score lies above the others, whose errors even out.  NaN for a number outside the vocabulary, which is never
// followed.
__device__ __forceinline__ double loss_score(const LossParams& p, int t, int id) {
    if (id >= p.V) return __builtin_nan("");
    const bf16 *x = p.X + (int64_t)t * p.width, *w = p.W + (int64_t)id * p.width;
    double s[2] = {0.0, 0.0};
#pragma unroll 4
    for (int c = threadIdx.x & 63; c < p.width >> 3; c += 64) {
        const intx4 u = *(const intx4*)(x + c * 8), v = *(const intx4*)(w + c * 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {                     // (a product of two bf16 is a float)
            s[0] += (double)(bf16_lo((unsigned)u[i]) * bf16_lo((unsigned)v[i]));
            s[1] += (double)(bf16_hi((unsigned)u[i]) * bf16_hi((unsigned)v[i]));
        }
    }
    double sum = s[0] + s[1];
#pragma unroll
    for (int m = 32; m; m >>= 1) sum += __shfl_xor(sum, m);
    return sum;
}
// A row that takes no part: zeros.
__device__ __forceinline__ void loss_no_row(const LossParams& p, int t) {
    const int lane = threadIdx.x & 63;
    if (lane == 0) p.row_loss[t] = 0.f;
    if (p.dX)
        for (int c = lane; c < p.width >> 3; c += 64) *(intx4*)(p.dX + (int64_t)t * p.width + c * 8) = intx4{0, 0, 0, 0};
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
// Workgroup `b` lists the rows of 256 that take part (and counts those before them itself); behind the lists, one a segment counts its rows.  IDS: of what the teachers' ids say, not yet of flags.
template <bool IDS>
__device__ __forceinline__ void loss_list(const LossParams& p, int b, int* lds) {
    const int lists = (p.T + 255) / 256;
    auto takes_part = [&](int t) __attribute__((always_inline)) {
        if constexpr (!IDS) return p.flags[t] >= 0;
        int most = -1;
#pragma unroll 8
        for (int j = 0; j < p.K; ++j) most = max(most, p.ids[(int64_t)t * p.K + j]);
        return most >= 0;
    };
    if (b < lists) {
        int before = 0;
        for (int t = threadIdx.x; t < b * 256; t += 256) before += takes_part(t);
        before = loss_count(before, lds);
        const int t = b * 256 + threadIdx.x;
        const bool part = t < p.T && takes_part(t);
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
    for (int t = p.off[i] + threadIdx.x; t < p.off[i + 1]; t += 256) n += takes_part(t);
    n = loss_count(n, lds);
    if (threadIdx.x == 0) p.gain[i] = p.mean ? p.losses[i].scale / (float)max(n, 1) : p.losses[i].scale;
}

// Labels: the lists, and a wavefront for each row's own score.  Latencies and 2 d elements a row: one row 4.8 us, 8192 of 4608 30.
SYMB_KERNEL __launch_bounds__(256) void symb_loss_labels_kernel(LossParams p) {
    __shared__ int lds[4];
    const int lists = (p.T + 255) / 256 + p.S;
    if ((int)blockIdx.x < lists) return loss_list<false>(p, blockIdx.x, lds);
    const int t = (blockIdx.x - lists) * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (t >= p.T) return;
    const int label = p.flags[t];
    if (label < 0) return loss_no_row(p, t);
    double z = loss_score(p, t, label), slope = 1.0;
    if (p.cap > 0.f) {
        const double y = z / p.cap, e = exp(-2.0 * fabs(y));
        slope = 4.0 * e / ((1.0 + e) * (1.0 + e));
        z = tanh(y) * p.cap;
    }
    z *= (double)kLog2e;
    if ((threadIdx.x & 63) == 0) {
        const float b = (float)z;
        p.info[t] = LossRow{kLog2e, b, seg_of_row(p.off, 0, p.S - 1, t), 1};
        p.label[t] = make_float2((float)slope, exp2f((float)(z - (double)b)));
    }
}
SYMB_KERNEL __launch_bounds__(256) void symb_loss_rows_kernel(LossParams p) {
    __shared__ int lds[4];
    loss_list<false>(p, blockIdx.x, lds);
}

// Teachers: a row's entries in the order of their ids, with their shares, the tiles of the vocabulary that they lie in, and the score of the one with the largest share.  A wavefront a row, behind
// the `lists` first workgroups, which list the rows.  In order, because a tile of the first product then finds its entries of a row side by side; by counting, entries squared / 64 steps a row.  One row of 20
// 8.8 us, 4096 of 64 18.5, 2048 of 128 24.
SYMB_KERNEL __launch_bounds__(256) void symb_loss_teacher_kernel(LossParams p, int lists) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    if ((int)blockIdx.x < lists) return loss_list<true>(p, blockIdx.x, (int*)smem);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), t = (blockIdx.x - lists) * 4 + wave;
    if (t >= p.T) return;
    const int K = p.K, pad = (K + 63) / 64 * 64;
    int* const list = (int*)smem + wave * 2 * pad;        // ids as they come (absent ones behind all others), then in order
    int* const order = list + pad;
    const int32_t* ids = p.ids + (int64_t)t * K;
    const float* l = p.teacher + (int64_t)t * K;
    const int seg = seg_of_row(p.off, 0, p.S - 1, t);
    const float T = p.losses[seg].temperature, to_t = 1.f / T;
    float most = -__builtin_inff(), first = 0.f;          // (first: this lane's first logit, all that it has of up to 64)
    int n = 0;
    bool outside = false;
    for (int j = lane; j < pad; j += 64) {
        const int id = j < K ? ids[j] : -1;
        const float v = j < K ? l[j] : 0.f;
        list[j] = id < 0 ? 0x7fffffff : min(id, 0x7ffffffe);
        if (j < 64) first = v;
        if (id >= 0) most = fmaxf(most, v);
        outside |= id >= p.V;
        n += __popcll(__ballot(id >= 0));
    }
    if (lane == 0) p.own_flags[t] = n ? 0 : -1;
    if (!n) return loss_no_row(p, t);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    most = across_wave(most, Max());
    auto raised = [&](int j) __attribute__((always_inline)) { return expf(((j < 64 ? first : l[j]) - most) * to_t); };
    // (a NaN among the logits makes the sum, and with it all shares, NaN)
    float sum = 0.f, best = -1.f;
    for (int j = lane; j < K; j += 64) sum += list[j] != 0x7fffffff ? raised(j) : 0.f;
    const float to_sum = 1.f / across_wave(sum, Add());
    int best_id = 0x7fffffff;
    for (int j = lane; j < K; j += 64) {
        const int id = list[j];
        if (id == 0x7fffffff) continue;
        int at = 0;                                       // entries before this one, in the order of ids and then as they come
        for (int k = 0; k < pad; k += 4) {
            const intx4 o = *(const intx4*)(list + k);
#pragma unroll
            for (int i = 0; i < 4; ++i) at += o[i] < id || (o[i] == id && k + i < j);
        }
        const float q = raised(j) * to_sum;
        order[at] = id;
        p.sorted[(int64_t)t * K + at] = id;
        p.shares[(int64_t)t * K + at] = q;
        if (q > best || (q == best && id < best_id)) best = q, best_id = id;
    }
    // the best entry's score
    const float top = across_wave(best, Max());
    int mine = best == top ? best_id : 0x7fffffff;
#pragma unroll
    for (int m = 32; m; m >>= 1) mine = min(mine, __shfl_xor(mine, m));
    outside = __any(outside || mine == 0x7fffffff);       // (all shares NaN: none is the largest)
    float s = __builtin_nanf(""), slope;
    if (!outside) {
        s = (float)loss_score(p, t, mine);
        if (p.cap > 0.f) s = loss_capped(s, p.cap, p.to_cap, slope);
    }
    const float a = kLog2e * to_t;
    if (lane == 0) p.info[t] = LossRow{a, s * a, seg, n};
    // starts[c]: entries in the tiles before c
    const int tiles = ((p.V - 1) >> p.tile_shift) + 1;
    uint16_t* const starts = p.starts + (int64_t)t * (tiles + 1);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    for (int k0 = 0; k0 <= n; k0 += 64) {
        const int k = k0 + lane;
        int from = 0, to = -1;
        if (k <= n) {
            from = k ? (min(order[k - 1], p.V - 1) >> p.tile_shift) + 1 : 0;
            to = k < n ? min(order[k], p.V - 1) >> p.tile_shift : tiles;
        }
        const bool wide = to - from >= 16;                // (the whole wavefront on it)
        if (!wide)
            for (int c = from; c <= to; ++c) starts[c] = (uint16_t)k;
        for (unsigned long long left = __ballot(wide); left; left &= left - 1) {
            const int of = __ffsll(left) - 1, at = __builtin_amdgcn_readlane(from, of), end = __builtin_amdgcn_readlane(to, of);
            for (int c = at + lane; c <= end; c += 64) starts[c] = (uint16_t)(k0 + of);
        }
    }
}

// What rounding four weights to bf16 leaves of them, as bf16.
__device__ __forceinline__ uint2 loss_second(const float (&v)[4], uint2 first) {
    return make_uint2(pack2_bf16(v[0] - bf16_lo(first.x), v[1] - bf16_hi(first.x)), pack2_bf16(v[2] - bf16_lo(first.y), v[3] - bf16_hi(first.y)));
}

// ---- products -------------------------------------------------------------------------------------------------------------------------
// A tile of Aop [rows][K] times Bop ([columns][K], or [K][columns] if NN) into the accumulation registers, with the loops of gemm16_asm.hpp: stages st0 .. st0 + KF - 1 of 64, and what K leaves
// behind the last whole stage if `tail`.  a_at(row): where a row of the tile starts, in elements from a_tile; b_tile: its first column at k = 0, `ldb` elements from the next (NN: from the next k);
// `columns`: how many there are.  The lane layout is that of symb_gemm16_kernel.
template <int MB, int NB, bool NN, class Row>
__device__ __forceinline__ void loss_tile(unsigned char* smem, const bf16* a_tile, Row a_at, const bf16* b_tile, int ldb, int columns, int st0, int KF, bool tail, int K) {
    using TT = Gemm16Tile<MB, NB>;
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
        if constexpr (TT::TALL) asm volatile(SYMB_GEMM16T_ZERO ::: SYMB_GEMM16T_ACLOBBERS);
        else if constexpr (NB == 8) asm volatile(SYMB_GEMM16_ZERO ::: SYMB_GEMM16_ACLOBBERS);
        else asm volatile(SYMB_GEMM16S_ZERO ::: SYMB_GEMM16S_ACLOBBERS);
    } else {
        // (the 256x128 loop wants its lane offsets and bases shifted, and starts each XCD at another eighth of the stages: see symb_gemm16_kernel)
        constexpr unsigned LOWER = TT::TALL ? 4096u : 0u;
        auto lower = [](int j) { return LOWER ? LOWER - 1024u * (unsigned)(j & 3) : 0u; };
        constexpr int NVB = NB > 4 ? NB : 4;
        unsigned vA[4], vB[NVB], ab[MB], bb[NB];
#pragma unroll
        for (int j = 0; j < 4; ++j) vA[j] = lds0 + frag_a(j >> 1, j & 1);
#pragma unroll
        for (int j = 0; j < NVB; ++j) vB[j] = lds0 + (NN ? frag_b_nn(j % NB) : frag_b_nt((j >> 1) & 1, j & 1));
#pragma unroll
        for (int j = 0; j < MB; ++j) {
            const int row = (wave * MB + j) * 8 + (lane >> 3), kc = (lane & 7) ^ swz_row(row);
            ab[j] = (a_at(row) + kc * 8) * 2u + lower(j);
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            if constexpr (!NN) {
                const int row = (wave * NB + j) * 8 + (lane >> 3), kc = (lane & 7) ^ swz_row(row);
                bb[j] = ((unsigned)min(row, columns - 1) * (unsigned)ldb + kc * 8) * 2u + lower(j);
            } else {
                constexpr int CPR = BN / 8;
                const int krow = (wave * NB + j) * (64 / CPR) + lane / CPR, nc = (lane % CPR) ^ swz_nmajor16(krow);
                bb[j] = ((unsigned)krow * (unsigned)ldb + (unsigned)min(nc * 8, columns - 8)) * 2u + lower(j);
            }
        }
        const int first = TT::TALL ? (int)((blockIdx.x & 7) * (unsigned)KF / 8) : 0;
        const unsigned long long ga = (unsigned long long)(a_tile + (size_t)(st0 + first) * 64) - LOWER;
        const unsigned long long gb = (unsigned long long)(b_tile + (size_t)(st0 + first) * 64 * (NN ? ldb : 1)) - LOWER;
        const unsigned stride_b = NN ? 128u * (unsigned)ldb : 128u;
        const unsigned swa = (unsigned)__builtin_amdgcn_readfirstlane((int)lds0 + wave * (1024 * MB));
        if constexpr (TT::TALL) {
            const unsigned swb = (unsigned)__builtin_amdgcn_readfirstlane((int)lds0 + wave * (1024 * NB));
#define SYMB_LOSS_LOOP_OPERANDS                                                                                     \
    :                                                                                                              \
    : "v"(vA[0]), "v"(vA[1]), "v"(vA[2]), "v"(vA[3]), "v"(vB[0]), "v"(vB[1]), "v"(vB[2]), "v"(vB[3]),              \
      "v"(ab[0]), "v"(ab[1]), "v"(ab[2]), "v"(ab[3]), "v"(ab[4]), "v"(ab[5]), "v"(ab[6]), "v"(ab[7]),              \
      "v"(bb[0]), "v"(bb[1]), "v"(bb[2]), "v"(bb[3]),                                                              \
      "s"(ga), "s"(gb), "s"(stride_b), "s"(KF), "s"(swa), "s"(swb), "s"(first)                                     \
    : "memory", "scc", SYMB_GEMM16T_SCLOBBERS, SYMB_GEMM16T_VCLOBBERS, SYMB_GEMM16T_ACLOBBERS
            if constexpr (NN) asm volatile(SYMB_GEMM16T_LOOP_NN SYMB_LOSS_LOOP_OPERANDS);
            else asm volatile(SYMB_GEMM16T_LOOP_NT SYMB_LOSS_LOOP_OPERANDS);
#undef SYMB_LOSS_LOOP_OPERANDS
        } else if constexpr (NB == 8) {
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
    constexpr int CA = BM * 8 / NT, CB = BN * 8 / NT, RSTEP = NT / 8, KSTEP = NT / (BN / 8);
    unsigned char *const sA = smem, *const sB = smem + TT::UNIT_A;
    const int lrow = tid >> 3, lkc = (tid & 7) * 8, nn_k = tid / (BN / 8), nn_nc = tid % (BN / 8);
    uint4 ra[CA], rb[CB];
#pragma unroll
    for (int i = 0; i < CA; ++i) ra[i] = ld_global_16(a_tile + a_at(lrow + i * RSTEP) + k0 + lkc, k0 + lkc < K);
#pragma unroll
    for (int i = 0; i < CB; ++i) {
        if constexpr (!NN) rb[i] = ld_global_16(b_tile + (size_t)min(lrow + i * RSTEP, columns - 1) * ldb + k0 + lkc, k0 + lkc < K);
        else {
            const int k = k0 + nn_k + i * KSTEP;
            rb[i] = ld_global_16(b_tile + (size_t)min(k, K - 1) * ldb + min(nn_nc * 8, columns - 8), k < K);
        }
    }
    const int a_lds0 = lds_off_kmajor(lrow, tid & 7), b_lds0 = NN ? lds_off_nmajor16<BN>(nn_k, nn_nc) : a_lds0;
#pragma unroll
    for (int i = 0; i < CA; ++i) *reinterpret_cast<uint4*>(sA + a_lds0 + i * RSTEP * 128) = ra[i];
#pragma unroll
    for (int i = 0; i < CB; ++i) *reinterpret_cast<uint4*>(sB + b_lds0 + i * (NN ? KSTEP * (BN * 2) : RSTEP * 128)) = rb[i];
    __syncthreads();
    const unsigned all = (1u << MB) - 1;
    for (int ks = 0; ks < (K - k0 + 31) >> 5; ++ks) {
        const unsigned va0 = lds0 + frag_a(ks, 0), va1 = lds0 + frag_a(ks, 1);
        if constexpr (!NN) {
            const unsigned vb0 = lds0 + TT::UNIT_A + frag_b_nt(ks, 0), vb1 = lds0 + TT::UNIT_A + frag_b_nt(ks, 1);
            if constexpr (TT::TALL)
                asm volatile(SYMB_GEMM16T_KSTEP32_NT : : "v"(va0), "v"(va1), "v"(vb0), "v"(vb1), "s"(all) : "memory", "scc", SYMB_GEMM16T_VCLOBBERS, SYMB_GEMM16T_ACLOBBERS);
            else if constexpr (NB == 8)
                asm volatile(SYMB_GEMM16_KSTEP32_NT : : "v"(va0), "v"(va1), "v"(vb0), "v"(vb1), "s"(all) : "memory", "scc", SYMB_GEMM16_VCLOBBERS, SYMB_GEMM16_ACLOBBERS);
            else
                asm volatile(SYMB_GEMM16S_KSTEP32_NT : : "v"(va0), "v"(va1), "v"(vb0), "v"(vb1), "s"(all) : "memory", "scc", SYMB_GEMM16S_VCLOBBERS, SYMB_GEMM16S_ACLOBBERS);
        } else {
            unsigned vb[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) vb[j] = lds0 + TT::UNIT_A + frag_b_nn(j) + ks * 32 * (BN * 2);
            if constexpr (TT::TALL)
                asm volatile(SYMB_GEMM16T_KSTEP32_NN : : "v"(va0), "v"(va1), "v"(vb[0]), "v"(vb[1]), "v"(vb[2]), "v"(vb[3]), "s"(all)
                             : "memory", "scc", SYMB_GEMM16T_VCLOBBERS, SYMB_GEMM16T_ACLOBBERS);
            else if constexpr (NB == 8)
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

// Element (j, e) of a lane's scores: half of what is left at every step.  (With masks that the compiler cannot see through: it makes selected values loads from a selected address, and the scores
// an array in scratch memory.)
template <int NB>
__device__ __forceinline__ float loss_pick(const float (&w)[NB][4], int j, int e) {
    auto mask = [](int bit) __attribute__((always_inline)) {
        int m = bit ? -1 : 0;
        asm volatile("" : "+v"(m));
        return m;
    };
    auto pick = [](int m, int yes, int no) __attribute__((always_inline)) { return (yes & m) | (no & ~m); };
    const int e0 = mask(e & 1), e1 = mask(e & 2), j0 = mask(j & 1), j1 = mask(j & 2), j2 = mask(j & 4);
    int v[NB];
    static_for<0, NB>([&](auto K) __attribute__((always_inline)) {
        constexpr int k = decltype(K)::value;
        v[k] = pick(e1, pick(e0, as_int(w[k][3]), as_int(w[k][2])), pick(e0, as_int(w[k][1]), as_int(w[k][0])));
    });
    if constexpr (NB == 8) static_for<0, 4>([&](auto K) __attribute__((always_inline)) { v[decltype(K)::value] = pick(j2, v[decltype(K)::value + 4], v[decltype(K)::value]); });
    return as_float(pick(j1, pick(j0, v[3], v[2]), pick(j0, v[1], v[0])));
}
// A tile row's entries of its teacher, behind the staged tile in LDS.  Their scores come out of the product itself: dot products of their own were 300 us of 1605 (4096 rows of 4096 over 32000, 64 entries), this
// costs the product some 20.
struct LossHits {
    int64_t at;                           // of the first one in `sorted`, `scores`
    int32_t n;
    int32_t id[4];                        // the first of them
    int32_t pad;
};

// X W^T of a chunk, a tile a workgroup: its rows' sums of weights, the scores of their teachers' entries, and the weights themselves where the gradient wants them.
template <int MB, int NB, bool GRAD, bool CAP, bool TEACHER>
SYMB_KERNEL __launch_bounds__(256) void symb_loss_scores_kernel(const LossParams p) {
    using TT = Gemm16Tile<MB, NB>;
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
    float a[MB], b[MB];
    int label[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int t = list[min(m0 + wm0 + 16 * i + l15, rows - 1)];
        a[i] = p.info[t].a;
        b[i] = p.info[t].b;
        if constexpr (!TEACHER) label[i] = p.flags[t] - (n0 + wn0 + 4 * lg);   // of block j, element e: 16 j + e
    }
    LossHits hits{};
    if (TEACHER && tid < BM && m0 + tid < rows) {
        const int t = list[m0 + tid];
        const uint16_t* const start = p.starts + (int64_t)t * (n_tiles + 1) + tn;
        const int at = start[0];
        hits.n = start[1] - at;
        hits.at = (int64_t)t * p.K + at;
#pragma unroll
        for (int k = 0; k < 4; ++k) hits.id[k] = p.sorted[(int64_t)t * p.K + min(at + k, p.K - 1)];
    }
    auto a_at = [&](int row) __attribute__((always_inline)) { return (unsigned)(list[min(m0 + row, rows - 1)] - first) * (unsigned)p.width; };
    loss_tile<MB, NB, false>(smem, p.X + (size_t)first * p.width, a_at, p.W + (size_t)n0 * p.width, p.width, p.V - n0, 0, p.width / 64, true, p.width);

    LossHits* const row_hits = reinterpret_cast<LossHits*>(smem + TT::C_BYTES);
    static_assert(TT::C_BYTES % 16 == 0 && TT::C_BYTES + BM * (int)sizeof(LossHits) <= TT::SMEM, "");
    if constexpr (TEACHER) {
        if (tid < BM) row_hits[tid] = hits;
        __syncthreads();
    }
    const unsigned c_lane = (unsigned)((wm0 + l15) * CP + (wn0 + lg * 4) * 2);
    const int left = p.V - (n0 + wn0 + 4 * lg);                                // columns of this lane: 16 j + e < left
    const bool edge = n0 + BN > p.V;
    float2* const stats = p.stats + (size_t)(2 * tn + (wave & 1)) * p.chunk + m0 + wm0;
    static_for<0, MB>([&](auto I) __attribute__((always_inline)) {
        constexpr int i = decltype(I)::value;
        float w[NB][4], slope[CAP ? NB : 1][4];
        auto scores = [&]() __attribute__((always_inline)) {
            static_for<0, NB>([&](auto J) __attribute__((always_inline)) {
                constexpr int j = decltype(J)::value;
                acc16_read4<4 * (NB * i + j)>(w[j][0], w[j][1], w[j][2], w[j][3]);
            });
        };
        // a z - b, the general way
        auto exponents = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (CAP) w[j][e] = loss_capped(w[j][e], p.cap, p.to_cap, slope[j][e]);
                    w[j][e] = fmaf(w[j][e], a[i], -b[i]);
                }
        };
        float sum;
        auto weights = [&](float shift) __attribute__((always_inline)) {
            float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) w[j][e] = __builtin_amdgcn_exp2f(w[j][e] - shift);
            if (edge)
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[j][e] = 16 * j + e < left ? w[j][e] : 0.f;
            if (!TEACHER && __any((unsigned)label[i] < 16u * NB)) {
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[e] += 16 * j + e == label[i] ? 0.f : w[j][e];
            } else {
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[e] += w[j][e];
            }
            sum = across_rows((s[0] + s[1]) + (s[2] + s[3]), Add());
        };
        scores();
        if constexpr (TEACHER) {
            const LossHits& hit = row_hits[wm0 + 16 * i + l15];
            const int n = hit.n;
#pragma unroll 1
            for (int k = 0; __any(k < n); ++k) {
                int c = -1;
                if (k < n) c = (k < 4 ? hit.id[k] : p.sorted[hit.at + k]) - (n0 + wn0);
                const bool mine = (unsigned)c < (unsigned)TT::WN && (c >> 2 & 3) == lg;
                if (!__any(mine)) continue;
                const float s = loss_pick<NB>(w, c >> 4, c & 3);
                if (mine) p.scores[hit.at + k] = s;
            }
        }
        if constexpr (CAP) {
            float top = 0.f;
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(w[j][e]));
            const float to_exp = a[i] * p.cap;
            if (__any(!(top <= kLossNear * p.cap) || !(to_exp < __builtin_inff()))) exponents();
            else {
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = w[j][e] * p.to_cap, th = loss_tanh(y);
                        slope[j][e] = fmaf(-th, th, 1.f);
                        w[j][e] = fmaf(th, to_exp, -b[i]);
                    }
            }
        } else exponents();
        float shift = 0.f;
        weights(0.f);
        if (__any(!(sum < 0x1p64f))) {                                         // scores far above the row's own entries (or NaN)
            const bool far = !(sum < 0x1p64f);
            scores();
            exponents();
            float most = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!edge || 16 * j + e < left) most = fmaxf(most, w[j][e]);
            most = across_rows(most, Max());
            shift = far ? most : 0.f;
            weights(shift);
        }
        if (lg == 0) stats[16 * i + l15] = make_float2(shift, sum);            // (rows behind the last one have room)
        if constexpr (GRAD) {
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                if constexpr (CAP)
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[j][e] *= slope[j][e];
                const uint2 first = make_uint2(pack2_bf16(w[j][0], w[j][1]), pack2_bf16(w[j][2], w[j][3]));
                // (of up to 64 rows the tile's lower half holds their second terms)
                if (MB == 4 && p.two) {
                    if (wm0 == 0) {
                        *reinterpret_cast<uint2*>(smem + c_lane + i * 16 * CP + j * 32) = first;
                        *reinterpret_cast<uint2*>(smem + c_lane + (kTwoRows + i * 16) * CP + j * 32) = loss_second(w[j], first);
                    }
                } else *reinterpret_cast<uint2*>(smem + c_lane + i * 16 * CP + j * 32) = first;
            }
        }
    });
    if constexpr (GRAD) {
        __syncthreads();
        constexpr int LPR = BN / 8, RPP = 256 / LPR;
        const int col = (lane % LPR) * 8, r0 = wave * (64 / LPR) + lane / LPR;
        const int held_rows = p.two ? kTwoRows + rows : rows;
        if (n0 + col < p.pitch) {
            bf16* const out = p.held + (size_t)m0 * p.pitch + n0 + col;
#pragma unroll 8
            for (int r = r0; r < BM; r += RPP)
                if (m0 + r < held_rows) *reinterpret_cast<uint4*>(out + (size_t)r * p.pitch) = *reinterpret_cast<const uint4*>(smem + r * CP + col * 2);
        }
    }
}

// The same for batches of up to 32 rows, where W's way from memory is all that counts.  A workgroup of eight wavefronts takes 64 columns: each wavefront every eighth 64 of the inner dimension, both operands
// from global memory straight into the matrix instruction's registers, the next 64 on their way meanwhile (up to 160 KiB a CU; the tiles of 128 columns have 32); the eight sums meet in LDS.
// RB: blocks of 16 rows.  One row of 4096 over 32000, W from HBM: 62 us the call, 74 with tiles, where 262 MB take 53 at the rate of a copy.
constexpr int kFewCols = 64, kFewRows = 32, kFewWaves = 8;
template <int RB, bool GRAD, bool TEACHER>
SYMB_KERNEL __launch_bounds__(64 * kFewWaves, RB == 1 ? 4 : 2) void symb_loss_few_kernel(const LossParams p) {
    constexpr int CB = kFewCols / 16, HALF = kFewWaves / 2;
    __shared__ floatx4 sums[HALF][RB * CB][64];
    __shared__ float part[2][16 * RB][CB];                // of 16 columns: sum of weights, largest exponent
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l15 = lane & 15, lg = lane >> 4;
    const int rows = loss_chunk_rows(p), n0 = blockIdx.x * kFewCols;
    if (rows <= 0) return;
    const int32_t* const list = p.rows + p.chunk0;
    int t[RB];
    const bf16 *x[RB], *w[CB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        t[r] = list[min(16 * r + l15, rows - 1)];
        x[r] = p.X + (size_t)t[r] * p.width + 16 * lg;
    }
#pragma unroll
    for (int c = 0; c < CB; ++c) w[c] = p.W + (size_t)min(n0 + 16 * c + l15, p.V - 1) * p.width + 16 * lg;
    // lane group g holds elements 16 g .. 16 g + 15 of 64, eight for each of two instructions
    struct Frags {
        bf16x8 x[RB][2], w[CB][2];
    };
    auto load = [&](Frags& f, int k) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int s = 0; s < 2; ++s) f.w[c][s] = *(const bf16x8*)(w[c] + k + 8 * s);
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int s = 0; s < 2; ++s) f.x[r][s] = *(const bf16x8*)(x[r] + k + 8 * s);
    };
    floatx4 acc[RB][CB] = {};
    auto products = [&](const Frags& f) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int c = 0; c < CB; ++c) acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.w[c][s], f.x[r][s], acc[r][c], 0, 0, 0);
    };
    const int whole = p.width / 64;
    Frags f, g;
    if (wave < whole) load(f, 64 * wave);
    for (int k = wave; k < whole; k += 2 * kFewWaves) {   // (behind the last 64 the last 64 again, not used)
        load(g, 64 * min(k + kFewWaves, whole - 1));
        __builtin_amdgcn_sched_barrier(0);
        products(f);
        if (k + kFewWaves >= whole) break;
        load(f, 64 * min(k + 2 * kFewWaves, whole - 1));
        __builtin_amdgcn_sched_barrier(0);
        products(g);
    }
    if (p.width % 64 && wave == whole % kFewWaves) {      // what is left of the inner dimension
        auto at = [&](const bf16* row, int s) __attribute__((always_inline)) {
            const int k = 64 * whole + 8 * s, last = p.width - 8 - 16 * lg;
            const bf16x8 v = *(const bf16x8*)(row + min(k, last));
            return k <= last ? v : bf16x8{};
        };
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int c = 0; c < CB; ++c) f.w[c][s] = at(w[c], s);
#pragma unroll
            for (int r = 0; r < RB; ++r) f.x[r][s] = at(x[r], s);
        }
        products(f);
    }
    // sums of all wavefronts: the upper ones to the lower ones, and those to whoever takes the block
    if (wave >= HALF)
#pragma unroll
        for (int q = 0; q < RB * CB; ++q) sums[wave - HALF][q][lane] = acc[q / CB][q % CB];
    __syncthreads();
    if (wave < HALF)
#pragma unroll
        for (int q = 0; q < RB * CB; ++q) {
            acc[q / CB][q % CB] += sums[wave][q][lane];
            sums[wave][q][lane] = acc[q / CB][q % CB];
        }
    __syncthreads();
    constexpr int MINE = (RB * CB + kFewWaves - 1) / kFewWaves;
    float v[MINE][4], slope[MINE][4];
    // a lane has row 16 r + l15, columns 16 c + 4 lg .. + 3 of its blocks
    auto block = [&](int k, auto f) __attribute__((always_inline)) {
        const int q = wave * MINE + k, r = q / CB, c = q % CB;
        if (q < RB * CB && 16 * r < rows) f(r, c, q, 16 * r + l15, n0 + 16 * c + 4 * lg);
    };
    auto row_of = [&](int r) __attribute__((always_inline)) { return list[min(16 * r + l15, rows - 1)]; };
    auto weights = [&](int k, int q, int row, int col, int label, float shift) __attribute__((always_inline)) {
        float sum = 0.f, most = -__builtin_inff();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool in = col + e < p.V;
            if (in) most = fmaxf(most, v[k][e]);
            const float u = in ? __builtin_amdgcn_exp2f(v[k][e] - shift) : 0.f;
            sum += col + e == label ? 0.f : u;
        }
        sum = across_rows(sum, Add());
        most = across_rows(most, Max());
        if (lg == 0) part[0][row][q % CB] = sum, part[1][row][q % CB] = most;
    };
#pragma unroll
    for (int k = 0; k < MINE; ++k)
        block(k, [&](int r, int c, int q, int row, int col) __attribute__((always_inline)) {
            const int t = row_of(r);
            const LossRow info = p.info[t];
            floatx4 s = sums[0][q][lane];
#pragma unroll
            for (int h = 1; h < HALF; ++h) s += sums[h][q][lane];
            if constexpr (TEACHER) {
                const uint16_t* const start = p.starts + (int64_t)t * ((p.V + kFewCols - 1) / kFewCols + 1) + blockIdx.x;
                const int64_t at = (int64_t)t * p.K;
                for (int j = start[0], end = row < rows ? start[1] : 0; j < end; ++j) {
                    const int i = p.sorted[at + j] - col;
                    if ((unsigned)i < 4u) p.scores[at + j] = i & 2 ? (i & 1 ? s[3] : s[2]) : (i & 1 ? s[1] : s[0]);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                slope[k][e] = 1.f;
                v[k][e] = fmaf(p.cap > 0.f ? loss_capped(s[e], p.cap, p.to_cap, slope[k][e]) : s[e], info.a, -info.b);
            }
            weights(k, q, row, col, TEACHER ? -1 : p.flags[t], 0.f);
        });
    __syncthreads();
    // scores far above a row's own entries (or NaN): smaller units, as in the tiles
    auto total = [&](int row) __attribute__((always_inline)) {
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < CB; ++c) s += part[0][row][c];
        return s;
    };
    float shift[MINE] = {};
    bool far = false;
#pragma unroll
    for (int k = 0; k < MINE; ++k)
        block(k, [&](int, int, int, int row, int) __attribute__((always_inline)) {
            if (total(row) < 0x1p64f) return;
            far = true;
            shift[k] = part[1][row][0];
#pragma unroll
            for (int c = 1; c < CB; ++c) shift[k] = fmaxf(shift[k], part[1][row][c]);
        });
    if (__syncthreads_or(far)) {
#pragma unroll
        for (int k = 0; k < MINE; ++k)
            block(k, [&](int r, int, int q, int row, int col) __attribute__((always_inline)) { weights(k, q, row, col, TEACHER ? -1 : p.flags[row_of(r)], shift[k]); });
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < MINE; ++k)
        block(k, [&](int, int c, int, int row, int col) __attribute__((always_inline)) {
            if (row >= rows) return;
            if (c == 0 && lg == 0) p.stats[(size_t)blockIdx.x * p.chunk + row] = make_float2(shift[k], total(row));
            if (!GRAD || col >= p.pitch) return;
            float u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = col + e < p.V ? __builtin_amdgcn_exp2f(v[k][e] - shift[k]) * slope[k][e] : 0.f;
            const uint2 first = make_uint2(pack2_bf16(u[0], u[1]), pack2_bf16(u[2], u[3]));
            *reinterpret_cast<uint2*>(p.held + (size_t)row * p.pitch + col) = first;
            *reinterpret_cast<uint2*>(p.held + (size_t)(kTwoRows + row) * p.pitch + col) = loss_second(u, first);
        });
}

// Parts that the second product's inner dimension (the vocabulary) is cut into: as few rounds of workgroups as possible, weighed against the partial tiles' way through memory.
// Nanoseconds: a stage of a tile of 256x256 and of 256x128, whose workgroup has a CU alone; of 128x128, of two workgroups that share a CU and of one that has it alone; the rest of a workgroup's
// time; a partial tile, written and read (of up to 64 rows kLossTwoNs).
constexpr int kLossParts = 128, kLossRoundNs = 5000, kLossTwoNs = 15;
template <int MB, int NB>
struct LossTile {
    static constexpr int kEdgeM = 32 * MB, kEdgeN = 32 * NB, kSlots = MB == 4 ? 512 : 256;
    static constexpr int kStageNs = NB == 8 ? 1400 : MB == 8 ? 750 : 1100, kLoneNs = MB == 4 ? 720 : kStageNs, kPartNs = NB == 8 ? 116 : 40;
    __host__ __device__ static constexpr int64_t tiles(int64_t rows, int64_t columns) { return (rows + kEdgeM - 1) / kEdgeM * ((columns + kEdgeN - 1) / kEdgeN); }
    __host__ __device__ static constexpr int64_t ns(int64_t tiles, int stages, int n, bool two) {
        return (tiles * n + kSlots - 1) / kSlots * ((int64_t)((stages + n - 1) / n) * (tiles * n <= kSlots / 2 ? kLoneNs : kStageNs) + kLossRoundNs) + tiles * n * (two ? kLossTwoNs : kPartNs);
    }
};
// room: partial tiles that fit the workspace.  (Four to eight rounds of workgroups even out whatever there is to even out.)
__host__ __device__ constexpr bool loss_grad_fits(int64_t tiles, int stages, int n, int64_t room) { return n == 1 || (tiles * n <= room && tiles * n <= 2048 && stages / n >= 4); }
enum LossTileKind : int32_t { kLossBig, kLossTall, kLossSmall };               // 256x256, 256x128, 128x128
template <class F>
__host__ __device__ __forceinline__ auto loss_tiled(int kind, F&& f) {
    return kind == kLossBig ? f(LossTile<8, 8>{}) : kind == kLossTall ? f(LossTile<8, 4>{}) : f(LossTile<4, 4>{});
}
template <class F>                        // (the second product)
__host__ __device__ __forceinline__ auto loss_grad_tiled(int kind, F&& f) {
    return kind == kLossBig ? f(LossTile<8, 8>{}) : f(LossTile<4, 4>{});
}

// ---- sums, losses, and the entries of q ---------------------------------------------------------------------------------------------
constexpr int kJoinRows = 16, kJoinSets = 32;
// Pairs (unit, sum): the sum counts in 2^unit.
__device__ __forceinline__ float loss_in(float2 s, float unit) { return s.x == unit ? s.y : s.y * exp2f(s.x - unit); }
// (3584 rows of 2000 parts 19 us; 256 rows of 394 7, a chain of loads and the launch.)
// 16 rows a workgroup of 512: the column parts' sums in a fixed order, the rows' losses, and their entries of p - q into the held weights.  `parts`: column parts of `cols` columns;
// finish: the segments' losses as well (one workgroup has all rows).  Beside that, for how many parts the gradient's product comes in.
template <class Tile>
__device__ __forceinline__ int loss_grad_parts(const LossParams& p, int rows) {
    const int64_t tiles = Tile::tiles(rows, p.width);
    const int stages = p.V / 64;
    float best = 3e38f;                                   // (nanoseconds)
    int n = 1;
    for (int k = 1 + (int)(threadIdx.x & 63); k <= kLossParts; k += 64) {
        const float ns = loss_grad_fits(tiles, stages, k, p.part_tiles) ? (float)Tile::ns(tiles, stages, k, p.two) * (1.f + 1e-4f * k) : 3e38f;
        if (ns < best) best = ns, n = k;
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) {
        const float other = __shfl_xor(best, m);
        const int k = __shfl_xor(n, m);
        if (other < best || (other == best && k < n)) best = other, n = k;
    }
    return n;
}
SYMB_KERNEL __launch_bounds__(kJoinRows* kJoinSets) void symb_loss_join_kernel(const LossParams p, int parts, int cols, bool finish) {
    __shared__ float2 lds[kJoinSets / 4][kJoinRows];
    __shared__ float row_unit[kJoinRows], row_sum[kJoinRows], row_gain[kJoinRows];
    __shared__ int row_t[kJoinRows];
    __shared__ LossRow row_info[kJoinRows];
    const int r = threadIdx.x % kJoinRows, set = threadIdx.x / kJoinRows, m0 = blockIdx.x * kJoinRows, m = m0 + r, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rows = loss_chunk_rows(p);
    if (m0 >= rows && !finish) return;
    if (p.dX && blockIdx.x == 0 && wave == kJoinSets / 4 - 1) {
        const int n = loss_grad_tiled(p.grad_tile, [&](auto tile) { return loss_grad_parts<decltype(tile)>(p, rows); });
        if (lane == 0) *p.part_count = n;
    }
    int t = 0;
    LossRow info{};
    float gain = 0.f;
    if (set == 0 && m < rows) {
        t = p.rows[p.chunk0 + m];
        info = p.info[t];
        gain = p.gain[info.seg];
    }
    float2 s = make_float2(0.f, 0.f);
    if (m < rows) {
        const float2* at = p.stats + (size_t)set * p.chunk + m;
        const size_t step = (size_t)kJoinSets * p.chunk;
        constexpr int AHEAD = 8;
        for (int c = set; c < parts; c += AHEAD * kJoinSets, at += AHEAD * step) {
            float2 v[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) v[k] = c + k * kJoinSets < parts ? at[k * step] : make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (v[k].x == s.x) s.y += v[k].y;
                else {
                    const float unit = fmaxf(s.x, v[k].x);
                    s = make_float2(unit, loss_in(s, unit) + loss_in(v[k], unit));
                }
            }
        }
    }
    const float top = across_rows(s.x, Max()), part = across_rows(loss_in(s, top), Add());
    if (lane < kJoinRows) lds[wave][r] = make_float2(top, part);
    __syncthreads();
    if (set == 0 && m < rows) {
        float unit = 0.f, l = 0.f;
#pragma unroll
        for (int k = 0; k < kJoinSets / 4; ++k) unit = fmaxf(unit, lds[k][r].x);
#pragma unroll
        for (int k = 0; k < kJoinSets / 4; ++k) l += loss_in(lds[k][r], unit);
        row_unit[r] = unit;
        row_sum[r] = l;
        row_t[r] = t;
        row_info[r] = info;
        if (!(fabsf(info.b) < __builtin_inff())) gain = l = __builtin_nanf("");          // (infinite scores among its entries)
        if (!p.ids) {
            const float mine = p.label[t].y * exp2f(-unit);
            p.row_loss[t] = unit == 0.f ? log1pf(l / mine) : unit * kLn2 + logf(l + mine) - logf(p.label[t].y);
            l += mine;
        } else gain *= kLog2e / info.a;
        if (p.dX) p.row_gain[m] = gain / l;
        row_gain[r] = l;
    }
    __syncthreads();
    const size_t second = (size_t)kTwoRows * p.pitch;
    auto put = [&](bf16* held, float v) __attribute__((always_inline)) {
        const bf16 first = (bf16)v;
        held[0] = first;
        if (p.two) held[second] = (bf16)(v - (float)first);
    };
    if (p.dX) {
        // columns that were held in other units than the row's
        for (int k = 0; k < kJoinRows && m0 + k < rows; ++k) {
            const float unit = row_unit[k];
            if (!(unit > 0.f)) continue;
            bf16* const held = p.held + (size_t)(m0 + k) * p.pitch;
            for (int c = threadIdx.x; c < p.pitch; c += kJoinRows * kJoinSets) {
                const float shift = c < p.V ? p.stats[(size_t)(c / cols) * p.chunk + m0 + k].x : unit;
                if (shift != unit) put(held + c, ((float)held[c] + (p.two ? (float)held[c + second] : 0.f)) * exp2f(shift - unit));
            }
        }
        __syncthreads();
        if (!p.ids && set == 0 && m < rows) {
            const int id = p.flags[t];
            if (id < p.V) put(p.held + (size_t)m * p.pitch + id, -row_sum[r] * p.label[t].x);
        }
    }
    if (p.ids)
        for (int k = wave; k < kJoinRows && m0 + k < rows; k += kJoinRows * kJoinSets / 64) {
            const LossRow row = row_info[k];
            const float unit = row_unit[k], l = row_gain[k], T = kLog2e / row.a;
            const int64_t at = (int64_t)row_t[k] * p.K;
            bf16* const held = p.held + (size_t)(m0 + k) * p.pitch;
            float base = 0.f;
            for (int j = lane; j < row.entries; j += 64) {
                const int id = p.sorted[at + j];
                if (id >= p.V) continue;                   // (the row is NaN already)
                float q = p.shares[at + j], z = p.scores[at + j], slope = 1.f;
                if (p.cap > 0.f) z = loss_capped(z, p.cap, p.to_cap, slope);
                z = fmaf(z, row.a, -row.b);
                if (!(q == 0.f)) base += q * (logf(q) - z * kLn2);
                if (!p.dX || (j && p.sorted[at + j - 1] == id)) continue;
                for (int o = j + 1; o < row.entries && p.sorted[at + o] == id; ++o) q += p.shares[at + o];     // (a token that the row names twice)
                put(held + id, (exp2f(z - unit) - q * l) * slope);
            }
            base = across_wave(base, Add());
            if (lane == 0) p.row_loss[row_t[k]] = T * T * (base + unit * kLn2 + logf(l));
        }
    if (!finish) return;
    __syncthreads();
    for (int i = threadIdx.x; i < p.S; i += kJoinRows * kJoinSets) {
        float sum = 0.f;
        int n = 0;
        for (int k = p.off[i]; k < p.off[i + 1]; ++k) {
            sum += p.row_loss[k];
            n += p.flags[k] >= 0;
        }
        p.loss[i] = p.mean ? sum / (float)max(n, 1) : sum;
    }
}

// ---- the gradient's product -----------------------------------------------------------------------------------------------------------
template <int MB, int NB>
SYMB_KERNEL __launch_bounds__(256) void symb_loss_grad_kernel(const LossParams p) {
    using TT = Gemm16Tile<MB, NB>;
    constexpr int BM = TT::BM, BN = TT::BN;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int own = loss_chunk_rows(p), rows = p.two ? kTwoRows + own : own;
    if (own <= 0) return;
    const int m_tiles = (rows + BM - 1) / BM, n_tiles = (p.width + BN - 1) / BN, tiles = m_tiles * n_tiles;
    const int n = *p.part_count, total = tiles * n, per_xcd = (total + 7) >> 3;
    const int lin = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || lin >= total) return;
    const int part = lin / tiles;
    int tm, tn;
    loss_place(lin % tiles, m_tiles, n_tiles, p.group_m, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN, stages = p.V / 64;
    const int st0 = (int)((int64_t)stages * part / n), st1 = (int)((int64_t)stages * (part + 1) / n);
    auto a_at = [&](int row) __attribute__((always_inline)) { return (unsigned)(min(m0 + row, rows - 1) - m0) * (unsigned)p.pitch; };
    loss_tile<MB, NB, true>(smem, p.held + (size_t)m0 * p.pitch, a_at, p.W + n0, p.width, p.width - n0, st0, st1 - st0, part == n - 1, p.V);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned lane_off = (unsigned)(wave * (MB * NB * 1024) + lane * 16);
    const unsigned long long mine = (unsigned long long)(p.parts + (size_t)(part * tiles + tm * n_tiles + tn) * (BM * BN));
    static_assert(!TT::TALL, "");
    if constexpr (MB == 4) {
        if (p.two) {
            // the second terms' product, of the wavefronts of the tile's lower half, to the first's, and no rows that there are not: 24 KiB of a tile's 64 for 37 rows
            static_assert(16 * MB == kTwoRows, "");
            floatx4* const second = reinterpret_cast<floatx4*>(smem) + (wave & 1) * (MB * NB * 64) + lane;
            auto blocks = [&](auto&& f) __attribute__((always_inline)) {
                static_for<0, MB>([&](auto I) __attribute__((always_inline)) {
                    if (16 * decltype(I)::value < own)
                        static_for<0, NB>([&](auto J) __attribute__((always_inline)) {
                            constexpr int block = NB * decltype(I)::value + decltype(J)::value;
                            float v[4];
                            acc16_read4<4 * block>(v[0], v[1], v[2], v[3]);
                            f(block, floatx4{v[0], v[1], v[2], v[3]});
                        });
                });
            };
            if (wave >= 2) blocks([&](int block, floatx4 v) __attribute__((always_inline)) { second[block * 64] = v; });
            __syncthreads();
            float* const to = p.parts + (size_t)(part * tiles + tm * n_tiles + tn) * (BM * BN) + (size_t)wave * (MB * NB * 256) + lane * 4;
            if (wave < 2) blocks([&](int block, floatx4 v) __attribute__((always_inline)) { *(floatx4*)(to + block * 256) = v + second[block * 64]; });
            return;
        }
    }
    if constexpr (NB == 8) asm volatile(SYMB_GEMM16_STORE_PARTIAL : : "v"(lane_off), "s"(mine) : "memory", SYMB_GEMM16_VCLOBBERS);
    else asm volatile(SYMB_GEMM16S_STORE_PARTIAL : : "v"(lane_off), "s"(mine) : "memory", SYMB_GEMM16S_VCLOBBERS);
}

// A segment's loss: its rows' in a fixed order.
__device__ __forceinline__ void loss_segment(const LossParams& p, int i, floatx4* room) {
    float* const lds = (float*)room;
    int* const counts = (int*)(room + 1);
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
SYMB_KERNEL __launch_bounds__(256) void symb_loss_segments_kernel(LossParams p) {
    __shared__ floatx4 lds[2];
    loss_segment(p, blockIdx.x, lds);
}

// The parts of a tile added in a fixed order, times the row's gain, to the rows they belong to.  A workgroup takes blocks of 16 x 16 of one wavefront's rows: four of them, or, of products in many
// parts, one whose parts its wavefronts share out (256 rows of 768 in 20 parts: 5.2 us, 15 without).  Workgroups from number `blocks` on: the segments' losses.  3584 rows of 4608: 27 us, 4.9 TB/s.
template <int MB, int NB, bool MANY>
SYMB_KERNEL __launch_bounds__(256) void symb_loss_reduce_kernel(const LossParams p, int blocks) {
    constexpr int BM = 32 * MB, BN = 32 * NB, GROUPS = MANY ? NB : NB / 4;
    __shared__ floatx4 lds[4][64];
    if ((int)blockIdx.x >= blocks) return loss_segment(p, blockIdx.x - blocks, lds[0]);
    const int rows = loss_chunk_rows(p);
    if (rows <= 0) return;
    const int n_tiles = (p.width + BN - 1) / BN, m_tiles = (rows + BM - 1) / BM, tiles = m_tiles * n_tiles;
    const int lane = threadIdx.x & 63, own = threadIdx.x >> 6, j = blockIdx.x % GROUPS * (MANY ? 1 : 4) + (MANY ? 0 : own);
    const int i = blockIdx.x / GROUPS % MB, wave = blockIdx.x / (GROUPS * MB) % 4, tile = blockIdx.x / (GROUPS * MB * 4);
    const int m0 = tile / n_tiles * BM + (wave >> 1) * (BM / 2) + 16 * i;
    if (tile >= tiles || m0 >= rows) return;
    const int m = m0 + (lane & 15), col = tile % n_tiles * BN + (wave & 1) * (BN / 2) + 16 * j + 4 * (lane >> 4);
    const int n = *p.part_count;
    const float* src = p.parts + (size_t)tile * (BM * BN) + (size_t)(wave * MB * NB + NB * i + j) * 256 + lane * 4;
    floatx4 s = floatx4{0, 0, 0, 0};
#pragma unroll 8
    for (int k = MANY ? own : 0; k < n; k += MANY ? 4 : 1) s += *(const floatx4*)(src + (size_t)k * tiles * (BM * BN));
    if constexpr (MANY) {
        lds[own][lane] = s;
        __syncthreads();
        if (own) return;
        s += lds[1][lane];
        s += lds[2][lane];
        s += lds[3][lane];
    }
    if (m >= rows || col >= p.width) return;
    const float gain = p.row_gain[m];
    *(uint2*)(p.dX + (size_t)p.rows[p.chunk0 + m] * p.width + col) = make_uint2(pack2_bf16(s[0] * gain, s[1] * gain), pack2_bf16(s[2] * gain, s[3] * gain));
}

}  // namespace symb
