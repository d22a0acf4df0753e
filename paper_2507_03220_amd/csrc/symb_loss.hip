// Host side of include/symb_loss.h: argument checks, the plan of a call and its launches.
#include "../../include/symb_loss.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>
#include <vector>

#include "loss_kernels.hpp"
#include "symb_context.hpp"

using namespace symb;

namespace {

symb_status check_loss(symb_handle h, const symb_loss_batch* b, int32_t entries) {
    if (!b) return fail(h, SYMB_ERR_INVALID_ARG, "batch is null");
    if (b->width <= 0 || b->width % 8) return fail(h, SYMB_ERR_INVALID_ARG, "width must be a positive multiple of 8");
    if (b->width > SYMB_LOSS_MAX_WIDTH) return fail(h, SYMB_ERR_UNSUPPORTED, "width %d exceeds SYMB_LOSS_MAX_WIDTH", b->width);
    if (b->vocab <= 0) return fail(h, SYMB_ERR_INVALID_ARG, "vocab must be positive");
    if (b->vocab > SYMB_LOSS_MAX_VOCAB) return fail(h, SYMB_ERR_UNSUPPORTED, "vocab %d exceeds SYMB_LOSS_MAX_VOCAB", b->vocab);
    if (b->reduction != SYMB_LOSS_MEAN && b->reduction != SYMB_LOSS_SUM) return fail(h, SYMB_ERR_INVALID_ARG, "unknown reduction %d", b->reduction);
    if (!(b->cap >= 0.f) || !std::isfinite(b->cap)) return fail(h, SYMB_ERR_INVALID_ARG, "cap must be finite and not negative");
    const symb_status st = check_segments(h, b->num_segments, b->seg_offsets);
    if (st != SYMB_OK) return st;
    if (b->num_segments && !b->losses) return fail(h, SYMB_ERR_INVALID_ARG, "losses is null");
    for (int i = 0; i < b->num_segments; ++i) {
        if (!std::isfinite(b->losses[i].scale)) return fail(h, SYMB_ERR_INVALID_ARG, "segment %d: scale must be finite", i);
        if (entries && (!(b->losses[i].temperature > 0.f) || !std::isfinite(b->losses[i].temperature)))
            return fail(h, SYMB_ERR_INVALID_ARG, "segment %d: temperature must be positive and finite", i);
        if (entries && (b->losses[i].temperature < 0x1p-20f || b->losses[i].temperature > 0x1p20f))        // (its square and its inverse go into fp32 products)
            return fail(h, SYMB_ERR_UNSUPPORTED, "segment %d: temperature %g, 2^-20 to 2^20 are supported", i, (double)b->losses[i].temperature);
    }
    if (entries < 0) return fail(h, SYMB_ERR_INVALID_ARG, "entries is negative");
    if (entries > SYMB_LOSS_MAX_ENTRIES) return fail(h, SYMB_ERR_UNSUPPORTED, "%d entries: SYMB_LOSS_MAX_ENTRIES at most", entries);
    const int64_t T = b->seg_offsets[b->num_segments];
    if (T > SYMB_LOSS_MAX_ROWS) return fail(h, SYMB_ERR_UNSUPPORTED, "%lld rows exceed SYMB_LOSS_MAX_ROWS", (long long)T);
    if (T * b->width >= ((int64_t)1 << 31)) return fail(h, SYMB_ERR_UNSUPPORTED, "%lld rows of %d: fewer than 2^31 elements at once", (long long)T, b->width);
    const size_t need = blob_bytes({{(size_t)b->num_segments + 1, sizeof(int32_t)}, {(size_t)b->num_segments, sizeof(LossDesc)}});
    if (need > kSlotBytes) return fail(h, SYMB_ERR_UNSUPPORTED, "batch descriptors need %zu bytes, capacity is %zu", need, kSlotBytes);
    return SYMB_OK;
}

// A call's chunks of rows, tiles, and the places of its workspace.
struct LossPlan {
    int chunk = 0, score_tile = kLossBig, grad_tile = kLossBig, pitch = 0, tile_cols = 0, column_parts = 0;
    int few = 0;                          // blocks of 16 rows of a batch that the kernel for few rows takes
    int64_t part_tiles = 0;
    size_t part_bytes = 0;
    bool two = false;                     // weights held in two terms
    bool many_parts = false;              // the second product's tiles come in many parts
    size_t rows = 0, flags = 0, count = 0, gain = 0, info = 0, label = 0, sorted = 0, shares = 0, scores = 0, starts = 0, row_loss = 0, stats = 0, row_gain = 0, held = 0, parts = 0, bytes = 0;
};
// What a call may hold: weights of a chunk of rows, and, where the losses alone are wanted, their sums.
constexpr int64_t kHeldBytes = (int64_t)2 << 30, kStatBytes = (int64_t)256 << 20;

constexpr int kLossListedRows = 512;

// Microseconds of the product with W of so many rows, in tiles of one kind; of the gradient's, in the number of parts that suits it best.
double score_us(int kind, int rows, const symb_loss_batch* b) {
    return loss_tiled(kind, [&](auto tile) {
        using L = decltype(tile);
        const int64_t tiles = L::tiles(rows, b->vocab);
        return 1e-3 * (double)((tiles + L::kSlots - 1) / L::kSlots) * ((b->width + 63) / 64 * (tiles <= L::kSlots / 2 ? L::kLoneNs : L::kStageNs) + (L::kSlots == 256 ? 8000 : 6000));
    });
}
double grad_us(int kind, int rows, const symb_loss_batch* b, bool two, int& n) {
    return loss_grad_tiled(kind, [&](auto tile) {
        using L = decltype(tile);
        const int64_t tiles = L::tiles(rows, b->width);
        int64_t least = INT64_MAX;
        for (int k = 1; k <= kLossParts && loss_grad_fits(tiles, b->vocab / 64, k, INT64_MAX); ++k) {
            const int64_t ns = L::ns(tiles, b->vocab / 64, k, two);
            if (ns + ns / 10000 * k < least) least = ns + ns / 10000 * k, n = k;
        }
        return 1e-3 * (double)least;
    });
}
// The kind that takes least, and that time.  (The second product in tiles of 256x128 was no faster anywhere.  The first, of 200 rows of 4096 over 32000: 74.4 us with them, 95.1 with those of
// 256x256, 90.3 with those of 128x128; 512 rows 126, 109, 160; 128 rows 85, 91, 76.)
int best_score(int rows, const symb_loss_batch* b, bool two, double& us) {
    int best = kLossSmall;
    us = score_us(best, rows, b);
    for (int kind = kLossBig; kind < kLossSmall && !two; ++kind)
        if (const double other = score_us(kind, rows, b); other < us) us = other, best = kind;
    return best;
}
int best_grad(int rows, const symb_loss_batch* b, bool two, int& n, double& us) {
    us = grad_us(kLossSmall, rows, b, two, n);
    int parts = 1;
    const double other = two ? us : grad_us(kLossBig, rows, b, false, parts);
    if (other >= us) return kLossSmall;
    n = parts;
    us = other;
    return kLossBig;
}

LossPlan plan_loss(const symb_loss_batch* b, int32_t entries, bool gradient) {
    LossPlan plan;
    const int64_t T = b->seg_offsets[b->num_segments], listed = T * entries;
    const int rows = (int)((T + 255) / 256 * 256);
    plan.pitch = (b->vocab + 63) / 64 * 64;
    // (a row's weights, or, of a small vocabulary, its fp32 product)
    const int64_t row_bytes = gradient ? std::max<int64_t>(plan.pitch * 2, (b->width + 255) / 256 * 1024) : ((int64_t)(b->vocab + 255) / 256) * 4 * (int64_t)sizeof(float2);
    const int most = (int)std::min<int64_t>(rows, std::max<int64_t>((gradient ? kHeldBytes : kStatBytes) / row_bytes / 256 * 256, 256));
    plan.two = gradient && T <= kTwoRows;
    // of the chunks that fit, the one whose whole chunks take least in all (each reads W once a product: 4.5 TB/s.  2048 rows of 4608 over 256000: 6.99 to 7.03 ms whole, 7.12 in 1792 and 256)
    const double read_us = (double)b->vocab * b->width * 2 / 4.5e6;
    int parts = 1;
    double least = 1e300;
    plan.chunk = most;
    const int step = std::max(256, most / 64 / 256 * 256);
    for (int c = step; c <= most; c += step) {
        const int whole = rows / c, rest = rows % c;
        auto us = [&](int r) {
            double score = 0.0, grad = 0.0;
            if (r) best_score(r, b, plan.two, score);
            if (r && gradient) best_grad(r, b, plan.two, parts, grad);
            return r ? std::max(score, read_us) + (gradient ? std::max(grad, read_us) : 0.0) + 15.0 : 0.0;
        };
        const double all = whole * us(c) + us(rest);
        if (all < least) least = all, plan.chunk = c;
    }
    const int first = (int)std::min<int64_t>(T, plan.chunk);
    double us = 0.0;
    plan.score_tile = best_score(first, b, plan.two, us);
    if (gradient) {
        // A row's few largest weights may be most of its gradient, and where rows are few their roundings do not even out: up to 64 rows (half of a tile of 128, whose other half costs nothing) hold
        // their weights in two bf16 terms.  One row: off by 1.7e-3 of it, what rounding dX costs, up to 3.7e-3 with one term; 256 rows with one term 2.4e-3.
        plan.grad_tile = best_grad(first, b, plan.two, parts, us);
        plan.many_parts = parts >= 8;
        loss_grad_tiled(plan.grad_tile, [&](auto tile) {
            using L = decltype(tile);
            // (room for more parts of fewer rows, where many of a batch take no part)
            plan.part_tiles = std::max<int64_t>(L::tiles(first, b->width) * parts, std::min<int64_t>(512, L::tiles(1, b->width) * std::max(b->vocab / 256, 1)));
            plan.part_bytes = (size_t)plan.part_tiles * L::kEdgeM * L::kEdgeN * sizeof(float);
        });
    }
    // The kernel for few rows: where rows are long or the tiles of 128 columns few.  Both sides, with W from HBM: 16 rows of 4096 over 32000 65 us with it, 75 with tiles; 32 rows 74, 76; of 6144 over
    // 49152 134, 142 and 149, 144; of 1024 over 50257 16 rows 45, 36; of 4096 over 12000 37, 65 and, 32 rows, 41, 66; of 768 over 4000 19, 20 and 23, 23.
    if (T <= kFewRows && (b->width >= 2048 || b->vocab <= 16384)) plan.few = T <= 16 ? 1 : 2;
    plan.tile_cols = plan.few ? kFewCols : plan.score_tile == kLossBig ? 256 : 128;
    const int column_tiles = (b->vocab + plan.tile_cols - 1) / plan.tile_cols;
    plan.column_parts = column_tiles * (plan.few ? 1 : 2);
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t o = at;
        at += align_up(n, 256);
        return o;
    };
    plan.rows = take(T * sizeof(int32_t));
    plan.flags = take(entries ? T * sizeof(int32_t) : 0);
    plan.count = take(2 * sizeof(int32_t));
    plan.gain = take(b->num_segments * sizeof(float));
    plan.info = take(T * sizeof(LossRow));
    plan.label = take(entries ? 0 : T * sizeof(float2));
    plan.sorted = take(listed * sizeof(int32_t));
    plan.shares = take(listed * sizeof(float));
    plan.scores = take(listed * sizeof(float));
    plan.starts = take(entries ? T * (column_tiles + 1) * sizeof(uint16_t) : 0);
    plan.row_loss = take(T * sizeof(float));
    plan.stats = take((size_t)plan.column_parts * plan.chunk * sizeof(float2));
    plan.row_gain = take(gradient ? plan.chunk * sizeof(float) : 0);
    plan.held = take(gradient ? (size_t)plan.chunk * plan.pitch * 2 : 0);
    plan.parts = take(plan.part_bytes);
    plan.bytes = T ? at : 0;
    return plan;
}

// A kernel of the tiles of gemm16_asm.hpp: its LDS once per context (the attribute belongs to the device the kernel is loaded on).
template <int MB, int NB, class F>
symb_status launch_tiles(symb_handle h, F kernel, int64_t tiles, const LossParams& p, hipStream_t s) {
    const void* k = reinterpret_cast<const void*>(kernel);
    constexpr int smem = Gemm16Tile<MB, NB>::SMEM;
    if (std::find(h->lds_attr_set.begin(), h->lds_attr_set.end(), k) == h->lds_attr_set.end()) {
        SYMB_HIP(h, hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, smem));
        h->lds_attr_set.push_back(k);
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(256), smem, s, p);
    SYMB_HIP(h, hipGetLastError());
    return SYMB_OK;
}
template <int MB, int NB>
symb_status launch_scores(symb_handle h, const LossParams& p, int rows, hipStream_t s, LossTile<MB, NB>) {
    const int64_t tiles = LossTile<MB, NB>::tiles(rows, p.V);
    auto by_teacher = [&](auto grad, auto cap) {
        constexpr bool G = decltype(grad)::value, C = decltype(cap)::value;
        return p.ids ? launch_tiles<MB, NB>(h, symb_loss_scores_kernel<MB, NB, G, C, true>, tiles, p, s) : launch_tiles<MB, NB>(h, symb_loss_scores_kernel<MB, NB, G, C, false>, tiles, p, s);
    };
    auto by_cap = [&](auto grad) { return p.cap > 0.f ? by_teacher(grad, std::true_type{}) : by_teacher(grad, std::false_type{}); };
    return p.dX ? by_cap(std::true_type{}) : by_cap(std::false_type{});
}
template <int RB>
symb_status launch_few(symb_handle h, const LossParams& p, hipStream_t s) {
    auto run = [&](auto grad, auto teacher) {
        hipLaunchKernelGGL((symb_loss_few_kernel<RB, decltype(grad)::value, decltype(teacher)::value>), dim3((p.V + kFewCols - 1) / kFewCols), dim3(64 * kFewWaves), 0, s, p);
    };
    if (p.dX) p.ids ? run(std::true_type{}, std::true_type{}) : run(std::true_type{}, std::false_type{});
    else p.ids ? run(std::false_type{}, std::true_type{}) : run(std::false_type{}, std::false_type{});
    SYMB_HIP(h, hipGetLastError());
    return SYMB_OK;
}
template <int MB, int NB>
symb_status launch_grad(symb_handle h, const LossParams& p, int rows, bool many_parts, bool segments, hipStream_t s, LossTile<MB, NB>) {
    const symb_status st = launch_tiles<MB, NB>(h, symb_loss_grad_kernel<MB, NB>, p.part_tiles, p, s);
    if (st != SYMB_OK) return st;
    const unsigned blocks = (unsigned)(LossTile<MB, NB>::tiles(rows, p.width) * 4 * MB * NB / (many_parts ? 1 : 4)), more = segments ? p.S : 0;
    if (many_parts) hipLaunchKernelGGL((symb_loss_reduce_kernel<MB, NB, true>), dim3(blocks + more), dim3(256), 0, s, p, (int)blocks);
    else hipLaunchKernelGGL((symb_loss_reduce_kernel<MB, NB, false>), dim3(blocks + more), dim3(256), 0, s, p, (int)blocks);
    SYMB_HIP(h, hipGetLastError());
    return SYMB_OK;
}

symb_status run_loss(symb_handle h, const symb_loss_batch* b, const void* X, const void* W, const int32_t* labels, const int32_t* ids, const float* logits, int32_t entries, float* loss,
                     float* row_loss, void* dX, void* ws, size_t ws_bytes, void* stream) {
    symb_status st = check_handle(h);
    if (st != SYMB_OK) return st;
    CallGuard guard(h);
    if ((st = check_loss(h, b, entries)) != SYMB_OK) return st;
    const int S = b->num_segments, T = b->seg_offsets[S];
    if (!S) return SYMB_OK;
    for (const void* ptr : {(const void*)loss, (const void*)row_loss, (const void*)labels, (const void*)ids, (const void*)logits})
        if ((uintptr_t)ptr & 3) return fail(h, SYMB_ERR_INVALID_ARG, "device pointers must be 4-byte aligned");
    if (T && (!X || !W || (entries ? !ids || !logits : !labels))) return fail(h, SYMB_ERR_INVALID_ARG, entries ? "X, W, ids and logits are required" : "X, W and labels are required");
    if (!loss && !row_loss && !dX) return fail(h, SYMB_ERR_INVALID_ARG, "neither losses nor a gradient are asked for");
    if (misaligned16(X) || misaligned16(W) || misaligned16(dX) || misaligned16(ws)) return fail(h, SYMB_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
    const LossPlan plan = plan_loss(b, entries, dX != nullptr);
    if (plan.bytes && (!ws || ws_bytes < plan.bytes)) return fail(h, SYMB_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes, %zu needed", ws ? ws_bytes : 0, plan.bytes);
    if (!T && !loss) return SYMB_OK;
    hipStream_t s = (hipStream_t)stream;
    std::vector<LossDesc> ld(S);
    for (int i = 0; i < S; ++i) ld[i] = LossDesc{b->losses[i].scale, b->losses[i].temperature};
    Blob blob;
    const size_t o_off = blob.add(b->seg_offsets, (size_t)S + 1), o_ld = blob.add(ld.data(), ld.size());
    unsigned char* dev = nullptr;
    if ((st = upload(h, blob, s, &dev)) != SYMB_OK) return st;
    unsigned char* const w = (unsigned char*)ws;
    LossParams p{};
    p.X = (const bf16*)X;
    p.W = (const bf16*)W;
    p.dX = (bf16*)dX;
    p.own_flags = (int32_t*)(w + plan.flags);
    p.flags = entries ? p.own_flags : labels;
    p.ids = ids;
    p.teacher = logits;
    p.loss = loss;
    p.row_loss = row_loss ? row_loss : (float*)(w + plan.row_loss);
    p.off = (const int32_t*)(dev + o_off);
    p.losses = (const LossDesc*)(dev + o_ld);
    p.rows = (int32_t*)(w + plan.rows);
    p.count = (int32_t*)(w + plan.count);
    p.part_count = p.count + 1;
    p.gain = (float*)(w + plan.gain);
    p.info = (LossRow*)(w + plan.info);
    p.label = (float2*)(w + plan.label);
    p.sorted = (int32_t*)(w + plan.sorted);
    p.shares = (float*)(w + plan.shares);
    p.scores = (float*)(w + plan.scores);
    p.starts = (uint16_t*)(w + plan.starts);
    p.stats = (float2*)(w + plan.stats);
    p.row_gain = (float*)(w + plan.row_gain);
    p.held = (bf16*)(w + plan.held);
    p.parts = (float*)(w + plan.parts);
    p.part_tiles = plan.part_tiles;
    p.T = T;
    p.S = S;
    p.V = b->vocab;
    p.pitch = plan.pitch;
    p.width = b->width;
    p.K = entries;
    p.tile_shift = plan.tile_cols == 64 ? 6 : plan.tile_cols == 128 ? 7 : 8;
    p.chunk = plan.chunk;
    p.group_m = 8;
    p.grad_tile = plan.grad_tile;
    p.two = plan.two;
    p.mean = b->reduction == SYMB_LOSS_MEAN;
    p.cap = b->cap;
    p.to_cap = b->cap > 0.f ? 1.f / b->cap : 0.f;
    const unsigned lists = (unsigned)((T + 255) / 256 + S), fours = (unsigned)((T + 3) / 4);
    if (entries && T) {
        // (few rows: the same launch lists them, of the ids themselves; every list of 256 reads those of all rows before it)
        const bool one = T <= kLossListedRows;
        hipLaunchKernelGGL(symb_loss_teacher_kernel, dim3(fours + (one ? lists : 0)), dim3(256), 4 * 2 * align_up(entries, 64) * sizeof(int32_t), s, p, one ? (int)lists : 0);
        SYMB_HIP(h, hipGetLastError());
        if (!one) {
            hipLaunchKernelGGL(symb_loss_rows_kernel, dim3(lists), dim3(256), 0, s, p);
            SYMB_HIP(h, hipGetLastError());
        }
    } else if (T) {
        hipLaunchKernelGGL(symb_loss_labels_kernel, dim3(lists + fours), dim3(256), 0, s, p);
        SYMB_HIP(h, hipGetLastError());
    }
    const bool finish = loss && T && T <= kJoinRows;
    for (int64_t at = 0; at < T; at += plan.chunk) {
        p.chunk0 = (int32_t)at;
        const int rows = (int)std::min<int64_t>(T - at, plan.chunk);
        if (plan.few) st = plan.few == 1 ? launch_few<1>(h, p, s) : launch_few<2>(h, p, s);
        else st = loss_tiled(plan.score_tile, [&](auto tile) { return launch_scores(h, p, rows, s, tile); });
        if (st != SYMB_OK) return st;
        hipLaunchKernelGGL(symb_loss_join_kernel, dim3((rows + kJoinRows - 1) / kJoinRows), dim3(kJoinRows * kJoinSets), 0, s, p, plan.column_parts, plan.few ? kFewCols : plan.tile_cols / 2, finish);
        SYMB_HIP(h, hipGetLastError());
        const bool segments = loss && !finish && at + rows == T;
        if (dX && (st = loss_grad_tiled(plan.grad_tile, [&](auto tile) { return launch_grad(h, p, rows, plan.many_parts, segments, s, tile); })) != SYMB_OK) return st;
    }
    if (loss && !finish && !(dX && T)) {
        hipLaunchKernelGGL(symb_loss_segments_kernel, dim3(S), dim3(256), 0, s, p);
        SYMB_HIP(h, hipGetLastError());
    }
    guard.completed = true;
    return seal_slot(h);
}

}  // namespace

extern "C" {

symb_status symb_loss_workspace_bytes(const symb_loss_batch* b, int32_t entries, int32_t gradient, size_t* out) {
    return guarded(nullptr, [&]() -> symb_status {
        if (!out) return fail(nullptr, SYMB_ERR_INVALID_ARG, "out is null");
        const symb_status st = check_loss(nullptr, b, entries);
        if (st != SYMB_OK) return st;
        *out = plan_loss(b, entries, gradient != 0).bytes;
        return SYMB_OK;
    });
}

symb_status symb_cross_entropy(symb_handle h, const symb_loss_batch* b, const void* X, const void* W, const int32_t* labels, float* loss, float* row_loss, void* dX, void* ws, size_t ws_bytes,
                               void* stream) {
    return guarded(h, [&]() -> symb_status { return run_loss(h, b, X, W, labels, nullptr, nullptr, 0, loss, row_loss, dX, ws, ws_bytes, stream); });
}

symb_status symb_distillation(symb_handle h, const symb_loss_batch* b, const void* X, const void* W, const int32_t* ids, const float* logits, int32_t entries, float* loss, float* row_loss,
                              void* dX, void* ws, size_t ws_bytes, void* stream) {
    return guarded(h, [&]() -> symb_status {
        if (entries < 1) return fail(h, SYMB_ERR_INVALID_ARG, "entries must be positive");
        return run_loss(h, b, X, W, nullptr, ids, logits, entries, loss, row_loss, dX, ws, ws_bytes, stream);
    });
}

}  // extern "C"
