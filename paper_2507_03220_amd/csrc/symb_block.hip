// Host side of include/symb_block.h: argument checks, work lists and launches of the norms and of the calls on the key/value cache.
#include "../../include/symb_block.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <initializer_list>
#include <new>
#include <utility>
#include <vector>

#include "kv_append_kernel.hpp"
#include "kv_attention_kernels.hpp"
#include "norm_kernels.hpp"
#include "symb_context.hpp"

using namespace symb;

namespace {

// Nothing throws across the C boundary: the work lists are the only allocations.
template <class F>
symb_status guarded(symb_handle h, F&& f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return fail(h, SYMB_ERR_UNSUPPORTED, "out of host memory for the batch's work lists");
    }
}

symb_status check_segments(symb_handle h, int32_t S, const int32_t* off) {
    if (S < 0) return fail(h, SYMB_ERR_INVALID_ARG, "num_segments is negative");
    if (!off) return fail(h, SYMB_ERR_INVALID_ARG, "seg_offsets is null");
    if (off[0] != 0) return fail(h, SYMB_ERR_BAD_SEGMENTS, "seg_offsets[0] must be 0");
    for (int i = 0; i < S; ++i)
        if (off[i + 1] < off[i]) return fail(h, SYMB_ERR_BAD_SEGMENTS, "seg_offsets decrease at segment %d", i);
    return SYMB_OK;
}

// The size of a Blob of these lists: what the workspace queries refuse as the calls do.
size_t blob_bytes(std::initializer_list<std::pair<size_t, size_t>> lists) {              // (entries, bytes of one)
    size_t n = 0;
    for (const auto& l : lists) n = align_up(n, 16) + std::max<size_t>(l.first, 1) * l.second;
    return n;
}

// ---- norms -----------------------------------------------------------------------------------
symb_status check_norm(symb_handle h, const symb_norm_batch* b) {
    if (!b) return fail(h, SYMB_ERR_INVALID_ARG, "batch is null");
    if (b->width <= 0 || b->width % 8) return fail(h, SYMB_ERR_INVALID_ARG, "width must be a positive multiple of 8");
    if (b->width > SYMB_NORM_MAX_WIDTH) return fail(h, SYMB_ERR_UNSUPPORTED, "width %d exceeds SYMB_NORM_MAX_WIDTH", b->width);
    if (b->kind != SYMB_NORM_LAYER && b->kind != SYMB_NORM_RMS) return fail(h, SYMB_ERR_INVALID_ARG, "unknown norm kind %d", b->kind);
    if (!(b->eps >= 0.f) || !std::isfinite(b->eps)) return fail(h, SYMB_ERR_INVALID_ARG, "eps must be finite and not negative");
    if (!std::isfinite(b->weight_base)) return fail(h, SYMB_ERR_INVALID_ARG, "weight_base must be finite");
    const symb_status st = check_segments(h, b->num_segments, b->seg_offsets);
    if (st != SYMB_OK) return st;
    if (b->num_segments && !b->norms) return fail(h, SYMB_ERR_INVALID_ARG, "norms is null");
    for (int i = 0; i < b->num_segments; ++i) {
        const symb_norm& n = b->norms[i];
        for (const void* ptr : {n.weight, n.bias, (const void*)n.dweight, (const void*)n.dbias})
            if (misaligned16(ptr)) return fail(h, SYMB_ERR_INVALID_ARG, "segment %d: norm pointer is not 16-byte aligned", i);
    }
    return SYMB_OK;
}

// The backward pass in chunks of rows.  Chunks of one group (the segments that name the same gradients) have their partial sums side by side, in the order
// of the batch, and are added in it.
struct NormPlan {
    std::vector<NormChunk> chunks;
    std::vector<NormGroup> groups;
    int parts = 0;
};
// Up to three workgroups a CU are on it together, so the rows are cut into 768 chunks at most, and into 512 or 256 where that many pay: a chunk's row takes 0.55 us, its partial sums 8 bytes a column
// and gradient at 4.9 TB/s, least in all with rows^2 = kNormParts (gradients) (rows of the batch) width to a chunk.  20480 rows of 2048 with bias (1290 chunks by this): 768 chunks 61.8 us, 512 66.3;
// 20480 of 4608 without (1219): 123.8, 122.0; 14 segments of 541 rows of 4096 (790): 47.7, 45.4; 5000 of 6144 with bias (367): 512 52.7, 256 49.7; 3000 of 4096 (500): 19.8, 20.6.
// A few chunks more than that, as segments' rounding up would have it, cost a round: 770 of them 50.6 us.
constexpr int kNormChunks = 768, kNormRows = 4;
constexpr double kNormParts = 3e-6;
symb_status plan_norm(symb_handle h, const symb_norm_batch* b, NormPlan& plan) {
    const int S = b->num_segments, T = b->seg_offsets[S];
    std::vector<int> order(S);
    for (int i = 0; i < S; ++i) order[i] = i;
    const symb_norm* n = b->norms;
    auto key = [&](int i) { return std::make_pair((uintptr_t)n[i].dweight, (uintptr_t)n[i].dbias); };
    std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return key(x) < key(y); });
    // a gradient named together with two different partners
    std::vector<std::pair<uintptr_t, uintptr_t>> seen;
    for (int i = 0; i < S; ++i) {
        if (i && key(order[i]) == key(order[i - 1])) continue;
        const auto k = key(order[i]);
        if (k.first) seen.emplace_back(k.first, i);
        if (k.second) seen.emplace_back(k.second, i);
    }
    std::sort(seen.begin(), seen.end());
    for (size_t i = 1; i < seen.size(); ++i)
        if (seen[i].first == seen[i - 1].first) return fail(h, SYMB_ERR_INVALID_ARG, "two segments share one of dweight and dbias, but not both");
    bool dw = false, db = false;
    int longest = 0;
    for (int i = 0; i < S; ++i) {
        dw |= n[i].dweight != nullptr;
        db |= n[i].dbias != nullptr;
        longest = std::max(longest, b->seg_offsets[i + 1] - b->seg_offsets[i]);
    }
    const double fit = T / std::max(std::sqrt(kNormParts * (dw + db) * T * b->width), (double)kNormRows);
    const int chunks = fit > 1250 ? kNormChunks : fit > 384 ? kNormChunks * 2 / 3 : kNormChunks / 3;
    int rows = std::max(kNormRows, (T + chunks - 1) / chunks);
    auto count = [&](int per) {
        int64_t c = 0;
        for (int i = 0; i < S; ++i) c += (b->seg_offsets[i + 1] - b->seg_offsets[i] + per - 1) / per;
        return c;
    };
    if (rows < longest && count(longest) <= chunks)
        for (int high = longest; rows < high;) {
            const int mid = rows + (high - rows) / 2;
            if (count(mid) <= chunks) high = mid;
            else rows = mid + 1;
        }
    for (int at = 0; at < S;) {
        int to = at + 1;
        while (to < S && key(order[to]) == key(order[at])) ++to;
        const bool wanted = n[order[at]].dweight || n[order[at]].dbias;
        NormGroup g{(float*)n[order[at]].dweight, (float*)n[order[at]].dbias, plan.parts, 0};
        for (int i = at; i < to; ++i) {
            const int s = order[i];
            for (int r = b->seg_offsets[s]; r < b->seg_offsets[s + 1]; r += rows)
                plan.chunks.push_back(NormChunk{s, r, std::min(rows, b->seg_offsets[s + 1] - r), wanted ? plan.parts + g.parts++ : -1});
        }
        plan.parts += g.parts;
        if (wanted) plan.groups.push_back(g);
        at = to;
    }
    if (plan.groups.size() > 65535) return fail(h, SYMB_ERR_UNSUPPORTED, "%zu different weight gradients: 65535 at most", plan.groups.size());
    const size_t need = blob_bytes({{(size_t)S, sizeof(NormDesc)}, {plan.chunks.size(), sizeof(NormChunk)}, {plan.groups.size(), sizeof(NormGroup)}});
    if (need > kSlotBytes) return fail(h, SYMB_ERR_UNSUPPORTED, "batch descriptors need %zu bytes, capacity is %zu", need, kSlotBytes);
    return SYMB_OK;
}
size_t norm_part_bytes(const NormPlan& plan, int width) { return align_up((size_t)plan.parts * width * sizeof(float), 256); }

std::vector<NormDesc> norm_descs(const symb_norm_batch* b) {
    std::vector<NormDesc> d(b->num_segments);
    for (int i = 0; i < b->num_segments; ++i)
        d[i] = NormDesc{(const bf16*)b->norms[i].weight, (const bf16*)b->norms[i].bias, (float*)b->norms[i].dweight, (float*)b->norms[i].dbias};
    return d;
}

template <bool RMS, int WAVES, int NV>
void launch_norm_fwd(const NormFwdParams& p, hipStream_t s) {
    constexpr int rows = WAVES < 4 ? 4 / WAVES : 1;
    hipLaunchKernelGGL((symb_norm_fwd_kernel<RMS, WAVES, NV>), dim3((p.T + rows - 1) / rows), dim3(WAVES < 4 ? 256 : WAVES * 64), 0, s, p);
}
// One wavefront a row while its registers hold it well, four above (20000 rows of 768: 14.3 us with one, 20.8 with four; of 2048 34.7, 37.0; of 4096 71, 63.3), and no more vectors a lane than
// the width asks for where that tells (20000 rows of 512 10.7 us with one, 12.1 with four; of 4096 63.3 with two, 64.5 with four; of 4608 and 6144 three are no better than four).
template <bool RMS>
void launch_norm_fwd(const NormFwdParams& p, hipStream_t s) {
    const int vecs = p.width / 8;
    if (vecs <= 64) return launch_norm_fwd<RMS, 1, 1>(p, s);
    if (vecs <= 256) return launch_norm_fwd<RMS, 1, 4>(p, s);
    if (vecs <= 512) return launch_norm_fwd<RMS, 4, 2>(p, s);
    if (vecs <= 1024) return launch_norm_fwd<RMS, 4, 4>(p, s);
    return launch_norm_fwd<RMS, 4, 8>(p, s);
}
template <bool RMS, bool BIAS, int WAVES, int NV>
void launch_norm_bwd(const NormBwdParams& p, int chunks, hipStream_t s) {
    hipLaunchKernelGGL((symb_norm_bwd_kernel<RMS, BIAS, WAVES, NV>), dim3(chunks), dim3(WAVES * 64), 0, s, p);
}
// Likewise (20000 rows of 768 41 us with one vector, 76 with four; of 4096 110.1 with two, 112.2; 5000 of 16384 124 with eight wavefronts, 153 with four of eight vectors a lane).
template <bool RMS, bool BIAS>
void launch_norm_bwd(const NormBwdParams& p, int chunks, hipStream_t s) {
    const int vecs = p.width / 8;
    if (vecs <= 256) return launch_norm_bwd<RMS, BIAS, 4, 1>(p, chunks, s);
    if (vecs <= 512) return launch_norm_bwd<RMS, BIAS, 4, 2>(p, chunks, s);
    if (vecs <= 1024) return launch_norm_bwd<RMS, BIAS, 4, 4>(p, chunks, s);
    return launch_norm_bwd<RMS, BIAS, 8, 4>(p, chunks, s);
}

// ---- key/value cache --------------------------------------------------------------------------
symb_status check_kv(symb_handle h, const symb_kv_batch* b, const symb_kv_cache* c) {
    if (!b) return fail(h, SYMB_ERR_INVALID_ARG, "batch is null");
    if (!c) return fail(h, SYMB_ERR_INVALID_ARG, "cache is null");
    const symb_status st = check_segments(h, b->num_segments, b->seg_offsets);
    if (st != SYMB_OK) return st;
    if (c->num_pages <= 0 || c->kv_heads <= 0) return fail(h, SYMB_ERR_INVALID_ARG, "num_pages and kv_heads must be positive");
    if (c->kv_heads > 8192) return fail(h, SYMB_ERR_UNSUPPORTED, "%d key heads: 8192 at most", c->kv_heads);
    if (c->head_dim != 64 && c->head_dim != 128) return fail(h, SYMB_ERR_UNSUPPORTED, "head_dim %d: 64 or 128", c->head_dim);
    if (c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128)
        return fail(h, SYMB_ERR_UNSUPPORTED, "page_tokens %d: 32, 64 or 128", c->page_tokens);
    if (b->num_segments && !b->past) return fail(h, SYMB_ERR_INVALID_ARG, "past is null");
    if (b->table_stride < 0 || (int64_t)b->num_segments * b->table_stride > INT32_MAX)
        return fail(h, SYMB_ERR_UNSUPPORTED, "page table of %d x %d entries", b->num_segments, b->table_stride);
    for (int i = 0; i < b->num_segments; ++i) {
        const int64_t n = b->seg_offsets[i + 1] - b->seg_offsets[i], len = (int64_t)b->past[i] + n;
        if (b->past[i] < 0) return fail(h, SYMB_ERR_INVALID_ARG, "past of segment %d is negative", i);
        if (!n) continue;
        if (len > INT32_MAX - 1024) return fail(h, SYMB_ERR_UNSUPPORTED, "segment %d has %lld tokens", i, (long long)len);
        if ((len + c->page_tokens - 1) / c->page_tokens > b->table_stride)
            return fail(h, SYMB_ERR_INVALID_ARG, "segment %d has %lld tokens, its row of the page table %d pages", i, (long long)len, b->table_stride);
    }
    return SYMB_OK;
}
symb_status check_kv_pointers(symb_handle h, const symb_kv_batch* b, const symb_kv_cache* c) {
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return fail(h, SYMB_ERR_INVALID_ARG, "cache pointers are required");
    if (misaligned16(c->k) || misaligned16(c->v)) return fail(h, SYMB_ERR_INVALID_ARG, "cache pointers must be 16-byte aligned");
    if (!b->page_table || ((uintptr_t)b->page_table & 3)) return fail(h, SYMB_ERR_INVALID_ARG, "page_table is null or misaligned");
    return SYMB_OK;
}
symb_status check_rows(symb_handle h, const void* p, int64_t stride, int64_t width, const char* what) {
    if (!p) return fail(h, SYMB_ERR_INVALID_ARG, "%s is null", what);
    if (misaligned16(p)) return fail(h, SYMB_ERR_INVALID_ARG, "%s is not 16-byte aligned", what);
    if (stride < width || stride % 8) return fail(h, SYMB_ERR_INVALID_ARG, "%s has rows %lld elements apart: a multiple of 8, %lld at least", what, (long long)stride, (long long)width);
    return SYMB_OK;
}
int page_shift(const symb_kv_cache* c) { return c->page_tokens == 32 ? 5 : c->page_tokens == 64 ? 6 : 7; }

template <int D>
void launch_append(const KvAppendParams& p, int pages, bool few, int ny, hipStream_t s) {
    if (few) hipLaunchKernelGGL((symb_kv_append_kernel<D, 64>), dim3(pages, ny), dim3(64), 0, s, p);
    else hipLaunchKernelGGL((symb_kv_append_kernel<D, 256>), dim3(pages, ny), dim3(256), 0, s, p);
}

// The work of one attention call.
struct KvPlan {
    std::vector<KvItem> items[3];         // tiles and, behind them, items of up to 16 rows; items of 32 rows; of 48
    int tiles = 0;
    std::vector<KvJoinItem> joins;
    int join_rows = 0;                    // the most rows of one of them
    int64_t part_rows = 0;                // rows of partial results, of one key head
};
// The kernels of an attention call: runs of `rows` rows of a segment for a key head.  All go over the tokens in chunks of 64.
struct KvKernel {
    int rows;
    int slots;                            // workgroups that run at once: two a CU (of a head of 64 three fit; counted on, they gained nothing), one with the registers of 17 rows and more
    int worth;                            // chunks that a workgroup has to be spared for parts to pay
};
// Joining parts costs a launch and a pass over them, 5 to 8 us.  A chunk takes a workgroup's wavefront (one in four goes to each) 0.9 us with up to 16 rows, 1.6 and 2.5 with 32 and 48, and a
// tile's workgroup 1.2 us, 2.0 beside another on its CU.
constexpr KvKernel kKvKernels[4] = {{128, 512, 4}, {16, 512, 20}, {32, 256, 12}, {48, 256, 8}};
static_assert(kKvChunk == kKvTileChunk, "");
// Which of them a segment's rows go to: up to 16 rows the second, above tiles (from 49 rows) or the kernels of 32 and 48 rows, where their work, counted in chunks of 16 rows, is worth it.
// Those widen the values once for all their rows, but 16 rows at a time are more workgroups, four wavefronts side by side on a run's tokens, and no launch of their own.
// Up to 48 rows, both sides (48 query heads on one key head): 91 chunks 15.0 us with 48 rows, 9.4 with 16; 4850 22.6, 21.3; 14400 32.4, 43; 35800 52.5, 87.6.  (32 key heads): 7700 30.5, 24.0;
// 17700 39.4, 35.9; 43600 77.4, 82.4.  Prompts, where their runs of 16 rows fill the chip once at most: 1290 chunks in 512 runs 13.3 us in tiles, 9.5; 2400 in 256 20.0, 12.6; 6500 in 480 26.3, 18.9;
// 12900 in 384 24.3, 15.9; 38000 in 512 41, 56; more runs than that: 2700 in 1024 13.5, 15.1; 3700 in 1500 11.0, 18.6.
constexpr int64_t kKvWideWork = 12288, kKvFewRuns = 512;

// Chunks that a workgroup takes: as few as keep all workgroups on the chip at once, where that is possible and spares the longest run enough; else all of a run's, and where the runs
// alone are more than that, what leaves about that many.  (Tiles are not split then: they come longest first, and while some wait for a place the longest is not what the call waits for.
// 816 tiles of up to 59 chunks 102 us, split at 36 chunks 112; 768 of up to 128 219, split 250.)
int64_t plan_quota(const std::vector<int32_t>& chunks, int kv_heads, const KvKernel& k) {
    int64_t most = 1, sum = 0;
    for (const int32_t n : chunks) {
        most = std::max<int64_t>(most, n);
        sum += n;
    }
    if (k.rows > 48 && (int64_t)chunks.size() * kv_heads > k.slots) return most;
    int64_t low = std::max<int64_t>((sum * kv_heads + k.slots - 1) / k.slots, 4), high = most;
    if ((int64_t)chunks.size() * kv_heads <= k.slots)
        for (int64_t at = low; at < high;) {              // (the fewest in [low, most]: a part of every run is one workgroup for each head)
            const int64_t mid = (at + high) / 2;
            int64_t parts = 0;
            for (const int32_t n : chunks) parts += (n + mid - 1) / mid;
            if (parts * kv_heads <= k.slots) high = low = mid;
            else at = low = mid + 1;
        }
    return most - low < k.worth ? most : low;
}

symb_status plan_attention(symb_handle h, const symb_kv_batch* b, const symb_kv_cache* c, int q_heads, int window, KvPlan& plan) {
    const int group = q_heads / c->kv_heads;
    std::vector<KvItem> runs;
    std::vector<int32_t> chunks;
    int64_t work[2] = {0, 0}, tiled_runs = 0;                      // of up to 48 rows, of more
    for (int i = 0; i < b->num_segments; ++i) {
        const int64_t n = b->seg_offsets[i + 1] - b->seg_offsets[i], rows = n * group;
        if (rows <= kKvKernels[1].rows) continue;
        const bool tiled = rows > kKvKernels[3].rows;
        const int64_t begin = window ? std::max<int64_t>((int64_t)b->past[i] + 1 - window, 0) / kKvChunk * kKvChunk : 0, of16 = (rows + 15) / 16 * c->kv_heads;
        work[tiled] += (b->past[i] + n + kKvChunk - 1 - begin) / kKvChunk * of16;
        if (tiled) tiled_runs += of16;
    }
    const bool wide = work[0] >= kKvWideWork, tiles = work[1] >= kKvWideWork || tiled_runs > kKvFewRuns;
    auto kind_of = [&](int64_t rows) { return rows > kKvKernels[3].rows ? (tiles ? 0 : 1) : rows > kKvKernels[1].rows && wide ? (rows > kKvKernels[2].rows ? 3 : 2) : 1; };
    for (int kind = 0; kind < 4; ++kind) {
        const KvKernel& kernel = kKvKernels[kind];
        runs.clear();
        chunks.clear();
        for (int i = 0; i < b->num_segments; ++i) {
            const int64_t rows = (int64_t)(b->seg_offsets[i + 1] - b->seg_offsets[i]) * group;
            if (!rows || kind_of(rows) != kind) continue;
            for (int64_t r0 = 0; r0 < rows; r0 += kernel.rows) {
                const int64_t first = b->past[i] + r0 / group, last = b->past[i] + std::min(r0 + kernel.rows - 1, rows - 1) / group;
                const int64_t begin = window ? std::max<int64_t>(first + 1 - window, 0) / kKvChunk * kKvChunk : 0;
                runs.push_back(KvItem{i * b->table_stride, b->seg_offsets[i], (int32_t)rows, b->past[i], (int32_t)r0, (int32_t)begin, (int32_t)last + 1, -1});
                chunks.push_back((int32_t)((last + kKvChunk - begin) / kKvChunk));
            }
        }
        if (runs.empty()) continue;
        const int64_t quota = plan_quota(chunks, c->kv_heads, kernel);
        std::vector<KvItem>& items = plan.items[std::max(kind - 1, 0)];
        const size_t at = items.size();
        for (size_t j = 0; j < runs.size(); ++j) {
            const KvItem& run = runs[j];
            const int n = chunks[j], parts = (int)((n + quota - 1) / quota);
            if (parts <= 1) {
                items.push_back(run);
                continue;
            }
            for (int r = run.r0; r < std::min(run.r0 + kernel.rows, run.rows); r += 16) {
                plan.joins.push_back(KvJoinItem{run.row0, run.rows, r, (int32_t)(plan.part_rows + r - run.r0), parts, kernel.rows});
                plan.join_rows = std::max(plan.join_rows, std::min(16, run.rows - r));
            }
            for (int k = 0; k < parts; ++k) {
                KvItem it = run;
                it.begin = run.begin + (int)((int64_t)n * k / parts) * kKvChunk;
                if (k + 1 < parts) it.end = run.begin + (int)((int64_t)n * (k + 1) / parts) * kKvChunk;
                it.part = (int32_t)plan.part_rows;
                plan.part_rows += kernel.rows;
                items.push_back(it);
            }
        }
        // the longest first: what is left over at the end is short
        std::stable_sort(items.begin() + at, items.end(), [](const KvItem& x, const KvItem& y) { return x.end - x.begin > y.end - y.begin; });
        if (kind == 0) {
            // and where two tiles share a CU from the start, the longest with the shortest of them: the second 256 workgroups the other way round.  512 tiles of up to 128 chunks 191 us, 198 without
            const size_t n1 = 256 / std::min(c->kv_heads, 256);
            if (items.size() > n1) std::reverse(items.begin() + n1, items.begin() + std::min(items.size(), 2 * n1));
            plan.tiles = (int)items.size();
        }
    }
    size_t all = plan.joins.size();
    for (const auto& list : plan.items) all += list.size();
    if ((int64_t)all * c->kv_heads > INT32_MAX || plan.part_rows > INT32_MAX) return fail(h, SYMB_ERR_UNSUPPORTED, "%zu work items of %d key heads", all, c->kv_heads);
    const size_t need = blob_bytes({{plan.items[0].size(), sizeof(KvItem)}, {plan.items[1].size(), sizeof(KvItem)}, {plan.items[2].size(), sizeof(KvItem)}, {plan.joins.size(), sizeof(KvJoinItem)}});
    if (need > kSlotBytes) return fail(h, SYMB_ERR_UNSUPPORTED, "%zu work items need %zu bytes of descriptors, capacity is %zu", all, need, kSlotBytes);
    return SYMB_OK;
}
size_t part_ml_bytes(const KvPlan& plan, int kv_heads) { return align_up((size_t)plan.part_rows * kv_heads * 2 * sizeof(float), 256); }
size_t part_bytes(const KvPlan& plan, const symb_kv_cache* c) {
    return plan.part_rows ? part_ml_bytes(plan, c->kv_heads) + (size_t)plan.part_rows * c->kv_heads * c->head_dim * sizeof(float) : 0;
}
symb_status check_attention(symb_handle h, const symb_kv_batch* b, const symb_kv_cache* c, int32_t q_heads, int32_t window) {
    const symb_status st = check_kv(h, b, c);
    if (st != SYMB_OK) return st;
    if (q_heads <= 0 || q_heads % c->kv_heads) return fail(h, SYMB_ERR_INVALID_ARG, "q_heads must be a positive multiple of kv_heads");
    if (window < 0) return fail(h, SYMB_ERR_INVALID_ARG, "window is negative");
    int64_t least = 0;                                            // work items, before any list of them is made
    for (int i = 0; i < b->num_segments; ++i) {
        const int64_t rows = (int64_t)(b->seg_offsets[i + 1] - b->seg_offsets[i]) * (q_heads / c->kv_heads);
        if (rows > INT32_MAX - 1024) return fail(h, SYMB_ERR_UNSUPPORTED, "segment %d has too many rows", i);
        least += (rows + kKvTileRows - 1) / kKvTileRows;
    }
    if (least * (int64_t)sizeof(KvItem) > (int64_t)kSlotBytes) return fail(h, SYMB_ERR_UNSUPPORTED, "%lld work items at least, %zu fit the descriptors", (long long)least, kSlotBytes / sizeof(KvItem));
    return SYMB_OK;
}

// From this many rows on, the parts of 16 rows are joined in a workgroup; below, where rows are few and their parts many, a workgroup joins one.  Both sides: 24500 rows of two parts 7.4 us and
// 21.8; 12000 rows of a 30000 token context 130.7 and 136.6 in all; 4800 of 8000 42 and 39; 2300 of up to 16000 37.7 and 32.
constexpr int64_t kKvJoinRows = 8192;
template <int D, bool CAP>
symb_status launch_attention(symb_handle h, KvAttentionParams p, const KvPlan& plan, const KvItem* const (&items)[3], const KvJoinParams& jp, hipStream_t s) {
    for (int i = 0; i < 3; ++i) {
        if (plan.items[i].empty()) continue;
        p.items = items[i];
        p.tiles = i ? 0 : plan.tiles;
        const dim3 grid((unsigned)(plan.items[i].size() * p.kv_heads));
        if (i == 0) hipLaunchKernelGGL((symb_kv_attention_kernel<D, CAP>), grid, dim3(256), 0, s, p);
        else if (i == 1) hipLaunchKernelGGL((symb_kv_rows_kernel<D, 2, CAP>), grid, dim3(256), 0, s, p);
        else hipLaunchKernelGGL((symb_kv_rows_kernel<D, 3, CAP>), grid, dim3(256), 0, s, p);
        SYMB_HIP(h, hipGetLastError());
    }
    if (!plan.joins.empty()) {
        const int64_t n = (int64_t)plan.joins.size() * p.kv_heads;
        if (n * plan.join_rows >= kKvJoinRows) hipLaunchKernelGGL((symb_kv_join_rows_kernel<D>), dim3((unsigned)n), dim3(256), 0, s, jp);
        else hipLaunchKernelGGL((symb_kv_join_kernel<D>), dim3((unsigned)n, plan.join_rows), dim3(256), 0, s, jp);
        SYMB_HIP(h, hipGetLastError());
    }
    return SYMB_OK;
}

}  // namespace

extern "C" {

symb_status symb_norm_workspace_bytes(const symb_norm_batch* b, size_t* out) {
    return guarded(nullptr, [&]() -> symb_status {
        if (!out) return fail(nullptr, SYMB_ERR_INVALID_ARG, "out is null");
        symb_status st = check_norm(nullptr, b);
        if (st != SYMB_OK) return st;
        NormPlan plan;
        if ((st = plan_norm(nullptr, b, plan)) != SYMB_OK) return st;
        *out = 2 * norm_part_bytes(plan, b->width);
        return SYMB_OK;
    });
}

symb_status symb_norm_fwd(symb_handle h, const symb_norm_batch* b, const void* X, void* Y, void* stream) {
    return guarded(h, [&]() -> symb_status {
        symb_status st = check_handle(h);
        if (st != SYMB_OK) return st;
        CallGuard guard(h);
        if ((st = check_norm(h, b)) != SYMB_OK) return st;
        const int T = b->seg_offsets[b->num_segments];
        if (!T) return SYMB_OK;
        if (!X || !Y) return fail(h, SYMB_ERR_INVALID_ARG, "X and Y are required");
        if (misaligned16(X) || misaligned16(Y)) return fail(h, SYMB_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
        hipStream_t s = (hipStream_t)stream;
        const std::vector<NormDesc> nd = norm_descs(b);
        Blob blob;
        const size_t o_off = blob.add(b->seg_offsets, (size_t)b->num_segments + 1), o_nd = blob.add(nd.data(), nd.size());
        unsigned char* dev = nullptr;
        if ((st = upload(h, blob, s, &dev)) != SYMB_OK) return st;
        const NormFwdParams p{(const bf16*)X, (bf16*)Y, (const int32_t*)(dev + o_off), (const NormDesc*)(dev + o_nd), b->num_segments, T, b->width, b->eps, b->weight_base};
        if (b->kind == SYMB_NORM_RMS) launch_norm_fwd<true>(p, s);
        else launch_norm_fwd<false>(p, s);
        SYMB_HIP(h, hipGetLastError());
        guard.completed = true;
        return seal_slot(h);
    });
}

symb_status symb_norm_bwd(symb_handle h, const symb_norm_batch* b, const void* X, const void* dY, void* dX, uint32_t flags, void* ws, size_t ws_bytes, void* stream) {
    return guarded(h, [&]() -> symb_status {
        symb_status st = check_handle(h);
        if (st != SYMB_OK) return st;
        CallGuard guard(h);
        if ((st = check_norm(h, b)) != SYMB_OK) return st;
        if (flags != SYMB_GRAD_OVERWRITE && flags != SYMB_GRAD_ACCUMULATE) return fail(h, SYMB_ERR_INVALID_ARG, "unknown flags %u", flags);
        NormPlan plan;
        if ((st = plan_norm(h, b, plan)) != SYMB_OK) return st;
        const int T = b->seg_offsets[b->num_segments];
        if (!T && (plan.groups.empty() || flags == SYMB_GRAD_ACCUMULATE)) return SYMB_OK;
        if (T && (!X || !dY || !dX)) return fail(h, SYMB_ERR_INVALID_ARG, "X, dY and dX are required");
        if (misaligned16(X) || misaligned16(dY) || misaligned16(dX) || misaligned16(ws)) return fail(h, SYMB_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
        const size_t part = norm_part_bytes(plan, b->width);
        if (2 * part > ws_bytes || (part && !ws)) return fail(h, SYMB_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes, %zu needed", ws ? ws_bytes : 0, 2 * part);
        hipStream_t s = (hipStream_t)stream;
        const std::vector<NormDesc> nd = norm_descs(b);
        Blob blob;
        const size_t o_nd = blob.add(nd.data(), nd.size()), o_ch = blob.add(plan.chunks.data(), plan.chunks.size()), o_gr = blob.add(plan.groups.data(), plan.groups.size());
        unsigned char* dev = nullptr;
        if ((st = upload(h, blob, s, &dev)) != SYMB_OK) return st;
        float *part_w = (float*)ws, *part_b = (float*)((unsigned char*)ws + part);
        if (T) {
            const NormBwdParams p{(const bf16*)X, (const bf16*)dY, (bf16*)dX, (const NormDesc*)(dev + o_nd), (const NormChunk*)(dev + o_ch), part_w, part_b, b->width, b->eps, b->weight_base};
            const int n = (int)plan.chunks.size();
            const bool rms = b->kind == SYMB_NORM_RMS, bias = std::any_of(plan.groups.begin(), plan.groups.end(), [](const NormGroup& g) { return g.db; });
            if (bias) rms ? launch_norm_bwd<true, true>(p, n, s) : launch_norm_bwd<false, true>(p, n, s);
            else rms ? launch_norm_bwd<true, false>(p, n, s) : launch_norm_bwd<false, false>(p, n, s);
            SYMB_HIP(h, hipGetLastError());
        }
        if (!plan.groups.empty()) {
            const NormReduceParams p{part_w, part_b, (const NormGroup*)(dev + o_gr), b->width, flags == SYMB_GRAD_ACCUMULATE};
            hipLaunchKernelGGL(symb_norm_reduce_kernel, dim3((b->width + 63) / 64, (unsigned)plan.groups.size()), dim3(256), 0, s, p);
            SYMB_HIP(h, hipGetLastError());
        }
        guard.completed = true;
        return seal_slot(h);
    });
}

symb_status symb_kv_append(symb_handle h, const symb_kv_batch* b, const symb_kv_cache* cache, const symb_rotation* rotation, const void* q, int64_t q_stride, int32_t q_heads,
                           void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* stream) {
    return guarded(h, [&]() -> symb_status {
        symb_status st = check_handle(h);
        if (st != SYMB_OK) return st;
        CallGuard guard(h);
        if ((st = check_kv(h, b, cache)) != SYMB_OK) return st;
        if (q_heads < 0) return fail(h, SYMB_ERR_INVALID_ARG, "q_heads is negative");
        const int S = b->num_segments, P = cache->page_tokens, D = cache->head_dim;
        int64_t most = 0;
        for (int i = 0; i < S; ++i)
            if (b->seg_offsets[i + 1] > b->seg_offsets[i]) most = std::max<int64_t>(most, (int64_t)b->past[i] + b->seg_offsets[i + 1] - b->seg_offsets[i]);
        if (rotation) {
            if (rotation->dim <= 0 || rotation->dim % 16 || rotation->dim > D) return fail(h, SYMB_ERR_INVALID_ARG, "rotation of %d elements: a multiple of 16, at most head_dim", rotation->dim);
            if (rotation->pairs != SYMB_ROTATE_HALVES && rotation->pairs != SYMB_ROTATE_ADJACENT) return fail(h, SYMB_ERR_INVALID_ARG, "unknown pairing %d", rotation->pairs);
            if (rotation->positions < most) return fail(h, SYMB_ERR_INVALID_ARG, "rotation table of %d positions, %lld needed", rotation->positions, (long long)most);
        }
        if (b->seg_offsets[S] == 0) return SYMB_OK;
        if ((q_heads > 0) != (q != nullptr)) return fail(h, SYMB_ERR_INVALID_ARG, "q_heads is %d and q is %s", q_heads, q ? "given" : "null");
        if ((st = check_kv_pointers(h, b, cache)) != SYMB_OK) return st;
        if (rotation && (!rotation->table || misaligned16(rotation->table))) return fail(h, SYMB_ERR_INVALID_ARG, "rotation table is null or not 16-byte aligned");
        if ((st = check_rows(h, k, k_stride, (int64_t)cache->kv_heads * D, "k")) != SYMB_OK) return st;
        if ((st = check_rows(h, v, v_stride, (int64_t)cache->kv_heads * D, "v")) != SYMB_OK) return st;
        if (q && (st = check_rows(h, q, q_stride, (int64_t)q_heads * D, "q")) != SYMB_OK) return st;
        if (q && (st = check_rows(h, q_out, q_out_stride, (int64_t)q_heads * D, "q_out")) != SYMB_OK) return st;
        size_t count = 0;
        for (int i = 0; i < S; ++i)
            if (b->seg_offsets[i + 1] > b->seg_offsets[i])
                count += (size_t)(((int64_t)b->past[i] + b->seg_offsets[i + 1] - b->seg_offsets[i] - 1) / P - b->past[i] / P + 1);
        if (count * sizeof(KvPage) > kSlotBytes) return fail(h, SYMB_ERR_UNSUPPORTED, "new tokens in %zu pages, %zu fit the descriptors", count, kSlotBytes / sizeof(KvPage));
        std::vector<KvPage> pages;
        int rows = 0;
        for (int i = 0; i < S; ++i)
            for (int64_t at = 0, n = b->seg_offsets[i + 1] - b->seg_offsets[i]; at < n;) {
                const int64_t pos = b->past[i] + at, take = std::min(n - at, P - pos % P);
                pages.push_back(KvPage{(int32_t)((int64_t)i * b->table_stride + pos / P), (int32_t)(b->seg_offsets[i] + at), (int32_t)take, (int32_t)pos});
                rows = std::max(rows, (int)take);
                at += take;
            }
        const bool few = rows <= kKvFewRows;
        const int heads_q = few ? 1 : 8, q_groups = (q_heads + heads_q - 1) / heads_q;
        const int64_t ny = 2 * (int64_t)cache->kv_heads + q_groups;
        if (ny > 65535) return fail(h, SYMB_ERR_UNSUPPORTED, "%d query heads beside %d key heads", q_heads, cache->kv_heads);
        hipStream_t s = (hipStream_t)stream;
        Blob blob;
        const size_t o_pg = blob.add(pages.data(), pages.size());
        unsigned char* dev = nullptr;
        if ((st = upload(h, blob, s, &dev)) != SYMB_OK) return st;
        KvAppendParams p{};
        p.pages = (const KvPage*)(dev + o_pg);
        p.page_table = b->page_table;
        p.k = (unsigned char*)cache->k;
        p.v = (unsigned char*)cache->v;
        p.k_scale = (unsigned char*)cache->k_scale;
        p.v_scale = (unsigned char*)cache->v_scale;
        p.rotation = rotation ? (const float*)rotation->table : nullptr;
        p.q_in = (const bf16*)q;
        p.q_out = (bf16*)q_out;
        p.k_in = (const bf16*)k;
        p.v_in = (const bf16*)v;
        p.q_stride = q_stride;
        p.q_out_stride = q_out_stride;
        p.k_stride = k_stride;
        p.v_stride = v_stride;
        p.num_pages = cache->num_pages;
        p.kv_heads = cache->kv_heads;
        p.q_heads = q_heads;
        p.page_shift = page_shift(cache);
        p.turned = rotation ? rotation->dim : 0;
        p.adjacent = rotation && rotation->pairs == SYMB_ROTATE_ADJACENT;
        p.heads_q = heads_q;
        p.q_groups = q_groups;
        if (D == 128) launch_append<128>(p, (int)pages.size(), few, (int)ny, s);
        else launch_append<64>(p, (int)pages.size(), few, (int)ny, s);
        SYMB_HIP(h, hipGetLastError());
        guard.completed = true;
        return seal_slot(h);
    });
}

symb_status symb_kv_workspace_bytes(const symb_kv_batch* b, const symb_kv_cache* cache, int32_t q_heads, int32_t window, size_t* out) {
    return guarded(nullptr, [&]() -> symb_status {
        if (!out) return fail(nullptr, SYMB_ERR_INVALID_ARG, "out is null");
        symb_status st = check_attention(nullptr, b, cache, q_heads, window);
        if (st != SYMB_OK) return st;
        KvPlan plan;
        if ((st = plan_attention(nullptr, b, cache, q_heads, window, plan)) != SYMB_OK) return st;
        *out = part_bytes(plan, cache);
        return SYMB_OK;
    });
}

symb_status symb_kv_attention(symb_handle h, const symb_kv_batch* b, const symb_kv_cache* cache, const void* q, int64_t q_stride, int32_t q_heads, void* out, int64_t out_stride,
                              float scale, int32_t window, float cap, void* ws, size_t ws_bytes, void* stream) {
    return guarded(h, [&]() -> symb_status {
        symb_status st = check_handle(h);
        if (st != SYMB_OK) return st;
        CallGuard guard(h);
        if ((st = check_attention(h, b, cache, q_heads, window)) != SYMB_OK) return st;
        if (!(scale > 0.f) || !std::isfinite(scale)) return fail(h, SYMB_ERR_INVALID_ARG, "scale must be positive and finite");
        if (!(cap >= 0.f) || !std::isfinite(cap)) return fail(h, SYMB_ERR_INVALID_ARG, "cap must be finite and not negative");
        if (b->seg_offsets[b->num_segments] == 0) return SYMB_OK;
        if ((st = check_kv_pointers(h, b, cache)) != SYMB_OK) return st;
        const int D = cache->head_dim;
        if ((st = check_rows(h, q, q_stride, (int64_t)q_heads * D, "q")) != SYMB_OK) return st;
        if ((st = check_rows(h, out, out_stride, (int64_t)q_heads * D, "out")) != SYMB_OK) return st;
        KvPlan plan;
        if ((st = plan_attention(h, b, cache, q_heads, window, plan)) != SYMB_OK) return st;
        const size_t need = part_bytes(plan, cache);
        if (need && (!ws || ws_bytes < need)) return fail(h, SYMB_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes, %zu needed", ws ? ws_bytes : 0, need);
        if (need && misaligned16(ws)) return fail(h, SYMB_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
        hipStream_t s = (hipStream_t)stream;
        Blob blob;
        size_t o_items[3];
        for (int i = 0; i < 3; ++i) o_items[i] = blob.add(plan.items[i].data(), plan.items[i].size());
        const size_t o_join = blob.add(plan.joins.data(), plan.joins.size());
        unsigned char* dev = nullptr;
        if ((st = upload(h, blob, s, &dev)) != SYMB_OK) return st;
        constexpr float kLog2e = 1.442695041f;
        KvAttentionParams p{};
        p.page_table = b->page_table;
        p.k = (const unsigned char*)cache->k;
        p.v = (const unsigned char*)cache->v;
        p.k_scale = (const unsigned char*)cache->k_scale;
        p.v_scale = (const unsigned char*)cache->v_scale;
        p.q = (const bf16*)q;
        p.out = (bf16*)out;
        p.part_ml = (float*)ws;
        p.part_o = (float*)((unsigned char*)ws + part_ml_bytes(plan, cache->kv_heads));
        p.q_stride = q_stride;
        p.out_stride = out_stride;
        p.num_pages = cache->num_pages;
        p.kv_heads = cache->kv_heads;
        p.group = q_heads / cache->kv_heads;
        p.page_shift = page_shift(cache);
        p.window = window;
        p.part_rows = (int32_t)plan.part_rows;
        p.scale = scale * kLog2e;
        if (cap > 0.f) {                  // (a quotient beyond fp32 is held at its end: scores of zero stay zero)
            p.cap = std::min(cap / scale, FLT_MAX);
            p.to_cap = std::min(kKvRoot * (scale / cap), FLT_MAX);
        }
        const KvJoinParams jp{(const KvJoinItem*)(dev + o_join), p.part_o, p.part_ml, p.out, out_stride, p.kv_heads, p.group, p.part_rows};
        const KvItem* const items[3] = {(const KvItem*)(dev + o_items[0]), (const KvItem*)(dev + o_items[1]), (const KvItem*)(dev + o_items[2])};
        if (D == 128) st = cap > 0.f ? launch_attention<128, true>(h, p, plan, items, jp, s) : launch_attention<128, false>(h, p, plan, items, jp, s);
        else st = cap > 0.f ? launch_attention<64, true>(h, p, plan, items, jp, s) : launch_attention<64, false>(h, p, plan, items, jp, s);
        if (st != SYMB_OK) return st;
        guard.completed = true;
        return seal_slot(h);
    });
}

}  // extern "C"
