// Attention of drafted trees over the paged cache: the launch plan and the C entries (kernels: cs_tree_impl.h).
#include <algorithm>
#include <functional>
#include <new>
#include <string.h>
#include <vector>
#include "cs_plan.h"
#include "cs_tree.h"
#include "cs_tree_impl.h"

namespace cs {

constexpr int32_t kTreeLeastPiece = 256;                         // keys of a piece, about, at least
constexpr int32_t kTreeModelled = 2048;                          // workgroups of a kv head up to which launches are modelled

// How a batch is launched: a pure function of the host lengths, the shape and the chip.
struct TreePlan {
    int32_t tiles = 0;                                           // column tiles of a workgroup: 1, 2 (wavefronts share the keys), 4, 8 or 12 (they share the rows)
    bool cut = false;                                            // some sequence comes in pieces
    std::vector<uint32_t> items;                                 // in launch order: a sequence's pieces and, innermost, its blocks stand together
    std::vector<int32_t> launches;                               // first items of the launches
    size_t ml_bytes = 0, bytes = 0;                              // workspace: (max, sum) of the partials, all of it
};

static size_t align16(size_t x) { return (x + 15) & ~(size_t)15; }

static TreePlan plan_tree(const cs_batch* b, int32_t Hq, int32_t Hkv, int32_t D) {
    TreePlan p;
    const int32_t G = Hq / Hkv, S = b->num_seqs;
    int32_t most = 1;
    for (int32_t s = 0; s < S; ++s) {
        const TreeBlocks t = tree_blocks((b->h_cu_q_lens[s + 1] - b->h_cu_q_lens[s]) * G);
        most = std::max(most, t.tiles);
    }
    p.tiles = most <= 1 ? 1 : most <= 2 ? most : (most + 3) / 4 * 4;
    // Pieces: the length at which a model of the launch ends first.  Workgroups of the chip's slots take the pieces in order, the longest first;
    // a step costs what it does on a full chip (measured with 512 workgroups of 4064 and 8160 keys, 8 kv heads), and a piece of a cut sequence its partial
    // result and a share of the merge.  (A fixed rule, halving from 8192 keys until there were two
    // workgroups a CU: 705 us where this one had 543, 32 trees of 8-32 nodes, 64/8 heads, on 2K-32K keys.)
    const int32_t slots = std::max(1, device_cus() * (p.tiles == 2 && D == 128 ? 1 : 2) / Hkv);
    auto step_us = [&](const TreeBlocks& t) {
        if (p.tiles <= 2) return 1.25 * (D == 64 || p.tiles == 2 ? 0.5 : 1.0);
        const double bytes = 1.31 / t.blocks, products = 0.33 * ((t.tiles + 3) / 4 + 1);   // a sequence's blocks share what they read
        return (D == 64 ? 0.55 : 1.0) * std::max(bytes, products + 0.22 * bytes);
    };
    auto pieces_of = [&](int32_t s, int64_t split) {
        const int32_t q = b->h_cu_q_lens[s + 1] - b->h_cu_q_lens[s], n = b->h_ctx_lens[s] + q, blocks = tree_blocks(q * G).blocks;
        if (blocks == 0) return 0;
        int32_t k = std::min(std::max((int32_t)((n + split / 2) / split), 1), std::min(kTreeMaxPieces, kMaxArgItems / blocks));
        for (int32_t fewer = k; k > 1; k = fewer) {              // (rounding a piece's length up can leave the last one empty)
            const int32_t c = tree_chunk_keys(n, k);
            fewer = (int32_t)(((int64_t)n + c - 1) / c);
            if (fewer >= k) break;
        }
        return k;
    };
    int64_t longest = kTreeLeastPiece;
    for (int32_t s = 0; s < S; ++s)
        if (b->h_cu_q_lens[s + 1] > b->h_cu_q_lens[s]) longest = std::max<int64_t>(longest, b->h_ctx_lens[s] + b->h_cu_q_lens[s + 1] - b->h_cu_q_lens[s]);
    const int64_t whole = 2 * longest;                           // nothing is cut
    int64_t split = whole;
    double least = 0;
    std::vector<float> work, busy;
    for (int64_t trial = whole; trial >= kTreeLeastPiece; trial = trial == whole ? longest : trial * 4 / 5) {
        // what the launch cannot end before: the slots' share of the work, and the longest piece
        auto piece_us = [&](const TreeBlocks& t, int32_t keys) { return 8.0 + (keys + 31) / 32 * step_us(t); };
        double partials = 0, all = 0, longest_us = 0;
        size_t pieces = 0;
        for (int32_t s = 0; s < S; ++s) {
            const int32_t q = b->h_cu_q_lens[s + 1] - b->h_cu_q_lens[s], n = b->h_ctx_lens[s] + q, k = pieces_of(s, trial);
            if (k == 0) continue;
            const TreeBlocks t = tree_blocks(q * G);
            const int32_t chunk = tree_chunk_keys(n, k);
            const double full = piece_us(t, chunk), last = piece_us(t, n - (k - 1) * chunk);
            all += t.blocks * ((k - 1) * full + last);
            longest_us = std::max(longest_us, full);
            pieces += (size_t)k * t.blocks;
            if (k > 1) partials += (double)k * t.blocks * t.tiles;
        }
        if ((int64_t)pieces > kTreeModelled && trial != whole) break;         // (pieces enough for an even end)
        const double merges = partials > 0 ? 4.0 + partials * Hkv * 16 * D * 8 / 5e6 : 0;
        if (trial != whole && std::max(all / slots, longest_us) + merges >= least) continue;
        work.clear();
        for (int32_t s = 0; s < S; ++s) {
            const int32_t q = b->h_cu_q_lens[s + 1] - b->h_cu_q_lens[s], n = b->h_ctx_lens[s] + q, k = pieces_of(s, trial);
            if (k == 0) continue;
            const TreeBlocks t = tree_blocks(q * G);
            const int32_t chunk = tree_chunk_keys(n, k);
            for (int32_t i = 0; i < k; ++i) work.insert(work.end(), t.blocks, (float)piece_us(t, std::min(chunk, n - i * chunk)));
        }
        std::sort(work.begin(), work.end(), std::greater<float>());
        busy.assign(slots, 0.f);                                 // a heap of when the slots come free
        for (float w : work) {
            std::pop_heap(busy.begin(), busy.end(), std::greater<float>());
            busy.back() += w;
            std::push_heap(busy.begin(), busy.end(), std::greater<float>());
        }
        const double end = *std::max_element(busy.begin(), busy.end()) + merges;
        if (trial == whole || end < least) { least = end; split = trial; }
    }
    struct Seq { int32_t seq, pieces, blocks, keys; };
    std::vector<Seq> seqs;
    seqs.reserve(S);
    for (int32_t s = 0; s < S; ++s) {
        const int32_t q = b->h_cu_q_lens[s + 1] - b->h_cu_q_lens[s], n = b->h_ctx_lens[s] + q, k = pieces_of(s, split);
        if (k == 0) continue;
        seqs.push_back({s, k, tree_blocks(q * G).blocks, tree_chunk_keys(n, k)});
        p.cut = p.cut || k > 1;
    }
    std::stable_sort(seqs.begin(), seqs.end(), [](const Seq& x, const Seq& y) { return x.keys > y.keys; });    // the longest first
    for (const Seq& s : seqs) {
        if (p.launches.empty() || (int32_t)p.items.size() - p.launches.back() + s.pieces * s.blocks > kMaxArgItems) p.launches.push_back((int32_t)p.items.size());
        for (int32_t i = 0; i < s.pieces; ++i)
            for (int32_t k = 0; k < s.blocks; ++k) p.items.push_back(tree_word(s.seq, i, s.pieces, k));
    }
    if (p.cut) {
        const size_t rows = p.items.size() * Hkv * 16 * p.tiles;
        p.ml_bytes = align16(rows * 2 * sizeof(float));
        p.bytes = p.ml_bytes + align16(rows * D * sizeof(float));
    }
    return p;
}

// The last plans that the thread made (the workspace query and the calls of the next layers ask for the same one: 64 sequences
// cost the host 35 us to plan, 256 of them 150; 115 and 540 where every cut was played), keyed by everything a plan depends on, the lengths value by value.
struct TreeMemo {
    int32_t S = -1, Hq = 0, Hkv = 0, D = 0, cus = 0;
    std::vector<int32_t> ctx, cu;
    TreePlan plan;
};
static const TreePlan& tree_plan_for(const cs_batch* b, int32_t Hq, int32_t Hkv, int32_t D) {
    static thread_local TreeMemo memo[4];
    static thread_local int next = 0;
    const int32_t S = b->num_seqs, cus = device_cus();
    for (TreeMemo& m : memo)
        if (m.S == S && m.Hq == Hq && m.Hkv == Hkv && m.D == D && m.cus == cus && memcmp(m.ctx.data(), b->h_ctx_lens, sizeof(int32_t) * S) == 0 &&
            memcmp(m.cu.data(), b->h_cu_q_lens, sizeof(int32_t) * (S + 1)) == 0)
            return m.plan;
    TreeMemo& m = memo[next];
    next = (next + 1) % 4;
    m.S = -1;                                                    // (no plan while this one is made: memory may run out)
    m.plan = plan_tree(b, Hq, Hkv, D);
    m.ctx.assign(b->h_ctx_lens, b->h_ctx_lens + S);
    m.cu.assign(b->h_cu_q_lens, b->h_cu_q_lens + S + 1);
    m.Hq = Hq; m.Hkv = Hkv; m.D = D; m.cus = cus;
    m.S = S;
    return m.plan;
}

template <int D, class E, int PS>
static void launch_tree(const TreePlan& p, const cs_kv_pool& pool, const uint16_t* layer_base, const cs_batch& b, int32_t G, const uint64_t* mask, int32_t mask_words,
                        const uint16_t* q, uint16_t* out, float scale_log2e, const TreePartials& part, const TreeItems& items, int32_t n, hipStream_t st) {
    const int32_t spread = p.tiles > 2 ? tree_spread_items(n, pool.num_kv_heads) : 0;
    const dim3 grid((uint32_t)(spread > 0 ? spread : n) * (uint32_t)pool.num_kv_heads);
#define CS_LAUNCH_TREE(KERNEL, NC, ...)                                                                                              \
    hipLaunchKernelGGL((KERNEL<D, E, PS, NC>), grid, dim3(kDecodeThreads), 0, st, layer_base, pool.page_stride, pool.num_pages,        \
                       pool.num_kv_heads, G, b.block_tables, b.max_blocks_per_seq, b.ctx_lens, b.cu_q_lens, mask, mask_words, q, out, scale_log2e, part, __VA_ARGS__)
    const int32_t n_spread = spread > 0 ? n : 0;
    if (p.tiles == 1) CS_LAUNCH_TREE(tree_kernel, 1, items);
    else if (p.tiles == 2) CS_LAUNCH_TREE(tree_kernel, 2, items);
    else if (p.tiles == 4) CS_LAUNCH_TREE(tree_ring_kernel, 1, n_spread, items);
    else if (p.tiles == 8) CS_LAUNCH_TREE(tree_ring_kernel, 2, n_spread, items);
    else CS_LAUNCH_TREE(tree_ring_kernel, 3, n_spread, items);
#undef CS_LAUNCH_TREE
}

template <int D, class E>
static int run_tree(const TreePlan& p, const cs_kv_pool& pool, int32_t layer, const cs_batch& b, int32_t G, const uint64_t* mask, int32_t mask_words,
                    const uint16_t* q, uint16_t* out, float scale, void* workspace, hipStream_t st) {
    const TreePartials part = {p.cut ? (float*)((char*)workspace + p.ml_bytes) : nullptr, p.cut ? (float*)workspace : nullptr};
    const uint16_t* layer_base = (const uint16_t*)pool.base + (int64_t)layer * pool.layer_stride;
    for (size_t i = 0; i < p.launches.size(); ++i) {
        TreeItems items;
        items.base = p.launches[i];
        const int32_t end = i + 1 < p.launches.size() ? p.launches[i + 1] : (int32_t)p.items.size(), n = end - items.base;
        std::copy(p.items.begin() + items.base, p.items.begin() + end, items.e);
        const float f = scale * 1.44269504088896340736f;
        if (pool.page_size == 16) launch_tree<D, E, 16>(p, pool, layer_base, b, G, mask, mask_words, q, out, f, part, items, n, st);
        else                      launch_tree<D, E, 8>(p, pool, layer_base, b, G, mask, mask_words, q, out, f, part, items, n, st);
        TreeMerges merges;
        uint32_t cut = 0;
        for (int32_t j = 0; p.cut && j < n; ++j) {
            const TreeItem it = tree_item(items.e[j]);
            if (it.pieces > 1 && it.piece == 0) merges.e[cut++] = {items.e[j], items.base + j};
        }
        if (cut > 0)
            hipLaunchKernelGGL((tree_merge_kernel<D, E>), dim3(cut * (uint32_t)pool.num_kv_heads, (uint32_t)p.tiles), dim3(4 * D), 0, st,
                               pool.num_kv_heads, G, 16 * p.tiles, b.cu_q_lens, out, part, merges);
    }
    return check_launch("tree_kernel");
}

static int32_t most_new(const cs_batch* b) {
    int32_t most = 0;
    for (int32_t s = 0; s < b->num_seqs; ++s) most = std::max(most, b->h_cu_q_lens[s + 1] - b->h_cu_q_lens[s]);
    return most;
}

static int attention_tree(const cs_kv_pool* pool, int32_t layer, const cs_batch* batch, const void* q, void* out, int32_t Hq, float softmax_scale,
                          const uint64_t* mask, int32_t mask_words, void* workspace, size_t workspace_bytes, void* stream, bool f16) {
    int rc = validate_pool(pool);
    if (rc) return rc;
    if (layer < 0 || layer >= pool->num_layers) return CS_ERR_INVALID_ARG;
    const int32_t Hkv = pool->num_kv_heads, D = pool->head_dim;
    rc = attention_shape_ok(Hq, Hkv, D);
    if (rc) return rc;
    rc = validate_batch(pool, batch);
    if (rc) return rc;
    if (batch->num_tokens == 0) return CS_OK;
    const int32_t most = most_new(batch);
    if (most > CS_MAX_TREE || !lengths_fit(batch)) return CS_ERR_UNSUPPORTED;
    if (!q || !out || ((uintptr_t)q & 15) || ((uintptr_t)out & 15)) return CS_ERR_INVALID_ARG;
    if (!(softmax_scale > 0.f) || softmax_scale > 3.0e38f) return CS_ERR_INVALID_ARG;   // positive, finite
    if (mask && (((uintptr_t)mask & 7) || mask_words < (most + 63) / 64 || mask_words > kTreeWords)) return CS_ERR_INVALID_ARG;
    try {
        const TreePlan& p = tree_plan_for(batch, Hq, Hkv, D);
        if (p.bytes > 0 && (!workspace || ((uintptr_t)workspace & 15))) return CS_ERR_INVALID_ARG;
        if (workspace_bytes < p.bytes) return CS_ERR_WORKSPACE_TOO_SMALL;
        const int32_t G = Hq / Hkv;
        hipStream_t st = (hipStream_t)stream;
        const uint16_t* qp = (const uint16_t*)q;
        uint16_t* op = (uint16_t*)out;
        if (D == 128)
            return f16 ? run_tree<128, F16>(p, *pool, layer, *batch, G, mask, mask_words, qp, op, softmax_scale, workspace, st)
                       : run_tree<128, Bf16>(p, *pool, layer, *batch, G, mask, mask_words, qp, op, softmax_scale, workspace, st);
        return f16 ? run_tree<64, F16>(p, *pool, layer, *batch, G, mask, mask_words, qp, op, softmax_scale, workspace, st)
                   : run_tree<64, Bf16>(p, *pool, layer, *batch, G, mask, mask_words, qp, op, softmax_scale, workspace, st);
    } catch (const std::bad_alloc&) {
        return hip_failed(hipErrorOutOfMemory, "launch plan");
    }
}

}  // namespace cs

using namespace cs;

extern "C" {

size_t cs_paged_attention_tree_workspace_bytes(const cs_batch* batch, int32_t Hq, int32_t Hkv, int32_t D) {
    if (attention_shape_ok(Hq, Hkv, D) != CS_OK) return 0;
    if (validate_batch(nullptr, batch) != CS_OK || batch->num_seqs == 0 || most_new(batch) > CS_MAX_TREE || !lengths_fit(batch)) return 0;
    try { return tree_plan_for(batch, Hq, Hkv, D).bytes; } catch (const std::bad_alloc&) { return 0; }
}

int cs_paged_attention_tree(const cs_kv_pool* pool, int32_t layer, const cs_batch* batch, const void* q, void* out, int32_t num_q_heads, float softmax_scale,
                            const uint64_t* tree_mask, int32_t mask_words, void* workspace, size_t workspace_bytes, void* stream) {
    return attention_tree(pool, layer, batch, q, out, num_q_heads, softmax_scale, tree_mask, mask_words, workspace, workspace_bytes, stream, false);
}

int cs_paged_attention_tree_f16(const cs_kv_pool* pool, int32_t layer, const cs_batch* batch, const void* q, void* out, int32_t num_q_heads, float softmax_scale,
                                const uint64_t* tree_mask, int32_t mask_words, void* workspace, size_t workspace_bytes, void* stream) {
    return attention_tree(pool, layer, batch, q, out, num_q_heads, softmax_scale, tree_mask, mask_words, workspace, workspace_bytes, stream, true);
}

}  // extern "C"
