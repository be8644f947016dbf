// Attention of drafted trees over the paged cache: the new tokens of a sequence are the nodes of a tree, and a node sees the
// cached tokens and the nodes that its mask names (by default: the nodes before it and itself).
//
// All nodes of a sequence see the same cached K and V, so the rows of one product are (node, query head of the kv head): R = q * G
// rows, 16 of them a column tile of
//   S^T[key][row] = K . Q^T            v_mfma_f32_16x16x32, 16 keys at a time
//   O^T[d][row]  += V^T . P^T          v_mfma_f32_16x16x32, 32 keys: two steps' keys, four consecutive ones of either a lane group
// with an online softmax per row in fp32.  K and V come from HBM into the operand registers as in decode (cs_decode_impl.h: the page
// format is the operand layout), and each page read serves up to kTreeTiles column tiles: a workgroup is
// (sequence, kv head, key range, block of up to 64 rows), its wavefronts take 32-key steps in turn.  Bound by HBM up to some 128 rows a kv
// head and beyond that by the matrix unit and the softmax's vector instructions.
#pragma once
#include "cs_decode_impl.h"
#include "cs_tree.h"

namespace cs {

constexpr int kTreeKeys = 32;                                    // keys of a step
constexpr float kTreeSlack = 6.f;                                // a running maximum may lie this far (in powers of two) below the scores

// LDS of a workgroup.
template <int D, int NC>
struct TreeLds {
    u32x4 q[NC][D / 32][64];                                     // Q as the B operand, lane by lane
    uint64_t mask[16 * NC + 1][kTreeWords + 1];                  // masks of the block's nodes, a word of zeros behind each
    float o[kDecodeWaves][16][D + 4];                            // one tile's partial outputs of the wavefronts
    float m[kDecodeWaves][NC][16], l[kDecodeWaves][NC][16];
};

template <class E>
__device__ __forceinline__ bool not_finite(uint32_t w) {
    constexpr uint32_t hi = E::kInfinity << 16;
    return (w & E::kInfinity) == E::kInfinity || (w & hi) == hi;
}
// The halves of w that are +infinity or no number (sign 0), or -infinity or no number (sign 1), as 1.0.
template <class E>
__device__ __forceinline__ uint32_t odd_ones(uint32_t w, uint32_t sign) {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t h = w >> 16 * i & 0xffffu, a = h & 0x7fffu;
        if (a > E::kInfinity || (a == E::kInfinity && h >> 15 == sign)) r |= (E::kOnes & 0xffffu) << 16 * i;
    }
    return r;
}
template <class E>
__device__ __forceinline__ uint32_t finite_only(uint32_t w) {
    const uint32_t lo = (w & E::kInfinity) == E::kInfinity ? 0u : w & 0xffffu;
    const uint32_t hi = (w >> 16 & E::kInfinity) == E::kInfinity ? 0u : w & 0xffff0000u;
    return lo | hi;
}

// A wavefront's running state of NC column tiles.
template <int D, int NC>
struct TreeState {
    f32x4 o[NC][D / 16];
    float m[NC], l[NC];
};

// One step: 32 keys from tok0 on, in the registers of two 16-key steps.  kTail: some of them are nodes, or lie behind the last one.
template <int D, class E, int NC, bool kTail>
__device__ __forceinline__ void tree_step(TreeState<D, NC>& st, PageRegs<D>& a, PageRegs<D>& b, const TreeLds<D, NC>& lds, int32_t tiles,
                                          float scale_log2e, int32_t tok0, int32_t ctx, int32_t n_keys, int32_t G, int32_t tile0, int lane)
{
    const int32_t quad = (lane >> 4) * 4;
    bool odd = false;
    if constexpr (kTail) {
        // slots behind the last token hold whatever was there
        auto keep = [&](PageRegs<D>& r, int32_t row0) {
            const int32_t valid = n_keys - row0;
            const uint32_t m0 = valid >= 2 ? 0xffffffffu : (valid == 1 ? 0x0000ffffu : 0u);
            const uint32_t m1 = valid >= 4 ? 0xffffffffu : (valid == 3 ? 0x0000ffffu : 0u);
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                r.v[dt][0] &= m0; r.v[dt][1] &= m1;
                odd = odd || not_finite<E>(r.v[dt][0]) || not_finite<E>(r.v[dt][1]);
            }
        };
        keep(a, tok0 + quad);
        keep(b, tok0 + 16 + quad);
        odd = __any(odd);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (c >= tiles) continue;
        f32x4 sa = {0.f, 0.f, 0.f, 0.f}, sb = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) {
            const u32x4 qb = lds.q[c][kk][lane];
            sa = E::mfma32(a.k[kk], qb, sa);
            sb = E::mfma32(b.k[kk], qb, sb);
        }
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = sa[i] * scale_log2e; x[4 + i] = sb[i] * scale_log2e; }
        uint32_t seen = 0xffu;                                   // bit i: x[i]'s key
        if constexpr (kTail) {
            const int32_t row = (tile0 + c) * 16 + (lane & 15), node = row / G - tile0 * 16 / G;
            const int32_t j = tok0 + quad - ctx;                 // the first key as a node
            uint64_t w;
            if (j >= 64 * kTreeWords) w = 0;
            else if (j <= -32) w = ~0ull;
            else if (j < 0) w = lds.mask[node][0] << -j | ((1ull << -j) - 1);
            else w = (j & 63) ? lds.mask[node][j >> 6] >> (j & 63) | lds.mask[node][(j >> 6) + 1] << (64 - (j & 63)) : lds.mask[node][j >> 6];
            const int32_t left = n_keys - (tok0 + quad);         // keys from the lane's first on
            if (left < 32) w &= left <= 0 ? 0ull : (1ull << left) - 1;
            seen = (uint32_t)(w & 15u) | (uint32_t)(w >> 16 & 15u) << 4;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = seen >> i & 1u ? x[i] : -INFINITY;
        }
        float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        mx = xor_max(mx, 16);
        mx = xor_max(mx, 32);
        if (__any(mx > st.m[c] + kTreeSlack)) {                  // (-infinity + slack: the first key that a row sees)
            const float m_new = fmaxf(st.m[c], mx), mu = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = exp2f(st.m[c] - mu);             // 0 where nothing was seen before
            st.l[c] *= alpha;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) st.o[c][dt] *= alpha;
            st.m[c] = m_new;
        }
        const float mu = st.m[c] == -INFINITY ? 0.f : st.m[c];
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = exp2f(x[i] - mu);
        // weights rounded to the element type, the matrix unit's operand; the sum is of the same rounded weights
        const u32x4 pb = { E::pack(p[0], p[1]), E::pack(p[2], p[3]), E::pack(p[4], p[5]), E::pack(p[6], p[7]) };
        st.l[c] += (E::sum2(pb[0]) + E::sum2(pb[1])) + (E::sum2(pb[2]) + E::sum2(pb[3]));
        if (!kTail || !odd) {
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt)
                st.o[c][dt] = E::mfma32(u32x4{a.v[dt][0], a.v[dt][1], b.v[dt][0], b.v[dt][1]}, pb, st.o[c][dt]);
        } else {
            // A V that is infinite or no number belongs to the rows that see its key, and a product with a weight of zero would bring
            // it to all: the product is made of the finite values, and a row that sees others gets them by themselves.
            u32x4 one;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                one[i] = (seen >> 2 * i & 1u ? E::kOnes & 0xffffu : 0u) | (seen >> (2 * i + 1) & 1u ? E::kOnes & 0xffff0000u : 0u);
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                const u32x4 v = {a.v[dt][0], a.v[dt][1], b.v[dt][0], b.v[dt][1]};
                u32x4 fin, up, down;
#pragma unroll
                for (int i = 0; i < 4; ++i) { fin[i] = finite_only<E>(v[i]); up[i] = odd_ones<E>(v[i], 0); down[i] = odd_ones<E>(v[i], 1); }
                st.o[c][dt] = E::mfma32(fin, pb, st.o[c][dt]);
                const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                const f32x4 plus = E::mfma32(up, one, zero), minus = E::mfma32(down, one, zero);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (plus[i] > 0.f) st.o[c][dt][i] += INFINITY;
                    if (minus[i] > 0.f) st.o[c][dt][i] -= INFINITY;
                }
            }
        }
    }
}

// Where the items of a cut block leave their partials: floats [item][kv head][16 NC rows][D], and (max, sum) of the rows.
struct TreePartials {
    float *o, *ml;
};

template <int D, class E, int PS, int NC>
__global__ __launch_bounds__(kDecodeThreads, 1) void tree_kernel(
    const uint16_t* __restrict__ layer_base, int64_t page_stride, int32_t num_pages, int32_t Hkv, int32_t G,
    const int32_t* __restrict__ block_tables, int32_t max_blocks, const int32_t* __restrict__ ctx_lens, const int32_t* __restrict__ cu_q_lens,
    const uint64_t* __restrict__ mask, int32_t mask_words, const uint16_t* __restrict__ q, uint16_t* __restrict__ out,
    float scale_log2e, TreePartials part, const TreeItems items)
{
    __shared__ TreeLds<D, NC> lds;
    const int32_t item = (int32_t)blockIdx.x / Hkv, g = (int32_t)blockIdx.x - item * Hkv;
    const TreeItem it = tree_item(items.e[item]);
    const int32_t s = it.seq, t0 = cu_q_lens[s], q_len = cu_q_lens[s + 1] - t0, ctx = ctx_lens[s];
    const int32_t n_keys = ctx + q_len, rows = q_len * G;
    const TreeBlocks blocks = tree_blocks(rows);
    const int32_t tile0 = it.block * blocks.tiles, tiles = min(blocks.tiles, (rows + 15) / 16 - tile0);
    const int32_t chunk = tree_chunk_keys(n_keys, it.pieces);
    const int32_t key_begin = min(n_keys, it.piece * chunk), key_end = min(n_keys, key_begin + chunk);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t Hq = Hkv * G;
    const int32_t* table = block_tables + (int64_t)s * max_blocks;
    const int32_t n_entries = min((n_keys + PS - 1) / PS, max_blocks);

    // the loads of the first step go out before Q and the masks are there
    const int32_t step_end = min((n_keys + kPage - 1) >> 4, PS == 16 ? max_blocks : (n_entries + 1) >> 1);      // 16-key steps that hold keys
    auto id_at = [&](int32_t step) { return loadable<PS>(step_ids<PS>(table, step, step_end, n_entries), num_pages); };
    auto fetch = [&](PageRegs<D>& r, const StepIds<PS>& id) { load_page<D>(r, layer_base, page_stride, id, g, Hkv, lane); };
    PageRegs<D> a0, b0, a1, b1;
    const int32_t pairs = (key_end - key_begin + kTreeKeys - 1) / kTreeKeys, first = key_begin >> 4;
    int32_t pair = wave;
    StepIds<PS> ida = id_at(first + 2 * pair), idb = id_at(first + 2 * pair + 1);
    fetch(a0, ida);
    fetch(b0, idb);
    ida = id_at(first + 2 * (pair + kDecodeWaves));
    idb = id_at(first + 2 * (pair + kDecodeWaves) + 1);

    for (int32_t u = threadIdx.x; u < tiles * (D / 32) * 64; u += kDecodeThreads) {
        const int32_t l = u & 63, kk = (u >> 6) % (D / 32), c = (u >> 6) / (D / 32);
        const int32_t row = (tile0 + c) * 16 + (l & 15), node = row / G, head = row - node * G;
        u32x4 v = {0u, 0u, 0u, 0u};
        if (row < rows) v = *(const u32x4*)(q + ((int64_t)(t0 + node) * Hq + g * G + head) * D + kk * 32 + (l >> 4) * 8);
        lds.q[c][kk][l] = v;
    }
    if (key_end > ctx) {
        const int32_t node0 = tile0 * 16 / G, nodes = min((tile0 + tiles) * 16 / G, q_len - 1) - node0 + 1;
        for (int32_t u = threadIdx.x; u < (16 * NC + 1) * (kTreeWords + 1); u += kDecodeThreads) {
            const int32_t n = u / (kTreeWords + 1), w = u - n * (kTreeWords + 1);
            uint64_t bits = 0;
            if (n < nodes && w < kTreeWords) {
                const int32_t node = node0 + n;
                if (!mask) bits = node >= 64 * w + 63 ? ~0ull : node < 64 * w ? 0ull : (2ull << (node & 63)) - 1;
                else if (w < mask_words) bits = mask[(int64_t)(t0 + node) * mask_words + w];
            }
            lds.mask[n][w] = bits;
        }
    }
    TreeState<D, NC> st;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        st.m[c] = -INFINITY;
        st.l[c] = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st.o[c][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __syncthreads();

    auto stage = [&](PageRegs<D>& ua, PageRegs<D>& ub, PageRegs<D>& fa, PageRegs<D>& fb) {
        const StepIds<PS> na = id_at(first + 2 * (pair + 2 * kDecodeWaves)), nb = id_at(first + 2 * (pair + 2 * kDecodeWaves) + 1);
        fetch(fa, ida);
        fetch(fb, idb);
        tree_step<D, E, NC, false>(st, ua, ub, lds, tiles, scale_log2e, key_begin + pair * kTreeKeys, ctx, n_keys, G, tile0, lane);
        ida = na; idb = nb;
        pair += kDecodeWaves;
    };
    const int32_t plain = max(0, min(pairs, (ctx - key_begin) / kTreeKeys));                // steps whose keys every row sees
    bool second = false;                                         // which registers hold the step to come
    while (pair < plain) {
        stage(a0, b0, a1, b1);
        second = true;
        if (pair >= plain) break;
        stage(a1, b1, a0, b0);
        second = false;
    }
    if (second) { a0 = a1; b0 = b1; }
    for (; pair < pairs;) {
        tree_step<D, E, NC, true>(st, a0, b0, lds, tiles, scale_log2e, key_begin + pair * kTreeKeys, ctx, n_keys, G, tile0, lane);
        pair += kDecodeWaves;
        if (pair >= pairs) break;
        fetch(a0, ida);
        fetch(b0, idb);
        ida = id_at(first + 2 * (pair + kDecodeWaves));
        idb = id_at(first + 2 * (pair + kDecodeWaves) + 1);
    }

    // the wavefronts' states are joined tile by tile
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        st.l[c] += __shfl_xor(st.l[c], 16, 64);
        st.l[c] += __shfl_xor(st.l[c], 32, 64);
        if (lane < 16) { lds.m[wave][c][lane] = st.m[c]; lds.l[wave][c][lane] = st.l[c]; }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (c >= tiles) continue;
        __syncthreads();
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) *(f32x4*)&lds.o[wave][lane & 15][dt * 16 + (lane >> 4) * 4] = st.o[c][dt];
        __syncthreads();
        for (int32_t u = threadIdx.x; u < 16 * (D / 4); u += kDecodeThreads) {
            const int32_t r = u / (D / 4), d = (u - r * (D / 4)) * 4, row = (tile0 + c) * 16 + r;
            if (row >= rows) continue;
            float M = lds.m[0][c][r];
#pragma unroll
            for (int w = 1; w < kDecodeWaves; ++w) M = fmaxf(M, lds.m[w][c][r]);
            float L = 0.f;
            f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kDecodeWaves; ++w) {
                const float mw = lds.m[w][c][r];
                if (mw == -INFINITY && lds.l[w][c][r] == 0.f) continue;      // (not a weight of zero: an infinity in V stays one)
                const float f = exp2f(mw - M);
                L += lds.l[w][c][r] * f;
                O += *(const f32x4*)&lds.o[w][r][d] * f;
            }
            if (it.pieces == 1) {
                const int32_t node = row / G, head = row - node * G;
                u32x2 w = {0u, 0u};                              // a row that sees nothing: zeros
                if (L != 0.f) w = u32x2{ E::pack(O[0] / L, O[1] / L), E::pack(O[2] / L, O[3] / L) };
                *(u32x2*)(out + ((int64_t)(t0 + node) * Hq + g * G + head) * D + d) = w;
            } else {
                const int64_t at = ((int64_t)(items.base + item) * Hkv + g) * (16 * NC) + c * 16 + r;
                *(f32x4*)(part.o + at * D + d) = O;
                if (d == 0) { part.ml[at * 2] = M; part.ml[at * 2 + 1] = L; }
            }
        }
    }
}

// Joins the pieces of cut blocks: a workgroup for each column tile (grid.y) of each first piece and kv head, a thread for 4 features of a row.
template <int D, class E>
__global__ __launch_bounds__(kDecodeThreads) void tree_merge_kernel(
    int32_t Hkv, int32_t G, int32_t part_rows, const int32_t* __restrict__ cu_q_lens, uint16_t* __restrict__ out, TreePartials part, const TreeItems items)
{
    const int32_t item = (int32_t)blockIdx.x / Hkv, g = (int32_t)blockIdx.x - item * Hkv, c = blockIdx.y;
    const TreeItem it = tree_item(items.e[item]);
    if (it.pieces == 1 || it.piece != 0) return;
    const int32_t t0 = cu_q_lens[it.seq], rows = (cu_q_lens[it.seq + 1] - t0) * G, Hq = Hkv * G;
    const TreeBlocks blocks = tree_blocks(rows);
    if (c >= blocks.tiles) return;
    for (int32_t u = threadIdx.x; u < 16 * (D / 4); u += kDecodeThreads) {
        const int32_t r = u / (D / 4), d = (u - r * (D / 4)) * 4, row = (it.block * blocks.tiles + c) * 16 + r;
        if (row >= rows) continue;
        float M = -INFINITY, L = 0.f;
        f32x4 O = {0.f, 0.f, 0.f, 0.f};
        const int64_t at = ((int64_t)(items.base + item) * Hkv + g) * part_rows + c * 16 + r, next = (int64_t)blocks.blocks * Hkv * part_rows;
        for (int32_t i = 0; i < it.pieces; ++i) M = fmaxf(M, part.ml[(at + i * next) * 2]);
        for (int32_t i = 0; i < it.pieces; ++i) {
            const float m = part.ml[(at + i * next) * 2], l = part.ml[(at + i * next) * 2 + 1];
            const f32x4 o = *(const f32x4*)(part.o + (at + i * next) * D + d);
            if (m == -INFINITY && l == 0.f) continue;
            const float f = exp2f(m - M);
            L += l * f;
            O += o * f;
        }
        const int32_t node = row / G, head = row - node * G;
        u32x2 w = {0u, 0u};
        if (L != 0.f) w = u32x2{ E::pack(O[0] / L, O[1] / L), E::pack(O[2] / L, O[3] / L) };
        *(u32x2*)(out + ((int64_t)(t0 + node) * Hq + g * G + head) * D + d) = w;
    }
}

}  // namespace cs
