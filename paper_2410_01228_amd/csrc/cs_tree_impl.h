// Attention of drafted trees over the paged cache: the new tokens of a sequence are the nodes of a tree, and a node sees the
// cached tokens and the nodes that its mask names (by default: the nodes before it and itself).
//
// All nodes of a sequence see the same cached K and V, so the rows of one product are (node, query head of the kv head): R = q * G
// rows, 16 of them a column tile of
//   S^T[key][row] = K . Q^T            v_mfma_f32_16x16x32, 16 keys at a time
//   O^T[d][row]  += V^T . P^T          v_mfma_f32_16x16x32, 32 keys: two steps' keys, four consecutive ones of either a lane group
// with an online softmax per row in fp32.  K and V come from HBM into the operand registers as in decode (cs_decode_impl.h: the page
// format is the operand layout), and each page read serves up to kTreeTiles column tiles: a workgroup is
// (sequence, kv head, key range, block of up to 192 rows), and its wavefronts take 32-key steps in turn (up to 32 rows) or rows (beyond).  Bound by HBM up
// to some 128 rows a kv head, and beyond that by the matrix unit and the softmax's vector instructions at the clock that they leave the card.
#pragma once
#include <type_traits>
#include "cs_decode_impl.h"
#include "cs_prefill_impl.h"
#include "cs_tree.h"

namespace cs {

constexpr int kTreeKeys = 32;                                    // keys of a step
constexpr float kTreeSlack = 6.f;                                // a running maximum may lie this far (in powers of two) below the scores

// Wavefronts of a SIMD: outputs of NC tiles (D / 4 registers each), two steps of K and V (D / 2 each) and the rest.
constexpr int tree_waves(int D, int NC) { return D * NC >= 256 ? 1 : 2; }

// LDS of a workgroup.
template <int D, int NC>
struct TreeLds {
    u32x4 q[NC][D / 32][64];                                // Q as the B operand, lane by lane
    uint64_t mask[16 * NC + 1][kTreeWords + 1];                  // masks of the block's nodes, a word of zeros behind each
    alignas(16) float o[kDecodeWaves][16][D + 4];                // one tile's partial outputs of the wavefronts, four floats at a time
    float m[kDecodeWaves][NC][16], l[kDecodeWaves][NC][16];
    int32_t odd;                                                 // a step met a V that is not finite
};

template <class E>
__device__ __forceinline__ bool not_finite(uint32_t w) {
    constexpr uint32_t hi = E::kInfinity << 16;
    return ((w & E::kInfinity) == E::kInfinity) | ((w & hi) == hi);
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

// K and V of a step, as operands: 16-key step h in element h of k, V's four tokens of a lane group from either.
template <int D>
struct TreeKv {
    u32x4 k[2][D / 32];
    u32x2 v[2][D / 16];
    __device__ __forceinline__ u32x4 both(int dt) const { return u32x4{v[0][dt][0], v[0][dt][1], v[1][dt][0], v[1][dt][1]}; }
};

// A lane's addresses in a page, in bytes from its K and its V block.
template <int D, int PS> struct TreeLane {
    uint32_t k, v;
    __device__ __forceinline__ TreeLane(int lane) {
        if (PS == 16) { k = lane * 16; v = (((lane >> 5) * 16 + (lane & 15)) * 2 + ((lane >> 4) & 1)) * 8; }
        else          { k = ((lane >> 4) * 8 + (lane & 7)) * 16; v = ((lane & 15) * 2 + ((lane >> 4) & 1)) * 8; }
    }
};

// One 16-key step's K into k[h], V into half h of v.  (Pages of 8: see load_page.)
template <int D, int PS, int H>
__device__ __forceinline__ void load_k(TreeKv<D>& r, const uint16_t* __restrict__ layer_base, int64_t page_stride, StepIds<PS> id, int32_t g, const TreeLane<D, PS>& at, int lane)
{
    int32_t page = id.a;
    if constexpr (PS == 8) page = (lane & 8) ? id.b : id.a;
    const char* p = (const char*)(layer_base + (int64_t)page * page_stride + (int64_t)g * (PS * D)) + at.k;
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) r.k[H][kk] = __builtin_nontemporal_load((const u32x4*)(p + kk * (PS * 64)));
}
template <int D, int PS, int H>
__device__ __forceinline__ void load_v(TreeKv<D>& r, const uint16_t* __restrict__ layer_base, int64_t page_stride, StepIds<PS> id, int32_t g, int32_t Hkv, const TreeLane<D, PS>& at, int lane)
{
    int32_t page = id.a;
    if constexpr (PS == 8) page = (lane & 32) ? id.b : id.a;
    const char* p = (const char*)(layer_base + (int64_t)page * page_stride + (int64_t)(Hkv + g) * (PS * D)) + at.v;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) r.v[H][dt] = __builtin_nontemporal_load((const u32x2*)(p + dt * (PS * 32)));
}

// The four weights' sum of the lane's two dwords pairs, as they are after rounding (bf16), or before it (fp16: below 2^-14 the matrix unit keeps
// subnormal weights, v_dot2 would not).
template <class E>
__device__ __forceinline__ float sum_weights(const float (&p)[8], u32x4 pb, float l) {
    if constexpr (E::kInfinity == 0x7f80u) {
        typedef __bf16 x2 __attribute__((ext_vector_type(2)));
        const x2 one = __builtin_bit_cast(x2, E::kOnes);
#pragma unroll
        for (int i = 0; i < 4; ++i) l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(x2, (uint32_t)pb[i]), one, l, false);
        return l;
    } else {
        return l + (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])));
    }
}

// Scores of one tile: 32 keys in K's registers.
template <int D, class E>
__device__ __forceinline__ void tree_scores(const TreeKv<D>& r, const u32x4 (*q)[64], int lane, float (&x)[8])
{
    f32x4 sa = {0.f, 0.f, 0.f, 0.f}, sb = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) {
        const u32x4 qb = q[kk][lane];
        sa = E::mfma32(r.k[0][kk], qb, sa);
        sb = E::mfma32(r.k[1][kk], qb, sb);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = sa[i]; x[4 + i] = sb[i]; }
}

// The scores' weights, rounded to the element type: an operand of the product with V.  A score of -infinity (not seen, or so far off) weighs 0.
template <int D, class E, int NC>
__device__ __forceinline__ u32x4 tree_weights(TreeState<D, NC>& st, int c, const float (&x)[8], float scale_log2e)
{
    // A row's maximum moves only when a score of its own lies 2^6 above it, and only then do the lanes of a row look at each other's scores.  (The rows
    // beside it, which look too, keep theirs: what they do not see changes no bit of them.)
    const float mine = max8(x);
    if (__any(__builtin_fmaf(mine, scale_log2e, -st.m[c]) > kTreeSlack)) {
        float mx = mine * scale_log2e;
        mx = xor_max(mx, 16);
        mx = xor_max(mx, 32);
        const float m_new = mx - st.m[c] > kTreeSlack ? mx : st.m[c];
        const float alpha = exp2f(st.m[c] - m_new);              // 0 where nothing was seen before
        st.l[c] *= alpha;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st.o[c][dt] *= alpha;
        st.m[c] = m_new;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], scale_log2e, -st.m[c]));
    const u32x4 pb = { E::pack(p[0], p[1]), E::pack(p[2], p[3]), E::pack(p[4], p[5]), E::pack(p[6], p[7]) };
    st.l[c] = sum_weights<E>(p, pb, st.l[c]);
    return pb;
}

// Of the keys first .. first + 31 as nodes (negative: cached tokens), which a row of this mask sees; `left` of them are there.
__device__ __forceinline__ uint32_t seen_window(const uint64_t* words, int32_t first, int32_t left)
{
    uint64_t w;
    if (first >= 64 * kTreeWords) w = 0;
    else if (first <= -32) w = ~0ull;
    else if (first < 0) w = words[0] << -first | ((1ull << -first) - 1);
    else w = (first & 63) ? words[first >> 6] >> (first & 63) | words[(first >> 6) + 1] << (64 - (first & 63)) : words[first >> 6];
    if (left < 32) w &= left <= 0 ? 0ull : (1ull << left) - 1;
    return (uint32_t)w;
}

// One step of 32 keys that every row sees, T tiles: the scores of a tile are under way while the one before is weighed.
template <int D, class E, int NC, int T>
__device__ __forceinline__ void tree_step(TreeState<D, NC>& st, const TreeKv<D>& r, const u32x4 (*q)[D / 32][64], float scale_log2e, int lane)
{
    if constexpr (NC > 1) asm volatile("" ::: "memory");         // Q stays in LDS: the compiler would hold it in registers that there are not
    float x[2][8];
    tree_scores<D, E>(r, q[0], lane, x[0]);
#pragma unroll
    for (int c = 0; c < T; ++c) {
        if (c + 1 < T) tree_scores<D, E>(r, q[c + 1], lane, x[(c + 1) & 1]);
        const u32x4 pb = tree_weights<D, E, NC>(st, c, x[c & 1], scale_log2e);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st.o[c][dt] = E::mfma32(r.both(dt), pb, st.o[c][dt]);
    }
}

// One step some of whose keys are nodes or lie behind the last one: 32 keys from tok0 on.
template <int D, class E, int NC, class Lds>
__device__ __forceinline__ void tree_tail_step(TreeState<D, NC>& st, TreeKv<D>& r, Lds& lds, int32_t tiles, float scale_log2e,
                                               int32_t tok0, int32_t ctx, int32_t n_keys, int32_t G, int32_t tile0, int lane)
{
    const int32_t quad = (lane >> 4) * 4;
    bool odd = false;
    // slots behind the last token hold whatever was there
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int32_t valid = n_keys - (tok0 + 16 * h + quad);
        const uint32_t m0 = valid >= 2 ? 0xffffffffu : (valid == 1 ? 0x0000ffffu : 0u);
        const uint32_t m1 = valid >= 4 ? 0xffffffffu : (valid == 3 ? 0x0000ffffu : 0u);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
            r.v[h][dt][0] &= m0; r.v[h][dt][1] &= m1;
            odd |= not_finite<E>(r.v[h][dt][0]) | not_finite<E>(r.v[h][dt][1]);
        }
    }
    // A V that is infinite or no number belongs to the rows that see its key, and a product with a weight of zero would bring it to all: the
    // products are made of the finite values, and odd_values() gives the others to whom they belong.
    if (__any(odd)) {
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
            for (int h = 0; h < 2; ++h) r.v[h][dt] = u32x2{ finite_only<E>(r.v[h][dt][0]), finite_only<E>(r.v[h][dt][1]) };
        lds.odd = 1;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (c >= tiles) continue;
        asm volatile("" ::: "memory");
        float x[8];
        tree_scores<D, E>(r, lds.q[c], lane, x);
        const int32_t row = (tile0 + c) * 16 + (lane & 15), node = row / G - tile0 * 16 / G;
        const uint32_t w = seen_window(lds.mask[node], tok0 + quad - ctx, n_keys - (tok0 + quad));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = w >> i & 1u ? x[i] : -INFINITY;
            x[4 + i] = w >> (16 + i) & 1u ? x[4 + i] : -INFINITY;
        }
        const u32x4 pb = tree_weights<D, E, NC>(st, c, x, scale_log2e);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st.o[c][dt] = E::mfma32(r.both(dt), pb, st.o[c][dt]);
    }
}

// What the infinities and NaN in V of the keys first .. end - 1 add to features d .. d + 3 of a row: those of the keys that it sees.
template <int D, class E, int PS, class Lds>
__device__ __forceinline__ f32x4 odd_values(const Lds& lds, const uint16_t* __restrict__ layer_base, int64_t page_stride, int32_t num_pages,
                                                      const int32_t* __restrict__ table, int32_t max_blocks, int32_t Hkv, int32_t g, int32_t node, int32_t d,
                                                      int32_t first, int32_t end, int32_t ctx)
{
    f32x4 add = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int32_t key = first; key < end; ++key) {
        const int32_t j = key - ctx;
        if (j >= 0 && !(lds.mask[node][j >> 6] >> (j & 63) & 1u)) continue;
        const int32_t entry = key / PS, t = key - entry * PS, id = entry < max_blocks ? table[entry] : -1;
        if (id < 0 || id >= num_pages) continue;
        const uint16_t* v = layer_base + (int64_t)id * page_stride + (int64_t)(Hkv + g) * (PS * D);
        for (int i = 0; i < 4; ++i) {
            const uint32_t h = v[(((d + i) / 16 * (PS / 8) + t / 8) * 16 + (d + i) % 16) * 8 + t % 8], a = h & 0x7fffu;
            if (a > E::kInfinity) add[i] += __builtin_nanf("");
            else if (a == E::kInfinity) add[i] += h >> 15 ? -INFINITY : INFINITY;
        }
    }
    return add;
}

// Where the items of a cut block leave their partials: floats [item][kv head][16 NC rows][D], and (max, sum) of the rows.
struct TreePartials {
    float *o, *ml;
};

// One or two column tiles: the wavefronts share the keys, each with the next step's K and V on their way into registers while it multiplies one.  Read once and
// past the caches (4% faster than through them): 64 chains of 4-6 tokens on 512-4096, 32/8 heads, 100 us, 6.1 TB/s.
template <int D, class E, int PS, int NC>
__global__ __launch_bounds__(kDecodeThreads, (tree_waves(D, NC))) void tree_kernel(
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
    const TreeLane<D, PS> at(lane);
    // (a step behind the last one reads the last one's pages: its keys are masked, or it is never used; no branch, so that loads can be counted)
    auto id_at = [&](int32_t step) {
        const int32_t to = min(step, step_end - 1);
        StepIds<PS> id;
        if constexpr (PS == 16) {
            id.a = table[to];
        } else {
            id.a = table[2 * to];
            id.b = table[min(2 * to + 1, n_entries - 1)];
        }
        return loadable<PS>(id, num_pages);
    };
    const int32_t pairs = (key_end - key_begin + kTreeKeys - 1) / kTreeKeys, first = key_begin >> 4;
    int32_t pair = wave;
    TreeKv<D> r[2];
    auto get_k = [&](TreeKv<D>& to, int32_t step) {
        load_k<D, PS, 0>(to, layer_base, page_stride, id_at(first + 2 * step), g, at, lane);
        load_k<D, PS, 1>(to, layer_base, page_stride, id_at(first + 2 * step + 1), g, at, lane);
    };
    auto get_v = [&](TreeKv<D>& to, int32_t step) {
        load_v<D, PS, 0>(to, layer_base, page_stride, id_at(first + 2 * step), g, Hkv, at, lane);
        load_v<D, PS, 1>(to, layer_base, page_stride, id_at(first + 2 * step + 1), g, Hkv, at, lane);
    };
    get_k(r[0], pair);
    get_v(r[0], pair);

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
    if (threadIdx.x == 0) lds.odd = 0;
    TreeState<D, NC> st;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        st.m[c] = kLeastMax;
        st.l[c] = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st.o[c][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __syncthreads();

    const int32_t plain = max(0, min(pairs, (ctx - key_begin) / kTreeKeys));                // steps whose keys every row sees
    auto run = [&](auto t) {
        constexpr int T = decltype(t)::value;
        auto stage = [&](const TreeKv<D>& use, TreeKv<D>& fill) {                          // the next step is in flight while this one is multiplied
            get_k(fill, pair + kDecodeWaves);
            get_v(fill, pair + kDecodeWaves);
            tree_step<D, E, NC, T>(st, use, lds.q, scale_log2e, lane);
            pair += kDecodeWaves;
        };
        while (pair < plain) {
            stage(r[0], r[1]);
            if (pair >= plain) { r[0] = r[1]; break; }
            stage(r[1], r[0]);
        }
    };
    if (tiles == 1) run(std::integral_constant<int, 1>{});
    if constexpr (NC >= 2) if (tiles == 2) run(std::integral_constant<int, 2>{});
    for (; pair < pairs; pair += kDecodeWaves) {
        tree_tail_step<D, E, NC>(st, r[0], lds, tiles, scale_log2e, key_begin + pair * kTreeKeys, ctx, n_keys, G, tile0, lane);
        if (pair + kDecodeWaves < pairs) {
            get_k(r[0], pair + kDecodeWaves);
            get_v(r[0], pair + kDecodeWaves);
        }
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
            const int32_t i = u / (D / 4), d = (u - i * (D / 4)) * 4, row = (tile0 + c) * 16 + i;
            if (row >= rows) continue;
            float M = lds.m[0][c][i];
#pragma unroll
            for (int w = 1; w < kDecodeWaves; ++w) M = fmaxf(M, lds.m[w][c][i]);
            float L = 0.f;
            f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kDecodeWaves; ++w) {
                const float mw = lds.m[w][c][i], lw = lds.l[w][c][i];
                const float f = exp2f(mw - M);                   // (a wavefront that saw nothing has nothing to weigh)
                L += lw * f;
                O += *(const f32x4*)&lds.o[w][i][d] * f;
            }
            if (lds.odd) O += odd_values<D, E, PS>(lds, layer_base, page_stride, num_pages, table, max_blocks, Hkv, g, row / G - tile0 * 16 / G, d,
                                                   key_begin + plain * kTreeKeys, key_end, ctx);
            if (it.pieces == 1) {
                const int32_t node = row / G, head = row - node * G;
                u32x2 w = {0u, 0u};                              // a row that sees nothing: zeros
                if (L != 0.f) w = u32x2{ E::pack(O[0] / L, O[1] / L), E::pack(O[2] / L, O[3] / L) };
                *(u32x2*)(out + ((int64_t)(t0 + node) * Hq + g * G + head) * D + d) = w;
            } else {
                const int64_t at = ((int64_t)(items.base + item) * Hkv + g) * (16 * NC) + c * 16 + i;
                *(f32x4*)(part.o + at * D + d) = O;
                if (d == 0) { part.ml[at * 2] = M; part.ml[at * 2 + 1] = L; }
            }
        }
    }
}

// ------------------------------------------------------------------------------------
// More than two column tiles: the wavefronts share the rows instead of the keys.  A step's K and V are copied into an LDS ring by
// LDS-DMA, three steps ahead of the one that is multiplied, and every wavefront reads them from there for its one to three tiles; Q stays
// in registers.  (With the keys dealt to the wavefronts, as above, eight tiles' outputs leave registers for one step of K and V only,
// whose loads then wait for the step before: 32 trees of 8-32 nodes, 64/8 heads,
// on contexts of 2K-32K keys: 1173 us in that form, 536-549 in this one, whose copies and plan are the better for it too.)
//
// LDS arrangement of a step: K block of the first 16-key step, 64 bytes, K block of the second, the V blocks; each as in a page of
// 16 tokens.  Row r = 8 * step + 4 * half + i of score tile X (Y) is token 8 * half + i (+ 4) of its step, so that over X and Y a lane group
// owns 8 consecutive keys, one 16-byte unit of V.  (The 64 bytes put the two blocks' units of a read into different banks.)
// ------------------------------------------------------------------------------------
constexpr int kTreeRing = 4;
template <int D, int NC>
struct RingLds {
    static constexpr int kBlock = 16 * D * 2, kSlot = 4 * kBlock + 64;               // bytes
    alignas(16) char ring[kTreeRing][kSlot];
    uint64_t mask[16 * 4 * NC + 1][kTreeWords + 1];
};

template <int D, class E, int PS, int NC>
__global__ __launch_bounds__(kDecodeThreads, 2) void tree_ring_kernel(
    const uint16_t* __restrict__ layer_base, int64_t page_stride, int32_t num_pages, int32_t Hkv, int32_t G,
    const int32_t* __restrict__ block_tables, int32_t max_blocks, const int32_t* __restrict__ ctx_lens, const int32_t* __restrict__ cu_q_lens,
    const uint64_t* __restrict__ mask, int32_t mask_words, const uint16_t* __restrict__ q, uint16_t* __restrict__ out,
    float scale_log2e, TreePartials part, const int32_t n_spread, const TreeItems items)
{
    typedef RingLds<D, NC> Lds;
    __shared__ Lds lds;
    int32_t item = (int32_t)blockIdx.x / Hkv, g = (int32_t)blockIdx.x - item * Hkv;
    if (n_spread > 0) {                                          // (see tree_spread_items)
        const int32_t sets = 8 / Hkv, turn = (int32_t)(blockIdx.x >> 3), set = (int32_t)(blockIdx.x & 7) / Hkv;
        g = (int32_t)(blockIdx.x & 7) - set * Hkv;
        item = (turn / kTreeRun * sets + set) * kTreeRun + turn % kTreeRun;
        if (item >= n_spread) return;
    }
    const TreeItem it = tree_item(items.e[item]);
    const int32_t s = it.seq, t0 = cu_q_lens[s], q_len = cu_q_lens[s + 1] - t0, ctx = ctx_lens[s];
    const int32_t n_keys = ctx + q_len, rows = q_len * G;
    const TreeBlocks blocks = tree_blocks(rows);
    const int32_t tile0 = it.block * blocks.tiles, block_tiles = min(blocks.tiles, (rows + 15) / 16 - tile0);
    const int32_t chunk = tree_chunk_keys(n_keys, it.pieces);
    const int32_t key_begin = min(n_keys, it.piece * chunk), key_end = min(n_keys, key_begin + chunk);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t each = (block_tiles + kDecodeWaves - 1) / kDecodeWaves, tile = wave * each, tiles = max(0, min(each, block_tiles - tile));
    const int32_t Hq = Hkv * G;
    const int32_t* table = block_tables + (int64_t)s * max_blocks;
    const int32_t n_entries = min((n_keys + PS - 1) / PS, max_blocks);
    const int32_t step_end = min((n_keys + kPage - 1) >> 4, PS == 16 ? max_blocks : (n_entries + 1) >> 1);
    const int32_t steps = (key_end - key_begin + kTreeKeys - 1) / kTreeKeys, first = key_begin >> 4;

    // The wavefront's part of a step's copies: K (even wavefronts) or V of 16-key step wave / 2, a page or a pair of pages of 8.  A step
    // behind the sequence's last one reads that one again: its keys are masked.
    // Page offsets travel in lane registers, lane j's of 16-key step window + j (pages of 8: of its pair), and are read out with v_readlane: a
    // scalar load and the 64-bit product behind it, in front of every step's copies, held up the step by 600 cycles.
    constexpr int kCopies = Lds::kBlock / 1024;
    int32_t window = 0;                                          // 16-key step of lane 0, counted from the item's first
    uint32_t off_lo[PS == 16 ? 1 : 2], off_hi[PS == 16 ? 1 : 2];
    auto load_window = [&] {
        const int32_t to = min(first + window + lane, step_end - 1);
        StepIds<PS> id;
        if constexpr (PS == 16) {
            id.a = table[to];
        } else {
            id.a = table[2 * to];
            id.b = table[min(2 * to + 1, n_entries - 1)];
        }
        id = loadable<PS>(id, num_pages);
        const int64_t block = (int64_t)((wave & 1 ? Hkv : 0) + g) * (PS * D);
        auto put = [&](int k, int32_t page) {
            const uint64_t off = ((uint64_t)page * (uint64_t)page_stride + (uint64_t)block) * 2;
            off_lo[k] = (uint32_t)off;
            off_hi[k] = (uint32_t)(off >> 32);
        };
        put(0, id.a);
        if constexpr (PS == 8) put(1, id.b);
        // (the load is waited for here, not at every readlane)
        if constexpr (PS == 16) asm volatile("" : "+v"(off_lo[0]), "+v"(off_hi[0]));
        else asm volatile("" : "+v"(off_lo[0]), "+v"(off_hi[0]), "+v"(off_lo[1]), "+v"(off_hi[1]));
    };
    load_window();
    auto copy = [&](int32_t step) {
        if (2 * step - window >= 64) {                           // (steps only ever grow)
            window += 64;
            load_window();
        }
        const int32_t at = 2 * step - window + (wave >> 1);
        auto page_at = [&](int k) {
            const uint64_t off = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_hi[k], at) << 32 | (uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_lo[k], at);
            return (const char*)layer_base + off;
        };
        char* dst = lds.ring[(uint32_t)step % kTreeRing] + (wave & 1 ? 2 * Lds::kBlock + 64 + (wave >> 1) * Lds::kBlock : (wave >> 1) * (Lds::kBlock + 64));
        if constexpr (PS == 16) {
            const char* src = page_at(0);
#pragma unroll
            for (int i = 0; i < kCopies; ++i) lds_dma16_one_page(src + i * 1024, (uint32_t)lane * 16, dst + i * 1024);
        } else {
            // K: 8 units a feature block; V: 16 units a feature tile
            const uint32_t off = wave & 1 ? ((lane >> 5) * 16 + (lane & 15)) * 16 : ((lane >> 4) * 8 + (lane & 7)) * 16;
            const uint64_t src = (uint64_t)(uintptr_t)((wave & 1 ? lane & 16 : lane & 8) ? page_at(1) : page_at(0)) + off;
#pragma unroll
            for (int i = 0; i < kCopies; ++i) lds_dma16_lane_addr<0>(src + i * 512, dst + i * 1024);
        }
    };
#pragma unroll
    for (int i = 0; i < kTreeRing - 1; ++i)
        if (i < steps) copy(i);

    u32x4 qb[NC][D / 32];
    TreeState<D, NC> st;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int32_t row = (tile0 + tile + c) * 16 + (lane & 15), node = row / G, head = row - node * G;
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) {
            qb[c][kk] = u32x4{0u, 0u, 0u, 0u};
            if (c < tiles && row < rows) qb[c][kk] = *(const u32x4*)(q + ((int64_t)(t0 + node) * Hq + g * G + head) * D + kk * 32 + (lane >> 4) * 8);
        }
        st.m[c] = kLeastMax;
        st.l[c] = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st.o[c][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (key_end > ctx) {
        const int32_t node0 = tile0 * 16 / G, nodes = min((tile0 + block_tiles) * 16 / G, q_len - 1) - node0 + 1;
        for (int32_t u = threadIdx.x; u < (64 * NC + 1) * (kTreeWords + 1); u += kDecodeThreads) {
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

    // The step's copies have landed, the wavefront's by its own count and the others' by the barrier, behind which nobody reads the step
    // before any more: its slot takes the copies of three steps on.
    auto begin = [&](int32_t i) {
        const int32_t left = min(steps - 1 - i, kTreeRing - 2);  // steps behind this one whose copies are under way
        if (left >= 2) wait_vmcnt<2 * kCopies>();
        else if (left == 1) wait_vmcnt<kCopies>();
        else wait_vmcnt<0>();
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
    };
    auto ahead = [&](int32_t i) {
        if (i + kTreeRing - 1 < steps) copy(i + kTreeRing - 1);
    };
    const uint32_t k_at = (lane & 15) / 8 * (Lds::kBlock + 64) + ((lane >> 4) * 16 + ((lane >> 2) & 1) * 8 + (lane & 3)) * 16;
    const uint32_t v_at = 2 * Lds::kBlock + 64 + (lane >> 5) * Lds::kBlock + (((lane >> 4) & 1) * 16 + (lane & 15)) * 16;
    auto scores = [&](const char* slot, int c, float (&x)[8]) {
        f32x4 sx = {0.f, 0.f, 0.f, 0.f}, sy = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) {
            sx = E::mfma32(*(const u32x4*)(slot + k_at + kk * 1024), qb[c][kk], sx);
            sy = E::mfma32(*(const u32x4*)(slot + k_at + kk * 1024 + 64), qb[c][kk], sy);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[j] = sx[j]; x[4 + j] = sy[j]; }
    };
    bool odd = false;
    const int32_t plain = max(0, min(steps, (ctx - key_begin) / kTreeKeys));
    int32_t i = 0;
    auto run = [&](auto t) {
        constexpr int T = decltype(t)::value;
        for (; i < plain; ++i) {
            begin(i);
            const char* slot = lds.ring[(uint32_t)i % kTreeRing];
            float x[T > 0 ? T : 1][8];
            u32x4 pb[T > 0 ? T : 1];
#pragma unroll
            for (int c = 0; c < T; ++c) scores(slot, c, x[c]);
            ahead(i);                                            // (behind the first reads of this step)
#pragma unroll
            for (int c = 0; c < T; ++c) pb[c] = tree_weights<D, E, NC>(st, c, x[c], scale_log2e);
            if constexpr (T > 0) {
#pragma unroll
                for (int dt = 0; dt < D / 16; ++dt) {
                    const u32x4 v = *(const u32x4*)(slot + v_at + dt * 512);
#pragma unroll
                    for (int c = 0; c < T; ++c) st.o[c][dt] = E::mfma32(v, pb[c], st.o[c][dt]);
                }
            }
        }
    };
    if (tiles == 0) run(std::integral_constant<int, 0>{});
    if (tiles == 1) run(std::integral_constant<int, 1>{});
    if constexpr (NC >= 2) if (tiles == 2) run(std::integral_constant<int, 2>{});
    if constexpr (NC >= 3) if (tiles == 3) run(std::integral_constant<int, 3>{});
    for (; i < steps; ++i) {
        begin(i);
        ahead(i);
        const char* slot = lds.ring[(uint32_t)i % kTreeRing];
        const int32_t key0 = key_begin + i * kTreeKeys + (lane >> 4) * 8, valid = n_keys - key0;     // the lane's 8 keys
        u32x4 pb[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            pb[c] = u32x4{0u, 0u, 0u, 0u};
            if (c >= tiles) continue;
            float x[8];
            scores(slot, c, x);
            const int32_t row = (tile0 + tile + c) * 16 + (lane & 15), node = row / G - tile0 * 16 / G;
            const uint32_t w = seen_window(lds.mask[node], key0 - ctx, valid);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = w >> j & 1u ? x[j] : -INFINITY;
            pb[c] = tree_weights<D, E, NC>(st, c, x, scale_log2e);
        }
        // slots behind the last token hold whatever was there; infinities and NaN: see tree_tail_step
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
            u32x4 v = *(const u32x4*)(slot + v_at + dt * 512);
            bool here = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] &= valid >= 2 * j + 2 ? 0xffffffffu : (valid == 2 * j + 1 ? 0x0000ffffu : 0u);
                here |= not_finite<E>(v[j]);
            }
            if (__any(here)) {
                odd = true;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = finite_only<E>(v[j]);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (c < tiles) st.o[c][dt] = E::mfma32(v, pb[c], st.o[c][dt]);
        }
    }

#pragma unroll
    for (int c = 0; c < NC; ++c) {
        if (c >= tiles) continue;
        float L = st.l[c];
        L += __shfl_xor(L, 16, 64);
        L += __shfl_xor(L, 32, 64);
        const int32_t row = (tile0 + tile + c) * 16 + (lane & 15), node = row / G, head = row - node * G;
        if (row >= rows) continue;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
            const int32_t d = dt * 16 + (lane >> 4) * 4;
            f32x4 O = st.o[c][dt];
            if (odd) O += odd_values<D, E, PS>(lds, layer_base, page_stride, num_pages, table, max_blocks, Hkv, g, node - tile0 * 16 / G, d, key_begin + plain * kTreeKeys, key_end, ctx);
            if (it.pieces == 1) {
                u32x2 w = {0u, 0u};                              // a row that sees nothing: zeros
                if (L != 0.f) w = u32x2{ E::pack(O[0] / L, O[1] / L), E::pack(O[2] / L, O[3] / L) };
                *(u32x2*)(out + ((int64_t)(t0 + node) * Hq + g * G + head) * D + d) = w;
            } else {
                const int64_t at = ((int64_t)(items.base + item) * Hkv + g) * (64 * NC) + (tile + c) * 16 + (lane & 15);
                *(f32x4*)(part.o + at * D + d) = O;
                if (d == 0) { part.ml[at * 2] = st.m[c]; part.ml[at * 2 + 1] = L; }
            }
        }
    }
}

// Joins the pieces of cut blocks: a workgroup for each column tile (grid.y) of each cut block and kv head, a thread for 4 features of a row.
template <int D, class E>
__global__ __launch_bounds__(4 * D) void tree_merge_kernel(
    int32_t Hkv, int32_t G, int32_t part_rows, const int32_t* __restrict__ cu_q_lens, uint16_t* __restrict__ out, TreePartials part, const TreeMerges merges)
{
    const int32_t merge = (int32_t)blockIdx.x / Hkv, g = (int32_t)blockIdx.x - merge * Hkv, c = blockIdx.y;
    const TreeItem it = tree_item(merges.e[merge].word);
    const int32_t t0 = cu_q_lens[it.seq], rows = (cu_q_lens[it.seq + 1] - t0) * G, Hq = Hkv * G;
    const TreeBlocks blocks = tree_blocks(rows);
    if (c >= blocks.tiles) return;
    const int32_t r = (int32_t)threadIdx.x / (D / 4), d = ((int32_t)threadIdx.x - r * (D / 4)) * 4, row = (it.block * blocks.tiles + c) * 16 + r;
    if (row >= rows) return;
    float M = kLeastMax, L = 0.f;
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
    const int64_t at = ((int64_t)merges.e[merge].item * Hkv + g) * part_rows + c * 16 + r, next = (int64_t)blocks.blocks * Hkv * part_rows;
    // eight pieces' loads in flight at once; with more of them the maxima are read twice
    for (int32_t i0 = 0; it.pieces > 8 && i0 < it.pieces; i0 += 8) {
        float m[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = part.ml[(at + min(i0 + i, it.pieces - 1) * next) * 2];
#pragma unroll
        for (int i = 0; i < 8; ++i) M = fmaxf(M, m[i]);
    }
    for (int32_t i0 = 0; i0 < it.pieces; i0 += 8) {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        f32x2 ml[8];
        f32x4 o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {                        // (past the last piece: the last again)
            const int64_t p = at + min(i0 + i, it.pieces - 1) * next;
            ml[i] = *(const f32x2*)(part.ml + p * 2);
            o[i] = *(const f32x4*)(part.o + p * D + d);
        }
        if (it.pieces <= 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) M = fmaxf(M, ml[i][0]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i0 + i >= it.pieces) continue;
            const float f = exp2f(ml[i][0] - M);
            L += ml[i][1] * f;
            O += o[i] * f;
        }
    }
    const int32_t node = row / G, head = row - node * G;
    u32x2 w = {0u, 0u};
    if (L != 0.f) w = u32x2{ E::pack(O[0] / L, O[1] / L), E::pack(O[2] / L, O[3] / L) };
    *(u32x2*)(out + ((int64_t)(t0 + node) * Hq + g * G + head) * D + d) = w;
}

}  // namespace cs
