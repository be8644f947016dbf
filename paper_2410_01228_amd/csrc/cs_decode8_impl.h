// Decode path over a pool of 8-bit codes (see cs_decode_impl.h for the scheme, which is the same: a workgroup per
// (sequence, kv head, key range), pages straight from HBM into registers, online softmax in fp32).
//
// A code is half as long, so a step is two pages (32 keys) where the 16-bit path takes one: a wavefront has as many
// bytes in flight, and its running maximum and sum are touched half as often a key.  Codes are widened to the
// 16-bit type of Q in registers, with their block's scale (exactly: it is a power of two), and then
//   S^T[token][head] = K[token][:] . Q[head][:]            v_mfma_f32_16x16x32, D/32 for each page
//   O^T[d][head]    += V^T[d][32 tokens] . P^T[32 tokens][head]   v_mfma_f32_16x16x32, D/16
// The page format is made for it.  A 16-byte unit of K is 16 features of a token: the A operands of two products, over
// features (4u + lane/16)*16 + 0..7 and + 8..15, so Q is loaded in that order too.  A unit of V is 4 tokens of a feature in 4
// feature tiles: with the unit of the other page it holds the A operands of 4 products, tokens 4*(lane/16) .. +4 of either
// page -- the tokens whose weights the lane has, in the order that the C layout of S^T leaves them in.
#pragma once
#include "cs_decode_impl.h"

namespace cs {

constexpr int kStep8 = 2 * kPage;                     // keys per step

template <int D>
struct StepRegs8 {
    u32x4 k[2][D / 64];  // K units u*64 + lane of the two pages
    u32x4 v[2][D / 64];  // V units u*64 + lane
    float scale;         // lane & 3: K of the first page, K of the second, V of the first, V of the second
};

// The pages of step `step` of an item that begins at page page_begin: the second repeats the first where the item ends
// inside the step (what it brings is masked); invalid outside the item.
__device__ __forceinline__ StepIds<8> step_ids8(const int32_t* __restrict__ table, int32_t page, int32_t page_end) {
    StepIds<8> ids;
    ids.a = page < page_end ? table[page] : -1;
    ids.b = page + 1 < page_end ? table[page + 1] : ids.a;
    return ids;
}

// page_bytes: from a page to the next one.
template <int D>
__device__ __forceinline__ void load_step8(StepRegs8<D>& r, const char* __restrict__ layer_base, int64_t page_bytes, StepIds<8> ids,
                                           int32_t g, int32_t Hkv, int lane)
{
    const int32_t id[2] = {ids.a, ids.b};
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const char* kblk = layer_base + (int64_t)id[p] * page_bytes + g * (kPage * D);
        const char* vblk = kblk + Hkv * (kPage * D);
#pragma unroll
        for (int u = 0; u < D / 64; ++u) r.k[p][u] = __builtin_nontemporal_load((const u32x4*)kblk + u * 64 + lane);
#pragma unroll
        for (int u = 0; u < D / 64; ++u) r.v[p][u] = __builtin_nontemporal_load((const u32x4*)vblk + u * 64 + lane);
    }
    // (a vector load like the others: scalar loads return in any order, and a wait for this step's scales would be one for the
    // next step's too)
    const char* page = layer_base + (int64_t)((lane & 1) ? ids.b : ids.a) * page_bytes;
    r.scale = *(const float*)(page + 2 * Hkv * (kPage * D) + (((lane & 2) ? Hkv : 0) + g) * 4);
}

template <int D, class E>
__device__ __forceinline__ void process_step8(WaveState<D>& st, const StepRegs8<D>& r, const u32x4* qb,
                                              float scale_log2e, int32_t tok0, int32_t n_keys, int lane)
{
    float scale[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) scale[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, r.scale), i));
    float x[8];
    const int32_t row0 = tok0 + (lane >> 4) * 4;      // first of this lane's 4 tokens of the first page
    const bool tail = tok0 + kStep8 > n_keys;          // wave-uniform
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < D / 64; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t w0 = r.k[p][u][2 * h], w1 = r.k[p][u][2 * h + 1];
                const u32x4 a = {E::template widen<false>(w0, scale[p]), E::template widen<true>(w0, scale[p]),
                                 E::template widen<false>(w1, scale[p]), E::template widen<true>(w1, scale[p])};
                s = E::mfma32(a, qb[2 * u + h], s);
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[4 * p + i] = s[i] * scale_log2e;
            if (tail && row0 + 16 * p + i >= n_keys) x[4 * p + i] = -INFINITY;
        }
    }
    float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    mx = xor_max(mx, 16);
    mx = xor_max(mx, 32);
    const float m_new = fmaxf(st.m, mx);               // finite: token tok0 is always valid
    if (__any(m_new > st.m)) {
        const float alpha = exp2f(st.m - m_new);       // 0 on the first step (m = -inf)
        st.l *= alpha;
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) st.o[dt] *= alpha;
        st.m = m_new;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = exp2f(x[i] - st.m);
    const u32x4 pb = { E::pack(p[0], p[1]), E::pack(p[2], p[3]), E::pack(p[4], p[5]), E::pack(p[6], p[7]) };
    // the sum uses the same rounded weights that multiply V
    st.l += (E::sum2(pb[0]) + E::sum2(pb[1])) + (E::sum2(pb[2]) + E::sum2(pb[3]));
    // slots past the sequence end hold stale codes (possibly NaN): zero them so 0 * x stays 0
    uint32_t mask[2] = {0xffffffffu, 0xffffffffu};
    if (tail) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int32_t valid = n_keys - (row0 + 16 * h);    // tokens of this lane's group that exist
            mask[h] = valid >= 4 ? 0xffffffffu : valid <= 0 ? 0u : (1u << (8 * valid)) - 1;
        }
    }
#pragma unroll
    for (int u = 0; u < D / 64; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t w0 = r.v[0][u][e], w1 = r.v[1][u][e];
            if (tail) { w0 &= mask[0]; w1 &= mask[1]; }
            const u32x4 a = {E::template widen<false>(w0, scale[2]), E::template widen<true>(w0, scale[2]),
                             E::template widen<false>(w1, scale[3]), E::template widen<true>(w1, scale[3])};
            st.o[u * 4 + e] = E::mfma32(a, pb, st.o[u * 4 + e]);
        }
}

// The (item, kv head) of pair w of a grid: eight items at a time, their heads in turn, so that the heads of an item go to one XCD
// (workgroups are dealt round-robin to the 8 of them; fewer than eight items that are left over: head by head).  A page's scales are one
// cache line for all heads: with the heads of a page spread over the XCDs each L2 fetches it, 64 bytes of use to a head's 4 KiB (256
// decodes of 512-4096 keys, 32/8 heads, 199.6 -> 186.7 us, 6.71 TB/s; 64 of 4096, 96.0 -> 81.0; 32 of 300-3000, 30.3 -> 22.2; 300 of 50-500,
// 64/8, 38.2 -> 33.5; 64 of 1000-8000, 28/4, 58.7 -> 56.9).
__device__ __forceinline__ void pair_of8(int32_t w, int32_t Hkv, int32_t n_items, int32_t& item, int32_t& g) {
    item = w / Hkv;
    g = w - item * Hkv;
    const int32_t first = item & ~7;
    if (first + 8 <= n_items) {
        const int32_t r = w - first * Hkv;
        item = first + (r & 7);
        g = r >> 3;
    }
}

// decode_item for 8-bit pools: page_stride in units of 2 bytes.
//
// One form for every launch: a step ahead, with loads that the compiler can count (Loads::kLone there).  A workgroup
// takes half as long as over 16-bit pages, so more of a launch is the time of its last ones, alone on their CUs, and full chips
// do not mind.  This, skipped loads, two steps ahead, us: 256 decodes of 512-4096 keys, 32/8 heads, 187.6, 189.4, 192.2; of 1000-8000,
// 4/2 heads, 57.9, 58.7, 63.7; 300 of 50-500, 64/8, 33.7, 37.0, 43.4; 1 of 20000, 64/8, 20.1, 22.4, 21.4; 128 of 2K-32K beside a chunk of
// 1024 on 30720, 64/8, 1492, 1621, 1508.  (Four workgroups a CU would have 128 registers each, and spill.)
template <int D, class Src, class E>
__device__ __forceinline__ void decode_item8(
    DecodeLds<D>& lds,
    const uint16_t* __restrict__ layer_base, int64_t page_stride, int32_t num_pages,
    int32_t Hkv, int32_t G,
    const int32_t* __restrict__ block_tables, int32_t max_blocks,
    const Src& src,
    const int32_t* __restrict__ ctx_lens, const int32_t* __restrict__ cu_q_lens,
    const uint16_t* __restrict__ q, uint16_t* __restrict__ out,
    float scale_log2e, const DecodePartials& part,
    int32_t item, int32_t g)
{
    DecodeItem it;
    if (!fetch_item(src, item, ctx_lens, cu_q_lens, it)) return;
    const int32_t s = it.seq, t = it.token, n_keys = it.n_keys;
    const int32_t page_begin = it.key_begin >> 4;
    // an item can come out empty when a short sequence is cut very finely
    const int32_t page_end = it.key_end > it.key_begin ? min((it.key_end + kPage - 1) >> 4, max_blocks) : page_begin;
    // keys the item may see: its last step may reach into the next piece's pages
    const int32_t end_key = min(n_keys, page_end * kPage);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t* table = block_tables + (int64_t)s * max_blocks;
    const int32_t Hq = Hkv * G;

    // Q as the B operand, in the order of K's features (above); heads >= G are zero rows.
    u32x4 qb[D / 32];
    {
        const int head = lane & 15;
        const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            u32x4 v = zero;
            if (head < G)
                v = *(const u32x4*)(q + ((int64_t)t * Hq + g * G + head) * D + ((j >> 1) * 4 + (lane >> 4)) * 16 + (j & 1) * 8);
            qb[j] = v;
        }
    }

    WaveState<D> st;
    st.m = -INFINITY;
    st.l = 0.f;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) st.o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};

    const char* base = (const char*)layer_base;
    const int64_t page_bytes = page_stride * 2;
    auto id_at = [&](int32_t p) { return step_ids8(table, p, page_end); };
    auto fetch = [&](StepRegs8<D>& r, const StepIds<8>& id) { load_step8<D>(r, base, page_bytes, loadable<8>(id, num_pages), g, Hkv, lane); };
    auto use = [&](const StepRegs8<D>& r, const StepIds<8>& id, int32_t pg) {
        if (step_ok<8>(id, num_pages)) process_step8<D, E>(st, r, qb, scale_log2e, pg << 4, end_key, lane);
    };
    constexpr int kStride = 2 * kDecodeWaves;                              // pages from a wavefront's step to its next
    int32_t pg = page_begin + 2 * wave;                                    // wave w takes the steps w, w + 4, ...
    StepRegs8<D> cur, nxt;
    StepIds<8> id_cur = id_at(pg), id_nxt = id_at(pg + kStride);
    if (pg < page_end) fetch(cur, id_cur);
    while (pg + kStride < page_end) {
        const StepIds<8> id_n2 = id_at(pg + 2 * kStride);
        fetch(nxt, id_nxt);
        use(cur, id_cur, pg);
        cur = nxt;
        id_cur = id_nxt;
        id_nxt = id_n2;
        pg += kStride;
    }
    if (pg < page_end) use(cur, id_cur, pg);                               // the wavefront's last step: nothing is loaded behind it
    leave_item<D, E>(lds, st, it, t, item, g, Hq, G, out, part, lane, wave);
}

}  // namespace cs
