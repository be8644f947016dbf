// Queries and keys on their way from the projection to the attention call: RMS norm of each head (optional), rotation by the
// token's position, and the append of K and V to the pages in the same pass.
//
//   y = x * w / sqrt(mean x^2 + eps)          (with a norm; y = x without)
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t = position * inv_freq[pair]
//
// fp32 from the 16-bit input on, rounded once at the end.  Positions reach 2^31, where a product in fp32 would be off by whole
// turns: the turns are counted in fp64 (an error of 2^31 / 2 pi * 2^-52, 1e-7 of a turn at most), and what is left of
// one, at most half, goes on in fp32.
//
// HBM-bound: each value is read and written once.  A thread has 8 features of a row, as two pieces of 4 (the two halves of four pairs).
// Where rows are written (Q, and K without a cache) a wavefront takes eight heads (16 of head dim 64) of one token, 2 KiB that lie
// side by side, so that its angles serve two rows of a lane, all of it is one trip to memory, and
// a launch has wavefronts enough to keep the memory busy (workgroups that walked 16 tokens' heads with the angles computed once ran at
// half the rate: 12K tokens appended, 32/8 heads, 96 us where this takes 65, at 4.7 TB/s).  Where K and V go to a page a workgroup takes its 16 tokens and a few heads.
#include <algorithm>
#include "cs_common.h"
#include "cs_elem.h"

namespace cs {

typedef uint32_t r_u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t r_u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 16;                                  // of a workgroup that fills a page
constexpr int kRopeRows = 2;                                     // rows of a thread

// What the kernel is told.  Strides in elements.
struct RopeArgs {
    const uint16_t *q, *k, *v, *q_norm, *k_norm;
    uint16_t *q_out, *k_out;                                     // k_out: rows, where nothing is appended
    int64_t q_stride, k_stride, v_stride;
    const float* inv_freq;
    const int32_t* positions;
    int64_t position_stride;
    float eps;
    int32_t rotary_dim, interleaved, num_axes, pairs0, pairs1;   // pairs0, pairs1: pairs of the first axis, of the first two
    int32_t T, Hq, Hkv;
    int32_t q_units, kv_units, kv_tokens;                        // wavefronts of a token: with heads of Q; with heads of K, of the tokens in front of kv_tokens
    // the append
    uint16_t* layer_base;
    int64_t page_stride;
    int32_t num_pages, page_size, S, max_blocks;
    const int32_t *block_tables, *ctx_lens, *cu_q_lens;
    int32_t slot_blocks, slot_groups;                            // workgroups of sequences with more than one new token: slots, parts of their heads
};

// Sum over the 16 (8) lanes that share a row, in each of them.
template <int kLanes>
__device__ __forceinline__ float row_sum(float v) {
    auto other = [](float x, auto ctrl) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true)); };
    v += other(v, std::integral_constant<int, 0xB1>{});          // lane ^ 1
    v += other(v, std::integral_constant<int, 0x4E>{});          // lane ^ 2
    v += other(v, std::integral_constant<int, 0x141>{});         // the other four of eight
    if (kLanes == 16) v += other(v, std::integral_constant<int, 0x140>{});   // the other eight of sixteen
    return v;
}

struct __attribute__((packed, aligned(4))) Freqs { float v[4]; };  // (inv_freq is aligned to 4 bytes)

// A thread's features of a row, and the angles of its token.
struct Turn {
    int32_t off0, off1;                                          // its two pieces of four features
    bool rotates, neighbours;                                    // pairs are (piece 0, piece 1), or neighbours inside a piece
    // The pieces of all threads lie side by side: rows are read and written 16 bytes a thread (12K tokens of 32/8 heads, rotated in pairs of neighbours, 50.5 us
    // with 8 bytes, 48 with 16; not rotated 51 and 46.  Heads rotated whole, 16 bytes a thread and the halves changing places between lanes: 49 with
    // either, and the append 67 us with 8, 71 with 16).
    bool wide;
    float c[4], s[4];
};

__device__ __forceinline__ void turn_places(Turn& r, const RopeArgs& a, int32_t j)
{
    r.rotates = 8 * j < a.rotary_dim;
    r.neighbours = a.interleaved != 0 || !r.rotates;
    r.wide = a.interleaved != 0 || a.rotary_dim == 0;
    r.off0 = r.neighbours ? 8 * j : 4 * j;
    r.off1 = r.neighbours ? 8 * j + 4 : a.rotary_dim / 2 + 4 * j;
}

__device__ __forceinline__ void turn_angles(Turn& r, const RopeArgs& a, int32_t j, int32_t t, int32_t position)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.c[i] = 1.f; r.s[i] = 0.f; }
    if (!r.rotates) return;
    // (a load of four frequencies and one of each axis's position; where the token is the wavefront's, those are scalar loads)
    int32_t axis[3] = {position, position, position};
    if (a.positions) {
        axis[0] = axis[1] = axis[2] = a.positions[t];
        if (a.num_axes > 1) axis[1] = axis[2] = a.positions[a.position_stride + t];
        if (a.num_axes > 2) axis[2] = a.positions[2 * a.position_stride + t];
    }
    const Freqs freq = *(const Freqs*)(a.inv_freq + 4 * j);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int32_t pair = 4 * j + i, at = pair < a.pairs0 ? axis[0] : pair < a.pairs1 ? axis[1] : axis[2];
        const double turns = (double)at * (double)freq.v[i] * 0.15915494309189535;   // 1 / 2 pi
        const float part = (float)(turns - rint(turns));
        r.s[i] = __builtin_amdgcn_sinf(part);                    // of a turn: off by 2^-22.9 at most over half a turn (measured at 2^22 points)
        r.c[i] = __builtin_amdgcn_cosf(part);
    }
}

// One row's 8 features: normed, rotated, rounded.  (Every fused multiply-add is spelled out: all kernels round alike.)
template <int D, class E>
__device__ __forceinline__ void turn_row(const Turn& r, bool normed, const r_u32x2* w, float eps, r_u32x2& x0, r_u32x2& x1)
{
    if (!normed && !r.rotates) return;                           // bits as they are
    float a[4], b[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        E::unpack(x0[i], a[2 * i], a[2 * i + 1]);
        E::unpack(x1[i], b[2 * i], b[2 * i + 1]);
    }
    if (normed) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = __builtin_fmaf(b[i], b[i], __builtin_fmaf(a[i], a[i], sum));
        const float f = rsqrtf(__builtin_fmaf(row_sum<D / 8>(sum), 1.f / D, eps));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float w0, w1;
            E::unpack(w[0][i], w0, w1);
            a[2 * i] *= f * w0; a[2 * i + 1] *= f * w1;
            E::unpack(w[1][i], w0, w1);
            b[2 * i] *= f * w0; b[2 * i + 1] *= f * w1;
        }
    }
    if (r.rotates) {
        if (r.neighbours) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float& lo = i < 2 ? a[2 * i] : b[2 * i - 4];
                float& hi = i < 2 ? a[2 * i + 1] : b[2 * i - 3];
                const float x = lo, y = hi;
                lo = __builtin_fmaf(x, r.c[i], -(y * r.s[i]));
                hi = __builtin_fmaf(y, r.c[i], x * r.s[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = a[i], y = b[i];
                a[i] = __builtin_fmaf(x, r.c[i], -(y * r.s[i]));
                b[i] = __builtin_fmaf(y, r.c[i], x * r.s[i]);
            }
        }
    }
    x0 = r_u32x2{ E::pack(a[0], a[1]), E::pack(a[2], a[3]) };
    x1 = r_u32x2{ E::pack(b[0], b[1]), E::pack(b[2], b[3]) };
}

// A thread's part of a norm's weights.
struct Weights {
    r_u32x2 w[2];
    bool there;
    __device__ __forceinline__ Weights(const Turn& r, const uint16_t* __restrict__ norm) : there(norm != nullptr) {
        w[0] = w[1] = r_u32x2{0u, 0u};
        if (norm) {
            w[0] = *(const r_u32x2*)(norm + r.off0);
            w[1] = *(const r_u32x2*)(norm + r.off1);
        }
    }
};

// kRopeRows rows of a thread, heads h, h + step, .. below end.
template <int D>
struct Rows {
    r_u32x2 x[kRopeRows][2];
    __device__ __forceinline__ Rows(const Turn& r, const uint16_t* __restrict__ src, int32_t h, int32_t step, int32_t end, bool there) {
#pragma unroll
        for (int i = 0; i < kRopeRows; ++i) {
            x[i][0] = x[i][1] = r_u32x2{0u, 0u};
            if (!there || h + i * step >= end) continue;
            const uint16_t* row = src + (h + i * step) * D;
            if (r.wide) {
                const r_u32x4 v = *(const r_u32x4*)(row + r.off0);
                x[i][0] = r_u32x2{v[0], v[1]};
                x[i][1] = r_u32x2{v[2], v[3]};
            } else {
                x[i][0] = *(const r_u32x2*)(row + r.off0);
                x[i][1] = *(const r_u32x2*)(row + r.off1);
            }
        }
    }
    template <class E, class Put>
    __device__ __forceinline__ void finish(const Turn& r, const Weights& w, float eps, int32_t h, int32_t step, int32_t end, bool there, Put put) {
#pragma unroll
        for (int i = 0; i < kRopeRows; ++i) {
            turn_row<D, E>(r, w.there, w.w, eps, x[i][0], x[i][1]);
            if (there && h + i * step < end) put(h + i * step, x[i][0], x[i][1]);
        }
    }
};

// The sequence of token t.  In an online-first batch it is usually sequence t: that is tried before bisecting the prefix sums.
__device__ __forceinline__ int32_t sequence_of(const RopeArgs& a, int32_t t) {
    const int32_t s = min(t, a.S - 1);
    if (a.cu_q_lens[s] <= t && t < a.cu_q_lens[s + 1]) return s;
    int32_t lo = 0, hi = a.S;                                    // cu[lo] <= t < cu[hi]
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (a.cu_q_lens[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
}

// One wavefront: heads of one token, from rows to rows; with a cache, K and V of a sequence's single token to its page.
template <int D, class E, bool kAppend>
__device__ __forceinline__ void rope_unit(const RopeArgs& a, int32_t unit)
{
    constexpr int kLanes = D / 8, kAtOnce = 64 / kLanes, kUnitHeads = kRopeRows * kAtOnce;
    const bool is_q = unit < a.T * a.q_units;
    const int32_t at = is_q ? unit : unit - a.T * a.q_units, each = is_q ? a.q_units : a.kv_units;
    const int32_t t = at / each, c = at - t * each;
    if (t >= (is_q ? a.T : a.kv_tokens)) return;
    const int32_t lane = threadIdx.x & 63, j = lane % kLanes;
    Turn r;
    turn_places(r, a, j);
    const int32_t H = is_q ? a.Hq : a.Hkv, h = c * kUnitHeads + lane / kLanes;
    Rows<D> rows(r, is_q ? a.q + t * a.q_stride : a.k + t * a.k_stride, h, kAtOnce, H, true);
    const Weights w(r, is_q ? a.q_norm : a.k_norm);
    int32_t position = 0, seq = 0;
    if (kAppend && (!a.positions || !is_q)) {
        seq = sequence_of(a, t);
        const int32_t first = a.cu_q_lens[seq];
        position = a.ctx_lens[seq] + (t - first);
        if (!is_q && a.cu_q_lens[seq + 1] - first != 1) return;  // more tokens than one: the workgroups that fill pages
    }
    if (is_q || !kAppend) {
        turn_angles(r, a, j, t, position);
        uint16_t* dst = (is_q ? a.q_out : a.k_out) + (int64_t)t * H * D;
        rows.template finish<E>(r, w, a.eps, h, kAtOnce, H, true, [&](int32_t head, r_u32x2 x0, r_u32x2 x1) {
            if (r.wide) {
                __builtin_nontemporal_store(r_u32x4{x0[0], x0[1], x1[0], x1[1]}, (r_u32x4*)(dst + head * D + r.off0));
                return;
            }
            __builtin_nontemporal_store(x0, (r_u32x2*)(dst + head * D + r.off0));
            __builtin_nontemporal_store(x1, (r_u32x2*)(dst + head * D + r.off1));
        });
        return;
    }
    r_u32x4 v[kRopeRows];
#pragma unroll
    for (int i = 0; i < kRopeRows; ++i) {
        v[i] = r_u32x4{0u, 0u, 0u, 0u};
        if (h + i * kAtOnce < H) v[i] = *(const r_u32x4*)(a.v + t * a.v_stride + (h + i * kAtOnce) * D + 8 * j);
    }
    const int32_t entry = position / a.page_size, slot = position - entry * a.page_size;
    const int32_t id = entry < a.max_blocks ? a.block_tables[(int64_t)seq * a.max_blocks + entry] : -1;
    turn_angles(r, a, j, t, position);
    if (id < 0 || id >= a.num_pages) return;
    uint16_t* page = a.layer_base + (int64_t)id * a.page_stride;
    const int32_t block_elems = a.page_size * D;
    rows.template finish<E>(r, w, a.eps, h, kAtOnce, H, true, [&](int32_t head, r_u32x2 x0, r_u32x2 x1) {
        // unit f / 8 of token `slot`, the half of it that the piece is
        uint16_t* blk = page + (int64_t)head * block_elems + slot * 8;
        if (r.wide) {
            *(r_u32x4*)(blk + j * a.page_size * 8) = r_u32x4{x0[0], x0[1], x1[0], x1[1]};
            return;
        }
        *(r_u32x2*)(blk + (r.off0 >> 3) * a.page_size * 8 + (r.off0 & 7)) = x0;
        *(r_u32x2*)(blk + (r.off1 >> 3) * a.page_size * 8 + (r.off1 & 7)) = x1;
    });
    // V as it is.  feature d of token t: (((d/16) * groups of 8 + t/8) * 16 + d%16) * 8 + t%8
#pragma unroll
    for (int i = 0; i < kRopeRows; ++i) {
        const int32_t head = h + i * kAtOnce;
        if (head >= H) break;
        uint16_t* dst = page + (int64_t)(a.Hkv + head) * block_elems + (((j >> 1) * (a.page_size >> 3) + (slot >> 3)) * 16 + (j & 1) * 8) * 8 + (slot & 7);
#pragma unroll
        for (int e = 0; e < 8; ++e) dst[e * 8] = (uint16_t)(v[i][e >> 1] >> (e & 1) * 16);
    }
}

// LDS of a workgroup that fills a page: rows of K and V, read and written 16 bytes at a time.
template <int D>
struct SlotLds {
    static constexpr int kHeads = kRopeThreads / (D / 8 * kRopeTokens);              // heads at once
    alignas(16) uint16_t k[kRopeRows][kHeads][kRopeTokens][D + 8];
    alignas(16) uint16_t v[kRopeRows][kHeads][kRopeTokens][D + 8];
};

// K and V of the 16 positions of a slot, heads kv0 .. of one part; kRopeRows * kHeads heads a round.
template <int D, class E>
__device__ __forceinline__ void rope_slot(const RopeArgs& a, int32_t block)
{
    constexpr int kLanes = D / 8;                                // threads of a row
    constexpr int kHeads = SlotLds<D>::kHeads;
    __shared__ SlotLds<D> lds;
    auto &k_tile = lds.k, &v_tile = lds.v;
    const int32_t tid = threadIdx.x, j = tid % kLanes, tok = tid / kLanes % kRopeTokens, sub = tid / (kLanes * kRopeTokens);
    const int32_t slot_id = block / a.slot_groups, part = block - slot_id * a.slot_groups;
    const int32_t kv0 = (int32_t)((int64_t)part * a.Hkv / a.slot_groups), kv1 = (int32_t)((int64_t)(part + 1) * a.Hkv / a.slot_groups);
    // start(s) = cu_q_lens[s] / 16 + 2 s, as in the append without rotation
    const OwnedBy own = owner_of(a.cu_q_lens, a.ctx_lens, 0, a.S, slot_id, [](int32_t c, int32_t i) { return (c >> 4) + 2 * i; });
    if (own.q_len <= 1) return;                                  // single tokens: rope_unit
    const int32_t first = own.ctx, last = first + own.q_len;     // the step fills positions [first, last)
    const int32_t p0 = ((first >> 4) + (slot_id - ((own.token >> 4) + 2 * own.seq))) << 4;
    if (p0 >= last) return;
    const int32_t position = p0 + tok, t = own.token + (position - first);
    const bool there = position >= first && position < last;
    Turn r;
    turn_places(r, a, j);
    const int64_t row = there ? t : own.token;
    const uint16_t *k_row = a.k + row * a.k_stride, *v_row = a.v + row * a.v_stride + 8 * j;
    const int32_t* table = a.block_tables + (int64_t)own.seq * a.max_blocks;
    auto page_of = [&](int32_t pos) -> uint16_t* {
        const int32_t entry = pos / a.page_size, id = entry < a.max_blocks ? table[entry] : -1;
        return id >= 0 && id < a.num_pages ? a.layer_base + (int64_t)id * a.page_stride : nullptr;
    };
    // a thread's part of the way out: of K the unit of features 8 fb .. + 7 of a token, of V that of one feature of the 8 positions of a half
    const int32_t k_tok = tid % kRopeTokens, fb = tid / kRopeTokens % kLanes, k_pos = p0 + k_tok;
    const int32_t f = tid % D, half = tid / D % 2, vpos = p0 + 8 * half, vgroups = a.page_size >> 3, block_elems = a.page_size * D;
    uint16_t *k_page = nullptr, *v_page = nullptr;
    const Weights w(r, a.k_norm);
    for (int32_t hb = kv0; hb < kv1; hb += kRopeRows * kHeads) {
        const int32_t h = hb + sub;
        Rows<D> k(r, k_row, h, kHeads, kv1, there);
        r_u32x4 v[kRopeRows];
#pragma unroll
        for (int i = 0; i < kRopeRows; ++i) {
            v[i] = r_u32x4{0u, 0u, 0u, 0u};
            if (there && h + i * kHeads < kv1) v[i] = *(const r_u32x4*)(v_row + (h + i * kHeads) * D);
        }
        if (hb == kv0) {
            if (k_pos >= first && k_pos < last) k_page = page_of(k_pos);
            if (vpos < last && vpos + 8 > first) v_page = page_of(vpos);
            turn_angles(r, a, j, (int32_t)row, position);
        } else {
            __syncthreads();                                     // everybody has read the tiles before
        }
#pragma unroll
        for (int i = 0; i < kRopeRows; ++i) *(r_u32x4*)&v_tile[i][sub][tok][8 * j] = v[i];
        k.template finish<E>(r, w, a.eps, h, kHeads, kv1, there, [&](int32_t head, r_u32x2 x0, r_u32x2 x1) {
            uint16_t* to = k_tile[(head - h) / kHeads][sub][tok];
            *(r_u32x2*)(to + r.off0) = x0;
            *(r_u32x2*)(to + r.off1) = x1;
        });
        // 16 rows become the page's units through LDS, so that stores are 16 bytes wide and a wavefront's lie side by side
        __syncthreads();
        if (k_page) {
#pragma unroll
            for (int i = 0; i < kRopeRows; ++i)
                if (h + i * kHeads < kv1)
                    *(r_u32x4*)(k_page + (int64_t)(h + i * kHeads) * block_elems + (fb * a.page_size + (k_pos & (a.page_size - 1))) * 8) = *(const r_u32x4*)&k_tile[i][sub][k_tok][8 * fb];
        }
        if (!v_page) continue;
#pragma unroll
        for (int i = 0; i < kRopeRows; ++i) {
            if (h + i * kHeads >= kv1) break;
            uint16_t* dst = v_page + (int64_t)(a.Hkv + h + i * kHeads) * block_elems + (((f >> 4) * vgroups + (a.page_size == 16 ? half : 0)) * 16 + (f & 15)) * 8;
            uint16_t e[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) e[n] = v_tile[i][sub][8 * half + n][f];
            if (vpos >= first && vpos + 8 <= last) {
                *(r_u32x4*)dst = r_u32x4{ (uint32_t)e[0] | (uint32_t)e[1] << 16, (uint32_t)e[2] | (uint32_t)e[3] << 16,
                                          (uint32_t)e[4] | (uint32_t)e[5] << 16, (uint32_t)e[6] | (uint32_t)e[7] << 16 };
            } else {
#pragma unroll
                for (int n = 0; n < 8; ++n)
                    if (vpos + n >= first && vpos + n < last) dst[n] = e[n];
            }
        }
    }
}

// The workgroups that fill pages first (with their chain of trips), then those of rows.
template <int D, class E, bool kAppend>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(const RopeArgs a)
{
    if constexpr (kAppend) {
        const int32_t slots = a.slot_blocks * a.slot_groups;
        if ((int32_t)blockIdx.x < slots) rope_slot<D, E>(a, (int32_t)blockIdx.x);
        else rope_unit<D, E, true>(a, ((int32_t)blockIdx.x - slots) * (kRopeThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    } else {
        rope_unit<D, E, false>(a, (int32_t)blockIdx.x * (kRopeThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    }
}

// kv_tokens: wavefronts for K too, of the tokens in front of this one (all of them without a cache; the last single one with it).
template <bool kAppend>
static int launch_rope(const RopeArgs& args, int32_t D, int32_t kv_tokens, bool f16, hipStream_t st) {
    RopeArgs a = args;
    const int32_t heads = kRopeRows * (512 / D);                 // of a wavefront
    a.q_units = (a.Hq + heads - 1) / heads;
    a.kv_units = (a.Hkv + heads - 1) / heads;
    a.kv_tokens = kv_tokens;
    const int64_t units = (int64_t)a.T * a.q_units + (int64_t)kv_tokens * a.kv_units, slots = (int64_t)a.slot_blocks * a.slot_groups, blocks = slots + (units + 3) / 4;
    if (units > 2147483647ll - 4 || blocks > 2147483647ll / kRopeThreads) return CS_ERR_UNSUPPORTED;     // (a launch holds fewer than 2^31 threads along x)
    const dim3 grid((uint32_t)blocks);
    if (D == 128) {
        if (f16) hipLaunchKernelGGL((rope_kernel<128, F16, kAppend>), grid, dim3(kRopeThreads), 0, st, a);
        else     hipLaunchKernelGGL((rope_kernel<128, Bf16, kAppend>), grid, dim3(kRopeThreads), 0, st, a);
    } else {
        if (f16) hipLaunchKernelGGL((rope_kernel<64, F16, kAppend>), grid, dim3(kRopeThreads), 0, st, a);
        else     hipLaunchKernelGGL((rope_kernel<64, Bf16, kAppend>), grid, dim3(kRopeThreads), 0, st, a);
    }
    return check_launch("rope_kernel");
}

static bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// The checks of what either call is given, and its part of the kernel's arguments.  may_count: positions may be left out.
static int fill_rope(const cs_rope* r, const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out,
                     int32_t T, int32_t Hq, int32_t Hkv, int32_t D, bool may_count, RopeArgs& a) {
    if (!r || !q || !k || !q_out) return CS_ERR_INVALID_ARG;
    if (Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0) return CS_ERR_INVALID_ARG;
    if (D != 64 && D != 128) return CS_ERR_UNSUPPORTED;
    if (r->rotary_dim < 0 || r->rotary_dim > D) return CS_ERR_INVALID_ARG;
    if (r->rotary_dim & 7) return CS_ERR_UNSUPPORTED;
    if (r->num_axes < 1 || r->num_axes > 3) return CS_ERR_INVALID_ARG;
    if (!(r->eps >= 0.f) || r->eps > 3.0e38f) return CS_ERR_INVALID_ARG;
    int32_t ends[3] = {r->rotary_dim / 2, r->rotary_dim / 2, r->rotary_dim / 2};
    if (r->num_axes > 1) {
        int64_t sum = 0;
        for (int32_t i = 0; i < r->num_axes; ++i) {
            if (r->axis_pairs[i] < 0) return CS_ERR_INVALID_ARG;
            sum += r->axis_pairs[i];
            ends[i] = (int32_t)std::min<int64_t>(sum, D);
        }
        if (sum != r->rotary_dim / 2) return CS_ERR_INVALID_ARG;
    }
    if (r->rotary_dim > 0) {
        if (!r->inv_freq || !aligned(r->inv_freq, 4) || !aligned(r->positions, 4)) return CS_ERR_INVALID_ARG;
        if (!r->positions && (!may_count || r->num_axes > 1)) return CS_ERR_INVALID_ARG;
        if (r->positions && r->num_axes > 1 && r->position_stride < T) return CS_ERR_INVALID_ARG;
    }
    const int64_t qw = (int64_t)Hq * D, kw = (int64_t)Hkv * D;
    if (q_stride < qw || k_stride < kw || ((q_stride | k_stride) & 7)) return CS_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(q_out, 16) || !aligned(r->q_norm, 8) || !aligned(r->k_norm, 8)) return CS_ERR_INVALID_ARG;
    a = RopeArgs{};
    a.q = (const uint16_t*)q; a.k = (const uint16_t*)k;
    a.q_norm = (const uint16_t*)r->q_norm; a.k_norm = (const uint16_t*)r->k_norm;
    a.q_out = (uint16_t*)q_out;
    a.q_stride = q_stride; a.k_stride = k_stride;
    a.inv_freq = r->inv_freq;
    a.positions = r->rotary_dim > 0 ? r->positions : nullptr;
    a.position_stride = r->position_stride;
    a.eps = r->eps;
    a.rotary_dim = r->rotary_dim; a.interleaved = r->interleaved;
    a.num_axes = r->num_axes; a.pairs0 = ends[0]; a.pairs1 = ends[1];
    a.T = T; a.Hq = Hq; a.Hkv = Hkv;
    return CS_OK;
}

static int qk_rope(const cs_rope* rope, int32_t T, int32_t Hq, int32_t Hkv, int32_t D, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                   void* q_out, void* k_out, void* stream, bool f16) {
    if (T < 0) return CS_ERR_INVALID_ARG;
    if (T == 0) return CS_OK;
    RopeArgs a;
    const int rc = fill_rope(rope, q, q_stride, k, k_stride, q_out, T, Hq, Hkv, D, false, a);
    if (rc) return rc;
    if (!k_out || !aligned(k_out, 16)) return CS_ERR_INVALID_ARG;
    a.k_out = (uint16_t*)k_out;
    return launch_rope<false>(a, D, T, f16, (hipStream_t)stream);
}

static int append_rope(const cs_kv_pool* pool, int32_t layer, const cs_batch* batch, const cs_rope* rope, int32_t Hq, const void* q, int64_t q_stride,
                       const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out, void* stream, bool f16) {
    int rc = validate_pool(pool);
    if (rc) return rc;
    if (layer < 0 || layer >= pool->num_layers) return CS_ERR_INVALID_ARG;
    rc = validate_batch(pool, batch);
    if (rc) return rc;
    if (batch->num_tokens == 0) return CS_OK;
    if (!lengths_fit(batch)) return CS_ERR_UNSUPPORTED;
    RopeArgs a;
    const int32_t Hkv = pool->num_kv_heads, D = pool->head_dim;
    rc = fill_rope(rope, q, q_stride, k, k_stride, q_out, batch->num_tokens, Hq, Hkv, D, true, a);
    if (rc) return rc;
    if (!v || !aligned(v, 16) || v_stride < (int64_t)Hkv * D || (v_stride & 7)) return CS_ERR_INVALID_ARG;
    a.v = (const uint16_t*)v; a.v_stride = v_stride;
    a.layer_base = (uint16_t*)pool->base + (int64_t)layer * pool->layer_stride;
    a.page_stride = pool->page_stride; a.num_pages = pool->num_pages; a.page_size = pool->page_size;
    a.S = batch->num_seqs; a.max_blocks = batch->max_blocks_per_seq;
    a.block_tables = batch->block_tables; a.ctx_lens = batch->ctx_lens; a.cu_q_lens = batch->cu_q_lens;
    int32_t single_end = 0;
    bool any_chunk = false;
    for (int32_t s = 0; s < a.S; ++s) {
        const int32_t n = batch->h_cu_q_lens[s + 1] - batch->h_cu_q_lens[s];
        if (n == 1) single_end = batch->h_cu_q_lens[s + 1];
        any_chunk |= n > 1;
    }
    a.slot_blocks = any_chunk ? a.T / 16 + 2 * a.S : 0;
    a.slot_groups = (Hkv + 256 / D - 1) / (256 / D);             // a round of heads each
    return launch_rope<true>(a, D, single_end, f16, (hipStream_t)stream);
}

}  // namespace cs

using namespace cs;

extern "C" {

int cs_qk_rope(const cs_rope* rope, int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
               const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out, void* k_out, void* stream) {
    return qk_rope(rope, num_tokens, num_q_heads, num_kv_heads, head_dim, q, q_stride, k, k_stride, q_out, k_out, stream, false);
}

int cs_qk_rope_f16(const cs_rope* rope, int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                   const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out, void* k_out, void* stream) {
    return qk_rope(rope, num_tokens, num_q_heads, num_kv_heads, head_dim, q, q_stride, k, k_stride, q_out, k_out, stream, true);
}

int cs_kv_append_rope(const cs_kv_pool* pool, int32_t layer, const cs_batch* batch, const cs_rope* rope, int32_t num_q_heads,
                      const void* q, int64_t q_stride, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                      void* q_out, void* stream) {
    return append_rope(pool, layer, batch, rope, num_q_heads, q, q_stride, k_new, k_stride, v_new, v_stride, q_out, stream, false);
}

int cs_kv_append_rope_f16(const cs_kv_pool* pool, int32_t layer, const cs_batch* batch, const cs_rope* rope, int32_t num_q_heads,
                          const void* q, int64_t q_stride, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                          void* q_out, void* stream) {
    return append_rope(pool, layer, batch, rope, num_q_heads, q, q_stride, k_new, k_stride, v_new, v_stride, q_out, stream, true);
}

}  // extern "C"
