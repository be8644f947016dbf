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
// HBM-bound: each value is read and written once.  A thread has 8 features of one token, as two pieces of 4 (the two halves of four
// pairs), and walks heads with the angles in its registers, so that a sine is computed once a token and not once a head.
#include <algorithm>
#include "cs_common.h"
#include "cs_elem.h"

namespace cs {

typedef uint32_t r_u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t r_u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 16;                                  // of a workgroup
constexpr int kRopeRows = 4;                                     // rows of a thread whose loads are in flight together

// What the kernel is told.  Strides in elements.
struct RopeArgs {
    const uint16_t *q, *k, *v, *q_norm, *k_norm;
    uint16_t *q_out, *k_out;                                     // k_out: rows, where nothing is appended
    int64_t q_stride, k_stride, v_stride;
    const float* inv_freq;
    const int32_t* positions;
    int64_t position_stride;
    float eps;
    int32_t rotary_dim, interleaved, pairs0, pairs1;             // pairs of the first two axes
    int32_t T, Hq, Hkv, groups;                                  // groups: parts that the heads are dealt in
    // the append
    uint16_t* layer_base;
    int64_t page_stride;
    int32_t num_pages, page_size, S, max_blocks;
    const int32_t *block_tables, *ctx_lens, *cu_q_lens;
    int32_t slot_blocks;                                         // workgroups of sequences with more than one new token
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

// A thread's features of a row, and the angles of its token.
struct Turn {
    int32_t off0, off1;                                          // its two pieces of four features
    bool rotates, neighbours;                                    // pairs are (piece 0, piece 1), or neighbours inside a piece
    float c[4], s[4];
};

template <int D>
__device__ __forceinline__ Turn turn_of(const RopeArgs& a, int32_t j, int32_t t, int32_t position)
{
    Turn r;
    r.rotates = 8 * j < a.rotary_dim;
    r.neighbours = a.interleaved != 0 || !r.rotates;
    r.off0 = r.neighbours ? 8 * j : 4 * j;
    r.off1 = r.neighbours ? 8 * j + 4 : a.rotary_dim / 2 + 4 * j;
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.c[i] = 1.f; r.s[i] = 0.f; }
    if (r.rotates) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t pair = 4 * j + i;
            int32_t at = position;
            if (a.positions) at = a.positions[(pair < a.pairs0 ? 0 : pair < a.pairs1 ? 1 : 2) * a.position_stride + t];
            const double turns = (double)at * (double)a.inv_freq[pair] * 0.15915494309189535;   // 1 / 2 pi
            const float part = (float)(turns - rint(turns));
            sincospif(2.f * part, &r.s[i], &r.c[i]);
        }
    }
    return r;
}

// One row's 8 features: normed, rotated, rounded.
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
        for (int i = 0; i < 4; ++i) sum += a[i] * a[i] + b[i] * b[i];
        const float f = 1.f / sqrtf(row_sum<D / 8>(sum) * (1.f / D) + eps);
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
                lo = x * r.c[i] - y * r.s[i];
                hi = y * r.c[i] + x * r.s[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = a[i], y = b[i];
                a[i] = x * r.c[i] - y * r.s[i];
                b[i] = y * r.c[i] + x * r.s[i];
            }
        }
    }
    x0 = r_u32x2{ E::pack(a[0], a[1]), E::pack(a[2], a[3]) };
    x1 = r_u32x2{ E::pack(b[0], b[1]), E::pack(b[2], b[3]) };
}

// Heads h0 + first, h0 + first + step, .. below h1 of one token: `src` its row of head 0, `put(head, piece 0, piece 1)` takes them away.
template <int D, class E, class Put>
__device__ __forceinline__ void turn_heads(const Turn& r, const uint16_t* __restrict__ src, const uint16_t* __restrict__ norm, float eps,
                                           int32_t first, int32_t end, int32_t step, bool there, Put put)
{
    r_u32x2 w[2] = {{0u, 0u}, {0u, 0u}};
    if (norm) {
        w[0] = *(const r_u32x2*)(norm + r.off0);
        w[1] = *(const r_u32x2*)(norm + r.off1);
    }
    for (int32_t h = first; h < end; h += kRopeRows * step) {
        r_u32x2 x[kRopeRows][2];
#pragma unroll
        for (int i = 0; i < kRopeRows; ++i) {
            const int32_t head = min(h + i * step, end - 1);
            x[i][0] = x[i][1] = r_u32x2{0u, 0u};
            if (there) {
                x[i][0] = *(const r_u32x2*)(src + head * D + r.off0);
                x[i][1] = *(const r_u32x2*)(src + head * D + r.off1);
            }
        }
#pragma unroll
        for (int i = 0; i < kRopeRows; ++i) {
            if (h + i * step >= end) break;
            turn_row<D, E>(r, norm != nullptr, w, eps, x[i][0], x[i][1]);
            if (there) put(h + i * step, x[i][0], x[i][1]);
        }
    }
}

// A workgroup: 16 tokens (of one page's positions, or packed ones), the heads of one of a.groups parts.
template <int D, class E, bool kAppend>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(const RopeArgs a)
{
    constexpr int kLanes = D / 8;                                // threads of a row
    constexpr int kHeads = kRopeThreads / (kLanes * kRopeTokens);// heads at once
    __shared__ uint16_t v_tile[2][kHeads][kRopeTokens][D + 8];
    const int32_t tid = threadIdx.x, j = tid % kLanes, tok = tid / kLanes % kRopeTokens, sub = tid / (kLanes * kRopeTokens);
    const int32_t kv0 = (int32_t)((int64_t)blockIdx.y * a.Hkv / a.groups), kv1 = (int32_t)((int64_t)(blockIdx.y + 1) * a.Hkv / a.groups);
    const int32_t G = a.Hq / a.Hkv;
    int32_t t = -1, position = 0, entry = -1, slot = 0, seq = 0;
    const bool slots = kAppend && (int32_t)blockIdx.x < a.slot_blocks;
    int32_t p0 = 0, first = 0, last = 0;                         // slots: first of the 16 positions; the step fills [first, last)
    if (slots) {
        // start(s) = cu_q_lens[s] / 16 + 2 s, as in the append without rotation
        const OwnedBy own = owner_of(a.cu_q_lens, a.ctx_lens, 0, a.S, (int32_t)blockIdx.x, [](int32_t c, int32_t i) { return (c >> 4) + 2 * i; });
        first = own.ctx;
        last = first + own.q_len;
        if (own.q_len <= 1) return;                              // single tokens: the workgroups behind these
        p0 = ((first >> 4) + ((int32_t)blockIdx.x - ((own.token >> 4) + 2 * own.seq))) << 4;
        if (p0 >= last) return;
        seq = own.seq;
        position = p0 + tok;
        if (position >= first && position < last) t = own.token + (position - first);
    } else {
        t = ((int32_t)blockIdx.x - (kAppend ? a.slot_blocks : 0)) * kRopeTokens + tok;
        if (t >= a.T) t = -1;
        if (kAppend && t >= 0) {
            // in an online-first batch token t is usually sequence t
            seq = min(t, a.S - 1);
            if (!(a.cu_q_lens[seq] <= t && t < a.cu_q_lens[seq + 1])) {
                int32_t lo = 0, hi = a.S;                        // cu[lo] <= t < cu[hi]
                while (hi - lo > 1) {
                    const int32_t mid = (lo + hi) >> 1;
                    if (a.cu_q_lens[mid] <= t) lo = mid; else hi = mid;
                }
                seq = lo;
            }
            position = a.ctx_lens[seq];
            if (a.cu_q_lens[seq + 1] - a.cu_q_lens[seq] != 1) t = -1;
        }
    }
    const bool there = t >= 0;
    uint16_t* page = nullptr;                                    // the token's page of this layer
    if (kAppend && there) {
        entry = position / a.page_size;
        slot = position - entry * a.page_size;
        const int32_t id = entry < a.max_blocks ? a.block_tables[(int64_t)seq * a.max_blocks + entry] : -1;
        if (id >= 0 && id < a.num_pages) page = a.layer_base + (int64_t)id * a.page_stride;
    }
    const Turn r = turn_of<D>(a, j, there ? t : 0, position);
    const int64_t row = there ? t : 0;
    turn_heads<D, E>(r, a.q + row * a.q_stride, a.q_norm, a.eps, kv0 * G + sub, kv1 * G, kHeads, there,
                     [&](int32_t h, r_u32x2 x0, r_u32x2 x1) {
        uint16_t* dst = a.q_out + (row * a.Hq + h) * D;
        *(r_u32x2*)(dst + r.off0) = x0;
        *(r_u32x2*)(dst + r.off1) = x1;
    });
    const int32_t block_elems = a.page_size * D;
    turn_heads<D, E>(r, a.k + row * a.k_stride, a.k_norm, a.eps, kv0 + sub, kv1, kHeads, there && (!kAppend || page),
                     [&](int32_t h, r_u32x2 x0, r_u32x2 x1) {
        if constexpr (kAppend) {
            // unit f / 8 of token `slot`, the half of it that the piece is
            uint16_t* blk = page + (int64_t)h * block_elems + slot * 8;
            *(r_u32x2*)(blk + (r.off0 >> 3) * a.page_size * 8 + (r.off0 & 7)) = x0;
            *(r_u32x2*)(blk + (r.off1 >> 3) * a.page_size * 8 + (r.off1 & 7)) = x1;
        } else {
            uint16_t* dst = a.k_out + (row * a.Hkv + h) * D;
            *(r_u32x2*)(dst + r.off0) = x0;
            *(r_u32x2*)(dst + r.off1) = x1;
        }
    });
    if constexpr (kAppend) {
        // V as it is.  feature d of token t: (((d/16) * groups of 8 + t/8) * 16 + d%16) * 8 + t%8
        const int32_t vgroups = a.page_size >> 3;
        const uint16_t* vrow = a.v + row * a.v_stride + 8 * j;
        if (!slots) {
            for (int32_t h = kv0 + sub; h < kv1; h += kHeads) {
                if (!page) break;
                const r_u32x4 x = *(const r_u32x4*)(vrow + h * D);
                uint16_t* dst = page + (int64_t)(a.Hkv + h) * block_elems + (((j >> 1) * vgroups + (slot >> 3)) * 16 + (j & 1) * 8) * 8 + (slot & 7);
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[e * 8] = (uint16_t)(x[e >> 1] >> (e & 1) * 16);
            }
            return;
        }
        // 16 rows become the page's units (one feature of 8 tokens each) through LDS, so that stores are 16 bytes wide
        const int32_t f = tid % D, half = tid / D % 2, vpos = p0 + 8 * half;
        const int32_t id_entry = vpos / a.page_size;
        const int32_t id = id_entry < a.max_blocks && vpos < last ? a.block_tables[(int64_t)seq * a.max_blocks + id_entry] : -1;
        const bool full = vpos >= first && vpos + 8 <= last;
        for (int32_t h = kv0, n = 0; h < kv1; h += kHeads, n ^= 1) {
            if (there && h + sub < kv1) *(r_u32x4*)&v_tile[n][sub][tok][8 * j] = *(const r_u32x4*)(vrow + (h + sub) * D);
            __syncthreads();
            if (id < 0 || id >= a.num_pages || h + sub >= kv1) continue;
            uint16_t* dst = a.layer_base + (int64_t)id * a.page_stride + (int64_t)(a.Hkv + h + sub) * block_elems +
                            (((f >> 4) * vgroups + (a.page_size == 16 ? half : 0)) * 16 + (f & 15)) * 8;
            uint16_t e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = v_tile[n][sub][8 * half + i][f];
            if (full) {
                *(r_u32x4*)dst = r_u32x4{ (uint32_t)e[0] | (uint32_t)e[1] << 16, (uint32_t)e[2] | (uint32_t)e[3] << 16,
                                          (uint32_t)e[4] | (uint32_t)e[5] << 16, (uint32_t)e[6] | (uint32_t)e[7] << 16 };
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (vpos + i >= first && vpos + i < last) dst[i] = e[i];
            }
        }
    }
}

// The parts that the heads are dealt in: enough workgroups for four a CU where there are heads enough.
static int32_t head_groups(int64_t blocks, int32_t Hkv) {
    const int64_t want = (4ll * device_cus() + blocks - 1) / std::max<int64_t>(blocks, 1);
    return (int32_t)std::min<int64_t>(std::max<int64_t>(want, 1), Hkv);
}

template <bool kAppend>
static int launch_rope(const RopeArgs& args, int32_t D, int64_t blocks, bool f16, hipStream_t st) {
    RopeArgs a = args;
    if (blocks > 2147483647ll / kRopeThreads) return CS_ERR_UNSUPPORTED;      // (a launch holds fewer than 2^31 threads along x)
    a.groups = std::min(head_groups(blocks, a.Hkv), 65535);
    const dim3 grid((uint32_t)blocks, (uint32_t)a.groups);
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
    a.pairs0 = ends[0]; a.pairs1 = ends[1];
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
    return launch_rope<false>(a, D, ((int64_t)T + kRopeTokens - 1) / kRopeTokens, f16, (hipStream_t)stream);
}

static int append_rope(const cs_kv_pool* pool, int32_t layer, const cs_batch* batch, const cs_rope* rope, int32_t Hq, const void* q, int64_t q_stride,
                       const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out, void* stream, bool f16) {
    int rc = validate_pool(pool);
    if (rc) return rc;
    if (layer < 0 || layer >= pool->num_layers) return CS_ERR_INVALID_ARG;
    rc = validate_batch(pool, batch);
    if (rc) return rc;
    if (batch->num_tokens == 0) return CS_OK;
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
    bool any_single = false, any_chunk = false;
    for (int32_t s = 0; s < a.S; ++s) {
        const int32_t n = batch->h_cu_q_lens[s + 1] - batch->h_cu_q_lens[s];
        any_single |= n == 1;
        any_chunk |= n > 1;
    }
    a.slot_blocks = any_chunk ? a.T / 16 + 2 * a.S : 0;
    return launch_rope<true>(a, D, (int64_t)a.slot_blocks + (any_single ? ((int64_t)a.T + kRopeTokens - 1) / kRopeTokens : 0), f16, (hipStream_t)stream);
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
