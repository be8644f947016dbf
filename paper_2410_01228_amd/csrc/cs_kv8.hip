// The 8-bit KV cache: the append that rounds new K/V rows to e4m3 codes with a power-of-two scale for each block, and the host
// side of its attention call (whose kernels are the 16-bit path's, instantiated for Kv8: cs_decode8_impl.h, cs_prefill_impl.h).
//
// A block is one page (16 tokens), K or V, one kv head.  Its scale is 2^e with the least e >= -100 that has all of the block's
// values within 448 * 2^e, the largest code; a code is the nearest e4m3 value to x / 2^e, ties to the even one.  A power of
// two, because then a token's code does not depend on who shares its block: raising e for a later token rescales the codes that
// are there without another rounding (except where they fall below the smallest normal code, 2^-6), the widening in
// the attention kernels is exact, and the range of e4m3 (2^-9 to 448) leaves so much room below that a finer scale would
// gain nothing: its steps are relative.
#include <algorithm>
#include <new>
#include "cs_common.h"
#include "cs_elem.h"
#include "cs_plan.h"

namespace cs {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int32_t kLeastExponent = -100, kMostExponent = 120;
constexpr float kMostCode = 448.f;
constexpr float kMostHalf = 61440.f;         // the largest value of 4 significant bits that half precision holds
constexpr float kMostBf16 = 0x1.ep127f;      // and bf16: 240 * 2^120 (above 248 * 2^120 the nearest code stands for 2^128)

// Where the blocks' scales begin in a page, in bytes.
__host__ __device__ inline int32_t scales_offset(int32_t Hkv, int32_t D) { return 2 * Hkv * (kPage * D); }

// The new rows' element type.  kMost: a block whose largest value is beyond it is a rare one (rare_size, rare_limit): values beyond the
// largest one of 4 significant bits, which end there, and infinities (bf16: they say nothing about the scale, and end at the
// block's largest code; fp16: values beyond kMostHalf like others).
struct RowBf16 {
    static constexpr float kMost = kMostBf16;
    static constexpr uint32_t kMostBits = 0x7f70;
    static __device__ __forceinline__ float value(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }
    static __device__ __forceinline__ void widen(uint32_t w, float& a, float& b) {
        a = __builtin_bit_cast(float, w << 16);
        b = __builtin_bit_cast(float, w & 0xffff0000u);
    }
    static __device__ __forceinline__ float rare_size(float x) { return fabsf(x) < INFINITY ? fminf(fabsf(x), kMost) : 0.f; }
    static __device__ __forceinline__ float rare_limit(float inv) { return fminf(kMostCode, kMost * inv); }
};
struct RowF16 {
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    static constexpr float kMost = kMostHalf;
    static constexpr uint32_t kMostBits = 0x7b80;
    static __device__ __forceinline__ float value(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }
    static __device__ __forceinline__ void widen(uint32_t w, float& a, float& b) {
        const x2 v = __builtin_bit_cast(x2, w);
        a = (float)v[0];
        b = (float)v[1];
    }
    static __device__ __forceinline__ float rare_size(float x) { return x == x ? fminf(fabsf(x), kMost) : 0.f; }
    static __device__ __forceinline__ float rare_limit(float inv) { return kMostHalf * inv; }
};

__device__ __forceinline__ float power(int32_t e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// The least exponent for a block whose largest value has these bits: 448 = 1.75 * 2^8.
__device__ __forceinline__ int32_t exponent_for(float top) {
    const uint32_t b = __builtin_bit_cast(uint32_t, top);
    return max((int32_t)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0), kLeastExponent);
}
__device__ __forceinline__ int32_t exponent_of(float scale) {
    return min(max((int32_t)((__builtin_bit_cast(uint32_t, scale) >> 23) & 255) - 127, kLeastExponent), kMostExponent);
}

// Scaled values of a rare block: none beyond the largest code that it may use; NaN stays NaN.
template <class Row, int N>
__device__ __forceinline__ void limit(float (&x)[N], float inv) {
    const float most = Row::rare_limit(inv);
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (fabsf(x[i]) > most) x[i] = copysignf(most, x[i]);
}
// The largest size among N words of two values, over the wavefront, and whether the block is a rare one.  Sizes of either type
// order like their bits, two at a time; beyond kMostBits come values beyond kMost, infinities and NaNs (which are no maximum).
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <class Row, int N>
__device__ __forceinline__ float largest(const uint32_t (&w)[N], bool& rare) {
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    uint32_t bits = max((uint32_t)m[0], (uint32_t)m[1]);
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) bits = max(bits, (uint32_t)__shfl_xor((int)bits, k, 64));
    rare = bits > Row::kMostBits;
    if (!rare) return Row::value(bits);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float a, b;
        Row::widen(w[i], a, b);
        top = fmaxf(top, fmaxf(Row::rare_size(a), Row::rare_size(b)));
    }
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k, 64));
    return top;
}
// Four values over the scale as four codes.
template <class Row>
__device__ __forceinline__ uint32_t codes4(uint32_t w0, uint32_t w1, float inv, bool rare) {
    float x[4];
    Row::widen(w0, x[0], x[1]);
    Row::widen(w1, x[2], x[3]);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= inv;
    if (rare) limit<Row>(x, inv);
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
}
// Four codes at a scale that is `factor` of theirs.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float factor) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * factor, lo[1] * factor, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * factor, hi[1] * factor, r, true);
}
// The factor from exponent e0 to e (2^-60 takes every code to zero).
__device__ __forceinline__ float rescale_factor(int32_t e0, int32_t e) { return power(max(e0 - e, -60)); }

// Bytes of a dword of 4 tokens that are below `n` (of the four).
__device__ __forceinline__ uint32_t first_bytes(int32_t n) {
    return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1;
}

constexpr int kAppend8SlotShift = 4;

constexpr int kAppend8Threads = 128;

// Chunks.  A workgroup owns one (page touched this step, kv head), one wavefront its K block, the other its V block; a lane has 16
// features of a token, at head dim 128 twice.  Bound by memory (three bytes a value) and, below some thousand tokens, by the
// trips to it: lengths, then rows, table entry and what the page holds.  Rows come in 16 bytes a lane, the codes leave as whole
// 16-byte units; V goes through LDS, where it is turned from 16 features of a token to 4 tokens of 4.  The wavefronts need
// nothing of each other: no barrier, and twice as many bytes under way as with a block shared by two of them (2048 tokens, 8
// heads, 5.4 -> 4.8 us; 31200 tokens 42.9 -> 40.8).  Rows are loaded through the caches: they come from a projection just done, which
// leaves them in the last level (31200 tokens 41.0 -> 31.4 us, 6.1 TB/s; 128 single tokens + 9900 in chunks 15.3 -> 12.0).  Two or four
// heads a workgroup are slower below some 10000 tokens (512: 3.7, 4.5, 6.6 us).
// Workgroup slots are dealt to sequences as start(s) = cu_q_lens[s]/16 + 2s, as in the 16-bit append.
template <class Row, int D>
__device__ __forceinline__ void append8_page(
    int32_t block, char* __restrict__ layer_base, int64_t page_bytes, int32_t num_pages, int32_t Hkv, int32_t S, int32_t first_seq, int32_t base_slot,
    const int32_t* __restrict__ block_tables, int32_t max_blocks, const int32_t* __restrict__ ctx_lens, const int32_t* __restrict__ cu_q_lens,
    const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new)
{
    constexpr int kUnits = D / 64;
    constexpr int kRowBytes = D + 16;                              // LDS row of a token's codes: 4 rows start 16 banks apart
    __shared__ __attribute__((aligned(16))) uint8_t turned[kPage * kRowBytes];
    const int32_t per = 8 * Hkv, group = block / per, in_group = block - group * per;   // a page's heads on one XCD
    const int32_t h = in_group >> 3, slot_id = base_slot + group * 8 + (in_group & 7);
    const OwnedBy own = owner_of(cu_q_lens, ctx_lens, first_seq, S - first_seq, slot_id, [](int32_t t, int32_t i) { return (t >> kAppend8SlotShift) + 2 * i; });
    const int32_t first = own.ctx, last = first + own.q_len;       // the step fills positions [first, last)
    if (own.q_len <= 1) return;                                    // single tokens: append8_token
    const int32_t blk = (first >> 4) + (slot_id - ((own.token >> kAppend8SlotShift) + 2 * own.seq));
    const int32_t p0 = blk << 4;
    if (first < 0 || p0 >= last || blk >= max_blocks) return;
    const bool is_v = threadIdx.x >= 64;
    const int32_t lane = threadIdx.x & 63, tok = lane & 15;
    const int32_t page = block_tables[(int64_t)own.seq * max_blocks + blk];
    const int32_t pos = p0 + tok;
    const bool is_new = pos >= first && pos < last;
    uint32_t w[8 * kUnits];
    const uint16_t* src = (is_v ? v_new : k_new) + ((int64_t)(own.token + pos - first) * Hkv + h) * D + (lane >> 4) * 16;
#pragma unroll
    for (int i = 0; i < 2 * kUnits; ++i) {
        u32x4 r = {0u, 0u, 0u, 0u};
        if (is_new) r = ((const u32x4*)(src + (i >> 1) * 64))[i & 1];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[4 * i + j] = r[j];
    }
    const bool page_ok = page >= 0 && page < num_pages;
    if (!page_ok) return;
    char* page_base = layer_base + (int64_t)page * page_bytes;
    u32x4* unit = (u32x4*)(page_base + ((is_v ? Hkv : 0) + h) * (kPage * D)) + lane;
    float* scale = (float*)(page_base + scales_offset(Hkv, D)) + (is_v ? Hkv : 0) + h;
    const int32_t held = min(max(first - p0, 0), kPage);           // tokens that the page holds already
    const int32_t upto = min(last - p0, kPage);
    // (what the block holds is asked for while the rows are on their way)
    u32x4 old[kUnits];
    float old_scale = 0.f;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        old[u] = u32x4{0u, 0u, 0u, 0u};
        if (is_v ? held > 0 || upto < kPage : held > 0) old[u] = unit[u * 64];
    }
    if (held > 0) old_scale = *scale;

    bool rare;
    const float top = largest<Row>(w, rare);
    int32_t e = exponent_for(top);
    const int32_t e_old = exponent_of(old_scale);
    if (held > 0) e = max(e, e_old);
    const float inv = power(-e);
    u32x4 c[kUnits];
#pragma unroll
    for (int i = 0; i < 4 * kUnits; ++i) c[i >> 2][i & 3] = codes4<Row>(w[2 * i], w[2 * i + 1], inv, rare);
    const bool raised = held > 0 && e > e_old;
    const float factor = rescale_factor(e_old, e);
    if (!is_v) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            if (is_new) unit[u * 64] = c[u];
            else if (raised && tok < held)
                unit[u * 64] = u32x4{rescale4(old[u][0], factor), rescale4(old[u][1], factor), rescale4(old[u][2], factor), rescale4(old[u][3], factor)};
        }
    } else {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) *(u32x4*)(turned + tok * kRowBytes + (u * 4 + (lane >> 4)) * 16) = c[u];
        // unit u*64 + lane: tokens 4 tg .. +4 of features u*64 + 16 i + f (a wavefront's LDS accesses stay in order)
        const int32_t f = lane & 15, tg = lane >> 4;
        const uint32_t below = first_bytes(held - 4 * tg), fresh = first_bytes(upto - 4 * tg) & ~below;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const uint8_t* from = turned + 4 * tg * kRowBytes + u * 64 + f;
            u32x4 n;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t v = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) v |= (uint32_t)from[j * kRowBytes + i * 16] << (8 * j);
                const uint32_t before = raised ? (rescale4(old[u][i], factor) & below) | (old[u][i] & ~below) : old[u][i];
                n[i] = (v & fresh) | (before & ~fresh);
            }
            if (fresh != 0 || (raised && below != 0)) unit[u * 64] = n;
        }
    }
    if (lane == 0 && (held == 0 || raised)) *scale = power(e);
}

// Single tokens (decode): a wavefront per (sequence, kv head), a lane D/64 features of K and of V.  Bound by latency: lengths,
// table entry and rows, the block's scale.  A token that raises its block's scale (rarely: the first of a page sets it)
// has the wavefront go over the block.
template <class Row, int D>
__device__ __forceinline__ void append8_token(
    int32_t wave, char* __restrict__ layer_base, int64_t page_bytes, int32_t num_pages, int32_t Hkv, int32_t first_seq, int32_t end_seq,
    const int32_t* __restrict__ block_tables, int32_t max_blocks, const int32_t* __restrict__ ctx_lens, const int32_t* __restrict__ cu_q_lens,
    const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new)
{
    const int32_t i = wave / Hkv, h = wave - i * Hkv, s = first_seq + i, lane = threadIdx.x & 63;
    if (s >= end_seq) return;
    const int32_t t = cu_q_lens[s], pos = ctx_lens[s];
    if (cu_q_lens[s + 1] - t != 1) return;
    const int32_t blk = pos >> 4, slot = pos & 15;
    if (pos < 0 || blk >= max_blocks) return;
    const int64_t src = ((int64_t)t * Hkv + h) * D;
    uint32_t kw, vw;
    if (D == 128) {
        kw = ((const uint32_t*)(k_new + src))[lane];
        vw = ((const uint32_t*)(v_new + src))[lane];
    } else {
        kw = k_new[src + lane];
        vw = v_new[src + lane];
    }
    const int32_t page = block_tables[(int64_t)s * max_blocks + blk];
    if (page < 0 || page >= num_pages) return;
    char* page_base = layer_base + (int64_t)page * page_bytes;
    float* scale = (float*)(page_base + scales_offset(Hkv, D)) + h;
    float old[2] = {0.f, 0.f};
    if (slot > 0) { old[0] = scale[0]; old[1] = scale[Hkv]; }
    uint32_t word[2] = {kw, vw}, code[2];
    int32_t e[2], e_old[2];
    bool raised[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const uint32_t w[1] = {word[b]};
        bool rare;
        const float top = largest<Row>(w, rare);
        e[b] = exponent_for(top);
        e_old[b] = exponent_of(old[b]);
        raised[b] = slot > 0 && e[b] > e_old[b];
        if (slot > 0) e[b] = max(e[b], e_old[b]);
        code[b] = codes4<Row>(word[b], 0u, power(-e[b]), rare);
        if (lane == 0 && (slot == 0 || raised[b])) scale[b * Hkv] = power(e[b]);
    }
    char* kblk = page_base + h * (kPage * D);
    char* vblk = kblk + Hkv * (kPage * D);
    if (raised[0]) {
        const float factor = rescale_factor(e_old[0], e[0]);
#pragma unroll
        for (int u = 0; u < D / 64; ++u) {
            if ((lane & 15) >= slot) continue;
            u32x4* p = (u32x4*)kblk + u * 64 + lane;
            const u32x4 w = *p;
            *p = u32x4{rescale4(w[0], factor), rescale4(w[1], factor), rescale4(w[2], factor), rescale4(w[3], factor)};
        }
    }
    // K: features 2 lane, 2 lane + 1 (head dim 64: lane) of unit (feature / 16) * 16 + slot
    if (D == 128) *(uint16_t*)(kblk + ((lane >> 3) * 16 + slot) * 16 + (lane & 7) * 2) = (uint16_t)code[0];
    else          *(uint8_t*)(kblk + ((lane >> 4) * 16 + slot) * 16 + (lane & 15)) = (uint8_t)code[0];
    if (raised[1]) {
        // whole units, the new token's codes fetched from the lanes that have them
        const float factor = rescale_factor(e_old[1], e[1]);
        const uint32_t below = first_bytes(slot - 4 * (lane >> 4));
        const uint32_t mine = first_bytes(slot + 1 - 4 * (lane >> 4)) & ~below;
#pragma unroll
        for (int u = 0; u < D / 64; ++u) {
            u32x4* p = (u32x4*)vblk + u * 64 + lane;
            u32x4 w = *p;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int d = u * 64 + j * 16 + (lane & 15);
                const uint32_t pair = (uint32_t)__shfl((int)code[1], D == 128 ? d >> 1 : d, 64);
                const uint32_t c = D == 128 && (d & 1) ? (pair >> 8) & 255u : pair & 255u;
                w[j] = (rescale4(w[j], factor) & below) | ((c * 0x01010101u) & mine) | (w[j] & ~(below | mine));
            }
            if ((below | mine) != 0) *p = w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            const int d = lane * (D / 64) + j;
            vblk[(((d >> 6) * 4 + (slot >> 2)) * 16 + (d & 15)) * 16 + ((d >> 4) & 3) * 4 + (slot & 3)] = (char)(code[1] >> (8 * j));
        }
    }
}

// Chunks first, single tokens behind them, in one launch.
template <class Row, int D>
__global__ __launch_bounds__(kAppend8Threads) void append8_kernel(
    char* __restrict__ layer_base, int64_t page_bytes, int32_t num_pages, int32_t Hkv, int32_t S, int32_t chunk_seq, int32_t base_slot,
    int32_t single_seq, int32_t single_end, const int32_t* __restrict__ block_tables, int32_t max_blocks,
    const int32_t* __restrict__ ctx_lens, const int32_t* __restrict__ cu_q_lens,
    const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new, uint32_t page_blocks)
{
    if (blockIdx.x < page_blocks)
        append8_page<Row, D>((int32_t)blockIdx.x, layer_base, page_bytes, num_pages, Hkv, S, chunk_seq, base_slot, block_tables, max_blocks,
                             ctx_lens, cu_q_lens, k_new, v_new);
    else
        append8_token<Row, D>((int32_t)((blockIdx.x - page_blocks) * (kAppend8Threads / 64) + (threadIdx.x >> 6)), layer_base, page_bytes, num_pages, Hkv,
                              single_seq, single_end, block_tables, max_blocks, ctx_lens, cu_q_lens, k_new, v_new);
}

static int validate_kv8(const cs_kv8_pool* p) {
    if (!p || !p->base) return CS_ERR_INVALID_ARG;
    if (p->num_layers <= 0 || p->num_pages <= 0 || p->num_kv_heads <= 0 || p->head_dim <= 0) return CS_ERR_INVALID_ARG;
    // (offsets inside a page are 32 bits)
    if ((p->head_dim != 64 && p->head_dim != 128) || p->num_kv_heads > 65535) return CS_ERR_UNSUPPORTED;
    if (p->page_stride < (int64_t)cs_kv8_page_bytes(p->num_kv_heads, p->head_dim) || (p->page_stride & 15) != 0) return CS_ERR_INVALID_ARG;
    if (p->page_stride > INT64_MAX / p->num_pages || p->layer_stride < (int64_t)p->num_pages * p->page_stride || (p->layer_stride & 15) != 0)
        return CS_ERR_INVALID_ARG;
    return ((uintptr_t)p->base & 15) ? CS_ERR_INVALID_ARG : CS_OK;
}

// The pool in the units of the attention launchers: 2 bytes.
static cs_kv_pool kv8_view(const cs_kv8_pool& p) {
    return cs_kv_pool{p.base, p.num_layers, p.num_pages, kPage, p.num_kv_heads, p.head_dim, p.layer_stride / 2, p.page_stride / 2};
}

static int append8(const cs_kv8_pool* pool, int32_t layer, const cs_batch* batch, const void* k_new, const void* v_new, void* stream, bool f16) {
    int rc = validate_kv8(pool);
    if (rc) return rc;
    if (layer < 0 || layer >= pool->num_layers) return CS_ERR_INVALID_ARG;
    rc = validate_batch(nullptr, batch);
    if (rc) return rc;
    if (batch->num_tokens == 0) return CS_OK;
    if (!k_new || !v_new || ((uintptr_t)k_new & 15) || ((uintptr_t)v_new & 15)) return CS_ERR_INVALID_ARG;
    const cs_batch& b = *batch;
    const int32_t Hkv = pool->num_kv_heads, D = pool->head_dim;
    // the sequences from the first to the last chunk, from the first to the last single token
    int32_t chunk0 = -1, chunk1 = -1, single0 = -1, single1 = -1;
    for (int32_t s = 0; s < b.num_seqs; ++s) {
        const int32_t ql = b.h_cu_q_lens[s + 1] - b.h_cu_q_lens[s];
        if (ql == 1) { if (single0 < 0) single0 = s; single1 = s + 1; }
        if (ql > 1) { if (chunk0 < 0) chunk0 = s; chunk1 = s + 1; }
    }
    const int32_t base_slot = chunk0 < 0 ? 0 : (b.h_cu_q_lens[chunk0] >> kAppend8SlotShift) + 2 * chunk0;
    const int64_t slots = chunk0 < 0 ? 0 : ((int64_t)(b.h_cu_q_lens[chunk1] >> kAppend8SlotShift) + 2 * chunk1 - base_slot + 7) & ~7ll;
    const int64_t page_blocks = slots * Hkv, waves = kAppend8Threads / 64;
    const int64_t token_blocks = single0 < 0 ? 0 : ((int64_t)(single1 - single0) * Hkv + waves - 1) / waves;
    if ((page_blocks + token_blocks) * kAppend8Threads > 4294967295ll) return CS_ERR_UNSUPPORTED;    // lanes of a launch
    char* base = (char*)pool->base + (int64_t)layer * pool->layer_stride;
#define CS_LAUNCH_APPEND8(ROW, DD)                                                                                      \
    hipLaunchKernelGGL((append8_kernel<ROW, DD>), dim3((uint32_t)(page_blocks + token_blocks)), dim3(kAppend8Threads), 0, (hipStream_t)stream, base, \
                       pool->page_stride, pool->num_pages, Hkv, chunk1, chunk0, base_slot, single0, single1, b.block_tables,     \
                       b.max_blocks_per_seq, b.ctx_lens, b.cu_q_lens, (const uint16_t*)k_new, (const uint16_t*)v_new, (uint32_t)page_blocks);
    if (D == 128) { if (f16) { CS_LAUNCH_APPEND8(RowF16, 128) } else { CS_LAUNCH_APPEND8(RowBf16, 128) } }
    else          { if (f16) { CS_LAUNCH_APPEND8(RowF16, 64) } else { CS_LAUNCH_APPEND8(RowBf16, 64) } }
#undef CS_LAUNCH_APPEND8
    return check_launch("8-bit append kernel");
}

// The plan of an attention call, null where the host has no memory for one (no exception leaves a C entry).
static const Plans* plans8(const cs_batch* b, int32_t Hq, int32_t Hkv, int32_t D) {
    try { return &plans_for(b, Hq, Hkv, D, 1, 1); } catch (const std::bad_alloc&) { return nullptr; }
}

static int attention_kv8(const cs_kv8_pool* pool, int32_t layer, const cs_batch* batch, const void* q, void* out, int32_t Hq, float softmax_scale,
                         void* workspace, size_t workspace_bytes, void* stream, bool f16) {
    int rc = validate_kv8(pool);
    if (rc) return rc;
    if (layer < 0 || layer >= pool->num_layers) return CS_ERR_INVALID_ARG;
    rc = attention_shape_ok(Hq, pool->num_kv_heads, pool->head_dim);
    if (rc) return rc;
    rc = validate_batch(nullptr, batch);
    if (rc) return rc;
    if (batch->num_tokens == 0) return CS_OK;
    if (!q || !out || ((uintptr_t)q & 15) || ((uintptr_t)out & 15)) return CS_ERR_INVALID_ARG;
    if (!(softmax_scale > 0.f) || softmax_scale > 3.0e38f) return CS_ERR_INVALID_ARG;   // positive, finite

    const cs_kv_pool view = kv8_view(*pool);
    const Plans* planned = plans8(batch, Hq, pool->num_kv_heads, pool->head_dim);
    if (!planned) return hip_failed(hipErrorOutOfMemory, "launch plan");
    const Plans& plans = *planned;
    const DecodePlan& d = plans.d;
    const PrefillPlan& p = plans.p;
    if (plans.need > 0 && (!workspace || ((uintptr_t)workspace & 15))) return CS_ERR_INVALID_ARG;
    if (workspace_bytes < plans.need) return CS_ERR_WORKSPACE_TOO_SMALL;
    hipStream_t st = (hipStream_t)stream;
    char* tiles_ws = (char*)workspace + plans.decode_bytes;
    if (plans.f.arrangement != 0) {
        // both kinds of work in one grid, then the merges that the grid does not do itself
        rc = launch_mixed_kv8(view, layer, *batch, d, p, q, out, Hq, softmax_scale, workspace, tiles_ws, st, f16, plans.f.prio,
                              plans.f.arrangement == 2 ? plans.f.persistent_wgs : 0);
        if (rc == CS_OK && p.max_ranges > 1 && !p.merges_in_place)
            rc = launch_prefill_merge(view, LayerSpan{1, 0, 0, 0}, *batch, p, out, Hq, tiles_ws, st, f16);
        if (rc || d.num_multi == 0 || d.merges_in_place) return rc;
        return launch_decode_kv8(view, layer, *batch, d, q, out, Hq, softmax_scale, workspace, st, f16, true);
    }
    if (d.num_prefill > 0) {
        rc = launch_prefill_kv8(view, layer, *batch, p, q, out, Hq, softmax_scale, tiles_ws, st, f16);
        if (rc) return rc;
    }
    return launch_decode_kv8(view, layer, *batch, d, q, out, Hq, softmax_scale, workspace, st, f16, false);
}

}  // namespace cs

using namespace cs;

extern "C" {

size_t cs_kv8_page_bytes(int32_t Hkv, int32_t D) {
    if (Hkv < 1 || Hkv > 65535 || (D != 64 && D != 128)) return 0;
    return ((size_t)scales_offset(Hkv, D) + 8 * (size_t)Hkv + 15) & ~(size_t)15;
}

int cs_kv8_append(const cs_kv8_pool* pool, int32_t layer, const cs_batch* batch, const void* k_new, const void* v_new, void* stream) {
    return append8(pool, layer, batch, k_new, v_new, stream, false);
}

int cs_kv8_append_f16(const cs_kv8_pool* pool, int32_t layer, const cs_batch* batch, const void* k_new, const void* v_new, void* stream) {
    return append8(pool, layer, batch, k_new, v_new, stream, true);
}

size_t cs_paged_attention_kv8_workspace_bytes(const cs_batch* batch, int32_t Hq, int32_t Hkv, int32_t D) {
    if (attention_shape_ok(Hq, Hkv, D) != CS_OK) return 0;
    if (validate_batch(nullptr, batch) != CS_OK || batch->num_seqs == 0) return 0;
    const Plans* plans = plans8(batch, Hq, Hkv, D);
    return plans ? plans->need : 0;
}

int cs_paged_attention_mixed_kv8(const cs_kv8_pool* pool, int32_t layer, const cs_batch* batch, const void* q, void* out, int32_t Hq,
                                 float softmax_scale, void* workspace, size_t workspace_bytes, void* stream) {
    return attention_kv8(pool, layer, batch, q, out, Hq, softmax_scale, workspace, workspace_bytes, stream, false);
}

int cs_paged_attention_mixed_kv8_f16(const cs_kv8_pool* pool, int32_t layer, const cs_batch* batch, const void* q, void* out, int32_t Hq,
                                     float softmax_scale, void* workspace, size_t workspace_bytes, void* stream) {
    return attention_kv8(pool, layer, batch, q, out, Hq, softmax_scale, workspace, workspace_bytes, stream, true);
}

int32_t cs_debug_mixed_kv8(const cs_batch* batch, int32_t Hq, int32_t Hkv, int32_t D, int32_t* ranges) {
    if (attention_shape_ok(Hq, Hkv, D) != CS_OK) return CS_ERR_INVALID_ARG;
    if (validate_batch(nullptr, batch) != CS_OK || batch->num_seqs == 0) return CS_ERR_INVALID_ARG;
    const Plans* plans = plans8(batch, Hq, Hkv, D);
    if (!plans) return hip_failed(hipErrorOutOfMemory, "launch plan");
    if (ranges) *ranges = std::max(plans->p.max_ranges, 1);
    return plans->f.arrangement;
}

int cs_kv8_page_space(const cs_kv8_pool* pool, cs_page_space* space) {
    const int rc = validate_kv8(pool);
    if (rc) return rc;
    if (!space) return CS_ERR_INVALID_ARG;
    *space = cs_page_space{pool->base, pool->num_layers, pool->num_pages, (int64_t)cs_kv8_page_bytes(pool->num_kv_heads, pool->head_dim),
                           pool->layer_stride, pool->page_stride};
    return CS_OK;
}

}  // extern "C"
