// Element types of the attention kernels.  The pool, Q and the output hold 16-bit floats:
// bf16 (the default) or IEEE half (the precision the paper's system served in, Sec. 6.1).
// Everything that depends on which -- the matrix instructions, the conversion from fp32, the
// widening back, the bit pattern of 1.0 -- is collected here; the copies (append, gather,
// restore) only move 16-bit words and do not care.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cs {

typedef uint32_t e_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t e_u32x2 __attribute__((ext_vector_type(2)));
typedef float e_f32x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
    typedef Bf16 Wide;
    static constexpr bool kEightBit = false;
    static constexpr int kCodes = 0;
    // two e4m3 codes of a dword (the lower or the upper half) times a power of two, exactly
    template <bool kUpper> static __device__ __forceinline__ uint32_t widen(uint32_t codes, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, kUpper));
    }
    static constexpr uint32_t kInfinity = 0x7f80u;                 // a half-word above it, sign aside, is no number
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    static constexpr uint32_t kOnes = 0x3f803f80u;                 // two 1.0
    // 16x16 tile, 32 values of the contraction per call: A and B hold 8 values per lane
    static __device__ __forceinline__ e_f32x4 mfma32(e_u32x4 a, e_u32x4 b, e_f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    // 16 values of the contraction per call: 4 values per lane
    static __device__ __forceinline__ e_f32x4 mfma16(e_u32x2 a, e_u32x2 b, e_f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s4, a), __builtin_bit_cast(s4, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ void unpack(uint32_t w, float& lo, float& hi) {
        lo = __builtin_bit_cast(float, w << 16);
        hi = __builtin_bit_cast(float, w & 0xffff0000u);
    }
    // two floats -> one dword, round to nearest even
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        x2 v = { (__bf16)lo, (__bf16)hi };
        return __builtin_bit_cast(uint32_t, v);
    }
    // exact sum of the two values of a dword
    static __device__ __forceinline__ float sum2(uint32_t w) {
        return __builtin_bit_cast(float, w << 16) + __builtin_bit_cast(float, w & 0xffff0000u);
    }
    // Whether the prefill kernel may scale Q once (by the softmax scale, rounded back to the
    // element type) instead of scaling every score: bf16's 8 mantissa bits do not stand the
    // second rounding on peaked softmaxes (max error 3e-2 to 8e-2 with queries scaled by 4-10).
    static constexpr bool kScaleFoldsIntoQ = false;
    static __device__ __forceinline__ uint32_t scale2(uint32_t w, float f) {
        return pack(__builtin_bit_cast(float, w << 16) * f, __builtin_bit_cast(float, w & 0xffff0000u) * f);
    }
};

struct F16 {
    typedef F16 Wide;
    static constexpr bool kEightBit = false;
    static constexpr int kCodes = 0;
    template <bool kUpper> static __device__ __forceinline__ uint32_t widen(uint32_t codes, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, kUpper));
    }
    static constexpr uint32_t kInfinity = 0x7c00u;
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x4 __attribute__((ext_vector_type(4)));
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    static constexpr uint32_t kOnes = 0x3c003c00u;
    static __device__ __forceinline__ e_f32x4 mfma32(e_u32x4 a, e_u32x4 b, e_f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ e_f32x4 mfma16(e_u32x2 a, e_u32x2 b, e_f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(x4, a), __builtin_bit_cast(x4, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ void unpack(uint32_t w, float& lo, float& hi) {
        const x2 v = __builtin_bit_cast(x2, w);
        lo = (float)v[0];
        hi = (float)v[1];
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        x2 v = { (_Float16)lo, (_Float16)hi };
        return __builtin_bit_cast(uint32_t, v);
    }
    static __device__ __forceinline__ float sum2(uint32_t w) {
        const x2 v = __builtin_bit_cast(x2, w);
        return (float)v[0] + (float)v[1];
    }
    // 11 mantissa bits stand it (max error 6e-3 with queries scaled by 6; one vector instruction
    // less per score)
    static constexpr bool kScaleFoldsIntoQ = true;
    static __device__ __forceinline__ uint32_t scale2(uint32_t w, float f) {
        const x2 v = __builtin_bit_cast(x2, w);
        return pack((float)v[0] * f, (float)v[1] * f);
    }
};

// The same over a pool of 8-bit codes (e4m3) with a power-of-two scale per block: Q, the weights and the
// output are E's, K and V are widened to E on their way into the matrix unit.  Widening is exact: a code has 4
// significant bits, and its scale only moves the exponent (half precision: as far as it reaches down to 2^-24; the
// append keeps values that would round up to 2^16 out).
template <class E> struct Kv8 : E {
    typedef E Wide;
    static constexpr bool kEightBit = true;
    static constexpr int kCodes = E::kInfinity == 0x7f80u ? 2 : 1;     // of a value of Q in prefill (QCodes), or 1: K is widened there
};

// Q as codes, for products with K's codes on the 8-bit matrix instruction (a tile of 16 x 16, 128 values of the contraction, with a scale
// of 2^e for each row and column).  A row of Q is scaled by a power of two to at most 448 and split: its nearest code,
// 16 times what is left of it as a code, and so on.  A code has 4 significant bits and a rest at most half a step of
// the code before, so two codes hold a bf16 (8 bits) without rounding where the first is a normal code: from 2^-13.8 of the row's
// largest value on (2^-6 of 225).  Below that the second code's grid, 2^-9 / 16, rounds: by 2^-14 of 225 at most, 2^-21.8 of the
// row's largest -- what fp32 sums of products with that value round by too, but in a row whose score does not hold
// that product (K is zero there) it is the row's error.  The scales put the parts back in their places.  Two parts take
// as long as the bf16 product of widened codes, without the widening and with half the bytes to read.  (A half has 11 bits: three
// codes, half as long again, and more registers than there are; there K is widened.  1024 tokens on 30720 keys, 64/8 heads, fp16: three
// codes 1016 us, K widened 924; 8 chunks of 2000-2600 on up to 4096, 32/8, 755 and 701.)
// Lane (column head or query = lane%16, group = lane/16) holds features 16*group .. +16 in the operand's lower half, 64 further on in the
// upper one; at head dim 64 the upper half is the next part, over the same codes of K.
typedef int32_t e_i32x8 __attribute__((ext_vector_type(8)));
template <int D, class E>
struct QCodes {
    static constexpr int kParts = 2, kProducts = D == 128 ? kParts : 1;
    e_u32x4 w[kProducts][2];
    uint32_t scale;                                    // byte p: of product p, exponent + 127

    // The codes of the row (zeros if not valid); all lanes take part.
    __device__ __forceinline__ void load(const uint16_t* row, bool valid, int lane) {
        constexpr int kUnits = D / 64;                 // 16 features each
        float x[kUnits * 16], top = 0.f;
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                e_u32x4 v = {0u, 0u, 0u, 0u};
                if (valid) v = *(const e_u32x4*)(row + (u * 4 + (lane >> 4)) * 16 + h * 8);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    E::unpack(v[e], x[u * 16 + h * 8 + 2 * e], x[u * 16 + h * 8 + 2 * e + 1]);
                }
            }
#pragma unroll
        for (int i = 0; i < kUnits * 16; ++i) top = fmaxf(top, fabsf(x[i]));
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const uint32_t bits = __builtin_bit_cast(uint32_t, top);
        const int32_t e = max((int32_t)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), -100);
        const float inv = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
#pragma unroll
        for (int i = 0; i < kUnits * 16; ++i) x[i] = __builtin_fmaf(x[i], inv, x[i] - x[i]);   // (an infinity becomes NaN: its scores are none either)
        const uint32_t e0 = (uint32_t)(e + 127);
        if (D == 128) scale = e0 | (e0 - 4) << 8;
        else scale = lane < 32 ? e0 : e0 - 4;          // of either half: lanes of groups 0-1, 2-3
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                e_u32x4 c;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float* y = x + u * 16 + 4 * i;
                    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
                    const int both = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
                    c[i] = (uint32_t)both;
                    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(both, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(both, true);
                    y[0] = (y[0] - a[0]) * 16.f; y[1] = (y[1] - a[1]) * 16.f;
                    y[2] = (y[2] - b[0]) * 16.f; y[3] = (y[3] - b[1]) * 16.f;
                }
                if (D == 128) w[p][u] = c;
                else w[0][p] = c;
            }
        }
    }

    // acc + K . Q^T of 16 tokens: k0, k1 the lane's codes of K (head dim 64: k0 is k1), k_scale the exponent + 127 of the lane's row.
    __device__ __forceinline__ e_f32x4 dot(e_u32x4 k0, e_u32x4 k1, uint32_t k_scale, e_f32x4 acc) const {
        const e_i32x8 a = join(k0, k1);
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, join(w[0][0], w[0][1]), acc, 0, 0, 0, (int)k_scale, 0, (int)scale);
        if constexpr (kProducts > 1)
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, join(w[1][0], w[1][1]), acc, 0, 0, 0, (int)k_scale, 1, (int)scale);
        return acc;
    }

private:
    static __device__ __forceinline__ e_i32x8 join(e_u32x4 a, e_u32x4 b) {
        return __builtin_bit_cast(e_i32x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

}  // namespace cs
