// Rows of a quantised KV cache on the device (attn_quant.hip, kvq_copy.hip).
//
// 32 consecutive dims of a row are a block: 32 codes, 8 bits (e4m3) or 4 bits
// (e2m1) each, and one byte b, the power of two 2^(b - 127) that they share
// (the OCP Microscaling formats MXFP8 and MXFP4). A block with largest
// magnitude A is held as
//   b = the smallest with A <= M 2^(b - 127), M = 448 or 6 the largest code,
//       but at least 10;  code = x 2^(127 - b), rounded to nearest, ties to even.
// With that b no code saturates, and A lies in the upper half of the codes'
// range. A power of two makes both directions exact but for that one rounding:
// every value that a block stands for has at most 4 significant bits, a
// magnitude of 2^-126 at least or 0, and so is a bf16 number (but for 2^128, to
// which magnitudes within 2^125 of it may round: infinity); the attention over
// a quantised cache multiplies exactly what is stored. It is also what
// the conversion instructions of gfx950 take (v_cvt_scalef32_pk_*: two values
// and their scale in one instruction).
// A block that holds an infinity or a NaN has b = 255 and codes 0, and reads
// as NaN: neither format has an infinity, and e2m1 has no NaN.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace sangam {

constexpr int kMxBlock = 32;       // dims of a block
constexpr uint32_t kMxNaN = 255u;  // scale byte of a block without values
constexpr uint32_t kMxMinScale = 10u;

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t mx_u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t mx_s16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t mx_u32x4 __attribute__((ext_vector_type(4)));

// (by value: a bit cast of a vector's element in place takes the first one)
__device__ __forceinline__ mx_bf16x2 mx_pair(uint32_t x) { return __builtin_bit_cast(mx_bf16x2, x); }
__device__ __forceinline__ mx_u16x2 mx_halves(uint32_t x) { return __builtin_bit_cast(mx_u16x2, x); }

// Eight codes (a piece of a block) from and to 8 bf16 values.
// 8 bits each
struct MxE4m3 {
    static constexpr int kWords = 2;            // of a piece
    static constexpr uint32_t kTop = 8u;        // the largest code is 1.75 * 2^8
    static constexpr uint32_t kTopBits = 0x60;  // .75 in the 7 fraction bits of a bf16
    static __device__ __forceinline__ mx_u32x4 read(const uint32_t (&c)[2], float scale) {
        return mx_u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], scale, false)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], scale, true)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], scale, false)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], scale, true))};
    }
    static __device__ __forceinline__ void write(uint32_t (&c)[2], mx_u32x4 x, float scale) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            mx_s16x2 p = {0, 0};
            p = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(p, mx_pair(x[2 * w]), scale, false);
            p = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(p, mx_pair(x[2 * w + 1]), scale, true);
            c[w] = __builtin_bit_cast(uint32_t, p);
        }
    }
};

// 4 bits each, the even one of two in the low half of a byte
struct MxE2m1 {
    static constexpr int kWords = 1;
    static constexpr uint32_t kTop = 2u;        // the largest code is 1.5 * 2^2
    static constexpr uint32_t kTopBits = 0x40;
    static __device__ __forceinline__ mx_u32x4 read(const uint32_t (&c)[1], float scale) {
        return mx_u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], scale, 0)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], scale, 1)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], scale, 2)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], scale, 3))};
    }
    static __device__ __forceinline__ void write(uint32_t (&c)[1], mx_u32x4 x, float scale) {
        uint32_t p = 0;
        p = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(p, mx_pair(x[0]), scale, 0);
        p = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(p, mx_pair(x[1]), scale, 1);
        p = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(p, mx_pair(x[2]), scale, 2);
        p = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(p, mx_pair(x[3]), scale, 3);
        c[0] = p;
    }
};

// The largest of the magnitudes of 8 bf16 values and of `m`, as bits (which
// compare as the magnitudes do; NaN above infinity above all numbers).
__device__ __forceinline__ mx_u16x2 mx_largest(mx_u16x2 m, mx_u32x4 x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) m = __builtin_elementwise_max(m, mx_halves(x[e] & 0x7FFF7FFFu));
    return m;
}

// Scale byte of a block whose largest magnitude has the bf16 bits `a`
template <typename Fmt>
__device__ __forceinline__ uint32_t mx_scale(uint32_t a) {
    if (a >= 0x7F80u) return kMxNaN;
    const int b = int(a >> 7) - int(Fmt::kTop) + int((a & 0x7Fu) > Fmt::kTopBits);
    return uint32_t(b > int(kMxMinScale) ? b : int(kMxMinScale));
}
__device__ __forceinline__ float mx_power(uint32_t scale) { return __uint_as_float(scale << 23); }

// 8 values of a block, or their codes
template <typename Fmt>
__device__ __forceinline__ mx_u32x4 mx_read(const uint32_t (&c)[Fmt::kWords], uint32_t scale) {
    return Fmt::read(c, mx_power(scale));  // (NaN for any code under 255: an exponent of all ones is a NaN scale)
}
template <typename Fmt>
__device__ __forceinline__ void mx_write(uint32_t (&c)[Fmt::kWords], mx_u32x4 x, uint32_t scale) {
    Fmt::write(c, x, mx_power(scale));
    if (scale == kMxNaN)
#pragma unroll
        for (int w = 0; w < Fmt::kWords; ++w) c[w] = 0;
}

// One block of a row: as it lies in memory, and its 32 values in four pieces of 8
template <typename Fmt>
struct MxBlock {
    static constexpr int kBytes = 16 * Fmt::kWords;
    mx_u32x4 codes[Fmt::kWords];
    uint32_t scale;

    // block `at` of a tensor's codes and scales
    __device__ __forceinline__ void load(const uint8_t* code, size_t at) {
#pragma unroll
        for (int w = 0; w < Fmt::kWords; ++w) codes[w] = *(const mx_u32x4*)(code + at * kBytes + 16 * w);
    }
    __device__ __forceinline__ void load(const uint8_t* code, const uint8_t* scales, size_t at) {
        load(code, at);
        scale = scales[at];
    }
    __device__ __forceinline__ void store(uint8_t* code, uint8_t* scales, size_t at) const {
#pragma unroll
        for (int w = 0; w < Fmt::kWords; ++w) *(mx_u32x4*)(code + at * kBytes + 16 * w) = codes[w];
        scales[at] = uint8_t(scale);
    }
    __device__ __forceinline__ mx_u32x4 piece(int j) const {
        uint32_t c[Fmt::kWords];
#pragma unroll
        for (int w = 0; w < Fmt::kWords; ++w) c[w] = codes[(j * Fmt::kWords + w) >> 2][(j * Fmt::kWords + w) & 3];
        return mx_read<Fmt>(c, scale);
    }
    __device__ __forceinline__ void quantise(const mx_u32x4 (&x)[4]) {
        mx_u16x2 m = {0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) m = mx_largest(m, x[j]);
        scale = mx_scale<Fmt>(m[0] > m[1] ? m[0] : m[1]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t c[Fmt::kWords];
            mx_write<Fmt>(c, x[j], scale);
#pragma unroll
            for (int w = 0; w < Fmt::kWords; ++w) codes[(j * Fmt::kWords + w) >> 2][(j * Fmt::kWords + w) & 3] = c[w];
        }
    }
};

}  // namespace sangam
