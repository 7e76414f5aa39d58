// Device-side pieces shared by the kernels of matrices in 8-bit floating point.
#pragma once
#include "f8_quotient.hpp"
#include "q4_common.hpp"

namespace nova {

// One operand of v_mfma_f32_16x16x128: lane 16 b + i holds row (column) i at 32 of the 128 positions of the sum.  Which 32 is the layout's choice, as long as
// both operands make the same one.
typedef int int8v __attribute__((ext_vector_type(8)));
union F8Fragment {
    uint4v half[2];
    int8v vec;
};

template <int FORMAT> constexpr float kLargestCode = FORMAT == NOVA_F8_E4M3 ? 448.0f : 57344.0f;

// Two ways to sum the 128 products of a chunk.
//   NARROW  on the codes themselves, at the matrix unit's full rate.  Of eight neighbouring products it cuts everything off, toward zero, below 2^-13 of the largest product
//           of the two codes' powers of two (subnormal codes count as the lowest normal ones), and adds such groups up in 24 bits.  That is 1.45e-5 of the sum's root mean
//           square on normal data, 3e-5 with a column in 200 20 times as large as the others, 5.4e-5 with 100 times, up to 7e-5 on log-normal magnitudes in E5M2: 0.07,
//           0.15, 0.26 and 0.35 of the root mean square of rounding to binary16, 0.01 to 0.05 of bfloat16's.  At the worst 7 2^-13 of that largest product per eight, all
//           of a sum where large products cancel.  For results in 16 bits of more than 64 rows, where the full way would take twice the time (8192 x 8192 x 8192 440 -> 883 us).
//   FULL    on the codes as binary16 numbers, which hold both formats' exactly, at half that rate: 1e-8 of the sum, as binary32 has it.  For results in binary32, and for up to
//           64 rows in every type, where the codes' bytes bind.
enum { F8_NARROW = 0, F8_FULL = 1 };

template <int FORMAT>
__device__ __forceinline__ half2v f16_pair(unsigned word, bool upper)
{
    if constexpr (FORMAT == NOVA_F8_E4M3)
        return upper ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, 1.0f, false);
    else
        return upper ? __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(word, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(word, 1.0f, false);
}

// A fragment as the matrix unit takes it
template <int FORMAT, int WAY>
struct F8Input {
    int8v codes;
    __device__ __forceinline__ void set(const F8Fragment &f) { codes = f.vec; }
};
template <int FORMAT>
struct F8Input<FORMAT, F8_FULL> {
    Fragment quarter[4];
    __device__ __forceinline__ void set(const F8Fragment &f)
    {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const unsigned word = (unsigned)f.vec[q];
            quarter[q / 2].words[q % 2 * 2] = __builtin_bit_cast(unsigned, f16_pair<FORMAT>(word, false));
            quarter[q / 2].words[q % 2 * 2 + 1] = __builtin_bit_cast(unsigned, f16_pair<FORMAT>(word, true));
        }
    }
};

// 16 x 16 sums over the 128 products of two fragments; lane 16 b + i gets those of row 4 b + v, column i, v = 0 .. 3
template <int FA, int FB, int WAY>
__device__ __forceinline__ float4v f8_products(const F8Input<FA, WAY> &a, const F8Input<FB, WAY> &b)
{
    float4v sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (WAY == F8_NARROW) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.codes, b.codes, sum, FA == NOVA_F8_E5M2, FB == NOVA_F8_E5M2, 0, 0, 0, 0);
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) sum = mfma<true>(a.quarter[q], b.quarter[q], sum);
        return sum;
    }
}

// Four binary32 values as four codes, rounded to nearest, ties to even
template <int FORMAT>
__device__ __forceinline__ unsigned f8_codes(float a, float b, float c, float d)
{
    if constexpr (FORMAT == NOVA_F8_E4M3)
        return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
    else
        return __builtin_amdgcn_cvt_pk_bf8_f32(c, d, __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false), true);
}

// Largest magnitude as bits (infinity is above every number, NaN above infinity) -> scale; a block that holds one of them has scale NaN
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
template <int FORMAT>
__device__ __forceinline__ float scale_of(unsigned bits)
{
    return bits < 0x7f800000u ? __uint_as_float(bits) / kLargestCode<FORMAT> : __builtin_nanf("");
}

// Codes of quotients by one scale as nova.h defines them: divided in binary32, kept within the largest code (a scale that is subnormal can be too small by half); 0 for
// scales of 0 and NaN.
template <int FORMAT>
struct F8Encoder : F8Divisor<float> {
    __device__ __forceinline__ explicit F8Encoder(float s) : F8Divisor<float>(s) {}
    __device__ __forceinline__ float kept(float v) const { return __builtin_amdgcn_fmed3f(quotient(v), -kLargestCode<FORMAT>, kLargestCode<FORMAT>); }
    // eight codes, in two words
    __device__ __forceinline__ void encode(const float (&v)[8], unsigned (&words)[2]) const
    {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const unsigned codes = f8_codes<FORMAT>(kept(v[4 * w]), kept(v[4 * w + 1]), kept(v[4 * w + 2]), kept(v[4 * w + 3]));
            words[w] = scale > 0.0f ? codes : 0;
        }
    }
    // two, in 16 bits
    __device__ __forceinline__ void encode(const float (&v)[2], uint16_t &half) const
    {
        const unsigned codes = f8_codes<FORMAT>(kept(v[0]), kept(v[1]), 0.0f, 0.0f);
        half = scale > 0.0f ? (uint16_t)codes : 0;
    }
};

// The largest value over the 16 lanes of a row of the wave
__device__ __forceinline__ unsigned largest_of_16(unsigned v)
{
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false));      // rotations by 8, 4, 2, 1
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, false));
    return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, false));
}

}  // namespace nova
