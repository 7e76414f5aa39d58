// Device-side pieces shared by the kernels of layers with 4-bit weights: the storage types by dtype code, and codes -> operands of the matrix unit.
#pragma once
#include "device_common.hpp"

namespace nova {

template <int DT> struct StorageOf;
template <> struct StorageOf<NOVA_F32> { typedef float type; };
template <> struct StorageOf<NOVA_F16> { typedef f16 type; };
template <> struct StorageOf<NOVA_BF16> { typedef bf16 type; };
template <int DT> using Storage = typename StorageOf<DT>::type;

typedef f16 half2v __attribute__((ext_vector_type(2)));
typedef f16 half8 __attribute__((ext_vector_type(8)));
typedef bf16 bhalf8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));
typedef unsigned short ushort8 __attribute__((ext_vector_type(8)));

// One operand of v_mfma_f32_16x16x32: lane 16 b + i holds row (column) i at positions 8 b .. 8 b + 7 of the sum.
union Fragment {
    unsigned words[4];
    uint4v vec;
    half8 h;
    bhalf8 b;
};

template <bool HALF>
__device__ __forceinline__ float4v mfma(const Fragment &a, const Fragment &b, float4v c)
{
    if constexpr (HALF) return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, b.h, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.b, b.b, c, 0, 0, 0);
}

// Eight codes of a word as binary16: the code with its sign bit flipped (c + 8) under the exponent of 1024 is 1024 + c + 8; 1032 comes off exactly.  One place
// higher it is 1024 + 16 (c + 8), of which a sixteenth less 72 is c.  Nine instructions: (w & a) ^ b is one if a and b are in vector registers (an
// instruction reads one scalar register at most), so a kernel puts the constants there once.
struct F16Codes {
    unsigned low, low_base, high, high_base;
    half2v sixteenth, offset, high_offset;

    static __device__ __forceinline__ unsigned in_vector(unsigned constant)
    {
        unsigned v;
        asm volatile("v_mov_b32 %0, %1" : "=v"(v) : "s"(constant));
        return v;
    }
    __device__ __forceinline__ F16Codes()
        : low(in_vector(0x000f000fu)), low_base(in_vector(0x64086408u)), high(in_vector(0x00f000f0u)), high_base(in_vector(0x64806480u)),
          sixteenth(__builtin_bit_cast(half2v, in_vector(0x2c002c00u))), offset(__builtin_bit_cast(half2v, in_vector(0xe408e408u))),
          high_offset(__builtin_bit_cast(half2v, in_vector(0xd480d480u)))
    {
    }
    __device__ __forceinline__ Fragment operator()(unsigned word) const
    {
        Fragment f;
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            const unsigned w = word >> (4 * j);
            f.words[j] = __builtin_bit_cast(unsigned, __builtin_bit_cast(half2v, (w & low) ^ low_base) + offset);
            f.words[j + 1] = __builtin_bit_cast(unsigned, __builtin_elementwise_fma(__builtin_bit_cast(half2v, (w & high) ^ high_base), sixteenth, high_offset));
        }
        return f;
    }
};

// ... as bfloat16, divided by 16: v_cvt_off_f32_i4 makes c / 16 of the low four bits of a byte (exact in bfloat16: 3 bits), and the high halves of two such
// binary32 values are the pair.  Thirteen instructions.
constexpr float kCodeUnit = 16.0f;
struct Bf16Codes {
    __device__ __forceinline__ Fragment operator()(unsigned word) const
    {
        Fragment f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned w = word >> (4 * (j % 2));
            const float even = __builtin_amdgcn_cvt_off_f32_i4((int)((w >> (8 * (j / 2))) & 0xff));
            const float odd = __builtin_amdgcn_cvt_off_f32_i4((int)((w >> (8 * (j / 2) + 16)) & 0xff));
            f.words[j] = __builtin_amdgcn_perm(__float_as_uint(odd), __float_as_uint(even), 0x07060302u);
        }
        return f;
    }
};

// Eight binary32 values as PIECES operands of bfloat16 whose sum they are: each piece but the last is the value cut off behind 8 bits of mantissa, so the
// rest is exact (and an infinity is all in the first piece); the last is the rest rounded.  Two pieces: within 2^-15 of the value; three: all of it, where it
// is 2^-109 or more (the last place of a piece is 2^-133 at the lowest).
typedef float float2v __attribute__((ext_vector_type(2)));
typedef bf16 bhalf2 __attribute__((ext_vector_type(2)));
template <int PIECES>
__device__ __forceinline__ void split_fragment(const float (&v)[8], Fragment (&f)[PIECES])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float even = v[2 * j], odd = v[2 * j + 1];
#pragma unroll
        for (int p = 0; p < PIECES - 1; ++p) {
            f[p].words[j] = __builtin_amdgcn_perm(__float_as_uint(odd), __float_as_uint(even), 0x07060302u);
            const float even_cut = __uint_as_float(__float_as_uint(even) & 0xffff0000u), odd_cut = __uint_as_float(__float_as_uint(odd) & 0xffff0000u);
            even = even == even_cut ? 0.0f : even - even_cut;
            odd = odd == odd_cut ? 0.0f : odd - odd_cut;
        }
        const float2v rest = {even, odd};
        f[PIECES - 1].words[j] = __builtin_bit_cast(unsigned, __builtin_convertvector(rest, bhalf2));
    }
}

// `count` consecutive elements from p on, at most 8; those behind them are zero.  The rows of a caller's matrix begin anywhere, so the 16- and 32-byte loads
// are unaligned ones.  Fewer than 8 are the end of what a load of the 8 up to there brings, if `before` says that 8 - count elements before p are the
// caller's as well.
template <typename T>
struct Eight { T v[8]; };
template <typename T>
__device__ __forceinline__ Eight<T> load_eight(const T *p, int count, bool before = false)
{
    Eight<T> e;
    if (count >= 8) {
        __builtin_memcpy(&e, p, sizeof e);
    } else if (sizeof(T) == 2 && before) {
        unsigned __int128 bits = 0;
        if (count > 0) {
            __builtin_memcpy(&bits, p + count - 8, sizeof bits);
            bits >>= 16 * (8 - count);
        }
        __builtin_memcpy(&e, &bits, sizeof e);
    } else {
#pragma unroll
        for (int v = 0; v < 8; ++v) e.v[v] = v < count ? p[v] : (T)0.0f;
    }
    return e;
}

}  // namespace nova
