// Quotients by one scale, as quantisation to 8-bit floating point needs them.  Plain C++ (constexpr functions serve the kernels too), so that f8_quotient_selftest.cpp can
// compare them with divisions on the CPU.
#pragma once

namespace nova {

// With the scale's inverse r, rounded, and a first quotient q = v r, q + (v - q s) r is v / s rounded once wherever that decides a code: f8_quotient_selftest.cpp compares it with
// the division for every significand of s and all v next to a border between codes, and the codes for scales of every exponent and for random pairs.  Values and scale are moved
// by a power of two first where something on the way could be subnormal that matters.  Six instructions with the code's bound, none of them a branch, where a division is ten.
// (A template, because a compiler may refuse a constexpr function that no constant expression can call.)
template <typename Float>
struct F8Divisor {
    Float scale, inverse, factor;
    constexpr explicit F8Divisor(Float s)
        : scale(s * factor_of(s)), inverse((Float)1 / scale), factor(factor_of(s)) {}
    static constexpr Float factor_of(Float s) { return s < (Float)0x1p-60 ? (Float)0x1p100 : s > (Float)0x1p100 ? (Float)0x1p-100 : (Float)1; }
    constexpr Float quotient(Float v) const
    {
        const Float moved = v * factor, q = moved * inverse;
        return __builtin_copysignf(__builtin_fmaf(__builtin_fmaf(-q, scale, moved), inverse, q), v);          // (a remainder of 0 makes -0 to 0)
    }
};

}  // namespace nova
