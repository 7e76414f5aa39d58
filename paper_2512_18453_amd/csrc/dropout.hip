// Dropout whose mask is a function of (seed, offset, row, column) and is never stored, and its gradient.
//
// Random words: Philox 4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; SC 2011).  One block of four words serves eight
// elements, 16 bits each; only where those 16 bits equal the threshold's upper 16 does the decision need the other 16, from a second block.
#include "q4_common.hpp"

namespace nova {

struct Words { unsigned w[4]; };

__device__ __forceinline__ unsigned xor3(unsigned a, unsigned b, unsigned c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

__device__ __forceinline__ Words philox(unsigned c0, unsigned c1, unsigned c2, unsigned c3, uint64_t seed)
{
    unsigned k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        const unsigned n0 = xor3((unsigned)(b >> 32), c1, k0), n2 = xor3((unsigned)(a >> 32), c3, k1);
        c0 = n0; c1 = (unsigned)b; c2 = n2; c3 = (unsigned)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// 8192 x 8192 in binary16, 10 % dropped: with a residual 64 us (403 MB, 6.3 TB/s; 85 where the results did not go past the caches), the gradient 60.5 with a third less to
// move: there the arithmetic of the words binds, some 230 instructions of a lane for eight elements.  Two groups per thread and turn, and workgroups that keep to one
// row, so that its addresses are the wave's, were slower (with the residual 86 and 70).
template <int DT>
__global__ void __launch_bounds__(256) dropout_kernel(const DropoutArgs a)
{
    typedef Storage<DT> T;
    typedef unsigned Stored __attribute__((ext_vector_type(sizeof(Eight<T>) / 4), aligned(sizeof(T))));
    const uint64_t offset = a.offset + (a.device_offset ? *a.device_offset : 0);
    const unsigned groups = ((unsigned)a.columns + 7) / 8;
    const uint64_t total = (uint64_t)a.rows * groups;
    const unsigned upper = (unsigned)(a.threshold >> 16), lower = (unsigned)(a.threshold & 0xffff);      // upper: up to 65536
    for (uint64_t idx = (uint64_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += (uint64_t)gridDim.x * 256) {
        const unsigned row = total >> 32 ? (unsigned)(idx / groups) : (unsigned)idx / groups, group = (unsigned)idx - row * groups;          // (the lower words)
        const int64_t column = (int64_t)group * 8;
        const int count = (int)min((int64_t)8, a.columns - column);
        const Eight<T> x = load_eight((const T *)a.x + row * a.ldx + column, count, column >= 8);
        Eight<T> other = {};
        if (a.residual) other = load_eight((const T *)a.residual + row * a.ldresidual + column, count, column >= 8);
        if (a.gate) other = load_eight((const T *)a.gate + row * a.ldgate + column, count, column >= 8);
        const Words bits = philox(group, row, (unsigned)offset, (unsigned)(offset >> 32), a.seed);
        // halves equal to the threshold's upper one: zeros among the differences' halves (a carry may find one too many, which costs time only)
        unsigned ties = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const unsigned difference = bits.w[w] ^ upper * 0x10001u;
            ties |= (difference - 0x10001u) & ~difference;
        }
        Words more = {{~0u, ~0u, ~0u, ~0u}};
        if (lower && (ties & 0x80008000u)) more = philox(group, row | 0x80000000u, (unsigned)offset, (unsigned)(offset >> 32), a.seed);
        Eight<T> y;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const unsigned half = bits.w[e / 2] >> (16 * (e % 2)) & 0xffff;
            bool keep = half > upper || (half == upper && (more.w[e / 2] >> (16 * (e % 2)) & 0xffff) >= lower);
            float v = (float)x.v[e];
            if (a.relu) v = v < 0.0f ? 0.0f : v;
            if (a.gate) keep = keep && (float)other.v[e] > 0.0f;
            v = keep ? v * a.factor : 0.0f;
            if (a.residual) v += (float)other.v[e];
            store_from_f32(&y.v[e], v);
        }
        T *const to = (T *)a.y + row * a.ldy + column;
        if (count == 8) {
            Stored whole;
            __builtin_memcpy(&whole, &y, sizeof y);
            __builtin_nontemporal_store(whole, (Stored *)to);
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < count) to[e] = y.v[e];
        }
    }
}

int launch_dropout(const DropoutArgs &a, int dtype, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    const uint64_t blocks = ((uint64_t)a.rows * (((unsigned)a.columns + 7) / 8) + 255) / 256;
    const unsigned grid = (unsigned)(blocks < (1 << 22) ? blocks : 1 << 22);
    if (dtype == NOVA_F32) dropout_kernel<NOVA_F32><<<grid, 256, 0, s>>>(a);
    else if (dtype == NOVA_F16) dropout_kernel<NOVA_F16><<<grid, 256, 0, s>>>(a);
    else dropout_kernel<NOVA_BF16><<<grid, 256, 0, s>>>(a);
    return (int)hipGetLastError();
}

}  // namespace nova
