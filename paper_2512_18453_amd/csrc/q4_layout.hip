// Layers with 4-bit weights: from weights or codes to the layout that the products read (nova_q4_pack in nova.h), and back.  Once per weight set, so
// these are the plain loops over the layout's words and scales: one thread per word of eight codes, one per scale.
#include "q4_common.hpp"

namespace nova {

// Index of the scale of output n and group g
__device__ __forceinline__ size_t q4_scale_index(const Q4Layout &q, int n, int g)
{
    if (q.backward) return (size_t)g * q.scale_pitch + n;
    const int per_chunk = kQ4Chunk / q.group;
    return ((size_t)(n / kQ4Rows) * q.scale_pitch + g / per_chunk * per_chunk) * kQ4Rows + n % kQ4Rows * per_chunk + g % per_chunk;
}

// Scale idx of the layout -> its output and group; false for padding
__device__ __forceinline__ bool q4_scale_at(const Q4Layout &q, size_t idx, int &n, int &g)
{
    if (q.backward) {
        n = (int)(idx % q.scale_pitch);
        g = (int)(idx / q.scale_pitch);
    } else {
        const int per_chunk = kQ4Chunk / q.group;
        const size_t chunk = idx / per_chunk / kQ4Rows;
        n = (int)(chunk / q.chunks) * kQ4Rows + (int)(idx / per_chunk % kQ4Rows);
        g = (int)(chunk % q.chunks) * per_chunk + (int)(idx % per_chunk);
    }
    return n < q.N && g < q.groups;
}

// Scales as given, or of weights: LANES = group / 8 lanes read a group, eight weights each
template <int DT, int LANES>
__global__ void __launch_bounds__(256) q4_scales_kernel(const Storage<DT> *__restrict__ src, Storage<DT> *__restrict__ scales, const Q4Layout q)
{
    const size_t step = (size_t)gridDim.x * (256 / LANES);
    for (size_t idx = (size_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; idx < q.scale_count; idx += step) {
        int n, g;
        const bool real = q4_scale_at(q, idx, n, g);
        if constexpr (LANES == 1) {
            scales[idx] = real ? src[(size_t)n * q.groups + g] : (Storage<DT>)0.0f;
        } else {
            const int lane = threadIdx.x % LANES, first = g * q.group + lane * 8;
            const Eight<Storage<DT>> w = load_eight(src + (size_t)n * q.K + first, real ? q.K - first : 0, first >= 8);
            unsigned largest = 0;                  // as bits: infinity is above every number, NaN above infinity
#pragma unroll
            for (int i = 0; i < 8; ++i) largest = max(largest, __float_as_uint((float)w.v[i]) & 0x7fffffffu);
#pragma unroll
            for (int across = LANES / 2; across; across /= 2) largest = max(largest, (unsigned)__shfl_xor((int)largest, across));
            const float s = largest < 0x7f800000u ? __uint_as_float(largest) / 7.0f : __builtin_nanf("");
            if (lane == 0) scales[idx] = (Storage<DT>)(real ? s : 0.0f);
        }
    }
}

template <int DT, bool QUANTIZE>
__global__ void __launch_bounds__(256) q4_codes_kernel(const void *__restrict__ src, const Storage<DT> *__restrict__ scales, unsigned *__restrict__ words,
                                                       const Q4Layout q)
{
    const size_t total = q.code_bytes / 4;
    for (size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += (size_t)gridDim.x * 256) {
        // the words of a panel in the order in which neighbouring threads read neighbouring weights: along a row forward, across the rows backward
        const int in_panel = idx % 256;
        const int w = q.backward ? in_panel / 64 : in_panel % 4, lane = q.backward ? in_panel % 64 : in_panel / 4;
        const size_t panel = idx / 256;
        const int row = (int)(panel / q.chunks) * kQ4Rows + lane % 16;
        const int first = (int)(panel % q.chunks) * kQ4Chunk + 32 * w + 8 * (lane / 16);
        const int count = row < q.rows ? min(q.reduction - first, 8) : 0;
        typedef std::conditional_t<QUANTIZE, Storage<DT>, int8_t> S;
        S v[8];
        const size_t at = q.backward ? (size_t)first * q.K + row : (size_t)row * q.K + first, step = q.backward ? q.K : 1;
        if (count == 8 && !q.backward) {
            __builtin_memcpy(v, (const S *)src + at, sizeof v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < count ? ((const S *)src)[at + i * step] : (S)0;
        }
        unsigned word = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int code = 0;
            if constexpr (QUANTIZE) {
                if (i < count) {
                    // (eight positions lie in one group forward; backward they are eight outputs of one input)
                    const float s = (float)scales[q4_scale_index(q, q.backward ? first + i : row, (q.backward ? row : first) / q.group)];
                    const float c = s > 0.0f ? rintf((float)v[i] / s) : 0.0f;                                  // s NaN or 0: code 0
                    code = (int)fminf(fmaxf(c, -8.0f), 7.0f);
                }
            } else {
                code = min(max((int)v[i], -8), 7);
            }
            word |= ((unsigned)code & 15u) << (4 * (i / 2) + 16 * (i % 2));
        }
        words[panel * 256 + lane * 4 + w] = word;
    }
}

template <int DT>
__global__ void __launch_bounds__(256) q4_unpack_kernel(const unsigned *__restrict__ words, const Storage<DT> *__restrict__ scales, int8_t *__restrict__ codes,
                                                        Storage<DT> *__restrict__ out_scales, const Q4Layout q)
{
    const size_t total = (size_t)q.N * q.K;
    for (size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += (size_t)gridDim.x * 256) {
        const int n = (int)(idx / q.K), k = (int)(idx % q.K);
        const int row = q.backward ? k : n, pos = q.backward ? n : k;
        const size_t panel = (size_t)(row / kQ4Rows) * q.chunks + pos / kQ4Chunk;
        const int lane = row % 16 + 16 * (pos % 32 / 8), w = pos % kQ4Chunk / 32, v = pos % 8;
        const unsigned word = words[panel * 256 + lane * 4 + w];
        codes[idx] = (int8_t)((int)(word << (28 - 4 * (v / 2) - 16 * (v % 2))) >> 28);
        if (out_scales && k % q.group == 0) out_scales[(size_t)n * q.groups + k / q.group] = scales[q4_scale_index(q, n, k / q.group)];
    }
}

static unsigned q4_blocks(size_t items)
{
    const size_t blocks = (items + 255) / 256;
    return (unsigned)(blocks < 65536 ? blocks : 65536);
}

template <int DT, bool QUANTIZE>
static int lay_out(const void *src, const void *scale_src, const Q4Layout &q, void *Wq, hipStream_t s)
{
    Storage<DT> *scales = (Storage<DT> *)((char *)Wq + q.code_bytes);
    const Storage<DT> *from = (const Storage<DT> *)scale_src;
    if (!QUANTIZE) q4_scales_kernel<DT, 1><<<q4_blocks(q.scale_count), 256, 0, s>>>(from, scales, q);
    else if (q.group == 32) q4_scales_kernel<DT, 4><<<q4_blocks(q.scale_count * 4), 256, 0, s>>>(from, scales, q);
    else if (q.group == 64) q4_scales_kernel<DT, 8><<<q4_blocks(q.scale_count * 8), 256, 0, s>>>(from, scales, q);
    else q4_scales_kernel<DT, 16><<<q4_blocks(q.scale_count * 16), 256, 0, s>>>(from, scales, q);
    NOVA_HIP_TRY(hipGetLastError());
    q4_codes_kernel<DT, QUANTIZE><<<q4_blocks(q.code_bytes / 4), 256, 0, s>>>(src, scales, (unsigned *)Wq, q);
    return (int)hipGetLastError();
}

int launch_q4_quantize(const void *w, const Q4Layout &q, int dtype, void *Wq, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == NOVA_F32) return lay_out<NOVA_F32, true>(w, w, q, Wq, s);
    if (dtype == NOVA_F16) return lay_out<NOVA_F16, true>(w, w, q, Wq, s);
    return lay_out<NOVA_BF16, true>(w, w, q, Wq, s);
}

int launch_q4_pack(const int8_t *codes, const void *scales, const Q4Layout &q, int dtype, void *Wq, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == NOVA_F32) return lay_out<NOVA_F32, false>(codes, scales, q, Wq, s);
    if (dtype == NOVA_F16) return lay_out<NOVA_F16, false>(codes, scales, q, Wq, s);
    return lay_out<NOVA_BF16, false>(codes, scales, q, Wq, s);
}

template <int DT>
static int unpack(const void *Wq, const Q4Layout &q, int8_t *codes, void *scales, hipStream_t s)
{
    q4_unpack_kernel<DT><<<q4_blocks((size_t)q.N * q.K), 256, 0, s>>>((const unsigned *)Wq, (const Storage<DT> *)((const char *)Wq + q.code_bytes), codes,
                                                                      (Storage<DT> *)scales, q);
    return (int)hipGetLastError();
}

int launch_q4_unpack(const void *Wq, const Q4Layout &q, int dtype, int8_t *codes, void *scales, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == NOVA_F32) return unpack<NOVA_F32>(Wq, q, codes, scales, s);
    if (dtype == NOVA_F16) return unpack<NOVA_F16>(Wq, q, codes, scales, s);
    return unpack<NOVA_BF16>(Wq, q, codes, scales, s);
}

}  // namespace nova
