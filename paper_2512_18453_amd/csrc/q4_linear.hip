// The products of layers with 4-bit weights: y = x W^T (+ bias, ReLU) and the gradient of x, dx = d W.
//
// A workgroup makes 16 rows by 16 columns of the result; its waves share the reduction, a panel of 16 columns by 128 positions (1 KB of codes) at a
// time, and add up through LDS in the order of their numbers.  Codes become operands in registers (q4_common.hpp).
//   forward   a group's products are summed on the matrix unit with the codes as integers and the sum is scaled in binary32
//   backward  the scales run along the reduction, so they go to the other operand: d * s in binary32, in two (three) bfloat16 pieces
#include "q4_common.hpp"

namespace nova {

constexpr int kWaves = 8;

// Operand pieces of eight elements of x: themselves, or three bfloat16 pieces of binary32
template <int DT> constexpr int forward_pieces = DT == NOVA_F32 ? 3 : 1;
template <int DT>
__device__ __forceinline__ void x_fragment(const Eight<Storage<DT>> &e, Fragment (&f)[forward_pieces<DT>])
{
    if constexpr (DT == NOVA_F32) split_fragment<3>(e.v, f);
    else __builtin_memcpy(&f[0], &e, 16);
}

template <bool HALF>
__device__ __forceinline__ Fragment codes_fragment(unsigned word)
{
    if constexpr (HALF) return codes_to_f16(word);
    else return codes_to_bf16_over_16(word);
}

// The waves' sums of a 16 x 16 tile, added in order; thread t < 256 gets row t / 16, column t % 16
__device__ __forceinline__ float sum_of_waves(float4v acc, float (*parts)[256])
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (int i = 0; i < 4; ++i) parts[wave][(lane / 16 * 4 + i) * 16 + lane % 16] = acc[i];
    __syncthreads();
    float sum = 0.0f;
    if (threadIdx.x < 256)
        for (int w = 0; w < kWaves; ++w) sum += parts[w][threadIdx.x];
    return sum;
}

template <int DT, int GROUP>
__global__ void __launch_bounds__(kWaves * 64)
q4_linear_kernel(const Storage<DT> *__restrict__ x, int64_t ldx, const char *__restrict__ Wq, const Storage<DT> *__restrict__ bias,
                 Storage<DT> *__restrict__ y, int64_t ldy, int M, const Q4Layout q, int relu)
{
    constexpr bool HALF = DT == NOVA_F16;
    constexpr int P = forward_pieces<DT>;
    __shared__ float parts[kWaves][256];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int tile = blockIdx.x % q.row_tiles, m0 = blockIdx.x / q.row_tiles * 16;
    const int m = m0 + lane % 16;
    const Storage<DT> *scales = (const Storage<DT> *)(Wq + q.code_bytes) + (size_t)tile * q.scale_pitch * kQ4Rows + lane % 16;
    float4v acc = {0, 0, 0, 0}, part;
    for (int c = wave; c < q.chunks; c += kWaves) {
        const uint4v codes = *(const uint4v *)(Wq + ((size_t)tile * q.chunks + c) * kQ4PanelBytes + lane * 16);
        for (int w = 0; w < 4; ++w) {
            const int k = c * kQ4Chunk + w * 32 + lane / 16 * 8;
            Fragment a[P];
            x_fragment<DT>(load_eight(x + (int64_t)m * ldx + k, m < M ? q.K - k : 0), a);
            const Fragment b = codes_fragment<HALF>(codes[w]);
            if (w * 32 % GROUP == 0) part = (float4v){0, 0, 0, 0};
#pragma unroll
            for (int p = 0; p < P; ++p) part = mfma<HALF>(a[p], b, part);
            if ((w + 1) * 32 % GROUP == 0) {
                const float s = (float)scales[(size_t)(c * (kQ4Chunk / GROUP) + w * 32 / GROUP) * kQ4Rows] * (HALF ? 1.0f : kCodeUnit);
                for (int i = 0; i < 4; ++i) acc[i] = fma32(s, part[i], acc[i]);
            }
        }
    }
    float sum = sum_of_waves(acc, parts);
    const int row = m0 + threadIdx.x / 16, n = tile * 16 + threadIdx.x % 16;
    if (threadIdx.x < 256 && row < M && n < q.N) {
        if (bias) sum += load_f32(bias + n);
        if (relu) sum = sum < 0.0f ? 0.0f : sum;
        store_from_f32(y + (int64_t)row * ldy + n, sum);
    }
}

template <int DT>
__global__ void __launch_bounds__(kWaves * 64)
q4_backward_kernel(const Storage<DT> *__restrict__ dy, int64_t lddy, const Storage<DT> *__restrict__ y, int64_t ldy, const char *__restrict__ Wq,
                   Storage<DT> *__restrict__ dx, int64_t lddx, int M, const Q4Layout q)
{
    constexpr int P = DT == NOVA_F32 ? 3 : 2;
    __shared__ float parts[kWaves][256];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int tile = blockIdx.x % q.row_tiles, m0 = blockIdx.x / q.row_tiles * 16;
    const int m = m0 + lane % 16;
    const Storage<DT> *scales = (const Storage<DT> *)(Wq + q.code_bytes) + (size_t)(tile * 16 / q.group) * q.scale_pitch;
    float4v acc = {0, 0, 0, 0};
    for (int c = wave; c < q.chunks; c += kWaves) {
        const uint4v codes = *(const uint4v *)(Wq + ((size_t)tile * q.chunks + c) * kQ4PanelBytes + lane * 16);
        for (int w = 0; w < 4; ++w) {
            const int n = c * kQ4Chunk + w * 32 + lane / 16 * 8, count = m < M ? q.N - n : 0;
            const Eight<Storage<DT>> d = load_eight(dy + (int64_t)m * lddy + n, count);
            const Eight<Storage<DT>> s = load_eight(scales + n, 8);
            float v[8];
            for (int i = 0; i < 8; ++i) v[i] = (float)d.v[i] * ((float)s.v[i] * kCodeUnit);
            if (y) {
                const Eight<Storage<DT>> r = load_eight(y + (int64_t)m * ldy + n, count);
                for (int i = 0; i < 8; ++i) v[i] = (float)r.v[i] > 0.0f ? v[i] : 0.0f;
            }
            Fragment a[P];
            split_fragment<P>(v, a);
            const Fragment b = codes_to_bf16_over_16(codes[w]);
#pragma unroll
            for (int p = P - 1; p >= 0; --p) acc = mfma<false>(a[p], b, acc);
        }
    }
    const float sum = sum_of_waves(acc, parts);
    const int row = m0 + threadIdx.x / 16, k = tile * 16 + threadIdx.x % 16;
    if (threadIdx.x < 256 && row < M && k < q.K) store_from_f32(dx + (int64_t)row * lddx + k, sum);
}

size_t q4_linear_workspace(int, const Q4Layout &, int) { return 0; }

// Rows in pieces that keep a launch below 2^31 threads
template <typename F>
static int in_row_pieces(int M, const Q4Layout &q, F &&launch)
{
    int64_t tiles = ((int64_t)1 << 31) / (kWaves * 64) / q.row_tiles;
    if (tiles < 1) tiles = 1;
    for (int64_t m0 = 0; m0 < M; m0 += tiles * 16) {
        const int rows = (int)(M - m0 < tiles * 16 ? M - m0 : tiles * 16);
        launch(m0, rows, (unsigned)(ceil_div(rows, 16) * (int64_t)q.row_tiles));
        NOVA_HIP_TRY(hipGetLastError());
    }
    return 0;
}

template <int DT, int GROUP>
static int linear(const void *x, int64_t ldx, const void *Wq, const void *bias, void *y, int64_t ldy, int M, const Q4Layout &q, int relu, hipStream_t s)
{
    return in_row_pieces(M, q, [&](int64_t m0, int rows, unsigned blocks) {
        q4_linear_kernel<DT, GROUP><<<blocks, kWaves * 64, 0, s>>>((const Storage<DT> *)x + m0 * ldx, ldx, (const char *)Wq, (const Storage<DT> *)bias,
                                                                   (Storage<DT> *)y + m0 * ldy, ldy, rows, q, relu);
    });
}

template <int DT>
static int linear_of_type(const void *x, int64_t ldx, const void *Wq, const void *bias, void *y, int64_t ldy, int M, const Q4Layout &q, int relu,
                          hipStream_t s)
{
    if (q.group == 32) return linear<DT, 32>(x, ldx, Wq, bias, y, ldy, M, q, relu, s);
    if (q.group == 64) return linear<DT, 64>(x, ldx, Wq, bias, y, ldy, M, q, relu, s);
    return linear<DT, 128>(x, ldx, Wq, bias, y, ldy, M, q, relu, s);
}

int launch_q4_linear(const void *x, int64_t ldx, const void *Wq, const void *bias, void *y, int64_t ldy, int M, const Q4Layout &q, int dtype, int flags,
                     void *, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    const int relu = (flags & NOVA_FLAG_RELU) != 0;
    if (dtype == NOVA_F32) return linear_of_type<NOVA_F32>(x, ldx, Wq, bias, y, ldy, M, q, relu, s);
    if (dtype == NOVA_F16) return linear_of_type<NOVA_F16>(x, ldx, Wq, bias, y, ldy, M, q, relu, s);
    return linear_of_type<NOVA_BF16>(x, ldx, Wq, bias, y, ldy, M, q, relu, s);
}

template <int DT>
static int backward_of_type(const void *dy, int64_t lddy, const void *y, int64_t ldy, const void *Wq, void *dx, int64_t lddx, int M, const Q4Layout &q,
                            hipStream_t s)
{
    return in_row_pieces(M, q, [&](int64_t m0, int rows, unsigned blocks) {
        q4_backward_kernel<DT><<<blocks, kWaves * 64, 0, s>>>((const Storage<DT> *)dy + m0 * lddy, lddy, y ? (const Storage<DT> *)y + m0 * ldy : nullptr,
                                                              ldy, (const char *)Wq, (Storage<DT> *)dx + m0 * lddx, lddx, rows, q);
    });
}

int launch_q4_linear_backward(const void *dy, int64_t lddy, const void *y, int64_t ldy, const void *Wq, void *dx, int64_t lddx, int M, const Q4Layout &q,
                              int dtype, void *, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == NOVA_F32) return backward_of_type<NOVA_F32>(dy, lddy, y, ldy, Wq, dx, lddx, M, q, s);
    if (dtype == NOVA_F16) return backward_of_type<NOVA_F16>(dy, lddy, y, ldy, Wq, dx, lddx, M, q, s);
    return backward_of_type<NOVA_BF16>(dy, lddy, y, ldy, Wq, dx, lddx, M, q, s);
}

}  // namespace nova
