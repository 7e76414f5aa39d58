// Products of matrices in 8-bit floating point: out[m][n] = sum over chunks c of 128 of  sA[m][c] sB[n][c] sum_k a[m][k] b[n][k].
//
// The products of a chunk are summed on the matrix unit, from zero, and the sum is scaled and added in binary32.  The matrix unit's rows are B's (n) and its
// columns A's (m): a lane then holds four neighbouring n of one m, so that A's scale is one number per lane and B's, where 128 rows share it, one per wave.
#include "f8_common.hpp"

namespace nova {

struct F8Call {
    const char *a, *b;
    const float *a_scales, *b_scales;
    const void *bias;
    void *out;
    float *partial;                               // [splits][M][N]
    int64_t ldout;
    int M, N, chunks, splits, split_chunks;
    int a_tiles, b_tiles, a_pitch, b_pitch, a_shift, b_shift;      // panels; scales from chunk to chunk; rows -> scales
    int dtype, flags;
};

__device__ __forceinline__ F8Fragment load_fragment(const char *panel, int lane)
{
    F8Fragment f;
    f.half[0] = *(const uint4v *)(panel + lane * 16);
    f.half[1] = *(const uint4v *)(panel + 1024 + lane * 16);
    return f;
}

template <typename T>
__device__ __forceinline__ void write_four(const F8Call &a, int64_t m, int n, float4v sum)
{
    const int count = min(4, a.N - n);
    T *to = (T *)a.out + m * a.ldout + n;
    T r[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        if (v < count) {
            float s = sum[v];
            if (a.bias) s += load_f32((const T *)a.bias + n + v);
            if (a.flags & NOVA_FLAG_ADD) s += load_f32(to + v);
            if (a.flags & NOVA_FLAG_RELU) s = s < 0.0f ? 0.0f : s;
            store_from_f32(&r[v], s);
        }
    }
    if (count == 4) {
        __builtin_memcpy(to, r, sizeof r);
    } else {
#pragma unroll
        for (int v = 0; v < 3; ++v)
            if (v < count) to[v] = r[v];
    }
}

__device__ __forceinline__ void write_result(const F8Call &a, int64_t m, int n, float4v sum)
{
    if (m >= a.M || n >= a.N) return;
    if (a.dtype == NOVA_F32) write_four<float>(a, m, n, sum);
    else if (a.dtype == NOVA_F16) write_four<f16>(a, m, n, sum);
    else write_four<bf16>(a, m, n, sum);
}

// A wave makes 16 MT x 16 NT results from operands that it loads itself
template <int MT, int NT, int FA, int FB, int WAY>
__global__ void __launch_bounds__(256) f8_wave_kernel(const F8Call a)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, i = lane % 16, b = lane / 16;
    const int across = (a.b_tiles + 4 * NT - 1) / (4 * NT);
    const int split = blockIdx.x % a.splits;
    const unsigned at = blockIdx.x / a.splits;
    const int n_tile = (int)(at % across) * 4 * NT + wave * NT, m_tile = (int)(at / across) * MT;
    if (n_tile >= a.b_tiles) return;
    float4v sum[MT][NT];
#pragma unroll
    for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int y = 0; y < NT; ++y) sum[x][y] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    const int last = min(a.chunks, (split + 1) * a.split_chunks);
    for (int c = split * a.split_chunks; c < last; ++c) {
        F8Input<FA, WAY> fa[MT];
        F8Input<FB, WAY> fb[NT];
        float sa[MT];
        float4v sb[NT];
#pragma unroll
        for (int x = 0; x < MT; ++x) {
            const int tile = min(m_tile + x, a.a_tiles - 1);
            fa[x].set(load_fragment(a.a + ((size_t)tile * a.chunks + c) * kF8PanelBytes, lane));
            sa[x] = a.a_scales[(size_t)c * a.a_pitch + ((tile * 16 + i) >> a.a_shift)];
        }
#pragma unroll
        for (int y = 0; y < NT; ++y) {
            const int tile = min(n_tile + y, a.b_tiles - 1);
            fb[y].set(load_fragment(a.b + ((size_t)tile * a.chunks + c) * kF8PanelBytes, lane));
#pragma unroll
            for (int v = 0; v < 4; ++v) sb[y][v] = a.b_scales[(size_t)c * a.b_pitch + ((tile * 16 + 4 * b + v) >> a.b_shift)];
        }
#pragma unroll
        for (int x = 0; x < MT; ++x)
#pragma unroll
            for (int y = 0; y < NT; ++y) {
                const float4v p = f8_products<FB, FA, WAY>(fb[y], fa[x]);
#pragma unroll
                for (int v = 0; v < 4; ++v) sum[x][y][v] = fma32(sa[x] * sb[y][v], p[v], sum[x][y][v]);
            }
    }
#pragma unroll
    for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int y = 0; y < NT; ++y) {
            const int64_t m = (int64_t)(m_tile + x) * 16 + i;
            const int n = (n_tile + y) * 16 + 4 * b;
            if (a.splits == 1) {
                write_result(a, m, n, sum[x][y]);
            } else if (m < a.M) {
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (n + v < a.N) a.partial[((size_t)split * a.M + m) * a.N + n + v] = sum[x][y][v];
            }
        }
}

// The pieces of a cut sum, in their order
__global__ void __launch_bounds__(256) f8_join_kernel(const F8Call a)
{
    const int groups = (a.N + 3) / 4;
    for (size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x; idx < (size_t)a.M * groups; idx += (size_t)gridDim.x * 256) {
        const int64_t m = idx / groups;
        const int n = (int)(idx % groups) * 4;
        float4v sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int split = 0; split < a.splits; ++split)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (n + v < a.N) sum[v] += a.partial[((size_t)split * a.M + m) * a.N + n + v];
        write_result(a, m, n, sum);
    }
}

struct F8Shape { int mt, splits, split_chunks; };

static F8Shape f8_shape(int M, int N, int K)
{
    F8Shape p;
    const int chunks = K / kF8Chunk + (K % kF8Chunk != 0);
    p.mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    const int64_t blocks = (((int64_t)M + 16 * p.mt - 1) / (16 * p.mt)) * ((N + 127) / 128);
    p.splits = 1;
    while (blocks * p.splits < 1024 && p.splits < 16 && p.splits * 8 <= chunks) p.splits *= 2;
    p.split_chunks = ceil_div(chunks, p.splits);
    p.splits = ceil_div(chunks, p.split_chunks);
    return p;
}

size_t f8_matmul_workspace(int M, int N, int K)
{
    const F8Shape p = f8_shape(M, N, K);
    return p.splits > 1 ? ((size_t)p.splits * M * N * 4 + 255) & ~(size_t)255 : 0;
}

template <int FA, int FB, int WAY>
static int run(const F8Call &a, const F8Shape &p, hipStream_t s)
{
    const int64_t across = (a.b_tiles + 7) / 8;
    const unsigned blocks = (unsigned)(across * ((a.a_tiles + p.mt - 1) / p.mt) * a.splits);
    if (p.mt == 1) f8_wave_kernel<1, 2, FA, FB, WAY><<<blocks, 256, 0, s>>>(a);
    else if (p.mt == 2) f8_wave_kernel<2, 2, FA, FB, WAY><<<blocks, 256, 0, s>>>(a);
    else f8_wave_kernel<4, 2, FA, FB, WAY><<<blocks, 256, 0, s>>>(a);
    NOVA_HIP_TRY(hipGetLastError());
    if (a.splits == 1) return 0;
    const size_t joins = ((size_t)a.M * ((a.N + 3) / 4) + 255) / 256;
    f8_join_kernel<<<(unsigned)(joins < 65536 ? joins : 65536), 256, 0, s>>>(a);
    return (int)hipGetLastError();
}

template <int FA, int FB>
static int run_way(const F8Call &a, const F8Shape &p, void *stream)
{
    return a.dtype == NOVA_F32 ? run<FA, FB, F8_FULL>(a, p, (hipStream_t)stream) : run<FA, FB, F8_NARROW>(a, p, (hipStream_t)stream);
}

int launch_f8_matmul(const F8Operand &a, const F8Operand &b, const void *bias, void *out, int64_t ldout, int dtype, int flags, void *workspace, void *stream)
{
    const F8Layout &la = a.layout, &lb = b.layout;
    const F8Shape p = f8_shape(la.rows, lb.rows, la.columns);
    const F8Call call = {(const char *)a.q, (const char *)b.q, (const float *)((const char *)a.q + la.code_bytes), (const float *)((const char *)b.q + lb.code_bytes),
                         bias, out, (float *)workspace, ldout, la.rows, lb.rows, la.chunks, p.splits, p.split_chunks, la.row_tiles, lb.row_tiles, la.scale_pitch,
                         lb.scale_pitch, la.block == 1 ? 0 : 7, lb.block == 1 ? 0 : 7, dtype, flags};
    if (a.format == NOVA_F8_E4M3)
        return b.format == NOVA_F8_E4M3 ? run_way<NOVA_F8_E4M3, NOVA_F8_E4M3>(call, p, stream) : run_way<NOVA_F8_E4M3, NOVA_F8_E5M2>(call, p, stream);
    return b.format == NOVA_F8_E4M3 ? run_way<NOVA_F8_E5M2, NOVA_F8_E4M3>(call, p, stream) : run_way<NOVA_F8_E5M2, NOVA_F8_E5M2>(call, p, stream);
}

}  // namespace nova
