// Matrices in 8-bit floating point: from rows of numbers to the layout that the products read (nova_f8_quantize in nova.h), from codes, and back.
//
// A workgroup takes 128 x 128 elements of the source, a thread 8 x 8 of them, and holds them in registers: what is largest in a row, a column or all of them
// is known before any is divided, and one read serves the layout of the rows, of the columns, and the columns' sums.  Codes go through LDS, where they are put
// in the panels' order, so that memory sees whole 16-byte pieces side by side.
#include "f8_common.hpp"

namespace nova {

constexpr int kTile = 128;

struct F8Quantize {
    F8Source src;
    char *rows_q, *columns_q;                     // layouts of the source and of its transpose; either may be null
    float *partial;                               // sums of the columns over 128 rows, or null
    int add;                                      // ... added to what is there
    F8Layout rows_layout, columns_layout;
    int tiles_across;
    int64_t tiles;
};

__device__ __forceinline__ float *f8_scales(char *q, const F8Layout &layout) { return (float *)(q + layout.code_bytes); }

// A tile's codes from LDS to the panels row_tile .. of a chunk
__device__ __forceinline__ void write_panels(const uint4v *staged, char *q, const F8Layout &layout, int row_tile, int chunk)
{
    for (int piece = threadIdx.x; piece < kTile * kTile / 16; piece += 256) {
        const int r = row_tile + piece / 128;
        if (r < layout.row_tiles) *(uint4v *)(q + ((size_t)r * layout.chunks + chunk) * kF8PanelBytes + piece % 128 * 16) = staged[piece];
    }
}

// Eight columns of COUNT rows from row on, STEP apart, `count` of which exist; elements whose gate is closed, and rows and columns behind the last, are zero.  (Rows behind
// the last are read from it, so that the loads of a thread are in one piece of code and wait together: 32 rows' transpose 14.2 us with a branch each.)
template <typename T, int COUNT, int STEP, bool GATED>
__device__ __forceinline__ void load_rows(const F8Source &src, int64_t row, int64_t column, float (&v)[COUNT][8])
{
    const int count = (int)min((int64_t)8, src.columns - column);
    Eight<T> x[COUNT], gate[COUNT];
    if (count == 8) {
#pragma unroll
        for (int k = 0; k < COUNT; ++k) {
            const int64_t r = min(row + k * STEP, (int64_t)src.rows - 1);
            __builtin_memcpy(&x[k], (const T *)src.x + r * src.ld + column, sizeof x[k]);
            if (GATED && src.gate) __builtin_memcpy(&gate[k], (const T *)src.gate + r * src.ldgate + column, sizeof x[k]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < COUNT; ++k) {
            const int64_t r = min(row + k * STEP, (int64_t)src.rows - 1);
            x[k] = load_eight((const T *)src.x + r * src.ld + column, count);
            if (GATED && src.gate) gate[k] = load_eight((const T *)src.gate + r * src.ldgate + column, count);
        }
    }
#pragma unroll
    for (int k = 0; k < COUNT; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool open = row + k * STEP < src.rows && !(GATED && src.gate && !((float)gate[k].v[e] > 0.0f));
            v[k][e] = open ? (float)x[k].v[e] : 0.0f;
        }
}

// A scale per row and chunk, and nothing but the rows' layout: a panel is one wave's
template <int DT, int FORMAT>
__global__ void __launch_bounds__(256) f8_quantize_rows_kernel(const F8Quantize a)
{
    typedef Storage<DT> T;
    __shared__ uint4v staged[4][kF8PanelBytes / 16];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, j = lane % 16, g = lane / 16;
    const F8Layout &q = a.rows_layout;
    const size_t panels = (size_t)q.row_tiles * q.chunks;
    for (size_t panel = (size_t)blockIdx.x * 4 + wave; panel < panels; panel += (size_t)gridDim.x * 4) {
        const int chunk = (int)(panel % q.chunks);
        const int64_t row = (int64_t)(panel / q.chunks) * kF8Rows + g;
        const int64_t column = (int64_t)chunk * kF8Chunk + 8 * j;
        float v[4][8];
        load_rows<T, 4, 4, false>(a.src, row, column, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            unsigned m = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max(m, magnitude(v[k][e]));
            const float s = scale_of<FORMAT>(largest_of_16(m));
            unsigned words[2];
            F8Encoder<FORMAT>(s).encode(v[k], words);
            __builtin_memcpy((uint64_t *)staged[wave] + (j / 2 % 2 * 1024 + (j / 4 * 16 + 4 * k + g) * 16 + j % 2 * 8) / 8, words, 8);
            if (j == 0) f8_scales(a.rows_q, q)[(size_t)chunk * q.scale_pitch + row + 4 * k] = s;
        }
        exchange_in_wave();
        uint4v *const to = (uint4v *)(a.rows_q + panel * kF8PanelBytes);
        to[lane] = staged[wave][lane];
        to[lane + 64] = staged[wave][lane + 64];
        exchange_in_wave();
    }
}

// BLOCK: 1 or 128.  WHAT: the rows' layout, the columns', or what there is of them and of the columns' sums, behind a gate if there is one
enum { F8_ROWS, F8_COLUMNS, F8_GRADIENT };
template <int DT, int FORMAT, int BLOCK, int WHAT>
__global__ void __launch_bounds__(256) f8_quantize_kernel(const F8Quantize a)
{
    typedef Storage<DT> T;
    __shared__ uint4v staged[kTile * kTile / 16];
    __shared__ unsigned largest[4][kTile];
    __shared__ float sums[4][kTile];
    const bool rows = WHAT == F8_GRADIENT ? a.rows_q != nullptr : WHAT == F8_ROWS, columns = WHAT == F8_GRADIENT ? a.columns_q != nullptr : WHAT == F8_COLUMNS;
    const bool summed = WHAT == F8_GRADIENT && a.partial;
    const int t = threadIdx.x, j = t % 16, g = t / 16, wave = t / 64;
    for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const int tile_row = (int)(tile / a.tiles_across), tile_column = (int)(tile % a.tiles_across);
        const int64_t row = (int64_t)tile_row * kTile + 8 * g, column = (int64_t)tile_column * kTile + 8 * j;
        float v[8][8];
        load_rows<T, 8, 1, WHAT == F8_GRADIENT>(a.src, row, column, v);

        // the largest of each column, and with them of the tile
        __syncthreads();
        if (BLOCK > 1 || columns) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                unsigned m = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) m = max(m, magnitude(v[k][e]));
                m = max(m, (unsigned)__shfl_xor((int)m, 16));
                m = max(m, (unsigned)__shfl_xor((int)m, 32));
                if (t % 64 < 16) largest[wave][8 * j + e] = m;
            }
        }
        if (summed) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) s += v[k][e];
                s += __shfl_xor(s, 16);
                s += __shfl_xor(s, 32);
                if (t % 64 < 16) sums[wave][8 * j + e] = s;
            }
        }
        __syncthreads();
        if (summed && t < kTile && tile_column * (int64_t)kTile + t < a.src.columns) {
            const float s = (sums[0][t] + sums[1][t]) + (sums[2][t] + sums[3][t]);
            float *const to = a.partial + (size_t)tile_row * a.src.columns + tile_column * kTile + t;
            *to = a.add ? (float)((double)*to + s) : s;
        }
        float whole = 0.0f;
        if constexpr (BLOCK > 1) {
            unsigned m = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int w = 0; w < 4; ++w) m = max(m, largest[w][8 * j + e]);
            whole = scale_of<FORMAT>(largest_of_16(m));
        }

        if (rows) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float s = whole;
                if constexpr (BLOCK == 1) {
                    unsigned m = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) m = max(m, magnitude(v[k][e]));
                    s = scale_of<FORMAT>(largest_of_16(m));
                    if (j == 0 && row + k < a.rows_layout.scale_pitch)
                        f8_scales(a.rows_q, a.rows_layout)[(size_t)tile_column * a.rows_layout.scale_pitch + row + k] = s;
                }
                unsigned words[2];
                F8Encoder<FORMAT>(s).encode(v[k], words);
                __builtin_memcpy((uint64_t *)staged + (g / 2 * kF8PanelBytes + j / 2 % 2 * 1024 + (j / 4 * 16 + g % 2 * 8 + k) * 16 + j % 2 * 8) / 8, words, 8);
            }
            if (BLOCK > 1 && t == 0) f8_scales(a.rows_q, a.rows_layout)[(size_t)tile_column * a.rows_layout.scale_pitch + tile_row] = whole;
            __syncthreads();
            write_panels(staged, a.rows_q, a.rows_layout, tile_row * (kTile / kF8Rows), tile_column);
            __syncthreads();
        }
        if (columns) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float s = whole;
                if constexpr (BLOCK == 1) {
                    const int n = 8 * j + e;
                    s = scale_of<FORMAT>(max(max(largest[0][n], largest[1][n]), max(largest[2][n], largest[3][n])));
                    if (g == 0 && column + e < a.columns_layout.scale_pitch)
                        f8_scales(a.columns_q, a.columns_layout)[(size_t)tile_row * a.columns_layout.scale_pitch + column + e] = s;
                }
                const float column_values[8] = {v[0][e], v[1][e], v[2][e], v[3][e], v[4][e], v[5][e], v[6][e], v[7][e]};
                unsigned words[2];
                F8Encoder<FORMAT>(s).encode(column_values, words);
                __builtin_memcpy((uint64_t *)staged + (j / 2 * kF8PanelBytes + g / 2 % 2 * 1024 + (g / 4 * 16 + j % 2 * 8 + e) * 16 + g % 2 * 8) / 8, words, 8);
            }
            if (BLOCK > 1 && t == 0) f8_scales(a.columns_q, a.columns_layout)[(size_t)tile_row * a.columns_layout.scale_pitch + tile_column] = whole;
            __syncthreads();
            write_panels(staged, a.columns_q, a.columns_layout, tile_column * (kTile / kF8Rows), tile_row);
        }
    }
}

// out (+)= the pieces' sums, in their order
__global__ void __launch_bounds__(256) f8_sums_kernel(const float *__restrict__ partial, float *__restrict__ out, int pieces, int columns, int add)
{
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= columns) return;
    double s = add ? out[n] : 0.0;
    for (int p = 0; p < pieces; ++p) s += partial[(size_t)p * columns + n];
    out[n] = (float)s;
}

template <typename T>
__global__ void __launch_bounds__(256) f8_zero_kernel(T *__restrict__ out, int64_t ld, int rows, int columns)
{
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < (int64_t)rows * columns; i += (int64_t)gridDim.x * 256) out[i / columns * ld + i % columns] = (T)0;
}

// A thread per 16-byte piece of the layout, and per scale
__global__ void __launch_bounds__(256) f8_pack_kernel(const uint8_t *__restrict__ codes, const float *__restrict__ scales, char *__restrict__ q, const F8Layout layout,
                                                      int transposed)
{
    const size_t stride = (size_t)gridDim.x * 256, first = (size_t)blockIdx.x * 256 + threadIdx.x;
    for (size_t idx = first; idx < layout.code_bytes / 16; idx += stride) {
        const int piece = idx % 128, lane = piece % 64;
        const size_t panel = idx / 128;
        const int64_t row = (int64_t)(panel / layout.chunks) * kF8Rows + lane % 16;
        const int64_t column = (int64_t)(panel % layout.chunks) * kF8Chunk + lane / 16 * 32 + piece / 64 * 16;
        uint8_t v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const bool real = row < layout.rows && column + i < layout.columns;
            v[i] = real ? codes[transposed ? (column + i) * layout.rows + row : row * layout.columns + column + i] : (uint8_t)0;
        }
        __builtin_memcpy(q + idx * 16, v, 16);
    }
    const int bands = (int)(((int64_t)layout.rows + layout.block - 1) / layout.block);
    for (size_t idx = first; idx < layout.scale_count; idx += stride) {
        const size_t band = idx % layout.scale_pitch, chunk = idx / layout.scale_pitch;
        f8_scales(q, layout)[idx] = band < (size_t)bands ? scales[transposed ? chunk * bands + band : band * layout.chunks + chunk] : 0.0f;
    }
}

__global__ void __launch_bounds__(256) f8_unpack_kernel(const char *__restrict__ q, const F8Layout layout, uint8_t *__restrict__ codes, float *__restrict__ scales)
{
    // a workgroup's threads read whole panels, neighbours write neighbouring pieces of a row
    const size_t stride = (size_t)gridDim.x * 256, first = (size_t)blockIdx.x * 256 + threadIdx.x;
    for (size_t idx = first; idx < layout.code_bytes / 16; idx += stride) {
        const int piece = idx % 8, row_in = idx / 8 % 16;
        const size_t panel = idx / 128;
        const int64_t row = (int64_t)(panel / layout.chunks) * kF8Rows + row_in, column = (int64_t)(panel % layout.chunks) * kF8Chunk + piece * 16;
        if (row >= layout.rows || column >= layout.columns) continue;
        uint8_t v[16];
        __builtin_memcpy(v, q + panel * kF8PanelBytes + piece % 2 * 1024 + (piece / 2 * 16 + row_in) * 16, 16);
        uint8_t *to = codes + row * layout.columns + column;
        if (column + 16 <= layout.columns) {
            __builtin_memcpy(to, v, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 15; ++i)
                if (column + i < layout.columns) to[i] = v[i];
        }
    }
    if (!scales) return;
    const int64_t bands = ((int64_t)layout.rows + layout.block - 1) / layout.block;
    for (size_t idx = first; idx < (size_t)bands * layout.chunks; idx += stride)
        scales[idx] = ((const float *)(q + layout.code_bytes))[idx % layout.chunks * layout.scale_pitch + idx / layout.chunks];
}

static unsigned blocks_for(size_t threads) { return (unsigned)(threads > ((size_t)1 << 30) ? (1 << 22) : (threads + 255) / 256); }

template <int DT, int FORMAT>
static void run_quantize(const F8Quantize &a, int block, bool gradient, hipStream_t s)
{
    const unsigned blocks = (unsigned)(a.tiles < (1 << 22) ? a.tiles : 1 << 22);
    if (gradient) {
        f8_quantize_kernel<DT, FORMAT, 1, F8_GRADIENT><<<blocks, 256, 0, s>>>(a);
    } else if (block > 1) {
        if (a.rows_q) f8_quantize_kernel<DT, FORMAT, 128, F8_ROWS><<<blocks, 256, 0, s>>>(a);
        else f8_quantize_kernel<DT, FORMAT, 128, F8_COLUMNS><<<blocks, 256, 0, s>>>(a);
    } else if (a.rows_q) {
        const size_t wanted = ((size_t)a.rows_layout.row_tiles * a.rows_layout.chunks + 3) / 4;
        f8_quantize_rows_kernel<DT, FORMAT><<<(unsigned)(wanted < (1 << 22) ? wanted : 1 << 22), 256, 0, s>>>(a);
    } else {
        f8_quantize_kernel<DT, FORMAT, 1, F8_COLUMNS><<<blocks, 256, 0, s>>>(a);
    }
}

static int quantize(F8Quantize a, int format, int block, bool gradient, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    a.tiles_across = (int)(((int64_t)a.src.columns + kTile - 1) / kTile);
    a.tiles = (int64_t)a.tiles_across * (((int64_t)a.src.rows + kTile - 1) / kTile);
    const bool e4m3 = format == NOVA_F8_E4M3;
    if (a.src.dtype == NOVA_F32) e4m3 ? run_quantize<NOVA_F32, NOVA_F8_E4M3>(a, block, gradient, s) : run_quantize<NOVA_F32, NOVA_F8_E5M2>(a, block, gradient, s);
    else if (a.src.dtype == NOVA_F16) e4m3 ? run_quantize<NOVA_F16, NOVA_F8_E4M3>(a, block, gradient, s) : run_quantize<NOVA_F16, NOVA_F8_E5M2>(a, block, gradient, s);
    else e4m3 ? run_quantize<NOVA_BF16, NOVA_F8_E4M3>(a, block, gradient, s) : run_quantize<NOVA_BF16, NOVA_F8_E5M2>(a, block, gradient, s);
    return (int)hipGetLastError();
}

int launch_f8_quantize(const F8Source &x, const F8Layout &q, int format, int transposed, void *Xq, void *stream)
{
    F8Quantize a = {x, nullptr, nullptr, nullptr, 0, q, q, 0, 0};
    (transposed ? a.columns_q : a.rows_q) = (char *)Xq;
    return quantize(a, format, q.block, false, stream);
}

int launch_f8_quantize_both(const F8Source &x, int format, void *Xq, void *Xq_transposed, float *sums, float *partial, int add, void *stream)
{
    // (up to 128 rows the sums are whole)
    const bool whole = x.rows <= kTile;
    const F8Quantize a = {x, (char *)Xq, (char *)Xq_transposed, !sums ? nullptr : whole ? sums : partial, whole && add, make_f8_layout(x.rows, x.columns, 1),
                          make_f8_layout(x.columns, x.rows, 1), 0, 0};
    if (int err = quantize(a, format, 1, true, stream)) return err;
    if (!sums || whole) return 0;
    f8_sums_kernel<<<(x.columns + 255) / 256, 256, 0, (hipStream_t)stream>>>(partial, sums, a.columns_layout.chunks, x.columns, add);
    return (int)hipGetLastError();
}

int launch_f8_pack(const uint8_t *codes, const float *scales, const F8Layout &q, int transposed, void *Xq, void *stream)
{
    f8_pack_kernel<<<blocks_for(q.code_bytes / 16), 256, 0, (hipStream_t)stream>>>(codes, scales, (char *)Xq, q, transposed);
    return (int)hipGetLastError();
}

int launch_f8_unpack(const void *Xq, const F8Layout &q, uint8_t *codes, float *scales, void *stream)
{
    f8_unpack_kernel<<<blocks_for(q.code_bytes / 16), 256, 0, (hipStream_t)stream>>>((const char *)Xq, q, codes, scales);
    return (int)hipGetLastError();
}

int launch_f8_zero(void *out, int64_t ld, int rows, int columns, int dtype, void *stream)
{
    const unsigned blocks = blocks_for((size_t)rows * columns);
    if (dtype == NOVA_F32) f8_zero_kernel<<<blocks, 256, 0, (hipStream_t)stream>>>((unsigned *)out, ld, rows, columns);
    else f8_zero_kernel<<<blocks, 256, 0, (hipStream_t)stream>>>((unsigned short *)out, ld, rows, columns);
    return (int)hipGetLastError();
}

}  // namespace nova
