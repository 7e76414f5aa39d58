// Matrices in 8-bit floating point: from rows of numbers to the layout that the products read (nova_f8_quantize in nova.h), from codes, and back.
//
// A workgroup takes 128 x 128 elements of the source (32 x 128 where there are no more rows), a thread 8 x 8 (2 x 8) of them, and holds them in registers: what is largest in a row, a column or all of them
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

// Where a 16-byte piece of a tile's panel lies in LDS: neighbours in the eight bytes that a wave's lanes write at a time are a panel, or 256 bytes, apart, and would all lie
// in the same banks
__device__ __forceinline__ int staged_piece(int panel, int piece) { return panel * 128 + (piece ^ ((piece / 16 ^ panel) & 7)); }

// Layouts of 8 MB and more go past the caches: 4096 x 25088 in 128 x 128 56 -> 50 us, 2048 rows through a layer of 4096 x 4096, whose product reads them at once, 44.6 -> 42.9.
// Smaller ones stay in them (the backward pass of 512 rows through that layer 70 us, past the caches 75).
constexpr size_t kStreamedLayout = (size_t)8 << 20;

template <int FILLED, bool STREAMED>
__device__ __forceinline__ void copy_panels(const uint4v *staged, char *q, const F8Layout &layout, int row_tile, int chunk)
{
    for (int piece = threadIdx.x; piece < kTile * kTile / 16; piece += 256) {
        const int panel = piece / 128, r = row_tile + panel;
        if (r >= layout.row_tiles) continue;
        const uint4v codes = piece % 64 / 16 < FILLED ? staged[staged_piece(panel, piece % 128)] : uint4v{0, 0, 0, 0};
        uint4v *const to = (uint4v *)(q + ((size_t)r * layout.chunks + chunk) * kF8PanelBytes + piece % 128 * 16);
        if constexpr (STREAMED) __builtin_nontemporal_store(codes, to);
        else *to = codes;
    }
}

// A tile's codes from LDS to the panels row_tile .. of a chunk, of which the first FILLED of four quarters hold codes.  (Two loops: of two stores in one the compiler makes one
// that goes through the caches.)
template <int FILLED>
__device__ __forceinline__ void write_panels(const uint4v *staged, char *q, const F8Layout &layout, int row_tile, int chunk)
{
    if (layout.code_bytes >= kStreamedLayout) copy_panels<FILLED, true>(staged, q, layout, row_tile, chunk);
    else copy_panels<FILLED, false>(staged, q, layout, row_tile, chunk);
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
template <int DT, int FORMAT, bool STREAMED>
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
        if constexpr (STREAMED) {
            __builtin_nontemporal_store(staged[wave][lane], to + lane);
            __builtin_nontemporal_store(staged[wave][lane + 64], to + lane + 64);
        } else {
            to[lane] = staged[wave][lane];
            to[lane + 64] = staged[wave][lane + 64];
        }
        exchange_in_wave();
    }
}

// What a workgroup shares
struct F8Shared {
    uint4v staged[kTile * kTile / 16];
    unsigned largest[4][kTile];
    float sums[4][kTile];
};

// BLOCK: 1 or 128.  WHAT: the rows' layout, the columns', or what there is of them and of the columns' sums, behind a gate if there is one.  R: rows of a thread, 8, or
// 2 where the source has at most 32 rows.  The workgroup is number `block` of `blocks`.
enum { F8_ROWS, F8_COLUMNS, F8_GRADIENT };
template <int DT, int FORMAT, int BLOCK, int WHAT, int R>
__device__ __forceinline__ void f8_quantize_tiles(const F8Quantize &a, unsigned block, unsigned blocks, F8Shared &shared)
{
    typedef Storage<DT> T;
    static_assert(R == 8 || (R == 2 && BLOCK == 1), "rows of a thread");
    const bool rows = WHAT == F8_GRADIENT ? a.rows_q != nullptr : WHAT == F8_ROWS, columns = WHAT == F8_GRADIENT ? a.columns_q != nullptr : WHAT == F8_COLUMNS;
    const bool summed = WHAT == F8_GRADIENT && a.partial;
    const int t = threadIdx.x, j = t % 16, g = t / 16, wave = t / 64;
    char *const staged = (char *)shared.staged;
    for (int64_t tile = block; tile < a.tiles; tile += blocks) {
        const int tile_row = (int)(tile / a.tiles_across), tile_column = (int)(tile % a.tiles_across);
        const int64_t row = (int64_t)tile_row * kTile + R * g, column = (int64_t)tile_column * kTile + 8 * j;
        float v[R][8];
        load_rows<T, R, 1, WHAT == F8_GRADIENT>(a.src, row, column, v);

        // the largest of each column, and with them of the tile
        __syncthreads();
        if (BLOCK > 1 || columns) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                unsigned m = 0;
#pragma unroll
                for (int k = 0; k < R; ++k) m = max(m, magnitude(v[k][e]));
                m = max(m, (unsigned)__shfl_xor((int)m, 16));
                m = max(m, (unsigned)__shfl_xor((int)m, 32));
                if (t % 64 < 16) shared.largest[wave][8 * j + e] = m;
            }
        }
        if (summed) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < R; ++k) s += v[k][e];
                s += __shfl_xor(s, 16);
                s += __shfl_xor(s, 32);
                if (t % 64 < 16) shared.sums[wave][8 * j + e] = s;
            }
        }
        __syncthreads();
        if (summed && t < kTile && tile_column * (int64_t)kTile + t < a.src.columns) {
            const float s = (shared.sums[0][t] + shared.sums[1][t]) + (shared.sums[2][t] + shared.sums[3][t]);
            float *const to = a.partial + (size_t)tile_row * a.src.columns + tile_column * kTile + t;
            *to = a.add ? (float)((double)*to + s) : s;
        }
        float whole = 0.0f;
        if constexpr (BLOCK > 1) {
            unsigned m = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int w = 0; w < 4; ++w) m = max(m, shared.largest[w][8 * j + e]);
            whole = scale_of<FORMAT>(largest_of_16(m));
        }

        if (rows) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
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
                const int r = R * g + k, piece = j / 2 % 2 * 64 + j / 4 * 16 + r % 16;
                *(uint64_t *)(staged + staged_piece(r / 16, piece) * 16 + j % 2 * 8) = (uint64_t)words[1] << 32 | words[0];
            }
            if (BLOCK > 1 && t == 0) f8_scales(a.rows_q, a.rows_layout)[(size_t)tile_column * a.rows_layout.scale_pitch + tile_row] = whole;
            __syncthreads();
            write_panels<4>(shared.staged, a.rows_q, a.rows_layout, tile_row * (kTile / kF8Rows), tile_column);
            __syncthreads();
        }
        if (columns) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int n = 8 * j + e, first = R * g, piece = first / 16 % 2 * 64 + first / 32 * 16 + n % 16;
                float s = whole;
                if constexpr (BLOCK == 1) {
                    s = scale_of<FORMAT>(max(max(shared.largest[0][n], shared.largest[1][n]), max(shared.largest[2][n], shared.largest[3][n])));
                    if (g == 0 && column + e < a.columns_layout.scale_pitch)
                        f8_scales(a.columns_q, a.columns_layout)[(size_t)tile_row * a.columns_layout.scale_pitch + column + e] = s;
                }
                float of_column[R];
#pragma unroll
                for (int k = 0; k < R; ++k) of_column[k] = v[k][e];
                char *const to = staged + staged_piece(n / 16, piece) * 16 + first % 16;
                if constexpr (R == 8) {
                    unsigned words[2];
                    F8Encoder<FORMAT>(s).encode(of_column, words);
                    *(uint64_t *)to = (uint64_t)words[1] << 32 | words[0];
                } else {
                    F8Encoder<FORMAT>(s).encode(of_column, *(uint16_t *)to);
                }
            }
            if (BLOCK > 1 && t == 0) f8_scales(a.columns_q, a.columns_layout)[(size_t)tile_row * a.columns_layout.scale_pitch + tile_column] = whole;
            __syncthreads();
            write_panels<R == 8 ? 4 : 1>(shared.staged, a.columns_q, a.columns_layout, tile_column * (kTile / kF8Rows), tile_row);
        }
    }
}

template <int DT, int FORMAT, int BLOCK, int WHAT, int R>
__global__ void __launch_bounds__(256) f8_quantize_kernel(const F8Quantize a)
{
    __shared__ F8Shared shared;
    f8_quantize_tiles<DT, FORMAT, BLOCK, WHAT, R>(a, blockIdx.x, gridDim.x, shared);
}

// What a backward pass needs of the gradient, and of the layer's input, in one launch
template <int DT, int FORMAT, int R>
__global__ void __launch_bounds__(256, DT == NOVA_F32 ? 2 : 3) f8_quantize_backward_kernel(const F8Quantize d, const F8Quantize x, unsigned d_blocks)
{
    __shared__ F8Shared shared;
    if (blockIdx.x < d_blocks) f8_quantize_tiles<DT, FORMAT, 1, F8_GRADIENT, R>(d, blockIdx.x, d_blocks, shared);
    else f8_quantize_tiles<DT, NOVA_F8_E4M3, 1, F8_COLUMNS, R>(x, blockIdx.x - d_blocks, gridDim.x - d_blocks, shared);
}

// out (+)= the pieces' sums, in their order
__global__ void __launch_bounds__(256) f8_sums_kernel(const float *__restrict__ partial, float *__restrict__ out, int pieces, int columns, int add)
{
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= columns) return;
    double s = add ? out[n] : 0.0;
#pragma unroll 16
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
        // neighbours take neighbouring pieces of a row, or, transposed, neighbouring columns of the source
        const int at = idx % 128, row_in = transposed ? at % 16 : at / 8, eighth = transposed ? at / 16 : at % 8;
        const size_t panel = idx / 128;
        const int64_t row = (int64_t)(panel / layout.chunks) * kF8Rows + row_in, column = (int64_t)(panel % layout.chunks) * kF8Chunk + eighth * 16;
        uint8_t v[16];
        if (!transposed && row < layout.rows && column + 16 <= layout.columns) {
            __builtin_memcpy(v, codes + row * layout.columns + column, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const bool real = row < layout.rows && column + i < layout.columns;
                v[i] = real ? codes[transposed ? (column + i) * layout.rows + row : row * layout.columns + column + i] : (uint8_t)0;
            }
        }
        __builtin_memcpy(q + panel * kF8PanelBytes + eighth % 2 * 1024 + (eighth / 2 * 16 + row_in) * 16, v, 16);
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
            typedef unsigned Piece __attribute__((ext_vector_type(4), aligned(1)));
            Piece whole;
            __builtin_memcpy(&whole, v, 16);
            __builtin_nontemporal_store(whole, (Piece *)to);
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

static void count_tiles(F8Quantize &a)
{
    a.tiles_across = (int)(((int64_t)a.src.columns + kTile - 1) / kTile);
    a.tiles = (int64_t)a.tiles_across * (((int64_t)a.src.rows + kTile - 1) / kTile);
}
static unsigned tile_blocks(const F8Quantize &a) { return (unsigned)(a.tiles < (1 << 21) ? a.tiles : 1 << 21); }
constexpr int kFewRows = 32;

template <int DT, int FORMAT>
static void run_quantize(const F8Quantize &a, int block, hipStream_t s)
{
    const unsigned blocks = tile_blocks(a);
    if (block > 1) {
        if (a.rows_q) f8_quantize_kernel<DT, FORMAT, 128, F8_ROWS, 8><<<blocks, 256, 0, s>>>(a);
        else f8_quantize_kernel<DT, FORMAT, 128, F8_COLUMNS, 8><<<blocks, 256, 0, s>>>(a);
    } else if (a.rows_q) {
        const size_t wanted = ((size_t)a.rows_layout.row_tiles * a.rows_layout.chunks + 3) / 4;
        const unsigned panels_blocks = (unsigned)(wanted < (1 << 22) ? wanted : 1 << 22);
        if (a.rows_layout.code_bytes >= kStreamedLayout) f8_quantize_rows_kernel<DT, FORMAT, true><<<panels_blocks, 256, 0, s>>>(a);
        else f8_quantize_rows_kernel<DT, FORMAT, false><<<panels_blocks, 256, 0, s>>>(a);
    } else if (a.src.rows <= kFewRows) {
        f8_quantize_kernel<DT, FORMAT, 1, F8_COLUMNS, 2><<<blocks, 256, 0, s>>>(a);
    } else {
        f8_quantize_kernel<DT, FORMAT, 1, F8_COLUMNS, 8><<<blocks, 256, 0, s>>>(a);
    }
}

template <int DT, int FORMAT>
static void run_backward(const F8Quantize &d, const F8Quantize &x, hipStream_t s)
{
    const unsigned d_blocks = tile_blocks(d), blocks = d_blocks + (x.columns_q ? tile_blocks(x) : 0);
    if (d.src.rows <= kFewRows) f8_quantize_backward_kernel<DT, FORMAT, 2><<<blocks, 256, 0, s>>>(d, x, d_blocks);
    else f8_quantize_backward_kernel<DT, FORMAT, 8><<<blocks, 256, 0, s>>>(d, x, d_blocks);
}

// f(std::integral_constant of dtype, of format)
template <typename F>
static void by_type(int dtype, int format, F &&f)
{
    auto of_format = [&](auto dt) {
        if (format == NOVA_F8_E4M3) f(dt, std::integral_constant<int, NOVA_F8_E4M3>{});
        else f(dt, std::integral_constant<int, NOVA_F8_E5M2>{});
    };
    if (dtype == NOVA_F32) of_format(std::integral_constant<int, NOVA_F32>{});
    else if (dtype == NOVA_F16) of_format(std::integral_constant<int, NOVA_F16>{});
    else of_format(std::integral_constant<int, NOVA_BF16>{});
}

int launch_f8_quantize(const F8Source &x, const F8Layout &q, int format, int transposed, void *Xq, void *stream)
{
    F8Quantize a = {x, nullptr, nullptr, nullptr, 0, q, q, 0, 0};
    (transposed ? a.columns_q : a.rows_q) = (char *)Xq;
    count_tiles(a);
    by_type(x.dtype, format, [&](auto dt, auto f) { run_quantize<dt, f>(a, q.block, (hipStream_t)stream); });
    return (int)hipGetLastError();
}

int launch_f8_quantize_backward(const F8Source &d, int format, void *dq, void *dq_transposed, float *sums, float *partial, int add, const F8Source &x,
                                void *xq_transposed, void *stream)
{
    // (up to 128 rows the sums are whole)
    const bool whole = d.rows <= kTile;
    F8Quantize a = {d, (char *)dq, (char *)dq_transposed, !sums ? nullptr : whole ? sums : partial, whole && add, make_f8_layout(d.rows, d.columns, 1),
                    make_f8_layout(d.columns, d.rows, 1), 0, 0};
    F8Quantize b = {x, nullptr, (char *)xq_transposed, nullptr, 0, {}, {}, 0, 0};
    count_tiles(a);
    if (xq_transposed) {
        b.columns_layout = make_f8_layout(x.columns, x.rows, 1);
        count_tiles(b);
    }
    by_type(d.dtype, format, [&](auto dt, auto f) { run_backward<dt, f>(a, b, (hipStream_t)stream); });
    NOVA_HIP_TRY(hipGetLastError());
    if (!sums || whole) return 0;
    f8_sums_kernel<<<(d.columns + 255) / 256, 256, 0, (hipStream_t)stream>>>(partial, sums, a.columns_layout.chunks, d.columns, add);
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
