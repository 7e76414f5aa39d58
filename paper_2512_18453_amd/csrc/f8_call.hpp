// What a launch of a product in 8-bit floating point is given, and how a call's rows are cut into launches.  Plain C++ (constexpr functions serve the kernels too), so that
// f8_call_selftest.cpp walks through it without a GPU.
#pragma once
#include "internal.hpp"

namespace nova {

struct F8Call {
    const char *a, *b;
    const float *a_scales, *b_scales;
    const void *bias;
    void *out;
    float *partial;                               // pieces of a cut sum, [splits][rows][N] for all rows of the call
    int64_t ldout;
    int M, N, chunks, splits, split_chunks;
    int a_tiles, b_tiles, a_pitch, b_pitch, a_shift, b_shift;      // panels; scales from chunk to chunk; rows -> scales
    int dtype, flags;
    int a_left;                                   // scales of a chunk from a_scales on: a_pitch of them, less in launches that begin at a later row
    int rows;                                     // of the call; M of the launch
};

// Which of a chunk's `left` scales an operand's row takes.  Rows behind the last, which a tile may have and which are not stored, take the last.
constexpr int f8_scale_at(int row, int shift, int left) { return (row >> shift) < left ? row >> shift : left - 1; }

// Where piece `split` of a cut sum begins, for the rows of the launch
constexpr size_t f8_piece_at(const F8Call &a, int split) { return (size_t)split * a.rows * a.N; }

// Panels of rows of one launch: tiles of TILE panels, `across` workgroups for each, `most` workgroups in a launch (2^22 of 512 threads keep it below 2^32 threads)
constexpr int64_t kF8LaunchBlocks = (int64_t)1 << 22;
constexpr int64_t f8_launch_panels(int64_t across, int tile, int64_t most) { return (most / across > 0 ? most / across : 1) * tile; }

// The launch whose rows begin at panel `first`: `panels` of them, or what is left
inline F8Call f8_launch(const F8Call &a, int64_t first, int64_t panels)
{
    F8Call part = a;
    const int64_t rows = first * kF8Rows;
    part.a_tiles = (int)(a.a_tiles - first < panels ? a.a_tiles - first : panels);
    part.M = (int)(a.M - rows < part.a_tiles * (int64_t)kF8Rows ? a.M - rows : part.a_tiles * (int64_t)kF8Rows);
    part.a += (size_t)first * a.chunks * kF8PanelBytes;
    part.a_scales += rows >> a.a_shift;
    part.a_left -= (int)(rows >> a.a_shift);
    part.out = (char *)a.out + rows * a.ldout * (int64_t)dtype_size(a.dtype);
    if (a.splits > 1) part.partial += (size_t)rows * a.N;
    return part;
}

}  // namespace nova
