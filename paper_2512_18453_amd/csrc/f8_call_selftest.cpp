// Walks, on the CPU, through the addresses of products in 8-bit floating point whose rows are cut into launches: every scale that a lane of a tile's workgroup loads, every
// panel, and where results and pieces of cut sums go.  Buffers have exactly the documented sizes, so that under AddressSanitizer a read behind them ends the program.
#include <cstdio>
#include <vector>

#include "f8_call.hpp"

using namespace nova;

static int failures = 0;
#define EXPECT(cond)                                                          \
    do {                                                                      \
        if (!(cond)) { std::printf("f8_call_selftest: line %d: %s (M %d, N %d, block %d, tile %d, most %d)\n", __LINE__, #cond, M, N, block, tile, most); ++failures; return; } \
    } while (0)

static void walk(int M, int N, int chunks, int block, int tile, int most, int splits)
{
    const F8Layout layout = make_f8_layout(M, chunks * kF8Chunk, block);
    // a scale's value: its own number
    std::vector<float> scales(layout.scale_count);
    for (size_t i = 0; i < scales.size(); ++i) scales[i] = (float)i;
    std::vector<char> panels(layout.code_bytes), out((size_t)M * N * 2);
    std::vector<float> partial(splits > 1 ? (size_t)splits * M * N : 0);
    F8Call call = {};
    call.a = panels.data();
    call.a_scales = scales.data();
    call.out = out.data();
    call.partial = partial.data();
    call.ldout = N;
    call.M = call.rows = M;
    call.N = N;
    call.chunks = chunks;
    call.splits = splits;
    call.a_tiles = layout.row_tiles;
    call.a_pitch = call.a_left = layout.scale_pitch;
    call.a_shift = block == 1 ? 0 : 7;
    call.dtype = NOVA_F16;
    const int64_t across = (int64_t)(N + tile * kF8Rows - 1) / (tile * kF8Rows) * splits, step = f8_launch_panels(across, tile, most);
    int64_t seen = 0;
    for (int64_t first = 0; first < call.a_tiles; first += step) {
        const F8Call part = f8_launch(call, first, step);
        EXPECT(part.a_tiles > 0 && part.M > 0 && part.M <= part.a_tiles * kF8Rows && (part.a_tiles - 1) * kF8Rows < part.M);
        const int down = (part.a_tiles + tile - 1) / tile;
        EXPECT(across * down <= most || down == 1);
        for (int m_tile = 0; m_tile < down * tile; m_tile += tile)
            for (int wave = 0; 4 * wave < tile; ++wave)
                for (int lane = 0; lane < 64; ++lane) {
                    const int row = (m_tile + 4 * wave) * kF8Rows + lane, at = f8_scale_at(row, part.a_shift, part.a_left);
                    EXPECT(at >= 0);
                    for (int c = 0; c < chunks; ++c) {
                        const float got = (part.a_scales + (size_t)c * part.a_pitch)[at];          // (a read that must lie inside)
                        const int64_t whole = first * kF8Rows + row;
                        if (row < part.M) EXPECT(got == (float)((size_t)c * layout.scale_pitch + (whole >> call.a_shift)));
                    }
                }
        for (int t = 0; t < part.a_tiles; ++t)
            EXPECT(part.a + ((size_t)t * part.chunks + chunks - 1) * kF8PanelBytes == panels.data() + ((size_t)(first + t) * chunks + chunks - 1) * kF8PanelBytes);
        for (int m = 0; m < part.M; m += part.M > 1 ? part.M - 1 : 1) {
            const size_t whole = (size_t)first * kF8Rows + m;
            EXPECT((char *)part.out + ((size_t)m * part.ldout + N - 1) * 2 == out.data() + (whole * N + N - 1) * 2);
            if (splits > 1)
                for (int s = 0; s < splits; ++s) {
                    float *const at = part.partial + f8_piece_at(part, s) + (size_t)m * N + N - 1;
                    EXPECT(at == partial.data() + ((size_t)s * M + whole) * N + N - 1);
                    *at = 1.0f;
                }
        }
        seen += part.M;
    }
    EXPECT(seen == M);
}

int main()
{
    for (int tile : {8, 16})
        for (int block : {1, 128})
            for (int M : {1, 16, 17, 129, 257, 300, 513, 1000, 1041})
                for (int N : {1, 130, 700})
                    for (int chunks : {1, 3})
                        for (int splits : {1, 3})
                            for (int most : {1, 2, 7, 100}) walk(M, N, chunks, block, tile, most, splits);
    if (failures) return 1;
    std::printf("f8_call_selftest: ok\n");
    return 0;
}
