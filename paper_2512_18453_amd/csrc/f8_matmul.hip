// Products of matrices in 8-bit floating point: out[m][n] = sum over chunks c of 128 of  sA[m][c] sB[n][c] sum_k a[m][k] b[n][k].
//
// The products of a chunk are summed on the matrix unit, from zero, and the sum is scaled and added in binary32.  The matrix unit's rows are B's (n) and its
// columns A's (m): a lane then holds four neighbouring n of one m, so that A's scale is one number per lane and B's, where 128 rows share it, one per wave.
#include "f8_call.hpp"
#include "f8_common.hpp"

namespace nova {

__device__ __forceinline__ F8Fragment load_fragment(const char *panel, int lane)
{
    F8Fragment f;
    f.half[0] = *(const uint4v *)(panel + lane * 16);
    f.half[1] = *(const uint4v *)(panel + 1024 + lane * 16);
    return f;
}

// Where results go: COUNT neighbouring columns from n on, of the rows that a thread is given.  What does not change from row to row is decided once: checks for
// every element in the loop over rows made the results of a 256 x 256 tile take 11 us.
template <typename T, int COUNT>
struct F8Columns {
    T *to;                                        // column n of row 0
    int64_t ld;
    int count;                                    // of the COUNT columns exist
    bool add, relu;
    float bias[COUNT];

    __device__ __forceinline__ F8Columns(void *out, int64_t ldout, const void *bias_row, int flags, int N, int n)
        : to((T *)out + n), ld(ldout), count(min(COUNT, N - n)), add((flags & NOVA_FLAG_ADD) != 0), relu((flags & NOVA_FLAG_RELU) != 0)
    {
#pragma unroll
        for (int v = 0; v < COUNT; ++v) bias[v] = bias_row && v < count ? load_f32((const T *)bias_row + n + v) : 0.0f;
    }
    __device__ __forceinline__ void write(int64_t m, const float (&sum)[COUNT]) const
    {
        struct Results { T v[COUNT]; } r = {};
        T *const at = to + m * ld;
        if (add) {
            if (count == COUNT) {
                __builtin_memcpy(&r, at, sizeof r);
            } else {
#pragma unroll
                for (int v = 0; v < COUNT - 1; ++v)
                    if (v < count) r.v[v] = at[v];
            }
        }
#pragma unroll
        for (int v = 0; v < COUNT; ++v) {
            float s = sum[v] + bias[v];
            if (add) s += (float)r.v[v];
            if (relu) s = s < 0.0f ? 0.0f : s;
            store_from_f32(&r.v[v], s);
        }
        if (count == COUNT) {
            // (past the caches' own order of writing back: 8192 x 8192 results of one chunk 57.4 us without, 41.9 with)
            typedef unsigned Words __attribute__((ext_vector_type(sizeof r / 4), aligned(sizeof(T))));
            Words words;
            __builtin_memcpy(&words, &r, sizeof r);
            __builtin_nontemporal_store(words, (Words *)at);
        } else {
#pragma unroll
            for (int v = 0; v < COUNT - 1; ++v)
                if (v < count) at[v] = r.v[v];
        }
    }
};

// f(element of the results' type, where they go, elements from row to row, bias, flags): of the result, or of a piece of a cut sum.  WIDE: 1 where results are known to be
// binary32, 0 where they are known to have 16 bits
template <int WIDE = -1, typename F>
__device__ __forceinline__ void with_results(const F8Call &a, int split, F &&f)
{
    if (a.splits > 1) f(0.0f, a.partial + f8_piece_at(a, split), (int64_t)a.N, nullptr, 0);
    else if (WIDE < 0 ? a.dtype == NOVA_F32 : WIDE) f(0.0f, a.out, a.ldout, a.bias, a.flags);
    else if (a.dtype == NOVA_F16) f((f16)0.0f, a.out, a.ldout, a.bias, a.flags);
    else f((bf16)0.0f, a.out, a.ldout, a.bias, a.flags);
}

// Four results of a row
template <int WIDE = -1>
__device__ __forceinline__ void write_four(const F8Call &a, int split, int64_t m, int n, const float (&four)[4])
{
    if (m < a.M && n < a.N)
        with_results<WIDE>(a, split, [&](auto element, void *out, int64_t ld, const void *bias, int flags) __attribute__((always_inline)) {
            F8Columns<decltype(element), 4>(out, ld, bias, flags, a.N, n).write(m, four);
        });
}

struct F8Shape { int kind, mt, nt, waves, splits, split_chunks; };           // kind: 0 up to 64 rows, 1 tiles of 128 x 128, 2 of 256 x 256

// ---- up to 64 rows ----
//
// Bound by B's bytes.  A workgroup makes 16 NT columns for all rows; its waves take the chunks of those columns in turn, load B's panels straight into registers, AHEAD - 1 ahead, and
// add up through LDS in the order of their numbers.  A's panels come the same way from L2; or, with few rows, every workgroup quantises x by itself first, into LDS,
// which saves the launch that would do it.  Chunks are summed the full way whatever the results' type: next to the bytes the matrix unit's time is small (with results in binary16,
// the narrow way and the full one: 1 row by 25088 x 4096 22.4, 22.3 us; 32 rows 30.0, 30.3; 64 rows 43.9, 41.7; 32 by 4096 x 4096 11.2, 11.2; 64 13.9, 14.4; 1 by 4096 x 25088 19.6, 20.4).
constexpr int kLaidOut = -1;
struct F8RowsOf { const void *x; int64_t ld; int K; };           // what A is quantised from

// Whether it saves more than it costs: every workgroup does the same, and LDS holds no more than 32768 elements.  Up to four rows it does (in us, with a launch of its own
// first and without: 1 row by 32768 x 4096 32.6, 29.4; 1 by 25088 x 4096 25.7, 22.4; 4 by 4096 x 16384 21.3, 20.3); more rows save less of what is loaded of A (a panel has 16),
// and then the workgroups' elements count: 8 by 2048 x 4096 10.3, 7.9; 6 by 4096 x 4096 10.5, 10.0; 7 10.5, 10.7; 16 by 2048 x 4096 10.5, 10.5; 8 by 2048 x 16384 15.2, 16.9.
static bool quantised_on_the_way(int M, int N, const F8Shape &p)
{
    const size_t elements = (size_t)M * p.split_chunks * kF8Chunk, workgroups = (size_t)ceil_div(N, 16) * p.splits;
    return p.kind == 0 && p.mt == 1 && elements <= 32768 && (M <= 4 || elements * workgroups <= (size_t)6 << 20);
}

// MT panels of rows, NT of columns; WIDE: results in binary32; DT: kLaidOut, or the type of x
template <int MT, int NT, int FA, int FB, int WIDE, bool BAND, int DT>
__global__ void __launch_bounds__(512) f8_rows_kernel(const F8Call a, const F8RowsOf rows)
{
    constexpr bool FUSED = DT != kLaidOut;
    constexpr int AHEAD = MT == 4 ? 2 : MT == 2 ? 3 : 4;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64, i = lane % 16, b = lane / 16;
    const int across = (a.b_tiles + NT - 1) / NT, tile = (int)(blockIdx.x % across) * NT, split = blockIdx.x / across;
    const int first = split * a.split_chunks, count = min(a.chunks - first, a.split_chunks);
    const int steps = count > wave ? (count - wave + waves - 1) / waves : 0;
    const char *panels[NT];
#pragma unroll
    for (int y = 0; y < NT; ++y) panels[y] = a.b + ((size_t)min(tile + y, a.b_tiles - 1) * a.chunks + first) * kF8PanelBytes;          // (past the last: computed and not stored)
    float *const scales_in_lds = (float *)(lds + (size_t)count * a.M * kF8Chunk);

    struct Stage {
        F8Fragment b[NT], a[FUSED ? 1 : MT];
        float4v b_scale[NT];
        float a_scale[MT];
    };
    auto load = [&](int step, Stage &s) __attribute__((always_inline)) {
        // (past the last: the last once more, and not multiplied, so that no load is in a branch)
        const int c = wave + min(step, steps - 1) * waves;
        const float *const sb = a.b_scales + (size_t)(first + c) * a.b_pitch;
#pragma unroll
        for (int y = 0; y < NT; ++y) {
            const char *const at = panels[y] + (size_t)c * kF8PanelBytes + lane * 16u;
            s.b[y].half[0] = __builtin_nontemporal_load((const uint4v *)at);
            s.b[y].half[1] = __builtin_nontemporal_load((const uint4v *)(at + 1024));
            const int t = min(tile + y, a.b_tiles - 1);
            if constexpr (BAND) s.b_scale[y][0] = sb[(t * 16) >> a.b_shift];
            else s.b_scale[y] = *(const float4v *)(sb + t * 16 + 4 * b);
        }
        if constexpr (!FUSED) {
#pragma unroll
            for (int x = 0; x < MT; ++x) {
                const int t = min(x, a.a_tiles - 1);
                s.a[x] = load_fragment(a.a + ((size_t)t * a.chunks + first + c) * kF8PanelBytes, lane);
                s.a_scale[x] = a.a_scales[(size_t)(first + c) * a.a_pitch + ((t * 16 + i) >> a.a_shift)];
            }
        }
    };
    float4v sum[NT][MT];
#pragma unroll
    for (int y = 0; y < NT; ++y)
#pragma unroll
        for (int x = 0; x < MT; ++x) sum[y][x] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](int step, Stage &s) __attribute__((always_inline)) {
        if constexpr (FUSED) {
            const int at = (wave + step * waves) * a.M + min(i, a.M - 1);
            s.a[0].half[0] = *(const uint4v *)(lds + (size_t)at * kF8Chunk + b * 32);
            s.a[0].half[1] = *(const uint4v *)(lds + (size_t)at * kF8Chunk + b * 32 + 16);
            s.a_scale[0] = scales_in_lds[at];
        }
        F8Input<FB, F8_FULL> fb[NT];
#pragma unroll
        for (int y = 0; y < NT; ++y) fb[y].set(s.b[y]);
#pragma unroll
        for (int x = 0; x < MT; ++x) {
            F8Input<FA, F8_FULL> fa;
            fa.set(s.a[x]);
#pragma unroll
            for (int y = 0; y < NT; ++y) {
                const float4v p = f8_products<FB, FA, F8_FULL>(fb[y], fa);
#pragma unroll
                for (int v = 0; v < 4; ++v) sum[y][x][v] = fma32(s.a_scale[x] * s.b_scale[y][BAND ? 0 : v], p[v], sum[y][x][v]);
            }
        }
    };

    Stage stage[AHEAD];
    if (steps > 0) static_for<AHEAD - 1>([&](auto I) __attribute__((always_inline)) { load(I, stage[I]); });
    if constexpr (FUSED) {
        // sixteen lanes take a row's chunk, eight elements each
        for (int at = threadIdx.x / 16; at < count * a.M; at += blockDim.x / 16) {
            const int c = at / a.M, m = at % a.M, column = (first + c) * kF8Chunk + lane % 16 * 8;
            const Eight<Storage<DT>> x = load_eight((const Storage<DT> *)rows.x + m * rows.ld + column, rows.K - column, column >= 8 && column < rows.K);
            unsigned largest = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) largest = max(largest, magnitude((float)x.v[e]));
            const float scale = scale_of<FA>(largest_of_16(largest));
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)x.v[e];
            unsigned words[2];
            F8Encoder<FA>(scale).encode(v, words);
            __builtin_memcpy(__builtin_assume_aligned(lds + (size_t)at * kF8Chunk + lane % 16 * 8, 8), words, 8);
            if (lane % 16 == 0) scales_in_lds[at] = scale;
        }
        __syncthreads();
    }
    for (int step = 0; step < steps; step += AHEAD)
        static_for<AHEAD>([&](auto I) __attribute__((always_inline)) {
            load(step + I + AHEAD - 1, stage[(I + AHEAD - 1) % AHEAD]);
            if (step + I < steps) multiply(step + I, stage[I]);
        });

    if constexpr (FUSED) __syncthreads();
    float4v *const sums = (float4v *)lds;
#pragma unroll
    for (int y = 0; y < NT; ++y)
#pragma unroll
        for (int x = 0; x < MT; ++x) sums[((wave * NT + y) * MT + x) * 64 + lane] = sum[y][x];
    __syncthreads();
    for (int e = threadIdx.x; e < NT * MT * 64; e += blockDim.x) {
        float four[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int w = 0; w < waves; ++w) {
            const float4v part = sums[w * NT * MT * 64 + e];
#pragma unroll
            for (int v = 0; v < 4; ++v) four[v] += part[v];
        }
        const int m = e / 64 % MT * 16 + i, n = (tile + e / 64 / MT) * 16 + 4 * b;
        write_four<WIDE>(a, split, m, n, four);
    }
}

// ---- tiles ----
//
// A workgroup of WM x WN waves makes 16 WM MT rows by 16 WN NT columns.  A stage is a chunk of both operands' panels with their scales; stages come straight from global
// memory to LDS, one ahead of the one that is multiplied, and a panel lies there as it lies in memory: the 64 lanes of a wave read 1024 bytes side by side.
//
// 8192 x 8192 x 8192 to bfloat16 439 us (479 on another card), 2504 TFLOP/s where a large library product of that format with one scale per matrix reaches 2655; with a scale per row and chunk
// of B too, where a sum takes two vector instructions instead of one, 527.  LDS binds about as much as the matrix unit: a chunk of a 256 x 256 tile is 2048 clocks of matrix
// instructions, 64 KB written and 192 KB read at 128 bytes a clock.  128 x 128 tiles, two workgroups per compute unit, read a third more: 512 us.  A's panels loaded by
// each wave into registers instead took more of those than there are (813).
template <int WM_, int WN_, int MT_, int NT_>
struct F8Tile {
    static constexpr int WM = WM_, WN = WN_, MT = MT_, NT = NT_, WAVES = WM * WN, THREADS = WAVES * 64, A = WM * MT, B = WN * NT;        // panels
    static constexpr int PER_WAVE = (A + B) / WAVES, SCALE_LOADS = (A + B) / 4;                                                         // panels; 64 scales each
    static constexpr int PANELS = (A + B) * kF8PanelBytes, STAGE = PANELS + (A + B) * kF8Rows * 4, PITCH = NT * 64 + 16;
    static constexpr int LDS = 2 * STAGE > WAVES * 32 * PITCH ? 2 * STAGE : WAVES * 32 * PITCH;                                         // 32 rows of each wave's results
    static_assert(A % 4 == 0 && (A + B) % 4 == 0 && PER_WAVE * WAVES == A + B && PER_WAVE % 2 == 0 && A % PER_WAVE == 0 && SCALE_LOADS <= WAVES, "what a wave loads is of one operand");
};

// 64 words of 4 bytes, as global_to_lds16 takes 16
__device__ __forceinline__ void global_to_lds4(const void *uniform_base, unsigned byte_offset, unsigned lds_wave_base)
{
    unsigned saved_m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved_m0) : "s"(lds_wave_base), "v"(byte_offset), "s"(uniform_base) : "memory");
}

// BAND: one scale of B for the 16 NT columns of a wave
template <typename Shape, int FA, int FB, int WAY, bool BAND>
__global__ void __launch_bounds__(Shape::THREADS, 2) f8_tile_kernel(const F8Call a)
{
    constexpr int MT = Shape::MT, NT = Shape::NT, STAGE = Shape::STAGE;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), i = lane % 16, b = lane / 16;
    const int wm = wave / Shape::WN, wn = wave % Shape::WN;
    // eight tiles of rows go along the columns together: what an XCD works on at a time is a patch of tiles
    const unsigned across = (a.b_tiles + Shape::B - 1) / Shape::B, down = (a.a_tiles + Shape::A - 1) / Shape::A, tiles = across * down;
    const unsigned id = xcd_local_block_id(blockIdx.x, gridDim.x), split = id / tiles, tile = id % tiles;
    const unsigned first_row = tile / (8 * across) * 8, together = min(8u, down - first_row), in_group = tile % (8 * across);
    const int m_tile = (int)(first_row + in_group % together) * Shape::A, n_tile = (int)(in_group / together) * Shape::B;
    const int first = split * a.split_chunks, count = min(a.chunks - first, a.split_chunks);

    // what this wave loads: PW panels of A's and then B's, and of the scales of A's and then B's rows, 64 by 64, one piece (or none)
    constexpr int PW = Shape::PER_WAVE;
    const bool of_a = PW * wave < Shape::A, scales_of_a = 4 * wave < Shape::A;
    const int panel0 = of_a ? m_tile + PW * wave : n_tile + PW * wave - Shape::A, last = (of_a ? a.a_tiles : a.b_tiles) - 1;
    const char *panel[PW];
#pragma unroll
    for (int p = 0; p < PW; ++p)                                                             // (past the last: computed and not stored)
        panel[p] = uniform_pointer((of_a ? a.a : a.b) + ((size_t)min(panel0 + p, last) * a.chunks + first) * kF8PanelBytes);
    const int pitch = scales_of_a ? a.a_pitch : a.b_pitch, left = scales_of_a ? a.a_left : a.b_pitch, row0 = (scales_of_a ? m_tile + 4 * wave : n_tile + 4 * wave - Shape::A) * 16;
    const char *scales = uniform_pointer((const char *)((scales_of_a ? a.a_scales : a.b_scales) + (size_t)first * pitch));
    const unsigned scale_at = (unsigned)f8_scale_at(row0 + lane, scales_of_a ? a.a_shift : a.b_shift, left) * 4u;
    const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(size_t)((__attribute__((address_space(3))) const void *)lds));
    auto issue = [&](int stage) __attribute__((always_inline)) {
        const unsigned at = lds0 + (unsigned)(stage * STAGE);
#pragma unroll
        for (int p = 0; p < PW; p += 2) {
            const void *planes[4] = {panel[p], panel[p] + 1024, panel[p + 1], panel[p + 1] + 1024};
            global_to_lds16_run<4, 1024>(planes, lane * 16u, at + (unsigned)((PW * wave + p) * kF8PanelBytes));
        }
        if (Shape::SCALE_LOADS == Shape::WAVES || wave < Shape::SCALE_LOADS) global_to_lds4(scales, scale_at, at + (unsigned)(Shape::PANELS + wave * 256));
#pragma unroll
        for (int p = 0; p < PW; ++p) panel[p] += kF8PanelBytes;
        scales += (size_t)pitch * 4;
    };

    float4v sum[MT][NT];
#pragma unroll
    for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int y = 0; y < NT; ++y) sum[x][y] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](const char *stage) __attribute__((always_inline)) {
        const char *const pa = stage + wm * MT * kF8PanelBytes, *const pb = stage + (Shape::A + wn * NT) * kF8PanelBytes;
        const float *const sa = (const float *)(stage + Shape::PANELS) + wm * MT * 16, *const sb = (const float *)(stage + Shape::PANELS) + (Shape::A + wn * NT) * 16;
        F8Input<FA, WAY> fa[MT];
        F8Input<FB, WAY> fb[2];
        float s[MT];
        float4v more[3], p[3];
#pragma unroll
        for (int x = 0; x < MT; ++x) {
            fa[x].set(load_fragment(pa + x * kF8PanelBytes, lane));
            s[x] = sa[x * 16 + i] * (BAND ? sb[0] : 1.0f);
        }
        auto load_columns = [&](int y) __attribute__((always_inline)) {
            fb[y % 2].set(load_fragment(pb + y * kF8PanelBytes, lane));
            if constexpr (!BAND) more[y % 3] = *(const float4v *)(sb + y * 16 + 4 * b);
        };
        auto add = [&](int k, const float4v &products) __attribute__((always_inline)) {
            const int x = k % MT, y = k / MT;
#pragma unroll
            for (int v = 0; v < 4; ++v) sum[x][y][v] = fma32(BAND ? s[x] : s[x] * more[y % 3][v], products[v], sum[x][y][v]);
        };
        if constexpr (WAY == F8_NARROW) {
            // A wave issues its instructions in order, so each matrix instruction is followed by the additions of the one two before, whose sums have arrived.  (The empty
            // statements keep that order: the compiler gathers the additions behind the matrix instructions, with more sums in between than there are registers.)
            load_columns(0);
            static_for<MT * NT + 2>([&](auto K) __attribute__((always_inline)) {
                constexpr int k = K, x = k % MT, y = k / MT;
                if constexpr (k < MT * NT) {
                    asm volatile("" : "+v"(fa[x].codes));
                    p[k % 3] = f8_products<FB, FA, WAY>(fb[y % 2], fa[x]);
                    if constexpr (x == 0 && y + 1 < NT) load_columns(y + 1);
                }
                if constexpr (k >= 2) {
                    add(k - 2, p[(k - 2) % 3]);
                    asm volatile("" : "+v"(sum[(k - 2) % MT][(k - 2) / MT]));
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        } else {
            static_for<MT * NT>([&](auto K) __attribute__((always_inline)) {
                if constexpr (K % MT == 0) load_columns(K / MT);
                add(K, f8_products<FB, FA, WAY>(fb[K / MT % 2], fa[K % MT]));
            });
        }
    };

    auto step = [&](int c) __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");       // this wave's pieces of the stage have landed
        __syncthreads();                                         // everyone's have, and the other stage is read
        if (c + 1 < count) issue((c + 1) % 2);
        __builtin_amdgcn_sched_barrier(0);
        multiply(lds + c % 2 * STAGE);
    };
    issue(0);
    for (int c = 0; c < count; c += 2) {                         // (in pairs, so that which stage it is is known: 1024 x 4096 x 4096 32.5 -> 25.6 us)
        step(c);
        if (c + 1 < count) step(c + 1);
    }
    // Results leave as rows: a lane holds four columns of one row, and 16 rows side by side would go to memory as pieces of 32 bytes (8192 x 8192 results of one chunk
    // 69.3 us).  So a wave passes them through LDS, 32 rows at a time, and writes a row of its tile as a whole.
    constexpr int PITCH = Shape::PITCH;                          // bytes of a row
    static_assert(MT % 2 == 0, "rows in pairs of panels");
    __syncthreads();                                             // everyone has read the last stage
    char *const own = lds + wave * 32 * PITCH;
    with_results(a, (int)split, [&](auto element, void *out, int64_t ld, const void *bias, int flags) __attribute__((always_inline)) {
        typedef decltype(element) T;
        constexpr int COUNT = 16 / sizeof(T), LANES = NT * 16 / COUNT;                       // columns of a lane; lanes that write a row
        const int n = (n_tile + wn * NT) * 16 + lane % LANES * COUNT;
        const F8Columns<T, COUNT> columns(out, ld, bias, flags, a.N, n);
        static_for<MT / 2>([&](auto X) __attribute__((always_inline)) {
            constexpr int x = 2 * X;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int y = 0; y < NT; ++y) *(float4v *)(own + (h * 16 + i) * PITCH + y * 64 + b * 16) = sum[x + h][y];
            exchange_in_wave();
#pragma unroll
            for (int k = 0; k < 32 * LANES / 64; ++k) {
                const int r = lane / LANES + k * (64 / LANES);
                const int64_t m = (int64_t)(m_tile + wm * MT + x) * 16 + r;
                float results[COUNT];
#pragma unroll
                for (int q = 0; q < COUNT; q += 4) {
                    const float4v four = *(const float4v *)(own + r * PITCH + (lane % LANES * COUNT + q) * 4);
#pragma unroll
                    for (int v = 0; v < 4; ++v) results[q + v] = four[v];
                }
                if (m < a.M && n < a.N) columns.write(m, results);
            }
            exchange_in_wave();
        });
    });
}

// The pieces of a cut sum, in their order
__global__ void __launch_bounds__(256) f8_join_kernel(F8Call a)
{
    const int groups = (a.N + 3) / 4, splits = a.splits;
    a.splits = 1;
    for (size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x; idx < (size_t)a.M * groups; idx += (size_t)gridDim.x * 256) {
        const int64_t m = idx / groups;
        const int n = (int)(idx % groups) * 4;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int split = 0; split < splits; ++split)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (n + v < a.N) sum[v] += a.partial[f8_piece_at(a, split) + m * a.N + n + v];
        write_four(a, 0, m, n, sum);
    }
}

static F8Shape f8_shape(int M, int N, int K, bool full)
{
    F8Shape p = {};
    const int chunks = K / kF8Chunk + (K % kF8Chunk != 0);
    auto tiles = [&](int edge) { return ((int64_t)M + edge - 1) / edge * ((N + edge - 1) / edge); };
    p.splits = 1;
    if (M <= 64) {
        p.mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
        // More than 16 rows and 32 MB of weights: two panels of columns share the rows that a wave loads (32 rows by 25088 x 4096 32.8 -> 30.1 us, 64 by 4096 x 25088
        // 48 -> 39.5; 32 by 4096 x 4096, where workgroups count for more, 11.2 -> 12.3).  Fewer workgroups than compute units, of long sums, are cut.  A workgroup is
        // four waves (1 row by 4096 x 25088 20.2 us, with eight 21.8), eight where it has a compute unit for itself (1 by 25088 x 4096 22.4, with four 24.3).
        const int64_t panels = (N + 15) / 16;
        p.nt = p.mt > 1 && panels * chunks >= 16384 ? 2 : 1;
        const int64_t groups = (panels + p.nt - 1) / p.nt;
        while (groups * p.splits * 2 <= 256 && p.splits < 64 && chunks / (p.splits * 2) >= 32) p.splits *= 2;
        p.split_chunks = ceil_div(chunks, p.splits);
        p.waves = p.mt == 1 && groups * p.splits <= 256 && p.split_chunks >= 8 ? 8 : p.split_chunks >= 4 ? 4 : p.split_chunks;
    } else {
        // An estimate in us of each way.  128 x 128: one or two workgroups per compute unit, so a chunk of one or both; 256 x 256: one.  (From 1024 x 4096 x 4096 and
        // 8192 x 8192 x 8192, with 128 columns of B per scale.)  A cut sum's pieces are written and read, and another kernel joins them.  On 45 drawn calls of 65 to 4096 rows the
        // way and cut that it chooses took 1.016 times as long as the best of up to 16 tried, on the average, 1.13 at the most.
        double least = 0;
        for (int kind = 1; kind <= (full ? 1 : 2); ++kind)
            for (int splits = 1; splits <= 16 && splits <= chunks; ++splits) {
                const int k = ceil_div(chunks, splits);
                const int64_t blocks = tiles(kind == 1 ? 128 : 256) * splits, together = kind == 1 ? 512 : 256, rounds = blocks / together, rest = blocks % together;
                const double round = kind == 1 ? k * (full ? 1.72 : 1.0) + 5 : k * 1.5 + 7;
                const double part = kind == 1 && rest <= 256 ? k * (full ? 1.2 : 0.65) + 4 : round;
                const double time = rounds * round + (rest ? part : 0) + (splits > 1 ? 4 + splits * (0.4 + 2e-6 * M * N) : 0);
                if (least == 0 || time < least) least = time, p.kind = kind, p.splits = splits;
            }
        p.split_chunks = ceil_div(chunks, p.splits);
    }
    p.splits = ceil_div(chunks, p.split_chunks);
    return p;
}

size_t f8_matmul_workspace(int M, int N, int K, int dtype)
{
    const F8Shape p = f8_shape(M, N, K, dtype == NOVA_F32);
    return p.splits > 1 ? ((size_t)p.splits * M * N * 4 + 255) & ~(size_t)255 : 0;
}

template <typename Shape, int FA, int FB, int WAY, bool BAND>
static int run_tiles(const F8Call &a, hipStream_t s)
{
    const auto kernel = f8_tile_kernel<Shape, FA, FB, WAY, BAND>;
    NOVA_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, Shape::LDS));
    const int64_t across = (a.b_tiles + Shape::B - 1) / Shape::B * (int64_t)a.splits;
    const int64_t step = f8_launch_panels(across, Shape::A, kF8LaunchBlocks);
    for (int64_t first = 0; first < a.a_tiles; first += step) {
        const F8Call part = f8_launch(a, first, step);
        kernel<<<(unsigned)(across * ((part.a_tiles + Shape::A - 1) / Shape::A)), Shape::THREADS, Shape::LDS, s>>>(part);
        NOVA_HIP_TRY(hipGetLastError());
    }
    return 0;
}

template <int MT, int NT, int FA, int FB, int WIDE, bool BAND, int DT>
static int run_rows(const F8Call &a, const F8RowsOf &rows, const F8Shape &p, hipStream_t s)
{
    const auto kernel = f8_rows_kernel<MT, NT, FA, FB, WIDE, BAND, DT>;
    const size_t sums = (size_t)p.waves * MT * NT * 1024, operand = DT == kLaidOut ? 0 : (size_t)a.split_chunks * a.M * (kF8Chunk + 4);
    const size_t lds = sums > operand ? sums : operand;          // 33 KB at most
    kernel<<<(unsigned)((a.b_tiles + NT - 1) / NT * (int64_t)a.splits), p.waves * 64, lds, s>>>(a, rows);
    return (int)hipGetLastError();
}

template <int FA, int FB, int WAY, bool BAND>
static int run_band(const F8Call &a, const F8Shape &p, hipStream_t s)
{
    if (p.kind == 2) {
        if constexpr (WAY == F8_NARROW) return run_tiles<F8Tile<4, 2, 4, 8>, FA, FB, WAY, BAND>(a, s);
    }
    // Eight waves hide more of each other's waits: 517 x 5001 x 2055 to bfloat16 18.2 -> 14.9 us, to binary32 25.8 -> 24.1.  But as binary16 each wave makes its operands,
    // and where compute units hold two workgroups and sums are long, four are the faster (8192 x 8192 x 8192 937 -> 883, 4096 x 4096 x 1024 42.9 -> 41.8; but x 512 27.5, with
    // four 27.9, and the gradients of 32 rows by 25088 x 4096 122.6, with four 131.6).
    if (p.kind >= 1) {
        if constexpr (WAY == F8_NARROW) {
            return run_tiles<F8Tile<2, 4, 4, 2>, FA, FB, WAY, BAND>(a, s);
        } else {
            const int64_t blocks = (int64_t)((a.a_tiles + 7) / 8) * ((a.b_tiles + 7) / 8) * a.splits;
            return blocks <= 256 || a.split_chunks <= 6 ? run_tiles<F8Tile<4, 2, 2, 4>, FA, FB, WAY, BAND>(a, s) : run_tiles<F8Tile<2, 2, 4, 4>, FA, FB, WAY, BAND>(a, s);
        }
    }
    constexpr int WIDE = WAY == F8_FULL;
    if (p.mt == 1) return run_rows<1, 1, FA, FB, WIDE, BAND, kLaidOut>(a, {}, p, s);
    if (p.mt == 2) return p.nt == 1 ? run_rows<2, 1, FA, FB, WIDE, BAND, kLaidOut>(a, {}, p, s) : run_rows<2, 2, FA, FB, WIDE, BAND, kLaidOut>(a, {}, p, s);
    return p.nt == 1 ? run_rows<4, 1, FA, FB, WIDE, BAND, kLaidOut>(a, {}, p, s) : run_rows<4, 2, FA, FB, WIDE, BAND, kLaidOut>(a, {}, p, s);
}

template <int FA, int FB>
static int run(const F8Call &a, const F8Shape &p, hipStream_t s)
{
    const bool band = a.b_shift > 0;
    if (a.dtype == NOVA_F32) return band ? run_band<FA, FB, F8_FULL, true>(a, p, s) : run_band<FA, FB, F8_FULL, false>(a, p, s);
    return band ? run_band<FA, FB, F8_NARROW, true>(a, p, s) : run_band<FA, FB, F8_NARROW, false>(a, p, s);
}

static int join(const F8Call &a, hipStream_t s)
{
    if (a.splits == 1) return 0;
    const size_t blocks = ((size_t)a.M * ((a.N + 3) / 4) + 255) / 256;
    f8_join_kernel<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(a);
    return (int)hipGetLastError();
}

static F8Call make_call(const F8Operand &a, const F8Operand &b, const F8Shape &p, const void *bias, void *out, int64_t ldout, int dtype, int flags, void *workspace)
{
    const F8Layout &la = a.layout, &lb = b.layout;
    return {(const char *)a.q, (const char *)b.q, (const float *)((const char *)a.q + la.code_bytes), (const float *)((const char *)b.q + lb.code_bytes), bias, out,
            (float *)workspace, ldout, la.rows, lb.rows, la.chunks, p.splits, p.split_chunks, la.row_tiles, lb.row_tiles, la.scale_pitch, lb.scale_pitch,
            la.block == 1 ? 0 : 7, lb.block == 1 ? 0 : 7, dtype, flags, la.scale_pitch, la.rows};
}

int launch_f8_matmul(const F8Operand &a, const F8Operand &b, const void *bias, void *out, int64_t ldout, int dtype, int flags, void *workspace, void *stream)
{
    const F8Shape p = f8_shape(a.layout.rows, b.layout.rows, a.layout.columns, dtype == NOVA_F32);
    const F8Call call = make_call(a, b, p, bias, out, ldout, dtype, flags, workspace);
    hipStream_t s = (hipStream_t)stream;
    const int err = a.format == NOVA_F8_E4M3 ? b.format == NOVA_F8_E4M3 ? run<NOVA_F8_E4M3, NOVA_F8_E4M3>(call, p, s) : run<NOVA_F8_E4M3, NOVA_F8_E5M2>(call, p, s)
                    : b.format == NOVA_F8_E4M3 ? run<NOVA_F8_E5M2, NOVA_F8_E4M3>(call, p, s)
                                               : run<NOVA_F8_E5M2, NOVA_F8_E5M2>(call, p, s);
    return err ? err : join(call, s);
}

// The layer y = Q(x) W^T: x is quantised into `a` (a layout in the caller's workspace), or on the way
int launch_f8_linear(const F8Source &x, const F8Operand &a, const F8Operand &w, const void *bias, void *y, int64_t ldy, int flags, void *workspace, void *stream)
{
    const F8Shape p = f8_shape(x.rows, w.layout.rows, x.columns, x.dtype == NOVA_F32);
    if (quantised_on_the_way(x.rows, w.layout.rows, p)) {
        const F8Call call = make_call(a, w, p, bias, y, ldy, x.dtype, flags, workspace);
        const F8RowsOf rows = {x.x, x.ld, x.columns};
        hipStream_t s = (hipStream_t)stream;
        const int err = x.dtype == NOVA_F32   ? run_rows<1, 1, NOVA_F8_E4M3, NOVA_F8_E4M3, 1, true, NOVA_F32>(call, rows, p, s)
                        : x.dtype == NOVA_F16 ? run_rows<1, 1, NOVA_F8_E4M3, NOVA_F8_E4M3, 0, true, NOVA_F16>(call, rows, p, s)
                                              : run_rows<1, 1, NOVA_F8_E4M3, NOVA_F8_E4M3, 0, true, NOVA_BF16>(call, rows, p, s);
        return err ? err : join(call, s);
    }
    if (int err = launch_f8_quantize(x, a.layout, a.format, 0, const_cast<void *>(a.q), stream)) return err;
    return launch_f8_matmul(a, w, bias, y, ldy, x.dtype, flags, workspace, stream);
}

}  // namespace nova
