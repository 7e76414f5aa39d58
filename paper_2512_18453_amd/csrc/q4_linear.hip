// The products of layers with 4-bit weights: y = x W^T (+ bias, ReLU) and the gradient of x, dx = d W.
//
// Codes are read as panels of 16 columns by 128 positions of the reduction (1 KB, one 16-byte load per lane) and become operands of the matrix unit in
// registers (q4_common.hpp).
//   forward   a group's products are summed on the matrix unit with the codes as integers and the sum is scaled in binary32
//   backward  the scales run along the reduction, so they go to the other operand: d * s in binary32, in two (three) bfloat16 pieces.  Two hold a
//             product of two bfloat16 numbers; one of binary16 numbers has 22 bits and loses 6, to 2^-5 of what rounding the result does: a third
//             piece is half as much matrix work again, and pieces of binary16 lack its range
// Two kernels: for up to 16 rows (q4_few_rows_kernel) the codes' bytes bind and nothing else; more rows (q4_tile_kernel) are shared by four waves through LDS.
// Where the result's tiles give too few workgroups, the reduction is cut over workgroups too; a third kernel adds the pieces in order.
#include "q4_common.hpp"

namespace nova {

// (called from several places, a step that is a function of its own would keep its stage in memory)
#define NOVA_INLINE __attribute__((always_inline))

struct Q4Call {
    const void *x, *gate, *bias;                  // x: the rows' operand; gate: the layer's result (backward)
    const char *Wq;
    void *out;
    float *partial;                               // [splits][M][rows of the layout]
    int64_t ldx, ldgate, ldout;
    int M, relu, splits, split_chunks;
    Q4Layout q;
};

// The scales of one column's groups in a panel, side by side
template <typename T, int COUNT>
struct alignas(sizeof(T) * COUNT) Several { T v[COUNT]; };

// Operand pieces of a row's eight elements: forward themselves, or three bfloat16 pieces of binary32; backward of the product with the scales
template <int DT, bool BACK> constexpr int kPieces = DT == NOVA_F32 ? 3 : BACK ? 2 : 1;

template <bool HALF> using Codes = std::conditional_t<HALF, F16Codes, Bf16Codes>;
template <bool HALF> constexpr float kUnit = HALF ? 1.0f : kCodeUnit;        // what the sums over such codes are multiplied by, at the end

// Forward, a group's sum is formed before its scale comes to it, and with rows of binary32 or bfloat16 such a sum can pass binary32's range (|x| adding up to
// 7e38) where the result does not.  A workgroup whose results are not all finite makes them again, from rows that are a 256th, in which no group's sum passes
// it, and writes those that were not: what holds infinities or NaN takes twice as long, anything else the check: 1 x 4096 x 1000 in binary32 6.83 -> 7.06 us,
// 32 x 4096 x 4096 in bfloat16 10.8 -> 11.2, 1024 x 8192 x 8192 148.6 -> 149.7.
template <int DT, bool BACK> constexpr int kPasses = BACK || DT == NOVA_F16 ? 1 : 2;
constexpr float kShrunk = 1.0f / 256;
template <int DT, int PASS>
__device__ __forceinline__ void row_fragment(const Eight<Storage<DT>> &x, Fragment (&f)[kPieces<DT, false>])
{
    Eight<Storage<DT>> row = x;
    if constexpr (PASS > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) row.v[i] = (Storage<DT>)((float)x.v[i] * kShrunk);
    }
    if constexpr (DT == NOVA_F32) split_fragment<kPieces<DT, false>>(row.v, f);
    else __builtin_memcpy(&f[0], &row, 16);
}
// What the sums of a pass are multiplied by
template <bool HALF, int PASS> constexpr float kSumUnit = PASS > 0 ? kUnit<HALF> / kShrunk : kUnit<HALF>;
// The thread's number; in a second pass one that the compiler does not know from the first, so that it keeps nothing in registers from there
template <int PASS>
__device__ __forceinline__ int thread_of_pass()
{
    int t = threadIdx.x;
    if constexpr (PASS > 0) asm volatile("" : "+v"(t));
    return t;
}
// Whether a thread of the workgroup has results left; flag: 0 since a barrier
__device__ __forceinline__ bool left_in_workgroup(bool mine, int &flag)
{
    exchange_in_wave();                           // (the wave has read what it reads of LDS, here and behind)
    if (mine) flag = 1;
    __syncthreads();
    const bool any = flag != 0;
    exchange_in_wave();
    return any;
}

template <typename T>
__device__ __forceinline__ void write_result(const Q4Call &a, int m, int n, float sum)
{
    if (a.bias) sum += load_f32((const T *)a.bias + n);
    if (a.relu) sum = sum < 0.0f ? 0.0f : sum;
    store_from_f32((T *)a.out + m * a.ldout + n, sum);
}

// ---- forward, up to 16 rows ----
//
// A wave makes 16 columns for all rows; `sharing` waves of a workgroup take the panels of the same columns in turn and add up through LDS in the order of their
// numbers.  Bound by the codes' bytes: a wave has AHEAD panels on their way in registers, with the rows' operand that belongs to them.  That is loaded
// along the rows, 256 bytes of four rows at a time, and goes through a piece of LDS that is the wave's own to the lanes that need it: read from memory as the
// matrix unit takes it, 16 rows side by side, each four lanes lie in four cache lines, and one row of 25088 by 4096 took 16.5 us, 16 rows 27.  Now one row
// takes 11.4 us (53 MB, 4.6 TB/s) with three sets of weights in turn and 12.8 with six, which the last-level cache cannot keep; 8 rows by 8192 x 4096 7.2:
// every 16 columns read all rows once more from L2.  The codes are streamed past it (1.5 us more without).
template <int DT, int GROUP, int QUADS>
struct FewRowsStage {
    uint4v codes;
    Eight<Storage<DT>> x[QUADS];                  // of row 4 i + lane / 16: positions 8 (lane % 16) ..
    Several<Storage<DT>, kQ4Chunk / GROUP> scale;
};

// `open`: in, which of the thread's results to write (bit i: the i-th); out, which were not written because they are not finite
template <int DT, int GROUP, int QUADS, int PASS>
__device__ __forceinline__ unsigned q4_few_rows_pass(const Q4Call &a, int sharing, unsigned open)
{
    typedef Storage<DT> T;
    typedef FewRowsStage<DT, GROUP, QUADS> Stage;
    constexpr bool HALF = DT == NOVA_F16;
    constexpr int P = kPieces<DT, false>, SCALES = kQ4Chunk / GROUP, AHEAD = 4;
    constexpr int PLANE = QUADS * 4 * 256, OWN = P * PLANE > 1024 ? P * PLANE : 1024;        // bytes of a wave: the operand, later its sums
    extern __shared__ __align__(16) char lds[];
    const Q4Layout &q = a.q;
    const int thread = thread_of_pass<PASS>(), lane = thread % 64, wave = __builtin_amdgcn_readfirstlane(thread / 64), tiles = blockDim.x / 64 / sharing;
    const int tile0 = blockIdx.x * tiles;
    const int tile = min(tile0 + wave / sharing, q.row_tiles - 1);           // (past the last: computed and not stored)
    // whole panels of this wave, and the one that ends inside
    const int whole = q.reduction / kQ4Chunk, first = wave % sharing, count = whole > first ? (whole - first + sharing - 1) / sharing : 0;
    const bool ragged = whole < q.chunks && first == whole % sharing;
    const T *scales = (const T *)(a.Wq + q.code_bytes) + (size_t)tile * q.scale_pitch * kQ4Rows;
    const char *codes = a.Wq + (size_t)tile * q.chunks * kQ4PanelBytes;
    const T *x[QUADS];
#pragma unroll
    for (int i = 0; i < QUADS; ++i) x[i] = (const T *)a.x + min(4 * i + lane / 16, a.M - 1) * a.ldx + lane % 16 * 8;     // (as above)
    char *own = lds + wave * OWN;
    const Codes<HALF> codes_to_operand;

    auto load_panel = [&](int c, Stage &s) NOVA_INLINE {
        s.codes = __builtin_nontemporal_load((const uint4v *)(codes + (size_t)c * kQ4PanelBytes + lane * 16u));
        s.scale = ((const Several<T, SCALES> *)scales)[(size_t)c * kQ4Rows + lane % 16u];
    };
    auto load = [&](int i, Stage &s) NOVA_INLINE {
        // (past the last: the last once more, and not multiplied; with the load in a branch every step waits for all of them, one row 16.1 us against 11.4)
        const int c = first + min(i, count - 1) * sharing;
#pragma unroll
        for (int r = 0; r < QUADS; ++r) __builtin_memcpy(&s.x[r], x[r] + c * kQ4Chunk, sizeof s.x[r]);
        load_panel(c, s);
    };

    float4v acc = {0, 0, 0, 0}, part = {0, 0, 0, 0};
    auto multiply = [&](const Stage &s) NOVA_INLINE {
        // 16-byte block b of row r lies at block b ^ r % 8: eight rows that are read at a time lie in different banks.  (Four rows are each read by four lanes:
        // 3 cycles of conflicts per LDS instruction are counted there, some 400 of a wave's 24000.)
#pragma unroll
        for (int r = 0; r < QUADS; ++r) {
            const int row = 4 * r + lane / 16;
            Fragment f[P];
            row_fragment<DT, PASS>(s.x[r], f);
#pragma unroll
            for (int p = 0; p < P; ++p) *(uint4v *)(own + p * PLANE + row * 256 + ((lane % 16) ^ (row % 8)) * 16) = f[p].vec;
        }
        exchange_in_wave();
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int row = lane % (4 * QUADS);
            Fragment rows[P];
#pragma unroll
            for (int p = 0; p < P; ++p) rows[p].vec = *(const uint4v *)(own + p * PLANE + row * 256 + ((w * 4 + lane / 16) ^ (row % 8)) * 16);
            const Fragment columns = codes_to_operand(s.codes[w]);
            if (w * 32 % GROUP == 0) part = (float4v){0, 0, 0, 0};
#pragma unroll
            for (int p = 0; p < P; ++p) part = mfma<HALF>(rows[p], columns, part);
            if ((w + 1) * 32 % GROUP == 0) {
                const float scale = (float)s.scale.v[w * 32 / GROUP];
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] = fma32(scale, part[i], acc[i]);
            }
        }
        exchange_in_wave();
    };

    Stage stage[AHEAD];
    if (ragged) {
#pragma unroll
        for (int r = 0; r < QUADS; ++r) stage[AHEAD - 1].x[r] = load_eight(x[r] + whole * kQ4Chunk, q.reduction - (whole * kQ4Chunk + lane % 16 * 8), whole > 0);
        load_panel(whole, stage[AHEAD - 1]);
    }
    if (count > 0) static_for<AHEAD - 1>([&](auto I) { load(I, stage[I]); });
    if (ragged) multiply(stage[AHEAD - 1]);
    for (int i = 0; i < count; i += AHEAD)
        static_for<AHEAD>([&](auto I) {
            load(i + I + AHEAD - 1, stage[(I + AHEAD - 1) % AHEAD]);
            if (i + I < count) multiply(stage[I]);
        });
#pragma unroll
    for (int i = 0; i < 4; ++i) ((float *)own)[(lane / 16 * 4 + i) * 16 + lane % 16] = acc[i];
    __syncthreads();
    unsigned left = 0;
    for (int e = thread, bit = 1; e < tiles * 256; e += blockDim.x, bit *= 2) {
        float sum = 0.0f;
        for (int w = 0; w < sharing; ++w) sum += ((const float *)(lds + (e / 256 * sharing + w) * OWN))[e % 256];
        sum *= kSumUnit<HALF, PASS>;
        const int m = e % 256 / 16, n = (tile0 + e / 256) * 16 + e % 16;
        if (m >= a.M || n >= q.rows || (PASS > 0 && !(open & bit))) continue;
        if (PASS < kPasses<DT, false> - 1 && !__builtin_isfinite(sum)) left |= bit;
        else write_result<T>(a, m, n, sum);
    }
    return left;
}

template <int DT, int GROUP, int QUADS>
__global__ void __launch_bounds__(1024) q4_few_rows_kernel(const Q4Call a, int sharing)
{
    __shared__ int flag;
    if (kPasses<DT, false> > 1 && threadIdx.x == 0) flag = 0;
    const unsigned open = q4_few_rows_pass<DT, GROUP, QUADS, 0>(a, sharing, ~0u);
    if constexpr (kPasses<DT, false> > 1)
        if (left_in_workgroup(open != 0, flag)) q4_few_rows_pass<DT, GROUP, QUADS, 1>(a, sharing, open);
}

// ---- more rows, and the gradient ----
//
// A workgroup of four waves makes 16 MT rows by 64 NT columns: the rows' operand of 128 positions goes through LDS (as the matrix unit takes it: pieces, backward
// with the scales multiplied in, once for each of the VERSIONS groups that the columns lie in), every wave reads it whole and multiplies its own NT panels. Two
// such stages: one is filled while the other is multiplied; what fills them is loaded AHEAD - 1 stages before.  A row's 16-byte blocks are stored at
// block ^ row % 16, so the 16 rows that a fragment's load touches lie in different banks.
//
// Many rows: 1024 by 8192 x 8192 in bfloat16 146 us, 941 TFLOP/s where a large library product of that type reaches 1211.  A panel is made into operands once per
// 64 rows, three vector instructions for each of its matrix instructions, so both units are busy (without making operands it took 124 us); 256 columns halve the
// LDS reads of 128 (162 us); eight waves on 128 rows were slower (174 to 227), as all of them wait at one barrier, and so were matrix instructions of 32 by 32
// (151).  Few tiles: 32 rows of the first layer behind the VGG stack (53 MB) 18.9 us, of which the second launch and 8 MB of pieces take 6; four groups of waves
// per workgroup that shared a tile's stages instead of most of the cut gained nothing.  Gradient: twice the products, 512 rows by 4096 x 16384 148 us; the versions
// of smaller groups and the narrower tiles that go with them 215 us (64) and 378 (32).
template <int MT_, int NT_, int AHEAD_>
struct Tile {
    static constexpr int MT = MT_, NT = NT_, AHEAD = AHEAD_, ROWS = 16 * MT, PANELS = 4 * NT;
    template <bool BACK, int GROUP> static constexpr int versions = BACK && 16 * PANELS > GROUP ? 16 * PANELS / GROUP : 1;
    template <int DT, bool BACK, int GROUP> static constexpr unsigned lds_bytes = 2 * versions<BACK, GROUP> * kPieces<DT, BACK> * ROWS * 256;
    static_assert(AHEAD % 2 == 0, "two stages in LDS");
};

template <int DT, bool BACK, int GROUP, typename Shape>
struct TileStage {
    Eight<Storage<DT>> x[Shape::MT], gate[BACK ? Shape::MT : 1], row_scale[Shape::template versions<BACK, GROUP>];
    uint4v codes[Shape::NT];
    Several<Storage<DT>, kQ4Chunk / GROUP> scale[BACK ? 1 : Shape::NT];
};

// `open` as above, bit (4 t + i) NT + n
template <int DT, bool BACK, int GROUP, typename Shape, int PASS>
__device__ __forceinline__ uint64_t q4_tile_pass(const Q4Call &a, uint64_t open)
{
    typedef Storage<DT> T;
    typedef TileStage<DT, BACK, GROUP, Shape> Stage;
    constexpr int MT = Shape::MT, NT = Shape::NT, AHEAD = Shape::AHEAD;
    constexpr bool HALF = DT == NOVA_F16 && !BACK;
    constexpr int P = kPieces<DT, BACK>, SCALES = kQ4Chunk / GROUP, VERSIONS = Shape::template versions<BACK, GROUP>;
    static_assert(VERSIONS == 1 || NT * 16 <= GROUP, "a wave's columns lie in one group");
    constexpr int PLANE = Shape::ROWS * 256, LDS_STAGE = VERSIONS * P * PLANE;        // bytes
    extern __shared__ __align__(16) char lds[];
    const Q4Layout &q = a.q;
    const int thread = thread_of_pass<PASS>(), lane = thread % 64, wave = __builtin_amdgcn_readfirstlane(thread / 64);
    const int column_blocks = (q.row_tiles + Shape::PANELS - 1) / Shape::PANELS, row_blocks = (a.M + Shape::ROWS - 1) / Shape::ROWS;
    const unsigned id = xcd_local_block_id(blockIdx.x, gridDim.x);
    const int m0 = id % row_blocks * Shape::ROWS, block_tile = id / row_blocks % column_blocks * Shape::PANELS, split = id / row_blocks / column_blocks;
    const int tile0 = block_tile + wave * NT;
    // whole panels, and the one that ends inside
    const int whole = q.reduction / kQ4Chunk, first = split * a.split_chunks, count = min(whole - first, a.split_chunks);
    const bool ragged = whole < q.chunks && split == a.splits - 1;
    const T *scales = (const T *)(a.Wq + q.code_bytes);
    const Codes<HALF> codes_to_operand;

    // thread t stages row t / 16 of every 16, positions 8 (t % 16) ..
    const int my_row = thread / 16, my_pos = thread % 16 * 8;
    const T *x_row[MT], *gate_row[BACK ? MT : 1];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = min(m0 + t * 16 + my_row, a.M - 1);                // (past the last: computed and not stored)
        x_row[t] = (const T *)a.x + m * a.ldx + my_pos;
        if (BACK) gate_row[t] = (const T *)a.gate + m * a.ldgate + my_pos;
    }
    const char *panels[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) panels[n] = a.Wq + (size_t)min(tile0 + n, q.row_tiles - 1) * q.chunks * kQ4PanelBytes;       // (as above)
    auto load_panels = [&](int c, Stage &s) NOVA_INLINE {
        if constexpr (BACK) {
            const int group = block_tile * 16 / GROUP;
#pragma unroll
            for (int v = 0; v < VERSIONS; ++v)
                __builtin_memcpy(&s.row_scale[v], scales + (size_t)min(group + v, q.groups - 1) * q.scale_pitch + c * kQ4Chunk + my_pos, sizeof s.row_scale[v]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            s.codes[n] = *(const uint4v *)(panels[n] + (size_t)c * kQ4PanelBytes + lane * 16u);
            if constexpr (!BACK)
                s.scale[n] = ((const Several<T, SCALES> *)scales)[((size_t)min(tile0 + n, q.row_tiles - 1) * q.chunks + c) * kQ4Rows + lane % 16u];
        }
    };
    auto load = [&](int i, Stage &s) NOVA_INLINE {
        const int c = first + min(i, count - 1), at = c * kQ4Chunk;             // (past the last: the last once more, and not multiplied)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            __builtin_memcpy(&s.x[t], x_row[t] + at, sizeof s.x[t]);
            if (BACK && a.gate) __builtin_memcpy(&s.gate[t], gate_row[t] + at, sizeof s.x[t]);
        }
        load_panels(c, s);
    };
    auto fill = [&](char *stage, const Stage &s) NOVA_INLINE {
#pragma unroll
        for (int v = 0; v < VERSIONS; ++v)
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                Fragment f[P];
                if constexpr (BACK) {
                    float d[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] = (float)s.x[t].v[i];
                    if (a.gate) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) d[i] = (float)s.gate[t].v[i] > 0.0f ? d[i] : 0.0f;
                    }
                    // (behind the gate: zero times a scale that is no number is NaN)
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] *= (float)s.row_scale[v].v[i];
                    split_fragment<P>(d, f);
                } else {
                    row_fragment<DT, PASS>(s.x[t], f);
                }
#pragma unroll
                for (int p = 0; p < P; ++p)
                    *(uint4v *)(stage + (v * P + p) * PLANE + (t * 16 + my_row) * 256 + ((my_pos / 8) ^ my_row) * 16) = f[p].vec;
            }
    };

    float4v acc[MT][NT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[t][n] = (float4v){0, 0, 0, 0};
    const int version = VERSIONS > 1 ? wave * NT * 16 / GROUP : 0;
    auto read_rows = [&](const char *stage, int w, Fragment (&rows)[MT][P]) NOVA_INLINE {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int p = 0; p < P; ++p)
                rows[t][p].vec = *(const uint4v *)(stage + (version * P + p) * PLANE + (t * 16 + lane % 16) * 256 + ((w * 4 + lane / 16) ^ (lane % 16)) * 16);
    };
    auto multiply = [&](const char *stage, const Stage &s) NOVA_INLINE {
        if constexpr (BACK) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                Fragment rows[MT][P];
                read_rows(stage, w, rows);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const Fragment columns = codes_to_operand(s.codes[n][w]);
#pragma unroll
                    for (int p = P - 1; p >= 0; --p)
#pragma unroll
                        for (int t = 0; t < MT; ++t) acc[t][n] = mfma<false>(rows[t][p], columns, acc[t][n]);
                }
            }
        } else {
            float4v part[MT][NT];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                Fragment rows[MT][P];
                read_rows(stage, w, rows);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const Fragment columns = codes_to_operand(s.codes[n][w]);
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int t = 0; t < MT; ++t)
                            part[t][n] = mfma<HALF>(rows[t][p], columns, w * 32 % GROUP == 0 && p == 0 ? (float4v){0, 0, 0, 0} : part[t][n]);
                }
                if ((w + 1) * 32 % GROUP == 0) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const float scale = (float)s.scale[n].v[w * 32 / GROUP];
#pragma unroll
                        for (int t = 0; t < MT; ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[t][n][i] = fma32(scale, part[t][n][i], acc[t][n][i]);
                    }
                }
            }
        }
    };

    Stage stage[AHEAD];
    if (count > 0) static_for<AHEAD - 1>([&](auto I) { load(I, stage[I]); });
    if (ragged) {
        Stage &s = stage[AHEAD - 1];
        const int at = whole * kQ4Chunk;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            s.x[t] = load_eight(x_row[t] + at, q.reduction - (at + my_pos), whole > 0);
            if (BACK && a.gate) s.gate[t] = load_eight(gate_row[t] + at, q.reduction - (at + my_pos), whole > 0);
        }
        load_panels(whole, s);
        fill(lds + LDS_STAGE, s);
        __syncthreads();
        multiply(lds + LDS_STAGE, s);
    }
    if (count > 0) fill(lds, stage[0]);
    for (int i = 0; i < count; i += AHEAD)
        static_for<AHEAD>([&](auto I) {
            if (i + I < count) {
                load(i + I + AHEAD - 1, stage[(I + AHEAD - 1) % AHEAD]);
                __syncthreads();
                multiply(lds + I % 2 * LDS_STAGE, stage[I]);
                if (i + I + 1 < count) fill(lds + (I + 1) % 2 * LDS_STAGE, stage[(I + 1) % AHEAD]);
            }
        });

    uint64_t left = 0;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = m0 + t * 16 + lane / 16 * 4 + i;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int column = (tile0 + n) * 16 + lane % 16;
                const uint64_t bit = (uint64_t)1 << ((t * 4 + i) * NT + n);
                if (m >= a.M || column >= q.rows || (PASS > 0 && !(open & bit))) continue;
                const float sum = acc[t][n][i] * kSumUnit<HALF, PASS>;
                if (PASS < kPasses<DT, BACK> - 1 && !__builtin_isfinite(sum)) left |= bit;
                else if (a.splits > 1) a.partial[((size_t)split * a.M + m) * q.rows + column] = sum;
                else write_result<T>(a, m, column, sum);
            }
        }
    return left;
}

template <int DT, bool BACK, int GROUP, typename Shape>
__global__ void __launch_bounds__(256, 2) q4_tile_kernel(const Q4Call a)
{
    __shared__ int flag;
    if (kPasses<DT, BACK> > 1 && threadIdx.x == 0) flag = 0;
    const uint64_t open = q4_tile_pass<DT, BACK, GROUP, Shape, 0>(a, ~(uint64_t)0);
    if constexpr (kPasses<DT, BACK> > 1)
        if (left_in_workgroup(open != 0, flag)) q4_tile_pass<DT, BACK, GROUP, Shape, 1>(a, open);
}

// The pieces of a cut reduction, in order
template <int DT>
__global__ void __launch_bounds__(256) q4_join_kernel(const Q4Call a)
{
    typedef Storage<DT> T;
    const size_t total = (size_t)a.M * a.q.rows;
    for (size_t at = (size_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (size_t)gridDim.x * 256) {
        float sum = 0.0f;
        for (int s = 0; s < a.splits; s += 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = s + i < a.splits ? a.partial[(s + i) * total + at] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[i];
        }
        write_result<T>(a, (int)(at / a.q.rows), (int)(at % a.q.rows), sum);
    }
}

// How a call is cut: few rows (mt 0; nt: waves that share a tile's panels) or tiles of 16 mt rows by 64 nt columns; waves of a workgroup; pieces of the reduction.
struct Q4Shape { int mt, nt, waves, splits, split_chunks; };

// Time of a call with tiles, in us, as it measured on layers of 1000 to 25088 columns and positions at 12 to 512 rows (to some 15 %): 2 for the launch; the
// stages of a workgroup one after the other, each `stage` long on a compute unit of its own and 0.71 times the workgroups there where several share one, as
// many as the fullest unit has; and for a cut reduction a launch and the pieces, added one behind the other, written and read.
static double q4_tile_time(int M, const Q4Layout &q, int dtype, int mt, int nt, int splits)
{
    const int64_t row_blocks = ((int64_t)M + 16 * mt - 1) / (16 * mt), blocks = ceil_div(q.row_tiles, 4 * nt) * row_blocks * splits;
    const int64_t on_a_unit = (blocks + 255) / 256;
    double stage = nt == 4 ? 1.6 : mt == 4 ? 0.83 : mt == 2 ? 0.58 : 0.45;
    if (q.backward) stage = mt == 4 ? 1.62 : mt == 2 ? 1.0 : 0.7;
    if (dtype == NOVA_F32) stage *= 2;
    // (a unit holds two workgroups of the widest tile, three to five of the others)
    double load = nt == 4 ? (on_a_unit <= 1 ? 1 : 1.43 * ((on_a_unit + 1) / 2)) : 0.71 * on_a_unit;
    if (load < 1) load = 1;
    return 2 + ceil_div(q.chunks, splits) * stage * load + (splits > 1 ? 2.4 + 0.04 * splits + (double)splits * M * q.rows * 8 / 4e6 : 0);
}

static Q4Shape q4_shape(int M, const Q4Layout &q, int dtype)
{
    Q4Shape p;
    p.splits = 1;
    // Up to 16 rows without sharing them, where the rows' operand, read by every 16 columns, is little: 12 rows by 16384 x 4096 (100 MB of it) 12.3 us against 11.1
    // in tiles, 8 rows 10.3 against 10.7; 16 rows by 4096 x 4096 6.0 against 8.0.  Rows of an odd number of 16-bit elements begin between 32-bit words, which a
    // 16-byte load takes some twelve times as long over: 8 rows by 5000 x 3001 9.9 against 8.1 in tiles, by 1000 x 4097 5.7 against 6.4.  Many columns with
    // little to sum are sooner through in tiles: 6 rows by 30000 x 500 7.8 against 5.7, by 300 x 700 3.5 against 5.1.
    const double operand = (double)q.row_tiles * M * q.K * dtype_size(dtype) * (q.K * dtype_size(dtype) % 4 ? 12 : 1);
    // A long sum is left to few waves here and can be cut in tiles, where the columns are few enough that the pieces are: 16 rows by 25088 x 1000 in binary16
    // 19.9 us against 9.7, by 8192 x 1000 8.3 against 7.2, by 4096 x 1000 5.3 against 6.1; 8 rows 13.3 against 9.8, 6.1 against 6.9; 1 row 9.0 against 9.1.
    // Binary32, of three pieces: 1 row by 25088 x 10 20.2 against 8.9, by 8192 x 10 8.0 against 6.0, by 4096 x 1000 5.9 against 6.2; by 25088 x 4096 the same.
    const bool long_sums = q.row_tiles <= 128 && ((dtype == NOVA_F32 || M > 8) ? q.chunks >= 64 : M > 4 && q.chunks > 128);
    if (!q.backward && M <= (dtype == NOVA_F32 ? 4 : 16) && !long_sums && (M <= 4 || (operand < 100e6 && (q.chunks >= 16 || q.row_tiles <= 256)))) {
        p.mt = 0;
        p.nt = q.row_tiles <= 512 ? 8 : q.row_tiles <= 2048 ? 4 : 2;
        while (q.row_tiles > 512 && p.nt > 1 && p.nt * 2 > q.chunks) p.nt /= 2;
        p.waves = p.nt < 4 ? 4 : p.nt;
    } else {
        // (taller tiles take more registers than there are in binary32, and wider ones where a panel holds several groups; where the columns' scales come in two
        // versions, taller ones take so much LDS that a compute unit holds one workgroup: 700 rows by 4096 x 4096 backward 195 us against 148)
        const int tallest = (dtype == NOVA_F32 ? 2 : 4) / (q.backward && q.group == 32 ? 2 : 1);
        p.mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
        if (p.mt > tallest) p.mt = tallest;
        p.nt = q.backward && q.group < 128 ? 1 : 2;
        p.waves = 4;
        double least = q4_tile_time(M, q, dtype, p.mt, p.nt, 1);
        const int narrow = p.nt;
        for (int nt = narrow; nt <= (p.mt == 4 && !q.backward && q.group == 128 ? 4 : narrow); nt *= 2)
            for (int splits = 1; splits <= 64 && splits <= q.chunks; ++splits) {
                const double time = q4_tile_time(M, q, dtype, p.mt, nt, splits);
                if (time < least) least = time, p.nt = nt, p.splits = splits;
            }
    }
    p.split_chunks = ceil_div(q.chunks, p.splits);
    p.splits = ceil_div(q.chunks, p.split_chunks);
    return p;
}

size_t q4_linear_workspace(int M, const Q4Layout &q, int dtype)
{
    if (M == 0) return 0;
    const Q4Shape p = q4_shape(M, q, dtype);
    return p.splits > 1 ? (size_t)p.splits * M * q.rows * 4 : 0;
}

template <int DT>
static int join(const Q4Call &a, hipStream_t s)
{
    if (a.splits == 1) return 0;
    const size_t blocks = ((size_t)a.M * a.q.rows + 255) / 256;
    q4_join_kernel<DT><<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(a);
    return (int)hipGetLastError();
}

template <int DT, bool BACK, int GROUP, typename Shape>
static int run_tiles(const Q4Call &a, hipStream_t s)
{
    const auto kernel = q4_tile_kernel<DT, BACK, GROUP, Shape>;
    constexpr unsigned lds = Shape::template lds_bytes<DT, BACK, GROUP>;
    static_assert(lds <= 64 * 1024, "LDS of a workgroup");
    const int64_t columns = (int64_t)ceil_div(a.q.row_tiles, Shape::PANELS) * a.splits;
    int64_t tiles = ((int64_t)1 << 31) / 256 / columns;           // rows in pieces that keep a launch below 2^31 threads
    if (tiles < 1) tiles = 1;
    const int64_t M = a.M, step = tiles * Shape::ROWS;
    for (int64_t m0 = 0; m0 < M; m0 += step) {
        Q4Call part = a;
        part.M = (int)(M - m0 < step ? M - m0 : step);
        part.x = (const Storage<DT> *)a.x + m0 * a.ldx;
        if (a.gate) part.gate = (const Storage<DT> *)a.gate + m0 * a.ldgate;
        part.out = (Storage<DT> *)a.out + m0 * a.ldout;
        kernel<<<(unsigned)(columns * ceil_div(part.M, Shape::ROWS)), 256, lds, s>>>(part);
        NOVA_HIP_TRY(hipGetLastError());
        if (int err = join<DT>(part, s)) return err;
    }
    return 0;
}

template <int DT, int GROUP, int QUADS>
static void run_few_rows(const Q4Call &a, const Q4Shape &p, hipStream_t s)
{
    constexpr unsigned operand = kPieces<DT, false> * QUADS * 4 * 256, own = operand > 1024 ? operand : 1024;
    q4_few_rows_kernel<DT, GROUP, QUADS><<<ceil_div(a.q.row_tiles, p.waves / p.nt), p.waves * 64, p.waves * own, s>>>(a, p.nt);
}

template <int DT, bool BACK, int GROUP>
static int run_group(const Q4Call &a, const Q4Shape &p, hipStream_t s)
{
    if constexpr (!BACK) {
        if (p.mt == 0) {
            if (a.M <= 4) run_few_rows<DT, GROUP, 1>(a, p, s);
            else if constexpr (DT != NOVA_F32) {
                if (a.M <= 8) run_few_rows<DT, GROUP, 2>(a, p, s);
                else run_few_rows<DT, GROUP, 4>(a, p, s);
            }
            return (int)hipGetLastError();
        }
    }
    constexpr int NT = BACK && GROUP < 128 ? 1 : 2;
    if constexpr (DT != NOVA_F32 && !BACK && GROUP == 128)
        if (p.nt == 4) return run_tiles<DT, BACK, GROUP, Tile<4, 4, 2>>(a, s);
    if constexpr (DT != NOVA_F32 && !(BACK && GROUP == 32))
        if (p.mt == 4) return run_tiles<DT, BACK, GROUP, Tile<4, NT, 2>>(a, s);
    if constexpr (DT != NOVA_F32 || !(BACK && GROUP == 32))
        if (p.mt == 2) return run_tiles<DT, BACK, GROUP, Tile<2, NT, DT == NOVA_F32 ? 2 : 4>>(a, s);
    return run_tiles<DT, BACK, GROUP, Tile<1, NT, 2>>(a, s);
}

template <int DT, bool BACK>
static int run(Q4Call a, void *workspace, hipStream_t s)
{
    const Q4Shape p = q4_shape(a.M, a.q, DT);
    a.partial = (float *)workspace;
    a.splits = p.splits;
    a.split_chunks = p.split_chunks;
    if (a.q.group == 32) return run_group<DT, BACK, 32>(a, p, s);
    if (a.q.group == 64) return run_group<DT, BACK, 64>(a, p, s);
    return run_group<DT, BACK, 128>(a, p, s);
}

template <bool BACK>
static int run_type(const Q4Call &a, int dtype, void *workspace, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == NOVA_F32) return run<NOVA_F32, BACK>(a, workspace, s);
    if (dtype == NOVA_F16) return run<NOVA_F16, BACK>(a, workspace, s);
    return run<NOVA_BF16, BACK>(a, workspace, s);
}

int launch_q4_linear(const void *x, int64_t ldx, const void *Wq, const void *bias, void *y, int64_t ldy, int M, const Q4Layout &q, int dtype, int flags,
                     void *workspace, void *stream)
{
    const Q4Call a = {x, nullptr, bias, (const char *)Wq, y, nullptr, ldx, 0, ldy, M, (flags & NOVA_FLAG_RELU) != 0, 1, 0, q};
    return run_type<false>(a, dtype, workspace, stream);
}

int launch_q4_linear_backward(const void *dy, int64_t lddy, const void *y, int64_t ldy, const void *Wq, void *dx, int64_t lddx, int M, const Q4Layout &q,
                              int dtype, void *workspace, void *stream)
{
    const Q4Call a = {dy, y, nullptr, (const char *)Wq, dx, nullptr, lddy, ldy, lddx, M, 0, 1, 0, q};
    return run_type<true>(a, dtype, workspace, stream);
}

}  // namespace nova
