// Log probabilities of rows of logits, entropy, the largest alternatives, and the gradient of the first two (nova_logprobs in nova.h).
//
// With M the largest allowed logit and d = scale (x - M): L = ln sum e^d, H = L - sum e^d d / sum e^d.  All of it in one pass over a row: every lane keeps
// the largest logit m it has seen, s = sum e^d and u = sum e^d d relative to it, and when m grows by some D, s becomes s e^-D and u becomes (u - s D) e^-D.
// Rows are cut into slices where there are few of them; a second kernel joins the slices.
//
// Alternatives.  The pass leaves the largest logit of every lane and of every cell, the up to kCells parts that a lane's share is cut into.  If `least` is the
// top-th largest of the lane maxima, the slice holds `top` logits that reach it, so only cells whose maximum does are read again (with 131072
// logits and 8 alternatives some dozen of 4096; a slice of one step has its logits still in registers).  What reaches `least` in them is sorted by one wave.  Where that is more than kCandidates (equal logits over all of a row) or a NaN stands in the row, the waves go over the slice once more, keeping sorted lists.
#include "q4_common.hpp"

#include <algorithm>
#include <cmath>

namespace nova {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kVectors = 4;                       // 8-element pieces that a lane has in hand at a time
constexpr int kMaxWaves = 4;                      // of a workgroup that reads logits
constexpr int kJoinWaves = 16;
constexpr int kMaxSlices = 64;
constexpr int kCells = 16;                        // of a lane
constexpr int kCandidates = 512;                  // eight per lane of the wave that sorts them

typedef unsigned long long rank_t;

// Rank of a logit: greater for greater values, NaN one above +infinity, -0 and 0 alike, -infinity (and masked) 0; below it the index, smaller first.  The
// ranks of a row's entries that count are all different.
__device__ __forceinline__ unsigned value_rank(float v)
{
    unsigned bits = __float_as_uint(v);
    if (v == 0.0f) bits = 0;
    bits = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    return v != v ? 0xff800001u : v == -INFINITY ? 0 : bits;
}
__device__ __forceinline__ float value_of_rank(unsigned r)
{
    return r == 0xff800001u ? __builtin_nanf("") : r == 0 ? -INFINITY : __uint_as_float(r & 0x80000000u ? r & 0x7fffffffu : ~r);
}
// The lowest bit that tells two values of a type apart
template <int DT> constexpr int kRankBits = DT == NOVA_BF16 ? 16 : DT == NOVA_F16 ? 13 : 0;
__device__ __forceinline__ rank_t rank_of(unsigned value, unsigned index) { return value ? (rank_t)value << 32 | (0xffffffffu - index) : 0; }

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;                                      // (fmaxf makes every operand canonical first, an instruction each; NaN is looked for elsewhere)
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// The value of lane ^ STEP: moves inside 16 lanes and exchanges of 16 and 32 lanes, a few cycles each (through LDS it is a hundred)
template <int STEP>
__device__ __forceinline__ unsigned across(unsigned v)
{
    const int lane = threadIdx.x % 64;
    if constexpr (STEP == 1) return __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, false);             // quad_perm 1 0 3 2
    if constexpr (STEP == 2) return __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, false);             // quad_perm 2 3 0 1
    if constexpr (STEP == 4) {
        v = __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, false);                                       // lane ^ 7
        return __builtin_amdgcn_update_dpp(0, v, 0x1b, 0xf, 0xf, false);                                     // lane ^ 3
    }
    if constexpr (STEP == 8) return __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, false);            // rotation by 8 of 16
    if constexpr (STEP == 16) {
        const auto pair = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return lane & 16 ? pair[0] : pair[1];
    }
    if constexpr (STEP == 32) {
        const auto pair = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return lane & 32 ? pair[0] : pair[1];
    }
}
template <int STEP> __device__ __forceinline__ float across(float v) { return __uint_as_float(across<STEP>(__float_as_uint(v))); }
template <int STEP>
__device__ __forceinline__ rank_t across(rank_t v)
{
    return (rank_t)across<STEP>((unsigned)(v >> 32)) << 32 | across<STEP>((unsigned)v);
}

__device__ __forceinline__ rank_t read_lane(rank_t v, int lane)
{
    return (rank_t)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, lane);
}

// m, s, u of a part of a row (d in units of ln 2)
struct Sums {
    float m, s, u;
};
// Exponents of 2, scale log2 e times t: that factor is c + rest.  c alone is off by up to 1.2 units of 2^-24, alike for all entries of a row: at a scale of 0.9
// L and H of rows of 131071 logits were off by 4 and 28 such units where 32 bits throughout leave 1 and 2.  One more multiply per logit: 1024 rows of 131072
// bfloat16 logits 55.6 -> 57.5 us.  rest is above 0, so that what is infinite in t is so, with its sign, in both products.
struct Exponent {
    float c, rest;

    // bounded: the exponent in units of ln 2 as it counts in u, where it may meet a power of 0
    __device__ __forceinline__ float power(float t, float &bounded) const
    {
        const float d = fma32(t, c, t * rest);
        bounded = fmaxf(d, -1e4f);
        return __builtin_amdgcn_exp2f(d);
    }
};
__device__ __forceinline__ float finite_reference(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ Sums rebased(Sums p, float m, Exponent c)     // m >= p.m
{
    float D;
    const float f = c.power(p.m - finite_reference(m), D);
    return {m, p.s * f, fma32(p.s, D, p.u) * f};
}
__device__ __forceinline__ Sums joined(Sums p, Sums q, Exponent c)
{
    const float m = fmaxf(p.m, q.m);
    const Sums a = rebased(p, m, c), b = rebased(q, m, c);
    return {m, a.s + b.s, a.u + b.u};
}
__device__ __forceinline__ Sums over_wave(Sums p, Exponent c)
{
    static_for<6>([&](auto I) {
        constexpr int STEP = 32 >> I;
        p = joined(p, {across<STEP>(p.m), across<STEP>(p.s), across<STEP>(p.u)}, c);
    });
    return p;
}

// The best 64 of a wave, best first, one per lane (0: none)
struct Best {
    rank_t mine = 0;

    // wave-uniform r
    __device__ __forceinline__ void insert(rank_t r)
    {
        const int place = __popcll(__ballot(mine > r)), lane = threadIdx.x % 64;
        const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(mine >> 32), 0x138, 0xf, 0xf, false);       // of the lane below
        const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)mine, 0x138, 0xf, 0xf, false);
        mine = lane < place ? mine : lane == place ? r : (rank_t)hi << 32 | lo;
    }
    // another wave's list: the larger of each pair from both ends are the best 64, falling and then rising; six exchanges sort them
    __device__ __forceinline__ void merge(const rank_t *other)
    {
        const int lane = threadIdx.x % 64;
        const rank_t theirs = other[63 - lane];
        mine = mine > theirs ? mine : theirs;
        static_for<6>([&](auto I) {
            constexpr int STEP = 32 >> I;
            const rank_t theirs = across<STEP>(mine);
            mine = ((lane & STEP) == 0) == (mine > theirs) ? mine : theirs;
        });
    }
};

// The largest rank that at least `count` of the lanes' N ranks reach, from the top bit down to bit LOWEST
template <int LOWEST, typename R, int N>
__device__ __forceinline__ R reached_by(const R (&rank)[N], int count)
{
    R t = 0;
    for (int bit = (int)sizeof(R) * 8 - 1; bit >= LOWEST; --bit) {
        const R next = t | (R)1 << bit;
        int reaching = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) reaching += __popcll(__ballot(rank[i] >= next));
        if (reaching >= count) t = next;
        if (reaching == count) break;
    }
    return t;
}

// The best `top` of more candidates than lanes, one per lane, in any order
template <int N>
__device__ __forceinline__ rank_t best_of(const rank_t *candidates, int count, int top, rank_t *scratch)
{
    const int lane = threadIdx.x % 64;
    rank_t all[N];
#pragma unroll
    for (int i = 0; i < N; ++i) all[i] = i * 64 + lane < count ? candidates[i * 64 + lane] : 0;
    const rank_t least = reached_by<0>(all, top);
    int kept = 0;
    scratch[lane] = 0;
    exchange_in_wave();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const unsigned long long keep = __ballot(all[i] >= least);
        if (keep >> lane & 1) scratch[kept + __popcll(keep & ((1ull << lane) - 1))] = all[i];
        kept += __popcll(keep);
    }
    exchange_in_wave();
    const rank_t mine = scratch[lane];
    exchange_in_wave();
    return mine;
}

// The wave's candidates (count of them in `candidates`, all ranks different), the best `top` of them sorted, one per lane; scratch: 64 ranks
__device__ __forceinline__ rank_t sorted_best(const rank_t *candidates, int count, int top, rank_t *scratch)
{
    const int lane = threadIdx.x % 64;
    rank_t mine = lane < count ? candidates[lane] : 0;
    if (count > 64) {
        if (count <= 128) mine = best_of<2>(candidates, count, top, scratch);
        else mine = best_of<kCandidates / 64>(candidates, count, top, scratch);
        count = top;
    }
    int place = 0;
    for (int i = 0; i < count; ++i) place += read_lane(mine, i) > mine;
    scratch[lane] = 0;
    exchange_in_wave();
    if (lane < count) scratch[place] = mine;
    exchange_in_wave();
    return scratch[lane];
}

// What a row's sums and list give the caller
template <int DT, bool MASK>
__device__ __forceinline__ void write_row(const LogprobsArgs &a, int row, Sums p, rank_t best)
{
    const int lane = threadIdx.x % 64;
    const bool empty = p.m == -INFINITY && p.s == 0.0f, bad = !(p.s == p.s);
    const float log_sum = empty ? -INFINITY : kLn2 * __log2f(p.s), nan = __builtin_nanf("");
    if (lane == 0) {
        a.stats[2 * (int64_t)row] = bad ? nan : p.m;
        a.stats[2 * (int64_t)row + 1] = log_sum;
        if (a.entropy) a.entropy[row] = empty ? 0.0f : log_sum - kLn2 * (p.u / p.s);
        if (a.logprob) {
            const int64_t t = a.targets[row];
            float lp = t < 0 ? 0.0f : nan;
            if (t >= 0 && t < a.V) {
                const bool allowed = !MASK || a.mask[row * a.mask_stride + t];
                const float x = allowed ? load_f32((const Storage<DT> *)a.logits + row * a.stride + t) : -INFINITY;
                lp = bad ? nan : empty ? -INFINITY : fma32(x - p.m, a.scale, -log_sum);
            }
            a.logprob[row] = lp;
        }
    }
    if (lane < a.top) {
        const int64_t at = (int64_t)row * a.top + lane;
        a.top_ids[at] = best ? (int64_t)(0xffffffffu - (unsigned)best) : -1;
        a.top_logprobs[at] = bad ? nan : best ? fma32(value_of_rank((unsigned)(best >> 32)) - p.m, a.scale, -log_sum) : -INFINITY;
    }
}

// 16 bytes that are used once, from and to any element's address: past the caches.  1024 rows of 131072 bfloat16 logits forward 68 -> 51 us (52 with the
// exponents' second part), 256 rows (which the last-level cache could keep) 27 -> 22; written so the gradient 131 -> 92, 34 -> 25 us.  The gradient reads
// logits as usual: 256 rows 24.7 us against 26.6.
typedef unsigned loose16 __attribute__((ext_vector_type(4), aligned(2)));
template <typename T>
__device__ __forceinline__ void load_streamed(Eight<T> &e, const T *p)
{
#pragma unroll
    for (unsigned i = 0; i < sizeof e / 16; ++i) ((loose16 *)&e)[i] = __builtin_nontemporal_load((const loose16 *)p + i);
}
template <typename T>
__device__ __forceinline__ void store_streamed(T *p, const Eight<T> &e)
{
#pragma unroll
    for (unsigned i = 0; i < sizeof e / 16; ++i) __builtin_nontemporal_store(((const loose16 *)&e)[i], (loose16 *)p + i);
}

// Eight logits from `at` on with their mask; what is masked or not before `end` reads as -infinity
template <int DT, bool MASK, bool STREAMED>
struct MaskedEight {
    Eight<Storage<DT>> x;
    unsigned long long mask;

    __device__ __forceinline__ void load(const Storage<DT> *row, const uint8_t *row_mask, unsigned at, unsigned end)
    {
        if (at + 8 <= end) {
            if (STREAMED) load_streamed(x, row + at);
            else __builtin_memcpy(&x, row + at, sizeof x);
            if (MASK) __builtin_memcpy(&mask, row_mask + at, 8);
        } else {
            mask = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x.v[e] = at + e < end ? row[at + e] : (Storage<DT>)-INFINITY;
                if (MASK) mask |= (unsigned long long)(at + e < end ? row_mask[at + e] : 0) << (8 * e);
            }
        }
    }
    __device__ __forceinline__ bool allowed(int e) const { return !MASK || (mask >> (8 * e) & 0xff); }
    __device__ __forceinline__ float operator[](int e) const { return allowed(e) ? (float)x.v[e] : -INFINITY; }
};

// A slice's results in the workspace: Sums, then top ranks
__host__ __device__ inline size_t slice_bytes(int top) { return 16 + (size_t)top * 8; }

// Workgroup (row, slice): threads take pieces of 8 logits in turn, kVectors in hand
template <int DT, bool MASK, bool TOP, int WAVES>
__global__ void __launch_bounds__(WAVES * 64) logprobs_kernel(const LogprobsArgs a, int slices, int slice_length, char *__restrict__ workspace)
{
    constexpr int THREADS = WAVES * 64, CELLS = WAVES == 1 ? 1 : kCells;           // (one wave takes what it can have in hand)
    constexpr unsigned STRIDE = THREADS * 8, IN_HAND = kVectors * STRIDE;
    __shared__ Sums wave_sums[WAVES];
    __shared__ unsigned lane_ranks[TOP ? THREADS : 1];
    __shared__ float cell_largest[TOP ? CELLS : 1][TOP ? THREADS : 1];
    __shared__ unsigned short cells[TOP ? kCandidates : 1];
    __shared__ rank_t candidates[TOP ? kCandidates : 1], lists[TOP ? WAVES : 1][64];
    __shared__ int found_cells, found;
    const int row = blockIdx.x / slices, slice = blockIdx.x % slices;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const Storage<DT> *x = (const Storage<DT> *)a.logits + row * a.stride;
    const uint8_t *mask = MASK ? a.mask + row * a.mask_stride : nullptr;
    const unsigned begin = (unsigned)slice * slice_length, length = a.V - begin < (unsigned)slice_length ? a.V - begin : slice_length, end = begin + length;
    const unsigned chunks = (length + IN_HAND - 1) / IN_HAND, per_cell = (chunks + CELLS - 1) / CELLS;
    const Exponent c = {a.exponent, a.exponent_rest};

    typedef MaskedEight<DT, MASK, true> Piece;
    auto load_piece = [&](unsigned at, Piece &p) { p.load(x, mask, at, end); };
    Piece next[kVectors];
    auto fetch = [&](unsigned base) {
#pragma unroll
        for (int j = 0; j < kVectors; ++j) load_piece(base + j * STRIDE + threadIdx.x * 8, next[j]);
    };

    Sums mine = {-INFINITY, 0.0f, 0.0f};
    float in_cell = -INFINITY;
    if (TOP && threadIdx.x == 0) found_cells = found = 0;
    fetch(begin);
    float v[kVectors * 8];
    for (unsigned chunk = 0, left = per_cell, cell = 0; chunk < chunks; ++chunk) {
#pragma unroll
        for (int i = 0; i < kVectors * 8; ++i) v[i] = next[i / 8][i % 8];
        if (chunk + 1 < chunks) fetch(begin + (chunk + 1) * IN_HAND);
        float largest = v[0];
#pragma unroll
        for (int i = 1; i < kVectors * 8 - 1; i += 2) largest = max3(largest, v[i], v[i + 1]);
        largest = max3(largest, v[kVectors * 8 - 1], v[kVectors * 8 - 1]);
        mine = rebased(mine, max3(mine.m, largest, largest), c);
        const float ref = finite_reference(mine.m);
        float s[2] = {0, 0}, u[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < kVectors * 8; ++i) {
            float d;
            const float e = c.power(v[i] - ref, d);
            s[i % 2] += e;
            u[i % 2] = fma32(e, d, u[i % 2]);
        }
        mine.s += s[0] + s[1];
        mine.u += u[0] + u[1];
        if constexpr (TOP) {
            in_cell = max3(in_cell, largest, largest);
            if (--left == 0 || chunk + 1 == chunks) {
                cell_largest[cell++][threadIdx.x] = in_cell;
                in_cell = -INFINITY;
                left = per_cell;
            }
        }
    }

    Best best;
    if constexpr (TOP) {
        const unsigned used = (chunks + per_cell - 1) / per_cell;
        lane_ranks[threadIdx.x] = value_rank(mine.m);
        bool again = __syncthreads_or(mine.s != mine.s);
        unsigned ranks[WAVES];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) ranks[w] = lane_ranks[w * 64 + lane];
        const float least = value_of_rank(reached_by<kRankBits<DT>>(ranks, a.top));
        // a lane's logits that reach `least`, of which bit i of `reaching` says that logit(i) does, to the candidates
        auto note = [&](unsigned reaching, auto &&logit, auto &&index) {
            int place = reaching ? atomicAdd(&found, __popc(reaching)) : 0;
            static_for<kVectors * 8>([&](auto I) {
                if ((reaching >> I & 1) && place < kCandidates) candidates[place++] = rank_of(value_rank(logit(I)), index(I));
            });
        };
        if (WAVES > 1 && !again && chunks == 1) {  // they are still there (one wave is sooner through with reading a few again)
            unsigned reaching = 0;
#pragma unroll
            for (int i = 0; i < kVectors * 8; ++i) reaching |= (unsigned)(v[i] >= least && v[i] != -INFINITY) << i;
            note(reaching, [&](int i) { return v[i]; }, [&](int i) { return begin + i / 8 * STRIDE + threadIdx.x * 8 + i % 8; });
        } else if (!again) {
            for (unsigned i = 0; i < used; ++i) {
                const float largest = cell_largest[i][threadIdx.x];
                if (largest >= least && largest != -INFINITY) {
                    const int at = atomicAdd(&found_cells, 1);
                    if (at < kCandidates) cells[at] = (unsigned short)(i * THREADS + threadIdx.x);
                }
            }
            __syncthreads();
            again = found_cells > kCandidates;
            const unsigned pieces = per_cell * kVectors;
            const uint64_t items = again ? 0 : (uint64_t)found_cells * pieces;
            for (uint64_t item = threadIdx.x; item < items; item += THREADS) {
                const unsigned cell = cells[item / pieces], piece = (unsigned)(item % pieces);
                const unsigned chunk = cell / THREADS * per_cell + piece / kVectors;
                const unsigned at = begin + chunk * IN_HAND + piece % kVectors * STRIDE + cell % THREADS * 8;
                if (chunk >= chunks || at >= end) continue;
                Piece p;
                load_piece(at, p);
                unsigned reaching = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) reaching |= (unsigned)(p[e] >= least && p[e] != -INFINITY) << e;
                note(reaching, [&](int e) { return p[e % 8]; }, [&](int e) { return at + e % 8; });
            }
        }
        __syncthreads();
        again = again || found > kCandidates;
        if (!again) {
            if (wave == 0) best.mine = sorted_best(candidates, found, a.top, lists[0]);
        } else {
            rank_t last = 0;
            for (unsigned base = begin + wave * 64; base < end; base += THREADS) {
                const unsigned at = base + lane;
                rank_t r = 0;
                if (at < end && (!MASK || mask[at])) r = rank_of(value_rank(load_f32(x + at)), at);
                unsigned long long lanes = __ballot(r > last);
                while (lanes) {
                    const rank_t one = read_lane(r, __builtin_ctzll(lanes));
                    lanes &= lanes - 1;
                    if (one > last) {
                        best.insert(one);
                        last = read_lane(best.mine, a.top - 1);
                    }
                }
            }
            if (WAVES > 1) {
                lists[wave][lane] = best.mine;
                __syncthreads();
                if (wave == 0)
                    for (int w = 1; w < WAVES; ++w) best.merge(lists[w]);
            }
        }
    }
    mine = over_wave(mine, c);
    if (WAVES > 1) {
        if (lane == 0) wave_sums[wave] = mine;
        __syncthreads();
        if (wave > 0) return;
        for (int w = 1; w < WAVES; ++w) mine = joined(mine, wave_sums[w], c);
    }
    if (slices == 1) {
        write_row<DT, MASK>(a, row, mine, best.mine);
    } else {
        char *out = workspace + blockIdx.x * slice_bytes(a.top);
        if (lane == 0) *(Sums *)out = mine;
        if (TOP && lane < a.top) ((rank_t *)(out + 16))[lane] = best.mine;
    }
}

// Joins the slices of a row: the waves take slices in turn, then pair by pair, in an order that depends on nothing but their number
template <int DT, bool MASK>
__global__ void __launch_bounds__(kJoinWaves * 64) logprobs_join_kernel(const LogprobsArgs a, int slices, const char *__restrict__ workspace)
{
    __shared__ Sums wave_sums[kJoinWaves];
    __shared__ rank_t lists[kJoinWaves][64];
    const int row = blockIdx.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
    const Exponent c = {a.exponent, a.exponent_rest};
    const char *in = workspace + (size_t)row * slices * slice_bytes(a.top);
    Sums mine = {-INFINITY, 0.0f, 0.0f};
    Best best;
    for (int i = wave; i < slices; i += waves) {
        const char *part = in + i * slice_bytes(a.top);
        mine = joined(mine, *(const Sums *)part, c);
        if (a.top) {
            const rank_t r = lane < a.top ? ((const rank_t *)(part + 16))[lane] : 0;
            if (i == wave) {
                best.mine = r;
            } else {
                lists[wave][lane] = r;
                exchange_in_wave();
                best.merge(lists[wave]);
                exchange_in_wave();
            }
        }
    }
    for (int half = waves / 2; half; half /= 2) {
        __syncthreads();
        if (wave >= half && wave < 2 * half) {
            if (lane == 0) wave_sums[wave] = mine;
            lists[wave][lane] = best.mine;
        }
        __syncthreads();
        if (wave < half) {
            mine = joined(mine, wave_sums[wave + half], c);
            if (a.top) best.merge(lists[wave + half]);
        }
    }
    if (wave == 0) write_row<DT, MASK>(a, row, mine, best.mine);
}

// Gradient of a row: scale ((a [v = target]) - p (a + h (ln p + H))).  Workgroup (row, slice of kBackwardLength); every thread reads kVectors pieces of 8, writes them
// back.  Bound by memory: a logit is read and a gradient written once.
constexpr int kBackwardThreads = 256, kBackwardLength = kBackwardThreads * kVectors * 8;
template <int DT, bool MASK>
__global__ void __launch_bounds__(kBackwardThreads) logprobs_backward_kernel(const LogprobsBackwardArgs a, int slices)
{
    const int row = blockIdx.x / slices;
    const unsigned begin = blockIdx.x % slices * (unsigned)kBackwardLength, end = a.V - begin < (unsigned)kBackwardLength ? a.V : begin + kBackwardLength;
    const Storage<DT> *x = (const Storage<DT> *)a.logits + row * a.stride;
    Storage<DT> *dx = (Storage<DT> *)a.dlogits + row * a.dstride;
    const uint8_t *mask = MASK ? a.mask + row * a.mask_stride : nullptr;
    MaskedEight<DT, MASK, false> piece[kVectors];
#pragma unroll
    for (int j = 0; j < kVectors; ++j) piece[j].load(x, mask, begin + (j * kBackwardThreads + threadIdx.x) * 8, end);
    const float best = a.stats[2 * (int64_t)row], log_sum = a.stats[2 * (int64_t)row + 1];
    const int64_t t = a.targets ? a.targets[row] : -1;
    float g = a.g_logprob && t >= 0 ? a.g_logprob[row] : 0.0f;
    if (t >= a.V) g = __builtin_nanf("");
    const float h = a.g_entropy ? a.g_entropy[row] : 0.0f, H = h != 0.0f ? a.entropy[row] : 0.0f;
    const bool empty = best == -INFINITY && t < a.V;
    const float constant = fma32(h, H, g);
#pragma unroll
    for (int j = 0; j < kVectors; ++j) {
        const unsigned at = begin + (j * kBackwardThreads + threadIdx.x) * 8;
        if (at >= end) continue;
        Eight<Storage<DT>> out;
        const int64_t hit = t - at;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float lp = fma32((float)piece[j].x.v[e] - best, a.scale, -log_sum), p = __builtin_amdgcn_exp2f(lp * kLog2e);
            float d = -(p * fma32(h, fmaxf(lp, -1e4f), constant));
            if (hit == e) d = g + d;
            d *= a.scale;
            out.v[e] = (Storage<DT>)(piece[j].allowed(e) && !empty ? d : 0.0f);
        }
        if (at + 8 <= end) {
            store_streamed(dx + at, out);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < end) dx[at + e] = out.v[e];
        }
    }
}

// How a call is cut: threads of a workgroup, slices of a row and their length (whole pieces of what a workgroup has in hand).
struct LogprobsShape { int threads, slices, length; };
static LogprobsShape logprobs_shape(int rows, int V)
{
    LogprobsShape p;
    p.threads = V <= 64 * kVectors * 8 ? 64 : kMaxWaves * 64;
    const int in_hand = p.threads * kVectors * 8;
    int64_t slices = ((int64_t)V + in_hand - 1) / in_hand;
    const int64_t wanted = rows > 0 ? (1023 + (int64_t)rows) / rows : 1024;
    if (slices > wanted) slices = wanted;
    if (slices > kMaxSlices) slices = kMaxSlices;
    const int64_t each = (((int64_t)V + slices - 1) / slices + in_hand - 1) / in_hand * in_hand;
    p.length = (int)(each < INT32_MAX ? each : INT32_MAX);
    p.slices = (int)(((int64_t)V + p.length - 1) / p.length);
    return p;
}

size_t logprobs_workspace(int rows, int V, int top, int)
{
    const LogprobsShape p = logprobs_shape(rows, V);
    return p.slices > 1 ? (size_t)rows * p.slices * slice_bytes(top) : 0;
}

constexpr int kRowsPerLaunch = 1 << 22;           // below 2^31 threads

template <int DT, bool MASK>
static int forward_rows(const LogprobsArgs &a, const LogprobsShape &p, void *workspace, hipStream_t s)
{
    const unsigned blocks = (unsigned)a.rows * p.slices;
    auto launch = [&](auto top, auto waves) {
        logprobs_kernel<DT, MASK, top(), waves()><<<blocks, waves() * 64, 0, s>>>(a, p.slices, p.length, (char *)workspace);
    };
    using std::integral_constant;
    auto with_top = [&](auto waves) {
        if (a.top) launch(integral_constant<bool, true>{}, waves);
        else launch(integral_constant<bool, false>{}, waves);
    };
    if (p.threads == 64) with_top(integral_constant<int, 1>{});
    else with_top(integral_constant<int, kMaxWaves>{});
    NOVA_HIP_TRY(hipGetLastError());
    if (p.slices == 1) return 0;
    int waves = 1;
    while (waves < kJoinWaves && waves < p.slices) waves *= 2;
    logprobs_join_kernel<DT, MASK><<<a.rows, waves * 64, 0, s>>>(a, p.slices, (const char *)workspace);
    return (int)hipGetLastError();
}

template <int DT>
static int forward(const LogprobsArgs &a, void *workspace, hipStream_t s)
{
    const LogprobsShape shape = logprobs_shape(a.rows, a.V);
    const double exponent = a.scale * 1.4426950408889634074;
    float c = (float)exponent;
    if (c > exponent) c = std::nextafter(c, 0.0f);
    const float rest = std::max((float)(exponent - c), std::max(c * 0x1p-40f, 0x1p-149f));
    for (int64_t r0 = 0; r0 < a.rows; r0 += kRowsPerLaunch) {
        LogprobsArgs p = a;
        p.exponent = c;
        p.exponent_rest = rest;
        p.logits = (const Storage<DT> *)a.logits + r0 * a.stride;
        if (a.targets) p.targets += r0;
        if (a.mask) p.mask += r0 * a.mask_stride;
        if (a.logprob) p.logprob += r0;
        if (a.entropy) p.entropy += r0;
        p.stats += 2 * r0;
        if (a.top) p.top_logprobs += r0 * a.top, p.top_ids += r0 * a.top;
        p.rows = (int)(a.rows - r0 < kRowsPerLaunch ? a.rows - r0 : kRowsPerLaunch);
        const int err = a.mask ? forward_rows<DT, true>(p, shape, workspace, s) : forward_rows<DT, false>(p, shape, workspace, s);
        if (err) return err;
    }
    return 0;
}

int launch_logprobs(const LogprobsArgs &a, int dtype, void *workspace, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == NOVA_F32) return forward<NOVA_F32>(a, workspace, s);
    if (dtype == NOVA_F16) return forward<NOVA_F16>(a, workspace, s);
    return forward<NOVA_BF16>(a, workspace, s);
}

template <int DT>
static int backward(const LogprobsBackwardArgs &a, hipStream_t s)
{
    const int slices = (int)(((int64_t)a.V + kBackwardLength - 1) / kBackwardLength), rows_per_launch = slices < kRowsPerLaunch ? kRowsPerLaunch / slices : 1;
    for (int64_t r0 = 0; r0 < a.rows; r0 += rows_per_launch) {
        LogprobsBackwardArgs p = a;
        p.logits = (const Storage<DT> *)a.logits + r0 * a.stride;
        p.stats += 2 * r0;
        if (a.targets) p.targets += r0;
        if (a.g_logprob) p.g_logprob += r0;
        if (a.entropy) p.entropy += r0;
        if (a.g_entropy) p.g_entropy += r0;
        if (a.mask) p.mask += r0 * a.mask_stride;
        p.dlogits = (Storage<DT> *)a.dlogits + r0 * a.dstride;
        const unsigned blocks = (unsigned)(a.rows - r0 < rows_per_launch ? a.rows - r0 : rows_per_launch) * slices;
        if (a.mask) logprobs_backward_kernel<DT, true><<<blocks, kBackwardThreads, 0, s>>>(p, slices);
        else logprobs_backward_kernel<DT, false><<<blocks, kBackwardThreads, 0, s>>>(p, slices);
        NOVA_HIP_TRY(hipGetLastError());
    }
    return 0;
}

int launch_logprobs_backward(const LogprobsBackwardArgs &a, int dtype, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == NOVA_F32) return backward<NOVA_F32>(a, s);
    if (dtype == NOVA_F16) return backward<NOVA_F16>(a, s);
    return backward<NOVA_BF16>(a, s);
}

}  // namespace nova
