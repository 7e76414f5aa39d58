// Log probabilities of rows of logits, entropy, the largest alternatives, and the gradient of the first two (nova_logprobs in nova.h).
//
// With M the largest allowed logit and d = scale (x - M): L = ln sum e^d, H = L - sum e^d d / sum e^d.  One workgroup per row: a pass for M, one for the
// sums, one per alternative.
#include "q4_common.hpp"

namespace nova {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kThreads = 256;

// Rank of a logit: greater for greater values, NaN above everything, -0 and 0 alike, -infinity (and masked) 0; below it the index, smaller first.  Ranks of a
// row's entries are all different.
__device__ __forceinline__ unsigned long long rank_of(float v, unsigned index)
{
    if (v == -INFINITY) return 0;
    unsigned bits = __float_as_uint(v + 0.0f);
    bits = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    if (v != v) bits = 0xff800001u;               // one above +infinity
    return (unsigned long long)bits << 32 | (0xffffffffu - index);
}

template <typename T, typename F>
__device__ __forceinline__ T over_workgroup(T v, T *shared, F &&join)
{
    for (int step = 32; step; step >>= 1) v = join(v, (T)__shfl_xor(v, step));
    __syncthreads();
    if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = v;
    __syncthreads();
    v = shared[0];
    for (int w = 1; w < kThreads / 64; ++w) v = join(v, shared[w]);
    return v;
}

template <int DT, bool MASK>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(const LogprobsArgs a)
{
    __shared__ unsigned long long shared_rank[kThreads / 64];
    __shared__ float shared[kThreads / 64];
    const int row = blockIdx.x;
    const Storage<DT> *x = (const Storage<DT> *)a.logits + row * a.stride;
    const uint8_t *mask = MASK ? a.mask + row * a.mask_stride : nullptr;
    auto logit = [&](int v) { return !MASK || mask[v] ? load_f32(x + v) : -INFINITY; };
    auto sum = [](float p, float q) { return p + q; };
    float best = -INFINITY;
    for (int64_t v = threadIdx.x; v < a.V; v += kThreads) best = fmaxf(best, logit(v));
    best = over_workgroup(best, shared, [](float p, float q) { return fmaxf(p, q); });
    const float c = a.scale * kLog2e, ref = best == -INFINITY ? 0.0f : best;
    float s = 0.0f, u = 0.0f;
    for (int64_t v = threadIdx.x; v < a.V; v += kThreads) {
        const float d = (logit(v) - ref) * c, e = __builtin_amdgcn_exp2f(d);
        s += e;
        u = fma32(e, fmaxf(d, -1e4f), u);
    }
    s = over_workgroup(s, shared, sum);
    u = over_workgroup(u, shared, sum);
    const bool empty = best == -INFINITY && s == 0.0f;
    const float log_sum = empty ? -INFINITY : kLn2 * __log2f(s);
    if (threadIdx.x == 0) {
        a.stats[2 * (int64_t)row] = s == s ? best : __builtin_nanf("");
        a.stats[2 * (int64_t)row + 1] = log_sum;
        if (a.entropy) a.entropy[row] = empty ? 0.0f : log_sum - kLn2 * u / s;
        if (a.logprob) {
            const int64_t t = a.targets[row];
            a.logprob[row] = t < 0 ? 0.0f : t >= a.V ? __builtin_nanf("") : empty ? -INFINITY : (logit(t) - ref) * a.scale - log_sum;
        }
    }
    unsigned long long last = ~0ull;
    for (int j = 0; j < a.top; ++j) {
        unsigned long long next = 0;
        for (int64_t v = threadIdx.x; v < a.V; v += kThreads) {
            const unsigned long long r = rank_of(logit(v), (unsigned)v);
            if (r < last && r > next) next = r;
        }
        last = next = over_workgroup(next, shared_rank, [](unsigned long long p, unsigned long long q) { return p > q ? p : q; });
        if (threadIdx.x == 0) {
            const int64_t at = (int64_t)row * a.top + j, id = next ? (int64_t)(0xffffffffu - (unsigned)next) : -1;
            a.top_ids[at] = id;
            a.top_logprobs[at] = s != s ? __builtin_nanf("") : next ? (logit(id) - ref) * a.scale - log_sum : -INFINITY;
        }
    }
}

template <int DT, bool MASK>
__global__ void __launch_bounds__(kThreads) logprobs_backward_kernel(const LogprobsBackwardArgs a)
{
    const int row = blockIdx.x;
    const Storage<DT> *x = (const Storage<DT> *)a.logits + row * a.stride;
    Storage<DT> *dx = (Storage<DT> *)a.dlogits + row * a.dstride;
    const uint8_t *mask = MASK ? a.mask + row * a.mask_stride : nullptr;
    const float best = a.stats[2 * (int64_t)row], log_sum = a.stats[2 * (int64_t)row + 1];
    const bool empty = best == -INFINITY;
    const int64_t t = a.targets ? a.targets[row] : -1;
    float g = a.g_logprob && t >= 0 ? a.g_logprob[row] : 0.0f;
    if (t >= a.V) g = __builtin_nanf("");
    const float h = a.g_entropy ? a.g_entropy[row] : 0.0f, H = h != 0.0f ? a.entropy[row] : 0.0f;
    for (int64_t v = threadIdx.x; v < a.V; v += kThreads) {
        float d = 0.0f;
        if ((!MASK || mask[v]) && !(empty && t < a.V)) {
            const float lp = (load_f32(x + v) - best) * a.scale - log_sum, p = __builtin_amdgcn_exp2f(lp * kLog2e);
            d = g * ((v == t ? 1.0f : 0.0f) - p) - h * (p * (fmaxf(lp, -1e4f) + H));
            d *= a.scale;
        }
        store_from_f32(dx + v, d);
    }
}

size_t logprobs_workspace(int, int, int, int) { return 0; }

constexpr int kRowsPerLaunch = 1 << 22;           // below 2^31 threads

template <int DT>
static int forward(LogprobsArgs a, hipStream_t s)
{
    const int rows = a.rows;
    for (int64_t r0 = 0; r0 < rows; r0 += kRowsPerLaunch) {
        LogprobsArgs p = a;
        p.logits = (const Storage<DT> *)a.logits + r0 * a.stride;
        if (a.targets) p.targets += r0;
        if (a.mask) p.mask += r0 * a.mask_stride;
        if (a.logprob) p.logprob += r0;
        if (a.entropy) p.entropy += r0;
        p.stats += 2 * r0;
        if (a.top) p.top_logprobs += r0 * a.top, p.top_ids += r0 * a.top;
        const unsigned blocks = (unsigned)(rows - r0 < kRowsPerLaunch ? rows - r0 : kRowsPerLaunch);
        if (a.mask) logprobs_kernel<DT, true><<<blocks, kThreads, 0, s>>>(p);
        else logprobs_kernel<DT, false><<<blocks, kThreads, 0, s>>>(p);
        NOVA_HIP_TRY(hipGetLastError());
    }
    return 0;
}

int launch_logprobs(const LogprobsArgs &a, int dtype, void *, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (dtype == NOVA_F32) return forward<NOVA_F32>(a, s);
    if (dtype == NOVA_F16) return forward<NOVA_F16>(a, s);
    return forward<NOVA_BF16>(a, s);
}

template <int DT>
static int backward(LogprobsBackwardArgs a, hipStream_t s)
{
    const int rows = a.rows;
    for (int64_t r0 = 0; r0 < rows; r0 += kRowsPerLaunch) {
        LogprobsBackwardArgs p = a;
        p.logits = (const Storage<DT> *)a.logits + r0 * a.stride;
        p.stats += 2 * r0;
        if (a.targets) p.targets += r0;
        if (a.g_logprob) p.g_logprob += r0;
        if (a.entropy) p.entropy += r0;
        if (a.g_entropy) p.g_entropy += r0;
        if (a.mask) p.mask += r0 * a.mask_stride;
        p.dlogits = (Storage<DT> *)a.dlogits + r0 * a.dstride;
        const unsigned blocks = (unsigned)(rows - r0 < kRowsPerLaunch ? rows - r0 : kRowsPerLaunch);
        if (a.mask) logprobs_backward_kernel<DT, true><<<blocks, kThreads, 0, s>>>(p);
        else logprobs_backward_kernel<DT, false><<<blocks, kThreads, 0, s>>>(p);
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
