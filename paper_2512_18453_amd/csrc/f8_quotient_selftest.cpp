// Compares the quotients of quantisation to 8-bit floating point with the processor's divisions, which round once:
//   - bit for bit, for all 2^23 significands of the scale and the two numbers to either side of every border between codes (and on it).  Where nothing is subnormal, powers of
//     two change no significand, and the borders of both formats are the multiples of 1/16 from 1 to 2;
//   - as codes, for scales of every exponent, the subnormal ones, those beside the ends of the ranges that are moved and the largest among them, at all borders of both formats;
//   - as codes, for random pairs from all of binary32.
#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <random>
#include <thread>
#include <vector>

#include "f8_quotient.hpp"

using nova::F8Divisor;

struct Format { const char *name; int bits, lowest; float largest; };
static const Format formats[2] = {{"E4M3", 3, -6, 448.0f}, {"E5M2", 2, -14, 57344.0f}};

static uint32_t bits_of(float v) { uint32_t b; std::memcpy(&b, &v, 4); return b; }
static float from_bits(uint32_t b) { float v; std::memcpy(&v, &b, 4); return v; }

// The value of the code nearest to q, ties to even
static float code(float q, const Format &f)
{
    const float kept = std::fmin(std::fmax(q, -f.largest), f.largest);
    int exponent = 0;
    std::frexp(kept, &exponent);
    const int step = std::max(exponent - 1, f.lowest) - f.bits;
    return std::copysign((float)std::ldexp(std::nearbyint(std::ldexp((double)kept, -step)), step), kept);
}

// Numbers halfway between neighbouring codes
static std::vector<float> borders(const Format &f)
{
    std::vector<float> codes = {0.0f}, b;
    for (int e = f.lowest, m = 1; codes.back() < f.largest; ++m) {
        if (m == 2 << f.bits) m = 1 << f.bits, ++e;
        codes.push_back((float)std::ldexp(m, e - f.bits));
    }
    for (size_t i = 1; i < codes.size(); ++i) b.push_back((codes[i - 1] + codes[i]) / 2);
    return b;
}

static std::atomic<long long> failures{0}, compared{0};
static void report(const char *what, float v, float s, float got, float want)
{
    if (failures++ < 10) std::printf("f8_quotient_selftest: %s: %a / %a gave %a, not %a\n", what, v, s, got, want);
}

static void every_significand(uint32_t first, uint32_t last)
{
    long long n = 0;
    for (uint32_t m = first; m < last; ++m) {
        const float s = from_bits(0x3f800000u | m);
        const F8Divisor<float> d(s);
        float v[80], got[80], want[80];
        for (int b = 0; b < 16; ++b) {
            const uint32_t near = bits_of((float)((1.0 + b / 16.0) * (double)s));
            for (int k = 0; k < 5; ++k) v[5 * b + k] = from_bits(near + k - 2);
        }
        for (int i = 0; i < 80; ++i) got[i] = d.quotient(v[i]);
        for (int i = 0; i < 80; ++i) want[i] = v[i] / s;
        if (std::memcmp(got, want, sizeof got))
            for (int i = 0; i < 80; ++i)
                if (got[i] != want[i]) report("next to a border", v[i], s, got[i], want[i]);
        n += 80;
    }
    compared += n;
}

static void same_code(const char *what, float v, float s)
{
    const float got = F8Divisor<float>(s).quotient(v), want = v / s;
    for (const Format &f : formats)
        if (bits_of(code(got, f)) != bits_of(code(want, f))) report(what, v, s, code(got, f), code(want, f));
}

static void every_exponent(unsigned seed)
{
    std::mt19937 random(seed);
    std::vector<float> b = borders(formats[0]), more = borders(formats[1]);
    b.insert(b.end(), more.begin(), more.end());
    std::vector<float> scales = {from_bits(1), from_bits(2), from_bits(3), from_bits(0x007fffffu), from_bits(0x00800000u), from_bits(0x7f7fffffu) / 448.0f, from_bits(0x7f7fffffu) / 57344.0f};
    for (float end : {0x1p-60f, 0x1p100f})
        for (int k = -3; k <= 3; ++k) scales.push_back(from_bits(bits_of(end) + k));
    for (int e = 0; e < 23; ++e)
        for (int k = 0; k < 8; ++k) scales.push_back(from_bits((1u << e) + random() % (1u << e)));                 // subnormal
    for (uint32_t e = 1; e < 247; ++e)
        for (int k = 0; k < 8; ++k) scales.push_back(from_bits(e << 23 | (random() & 0x7fffff)));                   // (2^119 is above the largest scale)
    long long n = 0;
    for (float s : scales)
        for (float border : b) {
            const double at = (double)border * s;
            if (at >= 0x1.fffffep127) continue;
            const uint32_t near = bits_of((float)at);
            for (int k = -2; k <= 2; ++k) {
                if ((int64_t)near + k < 0 || near + k >= 0x7f800000u) continue;
                same_code("at a border", from_bits(near + k), s);
                same_code("at a border", -from_bits(near + k), s);
                n += 4;
            }
        }
    compared += n;
}

static void random_pairs(unsigned seed, int count)
{
    std::mt19937 random(seed);
    for (int i = 0; i < count; ++i) {
        const uint32_t s = random() % (246u << 23) + 1, span = random() % (36u << 23);
        // from far below the scale to 2^16 times it
        const int64_t v = (int64_t)s + (16 << 23) - span;
        if (v < 0 || v >= 0x7f800000) continue;
        same_code("random", from_bits((uint32_t)v | (random() & 0x80000000u)), from_bits(s));
    }
    compared += 2LL * count;
}

int main()
{
    constexpr int kThreads = 8;
    std::vector<std::thread> threads;
    for (int t = 0; t < kThreads; ++t)
        threads.emplace_back([t] {
            const uint32_t share = (1u << 23) / kThreads;
            every_significand(t * share, (t + 1) * share);
            every_exponent(t);
            random_pairs(100 + t, 2000000);
        });
    for (std::thread &t : threads) t.join();
    if (failures) return 1;
    std::printf("%lld quotients compared\nf8_quotient_selftest: ok\n", (long long)compared);
    return 0;
}
