// CPU-only check of what an 8-bit cache's values are made of: every 16-bit number over many scales, against the
// nearest e4m3 value of the exact quotient.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <random>

#include "../paper_2601_20309_amd/csrc/kv_decode_kernels.hpp"

#define CHECK(cond, ...)                                              \
    do {                                                              \
        if (!(cond)) {                                                \
            std::fprintf(stderr, "FAIL %s:%d: ", __FILE__, __LINE__); \
            std::fprintf(stderr, __VA_ARGS__);                        \
            std::fprintf(stderr, "\n");                               \
            std::exit(1);                                             \
        }                                                             \
    } while (0)

namespace {
// x to e4m3's nearest, ties to even, at most 448; x is exact or nowhere near half way between two values
double nearest(double x)
{
    const double a = std::fabs(x);
    if (!(a < 448.0)) return std::copysign(a >= 448.0 ? 448.0 : a, x);
    const double step = std::ldexp(1.0, std::max(std::ilogb(a > 0 ? a : 1e-300) - 3, -9));
    return std::copysign(std::nearbyint(a / step) * step, x);
}

float bf16(uint32_t bits)
{
    bits <<= 16;
    float f;
    memcpy(&f, &bits, 4);
    return f;
}

float fp16(uint32_t bits)
{
    const int e = (int)(bits >> 10 & 31u), m = (int)(bits & 1023u);
    const float a = e == 31 ? (m ? std::nanf("") : std::numeric_limits<float>::infinity()) : e ? std::ldexp(1024.f + (float)m, e - 25) : std::ldexp((float)m, -24);
    return bits >> 15 ? -a : a;
}

void check(float x, float scale, const dkv::Scale &s)
{
    float values[1] = {x}, quotients[1];
    dkv::over(values, s, quotients);
    const float q = quotients[0];
    if (std::isnan(x)) {
        CHECK(std::isnan(q), "NaN / %g", scale);
        return;
    }
    CHECK(std::fabs(q) <= 448.f, "%a / %a = %a", x, scale, q);
    // (a quotient of a 24-digit number by another is 2^-29 of it or more away from a number of 5 digits, or is it)
    const double want = nearest((double)x / (double)scale), got = nearest((double)q);
    CHECK(want == got && std::signbit(want) == std::signbit(q), "%a / %a: %g, not %g", x, scale, got, want);
}
}  // namespace

int main()
{
    std::mt19937 rng(1);
    const float plain[] = {1.f, 0.01f, 0.02f, 0.03f, 0.0125f, 0.1f, 0.3f, 0.7f, 1.75f, 3e-5f, 448.f, 1.9999999f, 2.f, 1e38f, 3.4e38f, 1.2e-38f, 3e-39f};
    for (int i = 0; i < 60; i++) {
        const float scale = i < 17 ? plain[i] : std::ldexp(1.f + (float)(rng() & 0x7FFFFFu) * 0x1p-23f, (int)(rng() % 40u) - 30);
        const dkv::Scale s = dkv::Scale::of(scale);
        for (uint32_t b = 0; b < 65536u; b++) {
            check(bf16(b), scale, s);
            check(fp16(b), scale, s);
        }
        // 32-bit values, as turned keys are: around the middles between two e4m3 values, times the scale
        for (int k = 0; k < 20000; k++) {
            const float middle = std::ldexp((float)(2u * (8u + rng() % 8u) + 1u), (int)(rng() % 14u) - 10);
            float x = middle * scale;
            for (int n = (int)(rng() % 7u) - 3; n != 0; n += n < 0 ? 1 : -1) x = std::nextafterf(x, n < 0 ? 0.f : std::numeric_limits<float>::infinity());
            if (std::isfinite(x) && x > 1e-30f) check(rng() & 1u ? x : -x, scale, s);
        }
    }
    std::printf("host scale ok\n");
    return 0;
}
