// Checks, on the host, of the recurrence's arithmetic that host and device share (cngp_recur.h): states as their rounding to fp16 and sixteen
// bits beside it, and where windows of rows fall among sequences of equal length.  Nothing is launched.  Exit code 0 = all hold.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "cngp_recur.h"

using namespace cngp;

static int g_bad = 0;
static void expect(const bool ok, const char *what, const double a, const double b) {
    if (!ok && g_bad++ < 20) std::fprintf(stderr, "%s: %.17g %.17g\n", what, a, b);
}

static float to_half(const float v) { return (float)(_Float16)v; }
static float half_step_up(const float h) {                // the next fp16 value away from zero
    const _Float16 x = (_Float16)h;
    uint16_t       u;
    std::memcpy(&u, &x, 2);
    ++u;
    _Float16 y;
    std::memcpy(&y, &u, 2);
    return (float)y;
}

// Every fp32 value of a sample comes back to two roundings of fp32 or 2^-39, from its rounding to fp16 and from the value next to that.
static void states_come_back() {
    for (uint64_t u = 0; u < 0x7f800000ull; u += 977) {   // the positive finite numbers
        float h;
        const uint32_t bits = (uint32_t)u;
        std::memcpy(&h, &bits, 4);
        for (const float v : {h, -h}) {
            const float    rounded = to_half(v);
            const uint16_t low = low_half(v);
            const double   back = with_low_half(rounded, low), off = std::fabs(back - (double)v);
            if (std::isinf(rounded)) {
                expect(off <= std::fabs((double)v) * 0x1p-7, "a state beyond fp16", v, back);
                continue;
            }
            const double bound = std::fabs((double)v) * 0x1p-23 + 0x1p-39;
            expect(off <= bound, "a state", v, back);
            const float next = half_step_up(rounded);
            if (!std::isinf(next) && rounded != 0.0f) expect(std::fabs((double)with_low_half(next, low) - (double)v) <= bound, "a state from the value next to its rounding", v, next);
        }
    }
    expect(with_low_half(0.0f, low_half(0.0f)) == 0.0f, "zero", 0.0, with_low_half(0.0f, low_half(0.0f)));
    expect(std::isinf(with_low_half(INFINITY, low_half(INFINITY))), "infinity", 0.0, 0.0);
    expect(with_low_half(-INFINITY, low_half(-INFINITY)) == -INFINITY, "minus infinity", 0.0, 0.0);
    expect(std::isnan(with_low_half(NAN, low_half(NAN))), "no number", 0.0, 0.0);
    expect(with_low_half(65504.0f, low_half(65519.996f)) == 65519.996f, "the largest that fp16 holds", 65519.996, with_low_half(65504.0f, low_half(65519.996f)));
}

// Where the windows' edges fall among sequences of equal length, against 64 bits, for counts of rows up to the most that a call may have.
static void edges_of_equal_sequences() {
    for (const int64_t most : {(int64_t)1000, (int64_t)1 << 30, (int64_t)1100000000, (int64_t)1500000000, (int64_t)1 << 31, kMostRows})
        for (const int64_t S : {(int64_t)1, (int64_t)2, (int64_t)3, (int64_t)7, (int64_t)1000, (int64_t)123457, most < kMostRows ? most : kMostRows}) {
            if (S > most) continue;
            const int64_t each = (most < kMostRows ? most : kMostRows) / S, N = each * S;
            const Order   o{nullptr, (pos)N, (pos)S, (pos)each, false};
            const auto    check = [&](const int64_t p) {
                if (p < 0 || p > N) return;
                const int64_t q = (p + each - 1) / each;
                pos           got = -7, at = -7;
                o.equal_from((pos)p, got, at);
                expect(got == q && at == q * each, "a window's edge", (double)p, (double)got);
            };
            for (int64_t k = 0; k <= 1024; ++k)
                for (const int64_t d : {-1, 0, 1}) {
                    check((N + 1023) / 1024 * k + d);      // edges of 1024 windows
                    check(S / 1024 * k * each + d);        // around where sequences start
                }
            for (int64_t d = 0; d < 3; ++d) check(N - d);
        }
}

int main() {
    states_come_back();
    edges_of_equal_sequences();
    if (g_bad) { std::fprintf(stderr, "%d checks of the recurrence's arithmetic fail\n", g_bad); return 1; }
    std::printf("the recurrence's arithmetic holds\n");
    return 0;
}
