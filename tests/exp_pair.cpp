// csrc/exp_pair.hpp on the host, against expl: for values v and sums lse in fp32, e^(v - lse) of the pair that v - lse is.  Prints the largest relative error,
// as a power of two, and returns 1 if it is above 2^-40.
#include <math.h>
#include <stdio.h>

#include <algorithm>
#include <random>

#define __device__
#define __forceinline__ inline
#include "../paper_2601_12212_amd/csrc/exp_pair.hpp"

int main() {
    std::mt19937_64 rng(1);
    const auto between = [&](double lo, double hi) { return (float)(lo + (hi - lo) * (double)(rng() >> 11) * 0x1p-53); };
    double worst = 0;
    const auto one = [&](float v, float lse) {
        const float hi = v - lse, back = hi - v;
        const long double want = expl((long double)v - (long double)lse);
        const double got = dt::exp_pair(hi, (v - (hi - back)) - (lse + back));
        worst = std::max(worst, fabs((double)((long double)got / want - 1)));
    };
    for (float range : {0.4f, 1.f, 4.f, 30.f, 51.f, 350.f})
        for (int i = 0; i < 1000000; ++i) {
            const float v = between(-range, range), lse = i & 1 ? between(-range, range) : 0.f;
            if (v - lse > -103.9f) one(v, lse);
        }
    for (int n = -149; n <= 1000; ++n)  // where the reduced argument is largest, and where it is next to 0
        for (int i = -400; i <= 400; ++i) {
            const float edge = (float)((n + 0.5) * 0.69314718055994531), near = (float)(n * 0.69314718055994531);
            one(std::max(edge, -103.9f) * (1 + i * 0x1p-23f), 0.f);
            one(std::max(near, -103.9f) * (1 + i * 0x1p-23f), 0.f);
        }
    const bool ends = dt::exp_pair(0.f, 0.f) == 1.0 && dt::exp_pair(-104.f, 0.f) == 0.0 && dt::exp_pair(-INFINITY, NAN) == 0.0 && dt::exp_pair(-3e38f, 0.f) == 0.0;
    printf("%.2f %s\n", log2(worst), ends ? "" : "ends");
    return worst <= 0x1p-40 && ends ? 0 : 1;
}
