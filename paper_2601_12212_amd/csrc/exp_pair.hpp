// e^(hi + lo) in pairs of fp32, for device code and for a test on the host (tests/exp_pair.cpp).
#pragma once

namespace dt {

// To 2^-40, since 1 - P is one of the teacher's probabilities; 0 below e^-104.  Cody and Waite's reduction: g = hi + lo - n ln 2, |g| <= 0.35, with ln 2 = A - B - C, where A
// and B have nine significant bits each, so that n A and n B are exact (|n| < 2^15) and hi - n A too.  Then 1 + g + g^2 (1/2 + g (1/6 + g (1/24 + g (1/120 + g r)))),
// r = 1/720 + ... + g^5 / 11! in fp32: its error is below 2^-23 r |g|^6 < 2^-41, what is left out g^12 / 12! < 2^-46.  (The library's function in
// 64 bits: its constants, two registers each, were kept by every thread for as long as its row.)
__device__ __forceinline__ double exp_pair(float hi, float lo) {
    if (!(hi > -104.f)) return 0.0;
    constexpr float A = 0.693359375f, B = 0x1.bdp-13f, C = 0x1.05c61p-29;
    const float n = rintf(hi * 1.44269504f);
    const double g = (double)fmaf(n, -A, hi) + (double)(n * B) + ((double)lo + (double)(n * C));
    const float v = (float)g;
    float r = fmaf(v, 2.5052108e-8f, 2.7557319e-7f);
    r = fmaf(v, r, 2.7557319e-6f);
    r = fmaf(v, r, 2.4801587e-5f);
    r = fmaf(v, r, 1.9841270e-4f);
    r = fmaf(v, r, 1.3888889e-3f);
    double q = fma(g, (double)r, 1.0 / 120);
    q = fma(g, q, 1.0 / 24);
    q = fma(g, q, 1.0 / 6);
    q = fma(g, q, 0.5);
    return ldexp(fma(g * g, q, 1.0 + g), (int)n);
}

}  // namespace dt
