// Weights to the 4-bit format, on the host (offline, like the other weight
// quantizers of the library): for every 32 neighbours of a row the smallest e
// with max|w| <= 6 2^e, and the nearest code to w / 2^e, ties to the even
// code.  Every step is exact: the division is by a power of two, in double.
#include <cmath>
#include <cstdint>

#include "winof4.h"

extern "C" wino_status w4_quantize_weights(const float* w, int32_t n, int32_t k, uint8_t* codes, uint8_t* scales) {
    if (!w || !codes || !scales) return WINO_EINVAL;
    if (n < 0 || k < 0 || k % 32 != 0) return WINO_EINVAL;
    const int64_t groups = (int64_t)n * (k / 32);
    for (int64_t i = 0; i < 32 * groups; ++i)
        if (!std::isfinite(w[i])) return WINO_EINVAL;
    static const double limit[7] = {0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0};   // halfway to the next code
    for (int64_t g = 0; g < groups; ++g) {
        const float* x = w + 32 * g;
        double amax = 0;
        for (int i = 0; i < 32; ++i) amax = std::fmax(amax, std::fabs((double)x[i]));
        int e = 0;
        if (amax > 0) {
            int ex;
            const double f = std::frexp(amax, &ex);        // amax = f 2^ex, 6 2^e = 3/4 2^(e + 3)
            e = f > 0.75 ? ex - 2 : ex - 3;
            if (e < -127) e = -127;
        }
        scales[g] = (uint8_t)(e + 127);
        for (int i = 0; i < 16; ++i) {
            uint8_t byte = 0;
            for (int j = 0; j < 2; ++j) {
                const double v = std::ldexp(std::fabs((double)x[2 * i + j]), -e);
                uint8_t c = 0;
                for (int t = 0; t < 7; ++t) c += (t & 1) ? v >= limit[t] : v > limit[t];
                if (std::signbit(x[2 * i + j])) c |= 8;
                byte |= (uint8_t)(c << (4 * j));
            }
            codes[16 * g + i] = byte;
        }
    }
    return WINO_OK;
}
