// Sizes in sdp_ops_plan.h on the CPU: products of three sizes against 128 bits,
// quotients rounded up against 64.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "sdp_ops_plan.h"

static int bad = 0;
#define EXPECT(c) \
    do { \
        if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); ++bad; } \
    } while (0)

int main() {
    const int64_t edge[] = {0,       1,       2,           3,           8,           64,          2047,       2048,
                            1 << 20, 1 << 26, (1 << 26) + 8, 1 << 27, 1 << 28, 1 << 30, INT32_MAX - 1, INT32_MAX};
    for (int64_t a : edge)
        for (int64_t b : edge)
            for (int64_t c : edge) {
                const __int128 want = (__int128)a * b * c, limit = (__int128)1 << 60;
                EXPECT(sdpops::product(a, b, c) == (want <= limit ? (int64_t)want : -1));
            }
    // 2^64, which is 0 in 64 bits
    EXPECT(sdpops::product(2048, 1 << 26, 1 << 27) == -1 && sdpops::product(64, 1 << 28, 1 << 30) == -1);
    for (int64_t a : edge)
        for (int64_t less = 0; less < 200 && less <= a; ++less)
            for (int32_t b : {1, 3, 16, 32, 128})
                EXPECT(sdpops::parts_of((int32_t)(a - less), b) == (a - less + b - 1) / b);
    if (!bad) std::printf("ok\n");
    return bad != 0;
}
