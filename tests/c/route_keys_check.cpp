// sdp_route_keys.h on the CPU: keys of every BF16 value in every place, and their order.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "sdp_route_keys.h"

using namespace sdpops;

static int bad = 0;
#define EXPECT(c) \
    do { \
        if (!(c) && ++bad < 20) std::printf("line %d: %s\n", __LINE__, #c); \
    } while (0)

static float of_bits(uint32_t b) {
    float v;
    std::memcpy(&v, &b, 4);
    return v;
}

int main() {
    const float inf = HUGE_VALF;
    std::srand(3);
    // a BF16 value keeps itself and its place; the larger of two is the larger key, the
    // lower place of two equals
    for (uint32_t b = 0; b < 65536; ++b) {
        const float v = of_bits(b << 16);
        if (v != v || v == inf) continue;
        for (uint32_t i = 0; i < 16; ++i) {
            const float key = key_of<true>(v, i);
            if (v == -inf) {
                EXPECT(key == v);
                continue;
            }
            EXPECT(place_of<true>(key) == i && without_place(key) == v);
            for (int n = 0; n < 8; ++n) {
                const uint32_t pick = (uint32_t)std::rand() & 7, j = (uint32_t)std::rand() & 15;
                // itself, its negative, zeros, its neighbours
                const uint32_t others[8] = {b, b ^ 0x8000, 0, 0x8000, b + 1, b - 1, (uint32_t)std::rand(), b};
                const float w = of_bits(others[pick] << 16);
                if (w != w || w == inf || w == -inf || i == j) continue;
                const bool first = v > w || (v == w && i < j);
                EXPECT((key > key_of<true>(w, j)) == first);
            }
        }
    }
    // any 32-bit value keeps its place and loses at most its last four bits
    for (int n = 0; n < 2000000; ++n) {
        const float v = n < 4 ? of_bits(n < 2 ? n << 31 : 0x7f7fffffu | (uint32_t)n << 31)
                              : of_bits((uint32_t)std::rand() << 16 ^ (uint32_t)std::rand());
        if (!std::isfinite(v)) continue;
        const uint32_t i = (uint32_t)n & 15;
        const float key = key_of<false>(v, i);
        EXPECT(std::isfinite(key) && place_of<false>(key) == i);
        EXPECT(std::fabs((double)without_place(key) - v) <= std::fabs((double)v) * 0x1p-19 + 15 * 0x1p-149);
    }
    EXPECT(key_of<false>(-inf, 3) == -inf);
    if (!bad) std::printf("ok\n");
    return bad != 0;
}
