// What groups are worth by their keys (sdp_route_keys.h) on the CPU: where two groups'
// worths come in another order than those of their scores and biases in 64 bits, the
// rooms of the two say so.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "sdp_route_keys.h"

using namespace sdpops;

static double uniform() { return (double)std::rand() / RAND_MAX; }

struct Group {
    Worth worth;
    double exact;
};

// Two experts of about these biases; the scores are off by up to 40 roundings of one in all.
static Group make(double b0, double b1, double spread, bool two) {
    Group g = {{0.0f, 0.0f}, 0.0};
    float key[2];
    const double share = uniform();
    for (int k = 0; k < 2; ++k) {
        const double score = 0.45 * uniform();
        const float bias = (float)((k ? b1 : b0) + spread * (uniform() - 0.5));
        const double off = 40 * 0x1p-24 * (2 * uniform() - 1) * (k ? share : 1 - share);
        key[k] = key_of<false>((float)(score + off) + bias, (uint32_t)std::rand() & 15);
        if (k == 0 || two) g.exact += score + (double)bias;
    }
    if (!two) key[1] = -HUGE_VALF;
    g.worth = worth_of(key[0], key[1]);
    return g;
}

int main() {
    int bad = 0, turned = 0;
    std::srand(5);
    for (double size : {0.0, 1e-3, 0.5, 2.0, 7.9, 16.0, 100.0, 5e3, 1e7, 1e30})
        for (int form = 0; form < 4; ++form)
            for (int n = 0; n < 200000; ++n) {
                const double b0 = form & 1 ? -size : size, b1 = form & 2 ? size : 0.4 - size;
                Group a = make(b0, b1, 1e-6 * size, n % 4 != 0), b = make(b0, b1, 1e-6 * size, n % 4 != 0);
                // as close as the keys are off
                const double shift = a.exact - b.exact;
                if (size < 1e6) {
                    const float by = (float)(shift * (1 + 4e-6 * (uniform() - 0.5)));
                    b.exact += by, b.worth.value += 0.5f * by;  // (half of the worth)
                }
                const bool other = (a.exact < b.exact) != (a.worth.value < b.worth.value);
                turned += other;
                bad += other && std::fabs((double)a.worth.value - b.worth.value) >
                                    ((double)a.worth.room + b.worth.room);
            }
    // at the ends of FP32: numbers, in the order of their sums in 64 bits
    const float most = 0x1.fffffep127f, ends[] = {-most, -0.7f * most, -1e30f, -1.0f, 0.0f, 2.0f, 1e30f, 0.7f * most, most};
    for (float a : ends)
        for (float b : ends)
            for (float c : ends)
                for (float d : ends) {
                    const Worth x = worth_of(a, b), y = worth_of(c, d);
                    bad += !std::isfinite(x.value) || !std::isfinite(x.room);
                    const double sx = (double)a + b, sy = (double)c + d;
                    bad += sx > sy && y.value > x.value && (double)y.value - y.room > (double)x.value + x.room;
                }
    const Worth none = worth_of(-HUGE_VALF, -HUGE_VALF), one = worth_of(-most, -HUGE_VALF);
    bad += none.value != -HUGE_VALF || none.room != 0.0f || one.value != -0.5f * most;
    if (turned < 1000) std::printf("only %d came in another order\n", turned);
    if (bad) std::printf("%d of %d are not seen\n", bad, turned);
    if (!bad && turned >= 1000) std::printf("ok\n");
    return bad != 0 || turned < 1000;
}
