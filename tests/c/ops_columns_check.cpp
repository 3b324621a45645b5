// Columns of one buffer in sdp_ops_plan.h on the CPU: what is said to share no element
// shares none, and blocks of columns of any widths are known as such.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <set>

#include "sdp_ops_plan.h"

using namespace sdpops;

static int bad = 0;
#define EXPECT(c) \
    do { \
        if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); ++bad; } \
    } while (0)

static std::set<int64_t> elements(int64_t at, const Layout &l) {
    std::set<int64_t> out;
    for (int64_t a = 0; a < l.ext[0]; ++a)
        for (int64_t b = 0; b < l.ext[1]; ++b)
            for (int64_t c = 0; c < l.ext[2]; ++c)
                for (int64_t i = 0; i < l.inner; ++i)
                    out.insert(at + a * l.stride[0] + b * l.stride[1] + c * l.stride[2] + i);
    return out;
}

int main() {
    const char *base = (const char *)0 + 4096;
    std::srand(11);
    auto r = [](int n) { return (int64_t)(std::rand() % n); };
    // rows of two tensors that step alike, of widths and numbers of their own
    int shown = 0, met = 0;
    for (int k = 0; k < 200000; ++k) {
        Layout a{{1 + r(3), 1 + r(4), 1 + r(3)}, {r(60), r(24), r(8)}, 1 + r(6)};
        Layout b{{1 + r(3), 1 + r(4), 1 + r(3)}, {a.stride[0], a.stride[1], r(8)}, 1 + r(6)};
        const int64_t pa = r(30), pb = r(30);
        const auto ea = elements(pa, a), eb = elements(pb, b);
        bool meet = false;
        for (int64_t e : ea) meet = meet || eb.count(e) != 0;
        met += meet;
        if (disjoint(base + 2 * pa, a, base + 2 * pb, b, 2)) {
            ++shown;
            EXPECT(!meet);
        }
    }
    EXPECT(shown > 1000 && met > 1000);
    // columns [at, at + width) of the rows of one buffer
    for (int64_t width : {1, 7, 64}) {
        for (int64_t other : {1, 5, 32, 100}) {
            const int64_t stride = width + other + 3;
            Layout x{{1, 50, 1}, {0, stride, 0}, width}, y{{1, 50, 1}, {0, stride, 0}, other};
            EXPECT(disjoint(base, x, base + 2 * width, y, 2) && disjoint(base + 2 * width, y, base, x, 2));
            EXPECT(disjoint(base, x, base + 2 * (width + 3), y, 2));
            EXPECT(!disjoint(base, x, base + 2 * (width - 1), y, 2));
            EXPECT(!disjoint(base, x, base + 2 * (width + 4), y, 2));  // into the next row
            EXPECT(!disjoint(base, x, base + 2 * width + 1, y, 2));
            Layout fewer = y;
            fewer.ext[1] = 3;
            EXPECT(disjoint(base, x, base + 2 * width, fewer, 2) && disjoint(base + 2 * width, fewer, base, x, 2));
            fewer.stride[1] += 1;
            EXPECT(!disjoint(base, x, base + 2 * width, fewer, 2));
        }
    }
    if (!bad) std::printf("ok\n");
    return bad != 0;
}
