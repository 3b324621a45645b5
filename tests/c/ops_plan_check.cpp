// sdp_ops_plan.h on the CPU: spans and overlaps, against an enumeration of
// every element.
#include <cstdio>
#include <cstdlib>
#include <set>

#include "sdp_ops_plan.h"

using namespace sdpops;

static int bad = 0;
#define EXPECT(c) \
    do { \
        if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); ++bad; } \
    } while (0)

static std::multiset<int64_t> elements(int64_t at, const Layout &l) {
    std::multiset<int64_t> out;
    for (int64_t a = 0; a < l.ext[0]; ++a)
        for (int64_t b = 0; b < l.ext[1]; ++b)
            for (int64_t c = 0; c < l.ext[2]; ++c)
                for (int64_t i = 0; i < l.inner; ++i)
                    out.insert(at + a * l.stride[0] + b * l.stride[1] + c * l.stride[2] + i);
    return out;
}

int main() {
    // random small layouts: what the tests promise holds for every element
    std::srand(7);
    int proved = 0, injected = 0;
    for (int k = 0; k < 200000; ++k) {
        auto r = [](int n) { return (int64_t)(std::rand() % n); };
        Layout a{{1 + r(3), 1 + r(3), 1 + r(3)}, {r(40), r(20), r(8)}, 1 + r(4)};
        Layout b = a;
        if (r(2)) b = Layout{{1 + r(3), 1 + r(3), 1 + r(3)}, {r(40), r(20), r(8)}, 1 + r(4)};
        b.ext[2] = 1 + r(3);
        const int64_t pa = r(60), pb = r(60);
        const auto ea = elements(pa, a), eb = elements(pb, b);
        EXPECT(span(a) == *ea.rbegin() - *ea.begin() + 1);
        if (injective(a)) {
            ++injected;
            EXPECT(std::set<int64_t>(ea.begin(), ea.end()).size() == ea.size());
        }
        if (disjoint((const char *)0 + 1000 + 2 * pa, a, (const char *)0 + 1000 + 2 * pb, b, 2)) {
            ++proved;
            for (int64_t e : ea) EXPECT(eb.count(e) == 0);
        }
    }
    EXPECT(proved > 1000 && injected > 1000);
    // the fused projection: q, k and v heads of one row, in both orders of tokens and heads
    for (int heads_first = 0; heads_first < 2; ++heads_first) {
        const int64_t s = heads_first ? 128 : 10 * 128, h = heads_first ? 77 * 128 : 128, b = 77 * 10 * 128;
        Layout q{{3, 77, 6}, {b, s, h}, 128}, kk{{3, 77, 2}, {b, s, h}, 128};
        const char *base = (const char *)0 + 4096;
        EXPECT(disjoint(base, q, base + 6 * h * 2, kk, 2) && disjoint(base + 6 * h * 2, kk, base, q, 2));
        EXPECT(!disjoint(base, q, base + 5 * h * 2, kk, 2));
        EXPECT(!disjoint(base, q, base + 9 * h * 2, kk, 2));
        EXPECT(same_tensor(base, q, base, q) && !same_tensor(base, q, base, kk) && !same_tensor(base, q, base + 2, q));
    }
    Layout huge{{1 << 30, 1 << 30, 4}, {(int64_t)1 << 40, (int64_t)1 << 40, 1}, 1}, neg{{2, 2, 2}, {8, -4, 2}, 1},
        none{{0, 5, 5}, {1, 1, 1}, 4};
    EXPECT(span(huge) == -1 && span(neg) == -1 && span(none) == 0 && injective(none));
    if (!bad) std::printf("ok\n");
    return bad != 0;
}
