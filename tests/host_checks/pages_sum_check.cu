// Host-side check of the sums that say who is served when pages are given out (pages_add): in whatever order a scan
// takes its terms, a prefix sum is the exact one, or kPagesNever where that is no less.  Built and run by
// tests/test_host_logic.py; needs no GPU.
#include <cstdio>
#include <random>
#include <vector>
#include "../../paper_2410_16663_b200/csrc/cache_pages.cuh"

static bool check(const std::vector<int>& x, int chunk) {
    long long exact = 0;
    int carry = 0;
    for (size_t i0 = 0; i0 < x.size(); i0 += chunk) {
        // a chunk by doubling distances, as the lanes of a warp do it, then what came before it
        std::vector<int> v(x.begin() + i0, x.begin() + (i0 + chunk < x.size() ? i0 + chunk : x.size()));
        for (size_t sh = 1; sh < v.size(); sh <<= 1)
            for (size_t i = v.size(); i-- > sh;) v[i] = fa::pages_add(v[i], v[i - sh]);
        for (size_t i = 0; i < v.size(); ++i) {
            exact += x[i0 + i];
            const int upto = fa::pages_add(carry, v[i]);
            if (upto != (exact < fa::kPagesNever ? exact : fa::kPagesNever)) {
                printf("FAIL at %zu: %d, exact %lld\n", i0 + i, upto, exact);
                return false;
            }
        }
        carry = fa::pages_add(carry, v.back());
    }
    return true;
}

int main() {
    std::mt19937 rng(1);
    for (int run = 0; run < 2000; ++run) {
        const unsigned most = run % 4 == 0 ? 0x7fffffffu : run % 4 == 1 ? 1u << 20 : run % 4 == 2 ? 600000u : 40u;
        std::vector<int> x(1 + rng() % 4096);
        for (int& v : x) v = rng() % 8 == 0 ? 0 : (int)(rng() % (most + 1u));
        if (!check(x, 1 << (rng() % 11))) return 1;
    }
    if (!check(std::vector<int>(4096, 0x7fffffff), 32) || !check(std::vector<int>(4096, 524288), 32) || !check({0x7ffffffe, 0, 1, 1}, 2)) return 1;
    printf("OK\n");
    return 0;
}
