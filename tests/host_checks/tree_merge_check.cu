// Host-side check of what the merge of the many-rows tree kernel takes from its table (tree_merge_there): every entry that
// a plan's CTAs write for a shared item passes, entries for an item with one part do not, and whatever else the workspace may
// hold where a CTA wrote nothing, what passes stays inside the outputs, the partial results and their log-sum-exps.
// Built and run by tests/test_host_logic.py; needs no GPU.
#include <cstdio>
#include <random>
#include <vector>
#include "../../paper_2410_16663_b200/csrc/decode_tree.cuh"

// The entries that the loading warps of all CTAs write, in both layouts, out of the plan alone.
static bool plan_entries_pass(const std::vector<int>& tiles, int items, int grid) {
    const int B = (int)tiles.size();
    int total = 0;
    for (int t : tiles) total += t > 0 ? (t + fa::kTreeItemCost) * items : 0;
    if (total == 0) return true;
    const fa::TreePlan plan(total, grid);
    std::vector<int> owner(total, -1);
    for (int c = 0; c < grid; ++c)
        for (int u = plan.begin(c); u < plan.begin(c + 1); ++u) owner[u] = c;
    for (int u = 0; u < total; ++u)
        if (owner[u] < 0 || owner[u] != plan.owner(u)) return false;
    int at = 0;
    for (int b = 0; b < B; ++b)
        for (int it = 0; tiles[b] > 0 && it < items; ++it, at += tiles[b] + fa::kTreeItemCost) {
            const int first = plan.owner(at + fa::kTreeItemCost), last = plan.owner(at + tiles[b] + fa::kTreeItemCost - 1);
            if (fa::tree_merge_there(make_int4(b, it, first, last), B, items, grid) != (first < last)) return false;
        }
    return true;
}

int main() {
    std::mt19937 rng(1);
    auto below = [&](int n) { return (int)(rng() % (unsigned)n); };
    for (int run = 0; run < 3000; ++run) {
        std::vector<int> tiles(1 + below(40));
        for (int& t : tiles) t = below(4) ? below(60) : 0;
        if (!plan_entries_pass(tiles, 1 + below(20), run % 2 ? 148 : 1 + below(300))) {
            printf("FAIL plan %d\n", run);
            return 1;
        }
    }
    // anything: the indices that the merge makes of it, against the sizes of what it indexes
    const int edge[] = {0, 1, -1, 2, 7, 8, 147, 148, 149, 295, 296, 0x7fffffff, (int)0x80000000, 0x7fc00000, (int)0xff800000, (int)0xffffffff, 1 << 30, 65536};
    long long passed = 0;
    for (int run = 0; run < 4000000; ++run) {
        const int B = 1 + below(70), T = 1 + below(256), g = 1 + below(16), Hkv = 1 + below(9), blocks = 1 + below(4), grid = below(2) ? 148 : 296;
        const int rows = (g * T + blocks - 1) / blocks;
        auto any = [&]() { return below(3) == 0 ? (int)rng() : below(2) ? edge[below(18)] : below(300); };
        const int4 m = make_int4(any(), any(), any(), any());
        if (!fa::tree_merge_there(m, B, Hkv * blocks, grid)) continue;
        ++passed;
        const int hk = m.y / blocks, R0 = m.y % blocks * rows, end = rows < g * T - R0 ? rows : g * T - R0;
        bool ok = m.w > m.z;
        for (int row : {0, end - 1}) {
            if (end <= 0) break;
            const long long token = (R0 + row) / g, head = hk * g + (R0 + row) % g;
            const long long out = ((long long)m.x * T + token) * (Hkv * g) + head, lse = ((long long)m.x * (Hkv * g) + head) * T + token;
            ok = ok && token < T && out >= 0 && out < (long long)B * T * Hkv * g && lse >= 0 && lse < (long long)B * T * Hkv * g;
        }
        for (long long part : {2ll * m.z + 1, 2ll * m.w}) ok = ok && part >= 0 && part < 2ll * grid;
        if (!ok) {
            printf("FAIL entry %d %d %d %d\n", m.x, m.y, m.z, m.w);
            return 1;
        }
    }
    if (passed < 1000) {
        printf("FAIL only %lld entries passed\n", passed);
        return 1;
    }
    printf("OK %lld\n", passed);
    return 0;
}
