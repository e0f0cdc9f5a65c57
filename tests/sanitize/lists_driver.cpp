// Host-only check of lists of rows and of copies (deft_lists.cpp), built with -fsanitize=address,undefined by
// tests/test_kv_lists.py.  Random copies, forks, chains and cycles are made chain by chain, chains in a random order and in
// turns, each as the kernel makes them (eight reads ahead of the writes, the held page first), and compared with all at once.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <numeric>
#include <random>
#include <set>

#include "deft_lists.h"

#define CHECK(x) do { if (!(x)) { std::printf("failed: %s, line %d\n", #x, __LINE__); std::exit(1); } } while (0)

template <typename T>
static std::vector<T> part(const deft_kv_list_s &l, size_t off, int n) {
    std::vector<T> x((size_t)n);
    if (n) std::memcpy(x.data(), l.image.data() + off, n * sizeof(T));
    return x;
}

static void copies(std::mt19937 &rng, int pool, int n, int kind) {
    std::vector<int32_t> src, dst, all((size_t)pool);
    std::iota(all.begin(), all.end(), 0);
    std::shuffle(all.begin(), all.end(), rng);
    for (int i = 0; i < n; ++i) {
        dst.push_back(all[i]);
        if (kind == 0) src.push_back((int32_t)(rng() % pool));                       // anything, copies to themselves included
        if (kind == 1) src.push_back(all[(i + 1) % n]);                              // one cycle
        if (kind == 2) src.push_back(i + 1 < pool ? all[i + 1] : all[i]);            // one chain
        if (kind == 3) src.push_back(all[n < pool ? n + (int)(rng() % (pool - n)) : i]);  // forks of pages that stay
        if (kind == 4) src.push_back(all[(i ^ 1) < n ? (i ^ 1) : i]);                // exchanges
    }
    deft_kv_list_t *list = nullptr;
    CHECK(deft_kv_copies(src.data(), dst.data(), n, pool, &list) == DEFT_OK);
    CHECK(list->image.size() % 16 == 0 && deft_kv_list_device_bytes(list) == list->image.size());
    const auto chains = part<deft::CopyChain>(*list, 0, list->heads);
    const auto steps = part<deft::CopyStep>(*list, list->off_entries, list->entries);
    std::vector<int> want((size_t)pool), got((size_t)pool);
    std::iota(got.begin(), got.end(), 0);
    want = got;
    for (int i = 0; i < n; ++i) want[dst[i]] = src[i];
    int total = 0, moved = 0;
    for (int i = 0; i < n; ++i) moved += src[i] != dst[i];
    // the state of each chain's thread, advanced in turns
    struct Thread { int at, n, held; bool begun; };
    std::vector<Thread> threads;
    for (const auto &c : chains) {
        CHECK(c.count >= 1 && c.first == std::clamp(c.first, 0, list->entries - c.count));
        total += c.count;
        threads.push_back({0, c.held ? c.count - 1 : c.count, 0, false});
    }
    CHECK(total == list->entries && total == moved);
    std::vector<int> live(threads.size());
    std::iota(live.begin(), live.end(), 0);
    while (!live.empty()) {
        const size_t pick = rng() % live.size();
        const int k = live[pick];
        Thread &t = threads[k];
        const deft::CopyStep *s = &steps[chains[k].first];
        if (!t.begun) {
            t.begun = true;
            if (chains[k].held) t.held = got[s[t.n].src];
            continue;
        }
        int x[8];
        const int m = std::min(8, t.n - t.at);
        for (int u = 0; u < m; ++u) x[u] = got[s[t.at + u].src];
        for (int u = 0; u < m; ++u) got[s[t.at + u].dst] = x[u];
        t.at += m;
        if (t.at < t.n) continue;
        if (chains[k].held) got[s[t.n].dst] = t.held;
        live.erase(live.begin() + pick);
    }
    CHECK(got == want);
    deft_kv_list_destroy(list);
}

static void rows(std::mt19937 &rng, int pool, int n, int block) {
    std::vector<int32_t> all((size_t)pool);
    std::iota(all.begin(), all.end(), 0);
    if (rng() % 3) std::shuffle(all.begin(), all.end(), rng);
    deft_kv_list_t *list = nullptr;
    CHECK(deft_kv_rows(all.data(), n, pool, block, &list) == DEFT_OK);
    const auto groups = part<deft::RowGroup>(*list, 0, list->heads);
    const auto entries = part<deft::RowEntry>(*list, list->off_entries, list->entries);
    CHECK(list->entries == n && list->pool == pool && list->block_rows == block && !list->copies);
    int at = 0;
    std::set<int> blocks;
    for (const auto &g : groups) {
        CHECK(g.first == at && g.count >= 1 && g.count <= block && blocks.insert(g.block).second);
        int low = block;
        for (int i = at; i < at + g.count; ++i) {
            CHECK(entries[i].row / block == g.block && all[entries[i].token] == entries[i].row);
            CHECK(i == at || entries[i].row > entries[i - 1].row);
            low = std::min(low, entries[i].row % block);
        }
        CHECK(low == g.low);
        at += g.count;
    }
    CHECK(at == n);
    deft_kv_list_destroy(list);
}

int main() {
    std::mt19937 rng(7);
    for (int i = 0; i < 3000; ++i) {
        const int pool = 1 + (int)(rng() % 60), n = (int)(rng() % (pool + 1));
        copies(rng, pool, n, i % 5);
        rows(rng, pool, n, 1 << (rng() % 7));
    }
    copies(rng, 200000, 200000, 1);
    copies(rng, 200000, 199999, 2);
    copies(rng, 50000, 50000, 0);
    std::printf("lists ok\n");
    return 0;
}
