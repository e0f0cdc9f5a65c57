// Host side of the calls that write and copy parts of a KV cache: lists of rows by block, orders of copies in which nothing is
// overwritten before it is read, and the copies that put a paged pool in order.  No device calls.
#include <algorithm>
#include <cstring>
#include <memory>
#include <new>

#include "deft_lists.h"

namespace {

template <typename Head, typename Entry>
void pack(deft_kv_list_s &list, const std::vector<Head> &heads, const std::vector<Entry> &entries) {
    static_assert(sizeof(Head) == 16 && sizeof(Entry) == 8, "heads are read as 128-bit words, entries as 64-bit ones");
    list.heads = (int32_t)heads.size();
    list.entries = (int32_t)entries.size();
    list.off_entries = heads.size() * sizeof(Head);
    const size_t bytes = list.off_entries + entries.size() * sizeof(Entry);
    list.image.assign(std::max<size_t>(16, (bytes + 15) / 16 * 16), 0);
    if (!heads.empty()) std::memcpy(list.image.data(), heads.data(), list.off_entries);
    if (!entries.empty()) std::memcpy(list.image.data() + list.off_entries, entries.data(), entries.size() * sizeof(Entry));
}

int build_rows(const int32_t *rows, int32_t n, int32_t n_pool_rows, int32_t block_rows, deft_kv_list_s &list) {
    using deft::RowEntry;
    std::vector<RowEntry> entries((size_t)n);
    bool ascending = true;
    for (int32_t i = 0; i < n; ++i) {
        if (rows[i] < 0 || rows[i] >= n_pool_rows) return DEFT_EINVAL;
        entries[i] = {rows[i], i};
        ascending = ascending && (i == 0 || rows[i - 1] < rows[i]);
    }
    if (!ascending) {
        std::sort(entries.begin(), entries.end(), [](const RowEntry &a, const RowEntry &b) { return a.row < b.row; });
        for (int32_t i = 1; i < n; ++i)
            if (entries[i].row == entries[i - 1].row) return DEFT_EINVAL;
    }
    std::vector<deft::RowGroup> groups;
    for (int32_t i = 0; i < n; ++i) {
        const int32_t block = entries[i].row / block_rows;
        if (groups.empty() || groups.back().block != block) groups.push_back({block, i, 0, entries[i].row % block_rows});
        ++groups.back().count;
    }
    list.pool = n_pool_rows;
    list.block_rows = block_rows;
    pack(list, groups, entries);
    return DEFT_OK;
}

// Every page has at most one copy into it, so the copies form trees that hang from pages nobody overwrites, and cycles with
// trees that hang from their pages.  A page's own copies out come before the copy into it: post-order in a tree; in a cycle, all
// hanging trees first, then against the direction of the copies; the last one reads a page that is overwritten by then, and is
// read at the chain's beginning.  What hangs from one page that is not overwritten can be done in any order: a chain to each.
int build_copies(const int32_t *src, const int32_t *dst, int32_t n, int32_t n_pool_pages, deft_kv_list_s &list) {
    using deft::CopyStep;
    // the pages that have a part in it, numbered by themselves: a few copies in a large pool cost what a few copies cost
    std::vector<int32_t> pages;
    pages.reserve(2 * (size_t)n);
    for (int32_t i = 0; i < n; ++i) {
        if (src[i] < 0 || src[i] >= n_pool_pages || dst[i] < 0 || dst[i] >= n_pool_pages) return DEFT_EINVAL;
        pages.push_back(src[i]);
        pages.push_back(dst[i]);
    }
    std::sort(pages.begin(), pages.end());
    pages.erase(std::unique(pages.begin(), pages.end()), pages.end());
    auto number = [&](int32_t page) { return (int32_t)(std::lower_bound(pages.begin(), pages.end(), page) - pages.begin()); };
    const int32_t n_pages = (int32_t)pages.size();
    std::vector<int32_t> from((size_t)n_pages, -1), first_out((size_t)n_pages, -1), next_out((size_t)n_pages, -1);
    for (int32_t i = 0; i < n; ++i) {
        const int32_t d = number(dst[i]);
        if (from[d] >= 0) return DEFT_EINVAL;
        from[d] = number(src[i]);
    }
    for (int32_t d = n_pages - 1; d >= 0; --d) {  // copies out of a page as a list of destinations
        if (from[d] < 0 || from[d] == d) continue;
        next_out[d] = first_out[from[d]];
        first_out[from[d]] = d;
    }
    std::vector<deft::CopyChain> chains;
    std::vector<CopyStep> steps;
    std::vector<char> done((size_t)n_pages, 0);  // pages the copy into which has its place
    std::vector<int32_t> path;
    // the copies below `top` and, last, the one into it; next: the copies out of a page that are still to come
    std::vector<int32_t> next(first_out);
    auto subtree = [&](int32_t top, bool into_top) {
        path.assign(1, top);
        while (!path.empty()) {
            const int32_t p = path.back(), c = next[p];
            if (c >= 0) {
                next[p] = next_out[c];
                if (!done[c]) path.push_back(c);
                continue;
            }
            path.pop_back();
            if (p == top && !into_top) continue;
            steps.push_back({pages[from[p]], pages[p]});
            done[p] = 1;
        }
    };
    auto open = [&] { chains.push_back({(int32_t)steps.size(), 0, 0, 0}); };
    auto close = [&] { chains.back().count = (int32_t)steps.size() - chains.back().first; };
    auto moved = [&](int32_t p) { return from[p] >= 0 && from[p] != p; };
    for (int32_t p = 0; p < n_pages; ++p) {
        if (moved(p)) continue;  // not overwritten: every copy out of it begins a chain
        for (int32_t c = first_out[p]; c >= 0; c = next_out[c]) {
            open();
            subtree(c, true);
            close();
        }
    }
    std::vector<int32_t> ring;
    for (int32_t p = 0; p < n_pages; ++p) {
        if (!moved(p) || done[p]) continue;
        // what is left are cycles and what hangs from them: go back until a page comes again, it is on the cycle
        ring.clear();
        int32_t x = p;
        while (!done[x]) {
            done[x] = 2;
            x = from[x];
        }
        for (const int32_t on = x; ring.empty() || x != on; x = from[x]) ring.push_back(x);  // against the copies' direction
        for (int32_t y = p; done[y] == 2; y = from[y]) done[y] = 0;
        for (int32_t y : ring) done[y] = 1;
        open();
        for (int32_t y : ring) subtree(y, false);
        for (int32_t y : ring) steps.push_back({pages[from[y]], pages[y]});
        close();
        chains.back().held = 1;
    }
    // long chains first: what a launch waits for starts at once
    std::stable_sort(chains.begin(), chains.end(), [](const deft::CopyChain &a, const deft::CopyChain &b) { return a.count > b.count; });
    list.copies = true;
    list.pool = n_pool_pages;
    pack(list, chains, steps);
    return DEFT_OK;
}

template <typename F>
int make_list(deft_kv_list_t **out, F &&build) {
    *out = nullptr;
    try {
        std::unique_ptr<deft_kv_list_s> list(new deft_kv_list_s);
        const int rc = build(*list);
        if (rc == DEFT_OK) *out = list.release();
        return rc;
    } catch (const std::bad_alloc &) {
        return DEFT_ENOMEM;
    } catch (...) {
        return DEFT_EINVAL;
    }
}

}  // namespace

extern "C" int deft_kv_rows(const int32_t *rows, int32_t n, int32_t n_pool_rows, int32_t block_rows, deft_kv_list_t **out) {
    if (!out) return DEFT_EINVAL;
    *out = nullptr;
    if (n < 0 || n_pool_rows < 0 || (n > 0 && !rows)) return DEFT_EINVAL;
    if (block_rows < 1 || block_rows > 64 || (block_rows & (block_rows - 1))) return DEFT_EINVAL;
    return make_list(out, [&](deft_kv_list_s &list) { return build_rows(rows, n, n_pool_rows, block_rows, list); });
}

extern "C" int deft_kv_copies(const int32_t *src, const int32_t *dst, int32_t n, int32_t n_pool_pages, deft_kv_list_t **out) {
    if (!out) return DEFT_EINVAL;
    *out = nullptr;
    if (n < 0 || n_pool_pages < 0 || (n > 0 && (!src || !dst))) return DEFT_EINVAL;
    return make_list(out, [&](deft_kv_list_s &list) { return build_copies(src, dst, n, n_pool_pages, list); });
}

extern "C" size_t deft_kv_list_device_bytes(const deft_kv_list_t *list) { return list ? list->image.size() : 0; }

extern "C" void deft_kv_list_destroy(deft_kv_list_t *list) { delete list; }

extern "C" int deft_compact_pages(const int32_t *node_page_ptr, const int32_t *page_ids, int32_t n_pool_pages, const int32_t *node_parent,
                                  int32_t n_nodes, int32_t *new_page_ids, int32_t *src, int32_t *dst, int32_t *n_copies) {
    if (!node_page_ptr || !node_parent || !n_copies || n_nodes < 1 || n_pool_pages < 0 || node_page_ptr[0] != 0) return DEFT_EINVAL;
    *n_copies = 0;
    for (int32_t u = 0; u < n_nodes; ++u) {
        if (node_page_ptr[u + 1] < node_page_ptr[u]) return DEFT_EINVAL;
        if (node_parent[u] < -1 || node_parent[u] >= n_nodes) return DEFT_EINVAL;
    }
    const int32_t n = node_page_ptr[n_nodes];
    if (n > n_pool_pages || (n > 0 && (!page_ids || !new_page_ids || !src || !dst))) return DEFT_EINVAL;
    try {
        std::vector<int32_t> owned(page_ids, page_ids + n);
        std::sort(owned.begin(), owned.end());
        if (n > 0 && (owned.front() < 0 || owned.back() >= n_pool_pages)) return DEFT_EINVAL;
        if (std::adjacent_find(owned.begin(), owned.end()) != owned.end()) return DEFT_EINVAL;
        // sibling lists in ascending order; roots are the children of node n_nodes
        std::vector<int32_t> child((size_t)n_nodes + 1, -1), sibling((size_t)n_nodes, -1), path;
        for (int32_t u = n_nodes - 1; u >= 0; --u) {
            const int32_t p = node_parent[u] < 0 ? n_nodes : node_parent[u];
            sibling[u] = child[p];
            child[p] = u;
        }
        std::vector<int32_t> order;
        if (child[n_nodes] >= 0) path.push_back(child[n_nodes]);
        while (!path.empty()) {
            const int32_t u = path.back();
            path.pop_back();
            order.push_back(u);
            if (sibling[u] >= 0) path.push_back(sibling[u]);
            if (child[u] >= 0) path.push_back(child[u]);
        }
        if ((int32_t)order.size() != n_nodes) return DEFT_EINVAL;  // a cycle is reached from no root
        int32_t at = 0, copies = 0;
        for (int32_t u : order)
            for (int32_t i = node_page_ptr[u]; i < node_page_ptr[u + 1]; ++i, ++at) {
                const int32_t old = page_ids[i];  // (before the new number is written: the two tables may be one)
                new_page_ids[i] = at;
                if (old == at) continue;
                src[copies] = old;
                dst[copies++] = at;
            }
        *n_copies = copies;
    } catch (...) {
        return DEFT_ENOMEM;
    }
    return DEFT_OK;
}
