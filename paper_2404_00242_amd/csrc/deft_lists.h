// Lists of cache rows and pages (deft_lists.cpp) as the kernels of deft_cache.hip read them.
#pragma once

#include <cstdint>
#include <vector>

#include "deft.h"

namespace deft {
// Rows that one call writes into one block.  Image of a row list: the groups, then the entries.
struct RowGroup {
    int32_t block, first, count, low;  // entries [first, first + count); low: lowest of their positions in the block
};
struct RowEntry {
    int32_t row, token;  // ascending rows
};
// Copies that one thread makes one after the other, in an order in which no page is overwritten before it was read.  With
// `held` the last one's page is read first, before anything is written.  Image of a list of copies: the chains, then the steps.
struct CopyChain {
    int32_t first, count, held, unused;
};
struct CopyStep {
    int32_t src, dst;
};
}  // namespace deft

struct deft_kv_list_s {
    bool copies = false;  // a list of copies, else of rows
    int32_t pool = 0;     // rows or pages of the pool
    int32_t block_rows = 0;
    int32_t heads = 0;    // groups or chains
    int32_t entries = 0;  // rows or copies to make
    size_t off_entries = 0;
    std::vector<uint8_t> image;  // whole 16-byte words, at least one
};
