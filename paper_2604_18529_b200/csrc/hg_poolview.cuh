// The paged KV pool as the residency and page operations see it.
#pragma once

#include <stdint.h>

namespace hg {

struct KvPoolView {
    uint16_t* k;
    uint16_t* v;
    const int32_t* block_table;   // may be NULL: identity paging
    int64_t page_stride, head_stride, tok_stride;
    int B, Hkv, D, page_size, page_shift, max_pages, num_pages;
};

}  // namespace hg
