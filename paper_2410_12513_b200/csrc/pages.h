// What the decode step sees of a page manager.
#pragma once
#include "first.h"

namespace first {

struct PagedView {
    const first_cache8* layers = nullptr;  // [L]
    const int32_t* pages = nullptr;        // dev [L][B][max_pages]
    int L = 0, B = 0, max_pages = 0;
};
PagedView paged_view(const first_pages* p);

}  // namespace first
