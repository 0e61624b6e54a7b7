// What the decode step sees of a page manager.
#pragma once
#include "first.h"

namespace first {

struct PagedView {
    const first_ctx* ctx = nullptr;
    uint64_t plan = 0;                     // plan_serial of the context after the last commit (0: none yet)
    const first_cache8* layers = nullptr;  // [L]
    const int32_t* pages = nullptr;        // dev [L][B][max_pages]
    int L = 0, B = 0, max_pages = 0;
};
PagedView paged_view(const first_pages* p);
uint32_t* device_flags(const first_ctx* c);
uint64_t plan_serial(const first_ctx* c);  // how many plans (masks) the context has been given

}  // namespace first
