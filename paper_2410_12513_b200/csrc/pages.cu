// Pages of 8-bit caches handed out to sequences: joins, forks that share pages, trims, compaction.
//
// "Inference for FiRST", item 2: a sequence's layer decisions are fixed on its prompt and a skipped (sequence, layer) needs
// no cache, so every layer has page lists of its own.  All bookkeeping is on the host; first_pages_commit brings the
// device's tables up to date (and copies the pages that have to be) on the caller's stream.
#include <algorithm>
#include <cstring>
#include <map>
#include <new>
#include <set>
#include <utility>
#include <vector>

#include "first.h"
#include "ops.h"
#include "pages.h"

using namespace first;

namespace {

// One changed sequence a blockIdx.x, one layer a blockIdx.y.  What changed, per sequence: slot, tokens (-1: leave len and pos), then
// for each layer 1 + max_pages words: how many pages, their ids.
__global__ void __launch_bounds__(128) pages_update(const int32_t* u, int B, int L, int max_pages, int page, int32_t* pages, int32_t* cap,
                                                    int32_t* len, int32_t* pos) {
    const int l = blockIdx.y;
    const int32_t* x = u + (int64_t)blockIdx.x * (2 + (int64_t)L * (1 + max_pages));
    const int slot = x[0], tokens = x[1];
    const int32_t* y = x + 2 + (int64_t)l * (1 + max_pages);
    const int64_t at = (int64_t)l * B + slot;
    for (int i = threadIdx.x; i < max_pages; i += 128) pages[at * max_pages + i] = y[1 + i];
    if (threadIdx.x == 0) {
        cap[at] = y[0] * page;
        if (tokens >= 0) {
            len[at] = y[0] > 0 || tokens == 0 ? tokens : 0;
            if (l == 0) pos[slot] = tokens;
        }
    }
}

struct Seq {
    bool live = false, dirty = false, moved = false;  // moved: the device's len and pos become `stored`
    int32_t tokens = 0, stored = 0, coming = 0;       // coming: of the tokens, those it was extended by since the last commit
    std::vector<uint8_t> keep;
    std::vector<std::vector<int32_t>> pages;  // [L]
};
struct Import {  // keys and values to take over from another cache when the tables are up to date
    int slot, src_seq;
    int32_t n;
    first_kv_cache src;
    std::vector<void*> k, v;
};
struct Move {
    int32_t layer, from, to;
};

}  // namespace

struct first_pages {
    first_ctx* ctx = nullptr;
    first_model_desc d{};
    int B = 0, L = 0, max_pages = 0, page = 0;
    std::vector<first_cache8> layers;
    std::vector<void*> k, v;
    std::vector<Seq> seq;
    std::vector<std::set<int32_t>> free_;           // [L], the lowest id first
    std::vector<std::vector<int32_t>> refs, limbo;  // [L]: sequences on a page; freed pages that a pending copy still reads
    std::vector<Move> moves;                        // pending copies: distinct targets, sources as they are on the device now
    std::vector<Import> imports;
    int32_t *pages_d = nullptr, *cap_d = nullptr, *len_d = nullptr, *pos_d = nullptr, *zero_d = nullptr, *update_d = nullptr, *moves_d = nullptr;
    int64_t* off_d = nullptr;
    int64_t moves_cap = 0;
    uint64_t plan = 0;  // the context's plan that is this manager's
};

namespace {

int pages_for(const first_pages* p, int64_t tokens) { return (int)((tokens + p->page - 1) / p->page); }

int32_t take(first_pages* p, int l) {  // (the caller has made sure that there is one)
    const int32_t id = *p->free_[l].begin();
    p->free_[l].erase(p->free_[l].begin());
    p->refs[l][id] = 1;
    return id;
}
void drop(first_pages* p, int l, int32_t id) {
    if (--p->refs[l][id] > 0) return;
    auto read = [&](int32_t page) {
        return std::any_of(p->moves.begin(), p->moves.end(), [&](const Move& m) { return m.layer == l && m.from == page; });
    };
    const auto copy = std::find_if(p->moves.begin(), p->moves.end(), [&](const Move& m) { return m.layer == l && m.to == id; });
    if (copy != p->moves.end()) {  // nobody wants the copy any more; its source may have waited for it alone
        const int32_t from = copy->from;
        *copy = p->moves.back();
        p->moves.pop_back();
        const auto waits = std::find(p->limbo[l].begin(), p->limbo[l].end(), from);
        if (waits != p->limbo[l].end() && !read(from)) {
            p->limbo[l].erase(waits);
            p->free_[l].insert(from);
        }
    }
    if (read(id)) p->limbo[l].push_back(id);
    else p->free_[l].insert(id);
}

// Pages for the sequence to reach `tokens`, its last page to itself (after there were found to be enough).
void grow(first_pages* p, Seq& s, int64_t tokens) {
    for (int l = 0; l < p->L; ++l) {
        if (!s.keep[l]) continue;
        auto& list = s.pages[l];
        if (tokens > s.tokens && s.tokens % p->page) {
            int32_t& last = list[s.tokens / p->page];
            if (p->refs[l][last] > 1) {  // shared: a copy of its own, of what the page holds on the device
                const int32_t to = take(p, l);  // (a page that is still to be copied to belongs to one sequence: forks wait for the commit)
                p->moves.push_back({l, last, to});
                --p->refs[l][last];
                last = to;
                s.dirty = true;
            }
        }
        while ((int)list.size() < pages_for(p, tokens)) {
            list.push_back(take(p, l));
            s.dirty = true;
        }
    }
}

int free_slot(const first_pages* p) {
    for (int b = 0; b < p->B; ++b)
        if (!p->seq[b].live) return b;
    return -1;
}

// Whether any two of the layers' arrays have memory in common.
bool overlap(const first_cache8* layers, int L) {
    std::vector<std::pair<uintptr_t, uintptr_t>> spans;
    for (int l = 0; l < L; ++l) {
        const first_cache8& c = layers[l];
        const uintptr_t heads = (uintptr_t)c.n_pages * c.n_kv_heads, bytes = heads * c.page * c.head_dim;
        if (!heads) continue;
        for (const void* x : {c.k, c.v}) spans.emplace_back(reinterpret_cast<uintptr_t>(x), reinterpret_cast<uintptr_t>(x) + bytes);
        for (const float* x : {c.k_scale, c.v_scale}) spans.emplace_back(reinterpret_cast<uintptr_t>(x), reinterpret_cast<uintptr_t>(x) + 4 * heads);
    }
    std::sort(spans.begin(), spans.end());
    for (size_t i = 1; i < spans.size(); ++i)
        if (spans[i].first < spans[i - 1].second) return true;
    return false;
}

bool is_live(const first_pages* p, int32_t slot) { return slot >= 0 && slot < p->B && p->seq[slot].live; }

}  // namespace

namespace first {

PagedView paged_view(const first_pages* p) {
    PagedView v;
    v.ctx = p->ctx;
    v.plan = p->plan;
    v.layers = p->layers.data();
    v.pages = p->pages_d;
    v.L = p->L;
    v.B = p->B;
    v.max_pages = p->max_pages;
    return v;
}

}  // namespace first

extern "C" {

int first_pages_create(first_ctx* ctx, int32_t max_seqs, int32_t max_pages, const first_cache8* layers, first_pages** out) {
    if (!ctx || !layers || !out || max_seqs <= 0 || max_pages <= 0) return FIRST_E_ARG;
    *out = nullptr;
    first_model_desc d{};
    int rc = first_get_desc(ctx, &d);
    if (rc) return rc;
    if (max_seqs > d.max_batch) return FIRST_E_CAPACITY;
    if (d.n_layers > 96) return FIRST_E_UNSUPPORTED;
    int64_t all = 0;
    for (int l = 0; l < d.n_layers; ++l) {
        if ((rc = check_cache8(layers + l))) return rc;
        if (layers[l].n_kv_heads != d.n_kv_heads || layers[l].head_dim != d.head_dim || layers[l].page != layers[0].page ||
            layers[l].format != layers[0].format)
            return FIRST_E_SHAPE;
        all += layers[l].n_pages;
    }
    if (max_pages > 65000 || (int64_t)max_pages * layers[0].page > (1 << 30) || all > (1 << 28) || (int64_t)max_seqs * d.n_layers * max_pages > (1 << 28)) return FIRST_E_CAPACITY;
    first_pages* p = new (std::nothrow) first_pages();
    if (!p) return FIRST_E_ARG;
    try {
        if (overlap(layers, d.n_layers)) {
            delete p;
            return FIRST_E_ARG;
        }
        p->ctx = ctx; p->d = d; p->B = max_seqs; p->L = d.n_layers; p->max_pages = max_pages; p->page = layers[0].page;
        p->layers.assign(layers, layers + p->L);
        p->seq.resize(p->B);
        p->free_.resize(p->L);
        p->refs.resize(p->L);
        p->limbo.resize(p->L);
        for (int l = 0; l < p->L; ++l) {
            p->k.push_back(layers[l].k);
            p->v.push_back(layers[l].v);
            p->refs[l].assign(layers[l].n_pages, 0);
            for (int i = 0; i < layers[l].n_pages; ++i) p->free_[l].insert(p->free_[l].end(), i);
        }
    } catch (...) {
        delete p;
        return FIRST_E_ARG;
    }
    const size_t LB = (size_t)p->L * p->B, table = LB * max_pages, update = (size_t)p->B * (2 + (size_t)p->L * (1 + max_pages));
    p->moves_cap = all / 2 + (int64_t)LB;
    bool ok = cudaMalloc(&p->pages_d, 4 * table) == cudaSuccess && cudaMalloc(&p->cap_d, 4 * LB) == cudaSuccess &&
              cudaMalloc(&p->len_d, 4 * LB) == cudaSuccess && cudaMalloc(&p->pos_d, 4 * (size_t)p->B) == cudaSuccess &&
              cudaMalloc(&p->zero_d, 4) == cudaSuccess && cudaMalloc(&p->update_d, 4 * update) == cudaSuccess &&
              cudaMalloc(&p->moves_d, 12 * (size_t)p->moves_cap) == cudaSuccess && cudaMalloc(&p->off_d, 8 * LB) == cudaSuccess;
    ok = ok && cudaMemset(p->pages_d, 0xff, 4 * table) == cudaSuccess && cudaMemset(p->cap_d, 0, 4 * LB) == cudaSuccess &&
         cudaMemset(p->len_d, 0, 4 * LB) == cudaSuccess && cudaMemset(p->pos_d, 0, 4 * (size_t)p->B) == cudaSuccess &&
         cudaMemset(p->zero_d, 0, 4) == cudaSuccess && cudaMemset(p->off_d, 0, 8 * LB) == cudaSuccess;
    if (!ok) { first_pages_destroy(p); return FIRST_E_CUDA; }
    *out = p;
    return FIRST_OK;
}

int first_pages_destroy(first_pages* p) {
    if (!p) return FIRST_OK;
    void* ptrs[] = {p->pages_d, p->cap_d, p->len_d, p->pos_d, p->zero_d, p->update_d, p->moves_d, p->off_d};
    for (void* q : ptrs)
        if (q) cudaFree(q);
    delete p;
    return FIRST_OK;
}

int first_pages_join(first_pages* p, const uint8_t* mask_row, const first_kv_cache* src, int32_t src_seq, int32_t n_tokens,
                     int32_t* slot_out) {
    if (!p || !mask_row || !slot_out || n_tokens < 0 || (!src && n_tokens > 0)) return FIRST_E_ARG;
    if (src && (src->per_layer || !src->k || !src->v || !src->slab_off || src->cap_total <= 0 || src_seq < 0 || n_tokens > src->cap_total)) return FIRST_E_ARG;
    for (int l = 0; l < p->L; ++l) {
        if (mask_row[l] > 1) return FIRST_E_ARG;
        if (src && mask_row[l] && (!src->k[l] || !src->v[l])) return FIRST_E_ARG;
    }
    if (pages_for(p, n_tokens) > p->max_pages) return FIRST_E_CAPACITY;
    const int slot = free_slot(p);
    if (slot < 0) return FIRST_E_CAPACITY;
    try {
        Seq s;
        s.live = s.dirty = s.moved = true;
        s.keep.assign(mask_row, mask_row + p->L);
        s.pages.resize(p->L);
        for (int l = 0; l < p->L; ++l)
            if (s.keep[l] && pages_for(p, n_tokens) > (int)p->free_[l].size()) return FIRST_E_CAPACITY;
        if (src && n_tokens > 0) {
            Import im{slot, src_seq, n_tokens, *src, {src->k, src->k + p->L}, {src->v, src->v + p->L}};
            p->imports.push_back(std::move(im));
        }
        grow(p, s, n_tokens);
        s.tokens = s.stored = n_tokens;
        p->seq[slot] = std::move(s);
    } catch (...) {
        return FIRST_E_ARG;
    }
    *slot_out = slot;
    return FIRST_OK;
}

int first_pages_fork(first_pages* p, int32_t slot, int32_t* slot_out) {
    if (!p || !slot_out || slot < 0 || slot >= p->B) return FIRST_E_ARG;
    if (!p->seq[slot].live || p->seq[slot].coming) return FIRST_E_STATE;
    for (const Import& im : p->imports)
        if (im.slot == slot) return FIRST_E_STATE;  // (its first tokens are not there yet)
    const int to = free_slot(p);
    if (to < 0) return FIRST_E_CAPACITY;
    try {
        Seq s = p->seq[slot];
        s.dirty = s.moved = true;
        s.stored = s.tokens;
        for (int l = 0; l < p->L; ++l)
            for (int32_t id : s.pages[l]) ++p->refs[l][id];
        p->seq[to] = std::move(s);
    } catch (...) {
        return FIRST_E_ARG;
    }
    *slot_out = to;
    return FIRST_OK;
}

int first_pages_extend(first_pages* p, int32_t slot, int32_t n_new) {
    if (!p || n_new < 0 || slot < -1 || slot >= p->B) return FIRST_E_ARG;
    if (slot >= 0 && !p->seq[slot].live) return FIRST_E_STATE;
    const int b0 = slot < 0 ? 0 : slot, b1 = slot < 0 ? p->B : slot + 1;
    try {
        for (int l = 0; l < p->L; ++l) {  // nothing is taken unless there is room for all
            int64_t need = 0;
            std::map<int32_t, int32_t> left;  // sequences still on a shared page, the earlier ones having copied it
            for (int b = b0; b < b1; ++b) {
                const Seq& s = p->seq[b];
                if (!s.live) continue;
                if (pages_for(p, (int64_t)s.tokens + n_new) > p->max_pages) return FIRST_E_CAPACITY;
                if (!s.keep[l]) continue;
                need += std::max(pages_for(p, (int64_t)s.tokens + n_new) - (int)s.pages[l].size(), 0);
                if (n_new == 0 || s.tokens % p->page == 0) continue;
                const int32_t last = s.pages[l][s.tokens / p->page];
                int32_t& refs = left.emplace(last, p->refs[l][last]).first->second;
                if (refs > 1) { ++need; --refs; }
            }
            if (need > (int64_t)p->free_[l].size()) return FIRST_E_CAPACITY;
        }
        for (int b = b0; b < b1; ++b) {
            Seq& s = p->seq[b];
            if (!s.live) continue;
            grow(p, s, (int64_t)s.tokens + n_new);
            s.tokens += n_new;
            s.coming += n_new;
        }
    } catch (...) {
        return FIRST_E_ARG;
    }
    return FIRST_OK;
}

int first_pages_trim(first_pages* p, int32_t slot, int32_t n_tokens) {
    if (!p || slot < 0 || slot >= p->B || n_tokens < 0) return FIRST_E_ARG;
    Seq& s = p->seq[slot];
    if (!s.live || s.coming) return FIRST_E_STATE;
    if (n_tokens > s.tokens) return FIRST_E_ARG;
    for (const Import& im : p->imports)
        if (im.slot == slot) return FIRST_E_STATE;
    for (int l = 0; l < p->L; ++l)
        while (s.keep[l] && (int)s.pages[l].size() > pages_for(p, n_tokens)) {
            drop(p, l, s.pages[l].back());
            s.pages[l].pop_back();
        }
    s.tokens = s.stored = n_tokens;
    s.dirty = s.moved = true;
    return FIRST_OK;
}

int first_pages_leave(first_pages* p, int32_t slot) {
    if (!p || slot < 0 || slot >= p->B) return FIRST_E_ARG;
    Seq& s = p->seq[slot];
    if (!s.live) return FIRST_E_STATE;
    for (size_t i = 0; i < p->imports.size(); ++i)
        if (p->imports[i].slot == slot) { p->imports.erase(p->imports.begin() + i); break; }
    for (int l = 0; l < p->L; ++l)
        for (int32_t id : s.pages[l]) drop(p, l, id);
    s = Seq();
    s.dirty = s.moved = true;
    return FIRST_OK;
}

int first_pages_commit(first_pages* p, void* stream) {
    if (!p) return FIRST_E_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(st, &cap) != cudaSuccess) return FIRST_E_CUDA;
    if (cap != cudaStreamCaptureStatusNone) return FIRST_E_STATE;  // (what is copied below is the host's of this moment)
    try {
        // pageable sources: the runtime takes its own copies before it returns
        if (!p->moves.empty()) {
            if ((int64_t)p->moves.size() > p->moves_cap) return FIRST_E_CAPACITY;
            if (cudaMemcpyAsync(p->moves_d, p->moves.data(), 12 * p->moves.size(), cudaMemcpyHostToDevice, st) != cudaSuccess) return FIRST_E_CUDA;
            const int rc = first_copy_pages(p->layers.data(), p->L, p->moves_d, (int64_t)p->moves.size(), nullptr, stream);
            if (rc) return rc;
            p->moves.clear();
            for (int l = 0; l < p->L; ++l) {
                for (int32_t id : p->limbo[l]) p->free_[l].insert(id);
                p->limbo[l].clear();
            }
        }
        std::vector<int32_t> u;
        int n = 0;
        for (int b = 0; b < p->B; ++b) {
            const Seq& s = p->seq[b];
            if (!s.dirty) continue;
            ++n;
            u.push_back(b);
            u.push_back(s.moved ? s.stored : -1);
            for (int l = 0; l < p->L; ++l) {
                const size_t have = s.live ? s.pages[l].size() : 0;
                u.push_back((int32_t)have);
                if (have) u.insert(u.end(), s.pages[l].begin(), s.pages[l].end());
                u.insert(u.end(), p->max_pages - have, -1);
            }
        }
        if (n) {
            if (cudaMemcpyAsync(p->update_d, u.data(), 4 * u.size(), cudaMemcpyHostToDevice, st) != cudaSuccess) return FIRST_E_CUDA;
            pages_update<<<dim3(n, p->L), 128, 0, st>>>(p->update_d, p->B, p->L, p->max_pages, p->page, p->pages_d, p->cap_d, p->len_d, p->pos_d);
            if (cudaGetLastError() != cudaSuccess) return FIRST_E_CUDA;
        }
        for (Seq& s : p->seq) {
            s.dirty = s.moved = false;
            s.coming = 0;
        }
        for (const Import& im : p->imports)
            for (int l = 0; l < p->L; ++l) {
                if (!p->seq[im.slot].keep[l]) continue;
                Seqs8 s;
                s.pages = p->pages_d + ((int64_t)l * p->B + im.slot) * p->max_pages;
                s.width = p->max_pages;
                s.len = p->zero_d;
                s.B = 1; s.total = s.max_new = s.each = im.n;
                s.row_off = im.src.slab_off + im.src_seq;
                s.row_total = im.src.cap_total;
                s.row_cap = im.src.slab_cap ? im.src.slab_cap + im.src_seq : nullptr;
                s.flags = device_flags(p->ctx);
                const bool f32 = p->d.dtype == FIRST_DTYPE_F32;
                const int64_t hd = p->d.head_dim;
                const Rows8 k{im.k[l], hd, im.src.cap_total * hd, f32}, v{im.v[l], hd, im.src.cap_total * hd, f32};
                if (append8_launch(cache8_of(p->layers[l]), s, k, v, st, false) != cudaSuccess) return FIRST_E_CUDA;
            }
        p->imports.clear();
        std::vector<uint8_t> mask((size_t)p->B * p->L, 0);
        for (int b = 0; b < p->B; ++b)
            if (p->seq[b].live) std::memcpy(&mask[(size_t)b * p->L], p->seq[b].keep.data(), p->L);
        const int rc = first_set_mask_host(p->ctx, mask.data(), p->B, stream);
        if (rc == FIRST_OK) p->plan = plan_serial(p->ctx);
        return rc;
    } catch (...) {
        return FIRST_E_ARG;
    }
}

int first_pages_compact(first_pages* p, void* stream) {
    if (!p) return FIRST_E_ARG;
    int rc = first_pages_commit(p, stream);  // copies that are pending go first
    if (rc) return rc;
    try {
        for (int l = 0; l < p->L; ++l) {
            int32_t top = p->layers[l].n_pages - 1;
            std::vector<int32_t> to(p->layers[l].n_pages, -1);
            bool any = false;
            for (;;) {
                while (top >= 0 && p->refs[l][top] == 0) --top;
                if (top < 0 || p->free_[l].empty() || *p->free_[l].begin() > top) break;
                const int32_t hole = *p->free_[l].begin();
                p->free_[l].erase(p->free_[l].begin());
                p->moves.push_back({l, top, hole});
                p->refs[l][hole] = p->refs[l][top];
                p->refs[l][top] = 0;
                to[top] = hole;
                any = true;
                p->limbo[l].push_back(top);
            }
            if (!any) continue;
            for (Seq& s : p->seq) {
                if (!s.live) continue;
                for (int32_t& id : s.pages[l])
                    if (to[id] >= 0) { id = to[id]; s.dirty = true; }
            }
        }
    } catch (...) {
        return FIRST_E_ARG;
    }
    return first_pages_commit(p, stream);
}

int first_pages_kv(first_pages* p, first_kv_cache* out) {
    if (!p || !out) return FIRST_E_ARG;
    std::memset(out, 0, sizeof *out);
    out->k = p->k.data();
    out->v = p->v.data();
    out->slab_off = p->off_d;
    out->slab_cap = p->cap_d;
    out->len = p->len_d;
    out->pos = p->pos_d;
    return FIRST_OK;
}

int first_pages_layer(first_pages* p, int32_t layer, first_cache8* cache, const int32_t** pages, int32_t* max_pages, int32_t** len) {
    if (!p || layer < 0 || layer >= p->L) return FIRST_E_ARG;
    if (cache) *cache = p->layers[layer];
    if (pages) *pages = p->pages_d + (int64_t)layer * p->B * p->max_pages;
    if (max_pages) *max_pages = p->max_pages;
    if (len) *len = p->len_d + (int64_t)layer * p->B;
    return FIRST_OK;
}

int first_pages_stats(first_pages* p, int32_t* pages_held, int32_t* highest, int32_t* live) {
    if (!p) return FIRST_E_ARG;
    for (int l = 0; l < p->L; ++l) {
        int32_t held = 0, top = -1;
        for (int32_t i = 0; i < p->layers[l].n_pages; ++i)
            if (p->refs[l][i] > 0) { ++held; top = i; }
        if (pages_held) pages_held[l] = held;
        if (highest) highest[l] = top;
    }
    if (live) {
        *live = 0;
        for (const Seq& s : p->seq) *live += s.live ? 1 : 0;
    }
    return FIRST_OK;
}

int first_pages_tokens(const first_pages* p, int32_t slot, int32_t* tokens) {
    if (!p || !tokens || slot < 0 || slot >= p->B) return FIRST_E_ARG;
    if (!is_live(p, slot)) return FIRST_E_STATE;
    *tokens = p->seq[slot].tokens;
    return FIRST_OK;
}

}  // extern "C"
