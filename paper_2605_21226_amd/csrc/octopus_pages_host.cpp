// Host side of the entry points on the pages themselves: checks of arguments, workspace, launches.
#include <algorithm>

#include "octopus_internal.h"

namespace octopus {
namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// Pages and table entries are counted in 32 bits; compaction adds the counts of as many workgroups as there are 4096 pages.
constexpr int32_t kMostPages = 1 << 24;
constexpr int64_t kMostEntries = 1 << 30;
bool pool_ok(int32_t n_pages) { return n_pages >= 1 && n_pages <= kMostPages; }
bool rows_ok(int32_t n_rows, int32_t max_pages) {
    return n_rows >= 1 && n_rows <= 65535 && max_pages >= 1 && max_pages <= INT32_MAX / OCTOPUS_TILE &&
           static_cast<int64_t>(n_rows) * max_pages <= kMostEntries;
}

// Sets the call's scratch regions and returns their size.
size_t carve(PagesCall *c, char *at, int32_t n_pages, int32_t n_seq, int32_t max_pages) {
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char *p = at + off;
        off += up256(bytes);
        return p;
    };
    c->writers = reinterpret_cast<int32_t *>(take(4 * static_cast<size_t>(n_pages)));
    c->first = reinterpret_cast<int32_t *>(take(4 * static_cast<size_t>(n_pages)));
    c->fresh = reinterpret_cast<int32_t *>(take(4 * static_cast<size_t>(n_pages)));
    c->info = reinterpret_cast<SlotPages *>(take(sizeof(SlotPages) * static_cast<size_t>(n_seq)));
    c->staged = reinterpret_cast<int32_t *>(take(4 * static_cast<size_t>(n_seq) * max_pages));
    return off;
}

}  // namespace
}  // namespace octopus

using namespace octopus;

extern "C" {

size_t octopus_pages_workspace(int32_t n_pages, int32_t n_seq, int32_t max_pages_per_seq) {
    if (!pool_ok(n_pages) || !rows_ok(n_seq, max_pages_per_seq)) return 0;
    PagesCall c{};
    return carve(&c, nullptr, n_pages, n_seq, max_pages_per_seq);
}

int octopus_pages_update(int32_t *refs, int32_t n_pages, int32_t *block_table, int32_t max_pages_per_seq, int32_t *lens, int32_t n_seq,
                         const int32_t *source, const int32_t *keep_lens, const int32_t *new_lens, int32_t *moves, void *workspace,
                         size_t workspace_bytes, void *stream) {
    if (refs == nullptr || block_table == nullptr || lens == nullptr || new_lens == nullptr || moves == nullptr) return OCTOPUS_EINVAL;
    if (!pool_ok(n_pages) || !rows_ok(n_seq, max_pages_per_seq)) return OCTOPUS_EINVAL;
    if (!aligned(refs, 16) || !aligned(block_table, 4) || !aligned(lens, 4) || !aligned(source, 4) || !aligned(keep_lens, 4) ||
        !aligned(new_lens, 4) || !aligned(moves, 4))
        return OCTOPUS_EINVAL;
    PagesCall c{};
    if (workspace == nullptr || !aligned(workspace, 256) ||
        workspace_bytes < carve(&c, static_cast<char *>(workspace), n_pages, n_seq, max_pages_per_seq))
        return OCTOPUS_EWORKSPACE;
    c.refs = refs;
    c.n_pages = n_pages;
    c.table = block_table;
    c.max_pages = max_pages_per_seq;
    c.lens = lens;
    c.n_seq = n_seq;
    c.source = source;
    c.keep_lens = keep_lens;
    c.new_lens = new_lens;
    c.moves = moves;
    return launch_pages_update(c, stream) == 0 ? OCTOPUS_OK : OCTOPUS_EHIP;
}

int octopus_pages_compact(int32_t *refs, int32_t n_pages, int32_t *page_map, int32_t *moves, void *workspace, size_t workspace_bytes,
                          void *stream) {
    if (refs == nullptr || page_map == nullptr || moves == nullptr || !pool_ok(n_pages)) return OCTOPUS_EINVAL;
    if (!aligned(refs, 16) || !aligned(page_map, 4) || !aligned(moves, 4)) return OCTOPUS_EINVAL;
    PagesCall c{};
    if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < carve(&c, static_cast<char *>(workspace), n_pages, 1, 1))
        return OCTOPUS_EWORKSPACE;
    c.refs = refs;
    c.n_pages = n_pages;
    c.page_map = page_map;
    c.moves = moves;
    return launch_pages_compact(c, stream) == 0 ? OCTOPUS_OK : OCTOPUS_EHIP;
}

int octopus_pages_rename(const int32_t *page_map, int32_t n_pages, int32_t *table, int32_t n_rows, int32_t max_pages_per_row,
                         const int32_t *lens, void *stream) {
    if (page_map == nullptr || table == nullptr || !pool_ok(n_pages) || !rows_ok(n_rows, max_pages_per_row)) return OCTOPUS_EINVAL;
    if (!aligned(page_map, 4) || !aligned(table, 4) || !aligned(lens, 4)) return OCTOPUS_EINVAL;
    PagesCall c{};
    c.n_pages = n_pages;
    c.page_map = const_cast<int32_t *>(page_map);
    c.table = table;
    c.n_seq = n_rows;
    c.max_pages = max_pages_per_row;
    c.lens = const_cast<int32_t *>(lens);
    return launch_pages_rename(c, stream) == 0 ? OCTOPUS_OK : OCTOPUS_EHIP;
}

int octopus_pages_copy(const octopus_pool_t *pools, int32_t n_pools, int32_t n_pages, const int32_t *moves, int32_t max_moves, void *stream) {
    if (pools == nullptr || moves == nullptr || n_pools < 1 || max_moves < 0 || !pool_ok(n_pages) || !aligned(moves, 4)) return OCTOPUS_EINVAL;
    for (int32_t p = 0; p < n_pools; ++p)
        if (pools[p].data == nullptr || !aligned(pools[p].data, 16) || pools[p].page_bytes < 16 || pools[p].page_bytes % 16 != 0 ||
            pools[p].page_bytes > (int64_t{1} << 40) / n_pages)
            return OCTOPUS_EINVAL;
    if (max_moves == 0) return OCTOPUS_OK;
    for (int32_t first = 0; first < n_pools; first += kCopyPools) {
        CopyCall c{};
        const int32_t n = std::min(n_pools - first, kCopyPools);
        for (int32_t p = 0; p < n; ++p) c.pools[p] = CopyPool{pools[first + p].data, pools[first + p].page_bytes};
        c.moves = moves;
        c.max_moves = max_moves;
        c.n_pages = n_pages;
        if (launch_pages_copy(c, n, stream) != 0) return OCTOPUS_EHIP;
    }
    return OCTOPUS_OK;
}

}  // extern "C"
