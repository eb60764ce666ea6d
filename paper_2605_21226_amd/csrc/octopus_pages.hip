// Who holds which page: forking, growing, trimming and freeing sequences (pages_update), moving the pages in use to the front of the
// pools (pages_compact), and copying the pages that either says (pages_copy).
//
// A page's count is the number of table entries that hold it, a page with none is free, and free pages are handed out lowest number
// first, in the order of slots.  No list of free pages is kept: the counts are the whole state, results depend on nothing but them,
// and a call that releases and takes the same pages again leaves everything as it was.
#include <hip/hip_runtime.h>

#include "octopus_internal.h"
#include "octopus_scan.hpp"

namespace octopus {
namespace {

__device__ __forceinline__ int pages_of(int tokens) { return (tokens + (OCTOPUS_TILE - 1)) / OCTOPUS_TILE; }
__device__ __forceinline__ int page_id(const PagesCall &c, int id) { return min(max(id, 0), c.n_pages - 1); }
// Counts that one workgroup changes and reads; a barrier stands between.  (A fence for the whole device takes microseconds each.)
__device__ __forceinline__ int32_t load_count(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void add_count(int32_t *p, int n) { __hip_atomic_fetch_add(p, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }

// What a slot has, keeps and is to have.
struct Slot {
    int32_t src;           // -1: nobody
    int32_t own;           // tokens that it held
    int32_t kept, want;    // tokens of its source that it keeps, tokens that it is to have
};
__device__ __forceinline__ Slot slot_of(const PagesCall &c, int s) {
    const int32_t most = c.max_pages * OCTOPUS_TILE;
    auto held = [&](int t) { return min(max(c.lens[t], 0), most); };
    Slot x;
    x.src = c.source != nullptr ? c.source[s] : s;
    if (x.src < 0 || x.src >= c.n_seq) x.src = -1;
    x.own = held(s);
    x.want = min(max(c.new_lens[s], 0), most);
    x.kept = min(x.src == s ? x.own : (x.src >= 0 ? held(x.src) : 0), x.want);
    if (c.keep_lens != nullptr) x.kept = min(x.kept, max(c.keep_lens[s], 0));
    return x;
}

// Rows that come from another slot: what they keep is set aside (the row that it comes from may change too), and the counts follow.  A
// thread has one entry of kShareSlots slots, whose reads are on their way at once; slots of one source that follow each other add to a page's
// count together (64 samples of a prompt of 1024 pages: this launch took 27 us with an atomic addition a slot; the whole call takes 14.1, with
// 16 slots a thread 18.6).
constexpr int kRowThreads = 256, kShareSlots = 4;
__global__ __launch_bounds__(kRowThreads) void pages_share_kernel(PagesCall c) {
    __shared__ Slot slots[kShareSlots];
    const int s0 = blockIdx.y * kShareSlots, j = blockIdx.x * kRowThreads + threadIdx.x;
    if (threadIdx.x < kShareSlots) slots[threadIdx.x] = s0 + static_cast<int>(threadIdx.x) < c.n_seq ? slot_of(c, s0 + threadIdx.x) : Slot{-1, 0, 0, 0};
    __syncthreads();
    int32_t lost[kShareSlots], taken[kShareSlots];     // page ids, -1: none
#pragma unroll
    for (int i = 0; i < kShareSlots; ++i) {            // (every read is of an entry that is there, so that none waits for a branch)
        const Slot x = slots[i];
        const int64_t own = static_cast<int64_t>(s0 + i) * c.max_pages + j, from = static_cast<int64_t>(x.src) * c.max_pages + j;
        lost[i] = c.table[j < pages_of(x.own) ? own : 0];
        taken[i] = c.table[x.src >= 0 && j < pages_of(x.kept) ? from : 0];
    }
#pragma unroll
    for (int i = 0; i < kShareSlots; ++i) {
        const Slot x = slots[i];
        const bool moved = x.src != s0 + i;
        lost[i] = j < pages_of(x.own) && (moved || j >= pages_of(x.kept)) ? page_id(c, lost[i]) : -1;
        taken[i] = moved && j < pages_of(x.kept) ? page_id(c, taken[i]) : -1;
    }
    int less = 0, more = 0;
#pragma unroll
    for (int i = 0; i < kShareSlots; ++i) {
        if (taken[i] >= 0) c.staged[static_cast<int64_t>(s0 + i) * c.max_pages + j] = taken[i];
        const bool stays = lost[i] == taken[i];        // (a slot that comes from one whose page it held already)
        if (lost[i] >= 0) {
            less += stays ? 0 : 1;
            if (less != 0 && (i + 1 == kShareSlots || lost[i + 1] != lost[i])) {
                atomicAdd(&c.refs[lost[i]], -less);
                less = 0;
            }
        }
        if (taken[i] >= 0) {
            more += stays ? 0 : 1;
            if (more != 0 && (i + 1 == kShareSlots || taken[i + 1] != taken[i])) {
                atomicAdd(&c.refs[taken[i]], more);
                more = 0;
            }
        }
    }
}

// Pages of `at` .. `at` + kPerThread - 1 that are free (bits).
constexpr int kPerThread = 16;
__device__ __forceinline__ uint32_t free_pages(const PagesCall &c, int64_t at) {
    uint32_t free = 0;
#pragma unroll
    for (int i = 0; i < kPerThread; i += 4) {
        if (at + i + 4 <= c.n_pages) {
            const int4 n = *reinterpret_cast<const int4 *>(c.refs + at + i);
            free |= ((n.x <= 0 ? 1u : 0u) | (n.y <= 0 ? 2u : 0u) | (n.z <= 0 ? 4u : 0u) | (n.w <= 0 ? 8u : 0u)) << i;
        } else {
            for (int k = i; k < i + 4; ++k)
                if (at + k < c.n_pages && c.refs[at + k] <= 0) free |= 1u << k;
        }
    }
    return free;
}

// Which pages are copied, which free pages go where: one workgroup, a thread per slot; more slots than threads (ONE false) in rounds of
// as many.  Its time is that of reads that wait for each other: the slots' lengths, their entries, the counts of those (and the first
// counts of the search), and the barriers between.
constexpr int kAssignThreads = 1024;
constexpr int kFew = 4;              // entries of a slot that its thread deals with by itself
// With few entries in all (ROWS) it takes the rows from their sources as well, kEntries entries a thread, which wait in registers until all
// rows have been read.
constexpr int kEntries = 8;
template <bool ONE, bool ROWS>
__global__ __launch_bounds__(kAssignThreads) void pages_assign_kernel(PagesCall c) {
    static_assert(ONE || !ROWS, "rows are looked up by a thread per slot");
    __shared__ int room[2][kAssignThreads / kScanLanes];
    __shared__ int first_of[kAssignThreads], entry_of[kAssignThreads], fresh[kAssignThreads];
    __shared__ int flags[4];
    // ONE: pages that several would write into, found by their number, with the writers' count and the first of them
    constexpr int kTable = 2 * kAssignThreads;
    __shared__ int page_at[ONE ? kTable : 1], writers_at[ONE ? kTable : 1], first_at[ONE ? kTable : 1];
    const int tid = threadIdx.x;
    if (tid < 4) flags[tid] = 0;
    if constexpr (ONE)
        for (int i = tid; i < kTable; i += kAssignThreads) {
            page_at[i] = -1;
            writers_at[i] = 0;
            first_at[i] = INT32_MAX;
        }
    __syncthreads();
    // whether it holds for any thread, in this turn of the loop or one before (all threads call it; a barrier)
    auto any = [&](int which, bool it) {
        if (it) flags[which] = 1;
        __syncthreads();
        const bool is = flags[which] != 0;
        if constexpr (!ONE) __syncthreads();     // (the next turn may set it)
        return is;
    };
    SlotPages mine{0, 0, -1, 0};         // ONE: the thread's slot
    auto slot = [&](int s) { return ONE ? mine : c.info[s]; };
    __shared__ Slot slots[ROWS ? kAssignThreads : 1];
    __shared__ int page_in[ROWS ? kAssignThreads : 1], pages_stay[ROWS ? kAssignThreads : 1];
    int32_t row[kEntries];               // ROWS: what the thread's entries become, -1: nothing new
    const int n_entries = ROWS ? c.n_seq * c.max_pages : 0;

    // f(slot, k, entry, n): the k-th of the slot's `count` items, the n-th of all of them; by all threads, whosever they are
    auto spread = [&](int base, int count, int entry, auto f) {
        int total;
        const int upto = block_scan<kAssignThreads>(count, room[0], &total);
        first_of[tid] = upto - count;
        entry_of[tid] = entry;
        __syncthreads();
        for (int n = tid; n < total; n += kAssignThreads) {
            int lo = 0;
#pragma unroll
            for (int step = kAssignThreads / 2; step > 0; step /= 2)
                if (first_of[lo + step] <= n) lo += step;
            f(base + lo, n - first_of[lo], entry_of[lo], n);
        }
        __syncthreads();
    };

    // what each slot keeps; entries that a row loses (those of other slots' rows have been dealt with)
    for (int base = 0; base < c.n_seq; base += kAssignThreads) {
        const int s = base + tid;
        int lost = 0, from = 0;
        if (s < c.n_seq) {
            const Slot x = slot_of(c, s);
            const SlotPages kept{x.kept, x.want, x.src, 0};
            if constexpr (ONE) mine = kept;
            else c.info[s] = kept;
            from = pages_of(x.kept);
            if (c.source == nullptr) lost = max(pages_of(x.own) - from, 0);
            if constexpr (ROWS) slots[tid] = x;
        }
        if (c.source != nullptr) continue;
        auto lose = [&](int of, int k, int entry, int) {
            add_count(&c.refs[page_id(c, c.table[static_cast<int64_t>(of) * c.max_pages + entry + k])], -1);
        };
        if (any(0, lost > kFew)) spread(base, lost, from, lose);
        else
            for (int k = 0; k < lost; ++k) lose(s, k, from, 0);
    }

    // A page that is written into, because what a slot keeps ends inside it, has to be the slot's own.  Of those that would write into the same
    // one, the lowest keeps it if nobody else holds it -- one that continues its own row before those that came to it -- and the others
    // take a copy.
    auto written = [&](int s, const SlotPages &x) {
        const int64_t at = static_cast<int64_t>(s) * c.max_pages + x.kept / OCTOPUS_TILE;
        return x.want > x.kept && x.kept % OCTOPUS_TILE != 0 ? page_id(c, x.src == s ? c.table[at] : c.staged[at]) : -1;
    };
    auto rank = [&](int s, const SlotPages &x) { return x.src == s ? s : c.n_seq + s; };
    int my_page = -1;                    // ONE: the page that the thread's slot writes into
    // (entry e of the table is entry j of slot s; the quotient's error is far below the half that is added, e < 2^13)
    const float per_entry = 1.0f / c.max_pages;
    auto slot_at = [&](int e) { return static_cast<int>((e + 0.5f) * per_entry); };
    if constexpr (ROWS) {
        static_assert(kEntries * kAssignThreads <= 1 << 13, "");
        __syncthreads();
        int32_t lost[kEntries];
#pragma unroll
        for (int i = 0; i < kEntries; ++i) {           // (every read is of an entry that is there)
            if (i * kAssignThreads >= n_entries) break;
            const int e = min(tid + i * kAssignThreads, n_entries - 1), s = slot_at(e), j = e - s * c.max_pages;
            const Slot x = slots[s];
            lost[i] = c.table[e];
            row[i] = c.table[x.src >= 0 ? x.src * c.max_pages + j : e];
        }
#pragma unroll
        for (int i = 0; i < kEntries; ++i) {
            if (i * kAssignThreads >= n_entries) break;
            const int e = tid + i * kAssignThreads, s = slot_at(min(e, n_entries - 1)), j = e - s * c.max_pages;
            const Slot x = slots[s];
            const bool there = e < n_entries, moved = x.src != s, keeps = there && j < pages_of(x.kept);
            lost[i] = there && j < pages_of(x.own) && (moved || !keeps) ? page_id(c, lost[i]) : -1;
            if (keeps && j == x.kept / OCTOPUS_TILE) page_in[s] = page_id(c, row[i]);
            row[i] = keeps && moved ? page_id(c, row[i]) : -1;
            if (lost[i] != row[i]) {                   // (a slot that comes from one whose page it held already: no change)
                if (lost[i] >= 0) add_count(&c.refs[lost[i]], -1);
                if (row[i] >= 0) add_count(&c.refs[row[i]], 1);
            }
        }
        __syncthreads();
        if (tid < c.n_seq && mine.want > mine.kept && mine.kept % OCTOPUS_TILE != 0) my_page = page_in[tid];
    } else if constexpr (ONE) {
        if (tid < c.n_seq) my_page = written(tid, mine);
    }
    auto page_of = [&](int s) { return ONE ? my_page : written(s, c.info[s]); };
    __syncthreads();
    uint32_t free = free_pages(c, tid * kPerThread);
    bool shared = false;
    int holders = 0;                     // ONE: of the page that the thread's slot writes into
    for (int s = tid; s < c.n_seq; s += kAssignThreads) {
        const int page = page_of(s);
        if (page >= 0) holders = load_count(&c.refs[page]);
        shared |= page >= 0 && holders > 1;
    }
    if constexpr (ONE) {
        if (any(1, shared)) {
            int at = 0;
            if (shared) {
                at = static_cast<uint32_t>(my_page) * 2654435761u >> 21;          // (a half empty table: a free place is found)
                static_assert(kTable == 1 << 11, "");
                for (int other; (other = atomicCAS(&page_at[at], -1, my_page)) != -1 && other != my_page;) at = (at + 1) % kTable;
                atomicAdd(&writers_at[at], 1);
                atomicMin(&first_at[at], rank(tid, mine));
            }
            __syncthreads();
            if (shared && (holders > writers_at[at] || first_at[at] != rank(tid, mine))) mine.copied = 1;
        }
    } else if (any(1, shared)) {
        for (int s = tid; s < c.n_seq; s += kAssignThreads) {
            const int page = page_of(s);
            if (page >= 0) {
                c.writers[page] = 0;
                c.first[page] = INT32_MAX;
            }
        }
        __syncthreads();
        for (int s = tid; s < c.n_seq; s += kAssignThreads) {
            const int page = page_of(s);
            if (page >= 0) {
                add_count(&c.writers[page], 1);
                __hip_atomic_fetch_min(&c.first[page], rank(s, slot(s)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            }
        }
        __syncthreads();
        for (int s = tid; s < c.n_seq; s += kAssignThreads) {
            const int page = page_of(s);
            if (page >= 0 && (load_count(&c.refs[page]) > load_count(&c.writers[page]) || load_count(&c.first[page]) != rank(s, slot(s)))) c.info[s].copied = 1;
        }
    }

    // pages that are asked for
    auto asked = [&](const SlotPages &x) { return x.want > x.kept ? pages_of(x.want) - pages_of(x.kept) + x.copied : 0; };
    int wanted = 0, copies = 0;
    int my_upto = 0;                     // ONE: pages asked for up to the thread's slot
    for (int base = 0; base < c.n_seq; base += kAssignThreads) {
        int total;
        my_upto = block_scan<kAssignThreads>(base + tid < c.n_seq ? asked(slot(base + tid)) : 0, room[0], &total);
        wanted += total;
    }

    // the lowest free ones, in order
    const bool in_lds = wanted <= kAssignThreads;
    int found = 0;
    for (int64_t base = 0; found < wanted && base < c.n_pages; base += kAssignThreads * kPerThread) {
        const int64_t at = base + tid * kPerThread;
        if (base != 0) free = free_pages(c, at);
        int total;
        int n = found + block_scan<kAssignThreads>(static_cast<int>(__popc(free)), room[1], &total) - static_cast<int>(__popc(free));
        for (; free != 0 && n < wanted; free &= free - 1, ++n) {
            const int page = static_cast<int>(at) + __ffs(free) - 1;
            if (in_lds) fresh[n] = page;
            else c.fresh[n] = page;
        }
        found += total;
    }
    const bool enough = found >= wanted;
    __syncthreads();
    auto fresh_page = [&](int n) { return in_lds ? fresh[n] : c.fresh[n]; };

    int given = 0;
    for (int base = 0; base < c.n_seq; base += kAssignThreads) {
        const int s = base + tid;
        SlotPages x = s < c.n_seq ? slot(s) : SlotPages{0, 0, 0, 0};
        if (!enough) x.copied = 0;
        if (s < c.n_seq) {
            c.lens[s] = enough ? x.want : x.kept;
            if (!ROWS && (!ONE || c.source != nullptr)) c.info[s] = x;
            if constexpr (ROWS) pages_stay[s] = pages_of(x.kept) - x.copied;
        }
        if (!enough || wanted == 0) continue;
        const int need = asked(x);
        int total = wanted, upto = my_upto, moved;
        if constexpr (!ONE) upto = block_scan<kAssignThreads>(need, room[0], &total);
        const int begin = given + upto - need;
        if (any(2, x.copied != 0)) {
            const int nth = copies + block_scan<kAssignThreads>(x.copied, room[1], &moved) - x.copied;
            if (x.copied != 0) {
                const int page = ONE ? my_page : written(s, x);
                c.moves[2 + 2 * nth] = page;
                c.moves[3 + 2 * nth] = fresh_page(begin);
                add_count(&c.refs[page], -1);
            }
            copies += moved;
        }
        auto give = [&](int of, int k, int entry, int n) {
            const int page = fresh_page(n);
            c.table[static_cast<int64_t>(of) * c.max_pages + entry + k] = page;
            c.refs[page] = 1;
        };
        const int entry = pages_of(x.kept) - x.copied;
        if (any(3, need > kFew))    // (a barrier stands between the reads of entries above and these writes)
            spread(base, need, entry, [&](int of, int k, int first, int n) { give(of, k, first, given + n); });
        else
            for (int k = 0; k < need; ++k) give(s, k, entry, begin + k);
        given += total;
    }
    if constexpr (ROWS) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEntries; ++i) {
            if (i * kAssignThreads >= n_entries) break;
            const int e = tid + i * kAssignThreads, s = slot_at(min(e, n_entries - 1));
            if (row[i] >= 0 && e - s * c.max_pages < pages_stay[s]) c.table[e] = row[i];     // (a copied page's entry has been written)
        }
    }
    if (tid == 0) {
        c.moves[0] = copies;
        c.moves[1] = enough ? 0 : wanted - found;
    }
}

// Rows that come from another slot, from where they were set aside; a copied page's entry has been written.
__global__ __launch_bounds__(kRowThreads) void pages_rows_kernel(PagesCall c) {
    const int s = blockIdx.y, j = blockIdx.x * kRowThreads + threadIdx.x;
    const SlotPages x = c.info[s];
    if (x.src == s || j >= pages_of(x.kept) - x.copied) return;
    const int64_t at = static_cast<int64_t>(s) * c.max_pages + j;
    c.table[at] = c.staged[at];
}

// Compaction: with n pages in use, the i-th highest of them goes to the i-th lowest free page as long as that is lower, that is, those
// from n on go below n; after it the pages in use are 0 .. n - 1.
// (pages past the last are neither in use nor free)
__device__ __forceinline__ uint32_t used_pages(const PagesCall &c, int64_t at) {
    const int64_t there = min(max(c.n_pages - at, static_cast<int64_t>(0)), static_cast<int64_t>(kPerThread));
    return ~free_pages(c, at) & ((1u << there) - 1u);
}
// Pages from `at` on, of which `used` are in use and `n` below them: their places in `moves`, and in the map those of the pages that stay
// (the others' are written with their moves, later).
__device__ __forceinline__ void pair_pages(const PagesCall &c, int64_t at, uint32_t used, int n, int n_used) {
    if (at >= c.n_pages) return;
    const int first = static_cast<int>(at), there = min(c.n_pages - first, kPerThread);
    if (there == kPerThread) {
        typedef int32_t ids_t __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int i = 0; i < kPerThread; i += 4) *reinterpret_cast<ids_t *>(c.page_map + first + i) = ids_t{first + i, first + i + 1, first + i + 2, first + i + 3};
    } else {
        for (int i = 0; i < there; ++i) c.page_map[first + i] = first + i;
    }
    const int below = min(max(n_used - first, 0), kPerThread);          // of these pages that lie below n_used
    const uint32_t all = (1u << there) - 1u, low = (1u << below) - 1u;
    for (uint32_t high = used & all & ~low; high != 0; high &= high - 1) {
        const int i = __ffs(high) - 1;
        c.moves[2 + 2 * (n_used - 1 - (n + static_cast<int>(__popc(used & ((1u << i) - 1u)))))] = first + i;
    }
    for (uint32_t free = ~used & all & low; free != 0; free &= free - 1) {
        const int i = __ffs(free) - 1;
        c.moves[3 + 2 * (first + i - (n + static_cast<int>(__popc(used & ((1u << i) - 1u)))))] = first + i;
    }
    if (first < n_used && n_used <= first + there) c.moves[0] = n_used - (n + static_cast<int>(__popc(used & low)));      // free pages below n_used
    if (at == 0) {
        c.moves[1] = n_used;
        if (n_used == 0) c.moves[0] = 0;
    }
}
__device__ __forceinline__ void apply_move(const PagesCall &c, int i) {
    const int from = c.moves[2 + 2 * i], to = c.moves[3 + 2 * i];
    c.refs[to] = c.refs[from];
    c.refs[from] = 0;
    c.page_map[from] = to;
}

// Pools of as many pages as one workgroup's threads look at once, 16384: one launch.  Larger ones: three, whose time hardly grows.  us a call in a
// captured graph, half of the pages in use, one launch / three: 1100 pages 3.6 / 7.2, 16384 10.1 / 8.4; with the workgroup going on in rounds
// of 16384, 32768 21 / 8.4 and 65536 39 / 8.7 (nine tenths in use 13 / 8.6 and 23 / 9.0).  An eager caller waits 7 us longer for three launches.
constexpr int kCompactPages = kAssignThreads * kPerThread;
__global__ __launch_bounds__(kAssignThreads) void pages_compact_kernel(PagesCall c) {
    __shared__ int room[kAssignThreads / kScanLanes];
    const int tid = threadIdx.x, at = tid * kPerThread;
    const uint32_t used = used_pages(c, at);
    const int own = static_cast<int>(__popc(used));
    int n_used;
    const int below = block_scan<kAssignThreads>(own, room, &n_used) - own;
    pair_pages(c, at, used, below, n_used);
    __syncthreads();
    const int n = __hip_atomic_load(c.moves, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    for (int i = tid; i < n; i += kAssignThreads) apply_move(c, i);
}

// More pages: a workgroup counts its pages, and then numbers them from the others' counts.
constexpr int kCountThreads = 256;
constexpr int kCounted = kCountThreads * kPerThread;   // pages a workgroup looks at
__global__ __launch_bounds__(kCountThreads) void pages_count_kernel(PagesCall c) {
    __shared__ int room[kCountThreads / kScanLanes];
    const uint32_t used = used_pages(c, static_cast<int64_t>(blockIdx.x) * kCounted + threadIdx.x * kPerThread);
    int total;
    block_scan<kCountThreads>(static_cast<int>(__popc(used)), room, &total);
    if (threadIdx.x == 0) c.writers[blockIdx.x] = total;
}

__global__ __launch_bounds__(kCountThreads) void pages_pair_kernel(PagesCall c) {
    __shared__ int room[kCountThreads / kScanLanes];
    int before = 0, all = 0;
    for (int b = threadIdx.x; b < static_cast<int>(gridDim.x); b += kCountThreads) {
        const int n = c.writers[b];
        all += n;
        before += b < static_cast<int>(blockIdx.x) ? n : 0;
    }
    int n_used, n_before, total;
    block_scan<kCountThreads>(all, room, &n_used);
    block_scan<kCountThreads>(before, room, &n_before);
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kCounted + threadIdx.x * kPerThread;
    const uint32_t used = used_pages(c, at);
    const int n = static_cast<int>(__popc(used));
    pair_pages(c, at, used, n_before + block_scan<kCountThreads>(n, room, &total) - n, n_used);
}

__global__ __launch_bounds__(kCountThreads) void pages_apply_kernel(PagesCall c) {
    const int i = blockIdx.x * kCountThreads + threadIdx.x;
    if (i < c.moves[0]) apply_move(c, i);
}

__global__ __launch_bounds__(kRowThreads) void pages_rename_kernel(PagesCall c) {
    const int s = blockIdx.y, j = blockIdx.x * kRowThreads + threadIdx.x;
    if (j >= c.max_pages) return;
    const int64_t at = static_cast<int64_t>(s) * c.max_pages + j;
    const int page = page_id(c, c.table[at]);        // (asked for beside the length)
    if (c.lens == nullptr || j < pages_of(min(max(c.lens[s], 0), c.max_pages * OCTOPUS_TILE))) c.table[at] = c.page_map[page];
}

// A pool's pages by blockIdx.y, pieces of 16 KB of the moved pages by blockIdx.x.  What is written streams past the caches, what is read
// does not, since samples of one prompt all read its last page.  Pages at random places, keys and values of eight kv heads at d = 128, 3 bits:
// 32 pages of eight layers (84 MB read and written) 28 us with ordinary stores, 16.5 with streaming ones, 63 copies of one page of sixteen 50 and 37,
// 141 pages of eight layers (370 MB) 93 and 82, 4.5 TB/s, where a copy of as much in one piece reaches 5.3; streaming reads too: 21, 57 and 83.
// (256 to 1024 threads and 1024 to 16384 workgroups lie within 5 % of each other; 32 KB a turn was slower.)
constexpr int kCopyThreads = 512, kCopyAhead = 2;
constexpr int kPieceWords = kCopyThreads * kCopyAhead;     // of 16 bytes
__global__ __launch_bounds__(kCopyThreads) void pages_copy_kernel(CopyCall c) {
    typedef uint32_t word_t __attribute__((ext_vector_type(4)));
    const CopyPool pool = c.pools[blockIdx.y];
    const int64_t words = pool.page_bytes / 16;
    const int pieces = static_cast<int>((words + kPieceWords - 1) / kPieceWords);
    const int n = min(max(c.moves[0], 0), c.max_moves);
    for (int64_t i = blockIdx.x; i < static_cast<int64_t>(n) * pieces; i += gridDim.x) {
        const int move = static_cast<int>(i / pieces);
        const int64_t first = (i % pieces) * kPieceWords + threadIdx.x;
        const uint32_t from = c.moves[2 + 2 * move], to = c.moves[3 + 2 * move];
        if (from >= static_cast<uint32_t>(c.n_pages) || to >= static_cast<uint32_t>(c.n_pages)) continue;
        const word_t *src = static_cast<const word_t *>(pool.data) + from * words;
        word_t *dst = static_cast<word_t *>(pool.data) + to * words;
        word_t x[kCopyAhead];
#pragma unroll
        for (int k = 0; k < kCopyAhead; ++k)
            if (first + k * kCopyThreads < words) x[k] = src[first + k * kCopyThreads];
#pragma unroll
        for (int k = 0; k < kCopyAhead; ++k)
            if (first + k * kCopyThreads < words) __builtin_nontemporal_store(x[k], &dst[first + k * kCopyThreads]);
    }
}

dim3 row_grid(const PagesCall &c) { return dim3((c.max_pages + kRowThreads - 1) / kRowThreads, c.n_seq); }

}  // namespace

int launch_pages_update(const PagesCall &c, void *stream) {
    const hipStream_t on = static_cast<hipStream_t>(stream);
    const dim3 rows = row_grid(c);
    const bool one = c.n_seq <= kAssignThreads, few = one && static_cast<int64_t>(c.n_seq) * c.max_pages <= kEntries * kAssignThreads;
    auto assign = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(1), dim3(kAssignThreads), 0, on, c); };
    if (c.source != nullptr && few) {
        assign(pages_assign_kernel<true, true>);
        return static_cast<int>(hipGetLastError());
    }
    if (c.source != nullptr) hipLaunchKernelGGL(pages_share_kernel, dim3(rows.x, (c.n_seq + kShareSlots - 1) / kShareSlots), dim3(kRowThreads), 0, on, c);
    if (one) assign(pages_assign_kernel<true, false>);
    else assign(pages_assign_kernel<false, false>);
    if (c.source != nullptr) hipLaunchKernelGGL(pages_rows_kernel, rows, dim3(kRowThreads), 0, on, c);
    return static_cast<int>(hipGetLastError());
}

int launch_pages_compact(const PagesCall &c, void *stream) {
    const hipStream_t on = static_cast<hipStream_t>(stream);
    if (c.n_pages <= kCompactPages) {
        hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(kAssignThreads), 0, on, c);
        return static_cast<int>(hipGetLastError());
    }
    const dim3 blocks((c.n_pages + kCounted - 1) / kCounted);
    hipLaunchKernelGGL(pages_count_kernel, blocks, dim3(kCountThreads), 0, on, c);
    hipLaunchKernelGGL(pages_pair_kernel, blocks, dim3(kCountThreads), 0, on, c);
    hipLaunchKernelGGL(pages_apply_kernel, dim3((c.n_pages / 2 + kCountThreads) / kCountThreads), dim3(kCountThreads), 0, on, c);
    return static_cast<int>(hipGetLastError());
}

int launch_pages_rename(const PagesCall &c, void *stream) {
    hipLaunchKernelGGL(pages_rename_kernel, row_grid(c), dim3(kRowThreads), 0, static_cast<hipStream_t>(stream), c);
    return static_cast<int>(hipGetLastError());
}

int launch_pages_copy(const CopyCall &c, int32_t n_pools, void *stream) {
    int64_t pieces = 1;
    for (int p = 0; p < n_pools; ++p) {
        const int64_t n = (c.pools[p].page_bytes / 16 + kPieceWords - 1) / kPieceWords;
        pieces = n > pieces ? n : pieces;
    }
    const int64_t most = 4096 / n_pools, all = pieces * c.max_moves;
    hipLaunchKernelGGL(pages_copy_kernel, dim3(static_cast<unsigned>(all < most ? all : most), n_pools), dim3(kCopyThreads), 0,
                       static_cast<hipStream_t>(stream), c);
    return static_cast<int>(hipGetLastError());
}

}  // namespace octopus
