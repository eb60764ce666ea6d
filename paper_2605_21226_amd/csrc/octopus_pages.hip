// Who holds which page: forking, growing, trimming and freeing sequences (pages_update), moving the pages in use to the front of the
// pools (pages_compact), and copying the pages that either says (pages_copy).
//
// A page's count is the number of table entries that hold it, a page with none is free, and free pages are handed out lowest number
// first, in the order of slots.  No list of free pages is kept: the counts are the whole state, results depend on nothing but them,
// and a call that releases and takes the same pages again leaves everything as it was.
#include <hip/hip_runtime.h>

#include "octopus_internal.h"

namespace octopus {
namespace {

constexpr int kLanes = 64;

// Inclusive sum over a wavefront's lanes.
__device__ __forceinline__ int wave_scan(int x, int lane) {
#pragma unroll
    for (int m = 1; m < kLanes; m *= 2) {
        const int other = __shfl_up(x, m, kLanes);
        x += lane >= m ? other : 0;
    }
    return x;
}

// Exclusive sums over a workgroup's threads, and everybody's sum.  (all threads call this; `room` is free again after the next barrier)
template <int THREADS>
__device__ __forceinline__ int block_scan(int x, int *room, int *total) {
    constexpr int WAVES = THREADS / kLanes;
    const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    const int upto = wave_scan(x, lane);
    __syncthreads();
    if (lane == kLanes - 1) room[wave] = upto;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const int n = room[w];
        before += w < wave ? n : 0;
        all += n;
    }
    *total = all;
    return before + upto - x;
}

__device__ __forceinline__ int pages_of(int tokens) { return (tokens + (OCTOPUS_TILE - 1)) / OCTOPUS_TILE; }
__device__ __forceinline__ int page_id(const PagesCall &c, int id) { return min(max(id, 0), c.n_pages - 1); }
// (counts change under atomics of this launch: a read goes to where those happen)
__device__ __forceinline__ int32_t load_count(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

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
// thread per entry.
constexpr int kRowThreads = 256;
__global__ __launch_bounds__(kRowThreads) void pages_share_kernel(PagesCall c) {
    const int s = blockIdx.y, j = blockIdx.x * kRowThreads + threadIdx.x;
    const Slot x = slot_of(c, s);
    const int kept = pages_of(x.kept), own = pages_of(x.own);
    const int64_t row = static_cast<int64_t>(s) * c.max_pages;
    const bool moved = x.src != s;
    if (j < own && (moved || j >= kept)) atomicAdd(&c.refs[page_id(c, c.table[row + j])], -1);
    if (moved && j < kept) {
        const int page = page_id(c, c.table[static_cast<int64_t>(x.src) * c.max_pages + j]);
        c.staged[row + j] = page;
        atomicAdd(&c.refs[page], 1);
    }
}

// Which pages are copied, which free pages go where: one workgroup, a thread per slot, in rounds of as many slots.
constexpr int kAssignThreads = 1024;
constexpr int kPerThread = 16;       // counts a thread reads at once in the search
__global__ __launch_bounds__(kAssignThreads) void pages_assign_kernel(PagesCall c) {
    __shared__ int room[kAssignThreads / kLanes];
    __shared__ int first_of[kAssignThreads], entry_of[kAssignThreads];
    const int tid = threadIdx.x;

    // f(slot, k, n): the k-th of the slot's `count` items, the n-th of this round; any thread, all of them at once
    auto each = [&](int base, int count, int entry, auto f) {
        int total;
        const int before = block_scan<kAssignThreads>(count, room, &total);
        if (total == 0) return;
        first_of[tid] = before;
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
            c.info[s] = SlotPages{x.kept, x.want, x.src, 0};
            from = pages_of(x.kept);
            lost = max(pages_of(x.own) - from, 0);
        }
        if (c.source == nullptr)
            each(base, lost, from, [&](int slot, int k, int entry, int) {
                atomicAdd(&c.refs[page_id(c, c.table[static_cast<int64_t>(slot) * c.max_pages + entry + k])], -1);
            });
    }
    __threadfence();
    __syncthreads();

    // A page that is written into, because what a slot keeps ends inside it, has to be the slot's own.  Of those that would write into the same
    // one, the lowest keeps it if nobody else holds it -- one that continues its own row before those that came to it -- and the others
    // take a copy.
    auto written = [&](int s, const SlotPages &x) {
        const int64_t at = static_cast<int64_t>(s) * c.max_pages + x.kept / OCTOPUS_TILE;
        return x.want > x.kept && x.kept % OCTOPUS_TILE != 0 ? page_id(c, x.src == s ? c.table[at] : c.staged[at]) : -1;
    };
    auto rank = [&](int s, const SlotPages &x) { return x.src == s ? s : c.n_seq + s; };
    bool shared = false;
    for (int s = tid; s < c.n_seq; s += kAssignThreads) {
        const int page = written(s, c.info[s]);
        shared |= page >= 0 && load_count(&c.refs[page]) > 1;
    }
    if (__syncthreads_or(shared)) {
        for (int s = tid; s < c.n_seq; s += kAssignThreads) {
            const int page = written(s, c.info[s]);
            if (page >= 0) {
                c.writers[page] = 0;
                c.first[page] = INT32_MAX;
            }
        }
        __threadfence();
        __syncthreads();
        for (int s = tid; s < c.n_seq; s += kAssignThreads) {
            const SlotPages x = c.info[s];
            const int page = written(s, x);
            if (page >= 0) {
                atomicAdd(&c.writers[page], 1);
                atomicMin(&c.first[page], rank(s, x));
            }
        }
        __threadfence();
        __syncthreads();
        for (int s = tid; s < c.n_seq; s += kAssignThreads) {
            const SlotPages x = c.info[s];
            const int page = written(s, x);
            if (page >= 0 && (load_count(&c.refs[page]) > load_count(&c.writers[page]) || load_count(&c.first[page]) != rank(s, x)))
                c.info[s].copied = 1;
        }
    }

    // pages that are asked for
    auto asked = [&](const SlotPages &x) { return x.want > x.kept ? pages_of(x.want) - pages_of(x.kept) + x.copied : 0; };
    int wanted = 0, copies = 0;
    for (int base = 0; base < c.n_seq; base += kAssignThreads) {
        const int s = base + tid;
        const SlotPages x = s < c.n_seq ? c.info[s] : SlotPages{0, 0, 0, 0};
        int total;
        block_scan<kAssignThreads>(asked(x), room, &total);
        wanted += total;
    }

    // the lowest free ones, in order
    int found = 0;
    for (int64_t base = 0; found < wanted && base < c.n_pages; base += kAssignThreads * kPerThread) {
        const int64_t at = base + tid * kPerThread;
        uint32_t free = 0;
        if (at + kPerThread <= c.n_pages) {
            int4 n[kPerThread / 4];
#pragma unroll
            for (int i = 0; i < kPerThread / 4; ++i) n[i] = *reinterpret_cast<const int4 *>(c.refs + at + 4 * i);
#pragma unroll
            for (int i = 0; i < kPerThread / 4; ++i)
                free |= ((n[i].x <= 0 ? 1u : 0u) | (n[i].y <= 0 ? 2u : 0u) | (n[i].z <= 0 ? 4u : 0u) | (n[i].w <= 0 ? 8u : 0u)) << (4 * i);
        } else {
            for (int i = 0; i < kPerThread; ++i)
                if (at + i < c.n_pages && c.refs[at + i] <= 0) free |= 1u << i;
        }
        int total;
        int n = found + block_scan<kAssignThreads>(__popc(free), room, &total);
        for (; free != 0 && n < wanted; free &= free - 1, ++n) c.fresh[n] = static_cast<int32_t>(at) + __ffs(free) - 1;
        found += total;
    }
    const bool enough = found >= wanted;
    __threadfence();
    __syncthreads();

    int given = 0;
    for (int base = 0; base < c.n_seq; base += kAssignThreads) {
        const int s = base + tid;
        SlotPages x = s < c.n_seq ? c.info[s] : SlotPages{0, 0, 0, 0};
        const int need = enough ? asked(x) : 0;
        if (!enough) x.copied = 0;
        int total, moved;
        const int begin = given + block_scan<kAssignThreads>(need, room, &total);
        const int nth = copies + block_scan<kAssignThreads>(x.copied, room, &moved);
        if (x.copied != 0) {
            const int page = written(s, x);
            c.moves[2 + 2 * nth] = page;
            c.moves[3 + 2 * nth] = c.fresh[begin];
            atomicAdd(&c.refs[page], -1);
        }
        each(base, need, pages_of(x.kept) - x.copied, [&](int slot, int k, int entry, int n) {   // (a barrier stands before its writes)
            const int page = c.fresh[given + n];
            c.table[static_cast<int64_t>(slot) * c.max_pages + entry + k] = page;
            c.refs[page] = 1;
        });
        if (s < c.n_seq) {
            c.lens[s] = enough ? x.want : x.kept;
            c.info[s] = x;
        }
        given += total;
        copies += moved;
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
// from n on go below n; after it the pages in use are 0 .. n - 1.  A workgroup counts its pages, and then numbers them from the others' counts.
constexpr int kCountThreads = 256;
constexpr int kCounted = kCountThreads * kPerThread;   // pages a workgroup looks at
__device__ __forceinline__ uint32_t used_pages(const PagesCall &c, int64_t at) {
    uint32_t used = 0;
#pragma unroll
    for (int i = 0; i < kPerThread; i += 4) {
        if (at + i + 4 <= c.n_pages) {
            const int4 n = *reinterpret_cast<const int4 *>(c.refs + at + i);
            used |= ((n.x > 0 ? 1u : 0u) | (n.y > 0 ? 2u : 0u) | (n.z > 0 ? 4u : 0u) | (n.w > 0 ? 8u : 0u)) << i;
        } else {
            for (int k = i; k < i + 4; ++k)
                if (at + k < c.n_pages && c.refs[at + k] > 0) used |= 1u << k;
        }
    }
    return used;
}

__global__ __launch_bounds__(kCountThreads) void pages_count_kernel(PagesCall c) {
    __shared__ int room[kCountThreads / kLanes];
    int total;
    block_scan<kCountThreads>(__popc(used_pages(c, static_cast<int64_t>(blockIdx.x) * kCounted + threadIdx.x * kPerThread)), room, &total);
    if (threadIdx.x == 0) c.writers[blockIdx.x] = total;
}

__global__ __launch_bounds__(kCountThreads) void pages_pair_kernel(PagesCall c) {
    __shared__ int room[kCountThreads / kLanes];
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
    int n = n_before + block_scan<kCountThreads>(__popc(used), room, &total);    // pages in use below this one
    for (int i = 0; i < kPerThread; ++i) {
        const int id = static_cast<int>(at) + i;
        if (id >= c.n_pages) break;
        const bool is = (used >> i) & 1u;
        c.page_map[id] = id;
        if (is && id >= n_used) c.moves[2 + 2 * (n_used - 1 - n)] = id;
        if (!is && id < n_used) c.moves[3 + 2 * (id - n)] = id;
        n += is ? 1 : 0;
        if (id == n_used - 1) c.moves[0] = n_used - n;      // free pages below n_used
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        c.moves[1] = n_used;
        if (n_used == 0) c.moves[0] = 0;
    }
}

__global__ __launch_bounds__(kCountThreads) void pages_apply_kernel(PagesCall c) {
    const int i = blockIdx.x * kCountThreads + threadIdx.x;
    if (i >= c.moves[0]) return;
    const int from = c.moves[2 + 2 * i], to = c.moves[3 + 2 * i];
    c.refs[to] = c.refs[from];
    c.refs[from] = 0;
    c.page_map[from] = to;
}

__global__ __launch_bounds__(kRowThreads) void pages_rename_kernel(PagesCall c) {
    const int s = blockIdx.y, j = blockIdx.x * kRowThreads + threadIdx.x;
    const int n = c.lens != nullptr ? min(pages_of(min(max(c.lens[s], 0), c.max_pages * OCTOPUS_TILE)), c.max_pages) : c.max_pages;
    if (j >= n) return;
    const int64_t at = static_cast<int64_t>(s) * c.max_pages + j;
    c.table[at] = c.page_map[page_id(c, c.table[at])];
}

// A pool's pages by blockIdx.y, pieces of 16 KB of the moved pages by blockIdx.x.
constexpr int kCopyThreads = 256, kCopyAhead = 4;
constexpr int kPieceWords = kCopyThreads * kCopyAhead;     // of 16 bytes
__global__ __launch_bounds__(kCopyThreads) void pages_copy_kernel(CopyCall c) {
    const CopyPool pool = c.pools[blockIdx.y];
    const int64_t words = pool.page_bytes / 16;
    const int pieces = static_cast<int>((words + kPieceWords - 1) / kPieceWords);
    const int n = min(max(c.moves[0], 0), c.max_moves);
    for (int64_t i = blockIdx.x; i < static_cast<int64_t>(n) * pieces; i += gridDim.x) {
        const int move = static_cast<int>(i / pieces);
        const int64_t first = (i % pieces) * kPieceWords + threadIdx.x;
        const uint32_t from = c.moves[2 + 2 * move], to = c.moves[3 + 2 * move];
        if (from >= static_cast<uint32_t>(c.n_pages) || to >= static_cast<uint32_t>(c.n_pages)) continue;
        const uint4 *src = static_cast<const uint4 *>(pool.data) + from * words;
        uint4 *dst = static_cast<uint4 *>(pool.data) + to * words;
        uint4 x[kCopyAhead];
#pragma unroll
        for (int k = 0; k < kCopyAhead; ++k)
            if (first + k * kCopyThreads < words) x[k] = src[first + k * kCopyThreads];
#pragma unroll
        for (int k = 0; k < kCopyAhead; ++k)
            if (first + k * kCopyThreads < words) dst[first + k * kCopyThreads] = x[k];
    }
}

dim3 row_grid(const PagesCall &c) { return dim3((c.max_pages + kRowThreads - 1) / kRowThreads, c.n_seq); }

}  // namespace

int launch_pages_update(const PagesCall &c, void *stream) {
    const hipStream_t on = static_cast<hipStream_t>(stream);
    if (c.source != nullptr) hipLaunchKernelGGL(pages_share_kernel, row_grid(c), dim3(kRowThreads), 0, on, c);
    hipLaunchKernelGGL(pages_assign_kernel, dim3(1), dim3(kAssignThreads), 0, on, c);
    if (c.source != nullptr) hipLaunchKernelGGL(pages_rows_kernel, row_grid(c), dim3(kRowThreads), 0, on, c);
    return static_cast<int>(hipGetLastError());
}

int launch_pages_compact(const PagesCall &c, void *stream) {
    const hipStream_t on = static_cast<hipStream_t>(stream);
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
