// Page tables of a beam search: forking with reference counts, and compaction
// of a pool.  Pages themselves are copied by kv_copy.hip.
//
// Everything is integers whose result does not depend on an order: counts by
// atomic adds, ranks by prefix sums.  A page's rank among the free (or used)
// ones is the sum of the counts of the blocks of pages before its own and its
// place in that; a block's free pages are listed in the pass that counts them,
// so a row that is to get the r-th free page finds its block in the counts'
// prefix sums and reads the page from the list.
//
// Three launches, as each needs the one before whole: tables and counts; what
// every row needs and what is free; the pages.  Bound by these launches until
// tables and pool are large.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ngpu_lm.h"
#include "reduce.h"

namespace ngpu {

constexpr int kPageThreads = 256;
constexpr int kPageWaves = kPageThreads / kWave;
constexpr int kRowBlock = kPageThreads;        // rows whose needs are summed together
constexpr int kTile = 4096;                    // pages a workgroup takes at a time: 16 a lane
constexpr int kMostPageBlocks = 1024;          // whose counts a workgroup holds

// Blocks of pages: at most kMostPageBlocks, of whole tiles.
struct PageBlocks {
    int64_t per;       // pages a block
    int count;
};
static PageBlocks page_blocks(int64_t num_pages) {
    const int64_t tiles = (num_pages + kTile - 1) / kTile;
    const int64_t each = std::max<int64_t>(1, (tiles + kMostPageBlocks - 1) / kMostPageBlocks);
    return {each * kTile, int((tiles + each - 1) / each)};
}

struct Fork {
    ngpu_kv_fork_t a;
    PageBlocks blocks;
    int64_t *start;      // [R] needs of the rows before in its row block
    int64_t *row_sums;   // [row blocks]
    int32_t *last;       // [R] the page that the row would write into and others may hold, -1: none
    int32_t *more;       // [R] fresh pages behind it, -1: not to be had (dropped)
    int32_t *from;       // [R] the page to copy, -1: none
    int32_t *counts;     // [page blocks] free pages
    int32_t *lists;      // [page blocks, per] free pages, ascending
};

// Sum over the workgroup's threads before this one; `total`: over all.
__device__ __forceinline__ int64_t scan_threads(int64_t x, int64_t &total) {
    __shared__ int64_t sums[kPageWaves];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int64_t upto = x;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int64_t below = __shfl_up(upto, d);
        upto += lane >= d ? below : 0;
    }
    __syncthreads();
    if (lane == kWave - 1) sums[wave] = upto;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kPageWaves; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    return before + upto - x;
}

__device__ __forceinline__ int below(unsigned long long mask) {   // bits of the lanes before this one
    return int(__builtin_amdgcn_mbcnt_hi(unsigned(mask >> 32), __builtin_amdgcn_mbcnt_lo(unsigned(mask), 0u)));
}

// The pages of a block for which `is` holds, in ascending order, a tile of coalesced loads at a time:
// take(page, its number among them).  Returns how many there are; for the whole workgroup.
template <class Is, class Take>
__device__ __forceinline__ int over_pages(const int32_t *refs, int64_t p0, int64_t p1, Is is, Take take) {
    constexpr int kSteps = kTile / kPageThreads;
    __shared__ int sums[2][kPageWaves];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int done = 0, turn = 0;
    for (int64_t t0 = p0; t0 < p1; t0 += kTile, turn ^= 1) {
        const int64_t w0 = t0 + wave * (kTile / kPageWaves) + lane;
        int r[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) r[i] = w0 + kWave * i < p1 ? refs[w0 + kWave * i] : 0;
        unsigned long long masks[kSteps];
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            masks[i] = __ballot(w0 + kWave * i < p1 && is(r[i], w0 + kWave * i));
            mine += __builtin_popcountll(masks[i]);
        }
        if (lane == 0) sums[turn][wave] = mine;
        __syncthreads();
        int at = done;
#pragma unroll
        for (int w = 0; w < kPageWaves; ++w) {
            at += w < wave ? sums[turn][w] : 0;
            done += sums[turn][w];
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (masks[i] >> lane & 1) take(w0 + kWave * i, at + below(masks[i]));
            at += __builtin_popcountll(masks[i]);
        }
    }
    return done;
}

__device__ __forceinline__ int64_t held_tokens(const ngpu_kv_fork_t &a, int64_t row) {
    return min(max(int64_t(a.lengths[row]), int64_t(0)), a.width * a.page_size);
}
__device__ __forceinline__ bool in_pool(const ngpu_kv_fork_t &a, int32_t page) { return page >= 0 && page < a.num_pages; }

// 1. A wavefront a row, the new ones first: a new row's entries, and an old row's part of the counts (children less one).
__global__ __launch_bounds__(kPageThreads) void fork_tables_kernel(Fork f, int64_t row0) {
    const ngpu_kv_fork_t &a = f.a;
    const int lane = threadIdx.x % kWave;
    const int64_t R = a.G * a.K, row = row0 + int64_t(blockIdx.x) * kPageWaves + threadIdx.x / kWave;
    if (row < R) {
        const int64_t g = row / a.K;
        const int32_t parent = a.parents[row];
        const bool live = parent >= 0 && parent < a.W;
        const int64_t old = g * a.W + (live ? parent : 0);
        const int64_t n = live ? held_tokens(a, old) : 0, have = (n + a.page_size - 1) / a.page_size;
        int64_t tokens = live ? (a.tokens ? int64_t(a.tokens[row]) : a.T) : 0;
        tokens = max(tokens, int64_t(0));
        const int64_t wanted = (n + tokens + a.page_size - 1) / a.page_size;
        const bool fits = wanted <= a.width;
        for (int64_t i = lane; i < a.width; i += kWave)
            a.out_pages[row * a.width + i] = i < have ? a.pages[old * a.pages_stride + i] : -1;
        if (lane == 0) {
            int32_t last = -1;
            if (fits && tokens > 0 && n % a.page_size != 0) last = a.pages[old * a.pages_stride + have - 1];
            f.last[row] = in_pool(a, last) ? last : -1;
            f.more[row] = fits ? int32_t(tokens > 0 ? wanted - have : 0) : -1;
            a.out_lengths[row] = int32_t(min(n, int64_t(INT32_MAX)));
        }
    } else if (row < R + a.G * a.W) {
        const int64_t old = row - R, g = old / a.W;
        const int32_t w = int32_t(old % a.W);
        int children = 0;
        for (int64_t j0 = 0; j0 < a.K; j0 += kWave)
            children += __builtin_popcountll(__ballot(j0 + lane < a.K && a.parents[g * a.K + min(j0 + lane, a.K - 1)] == w));
        const int64_t have = children > 0 ? (held_tokens(a, old) + a.page_size - 1) / a.page_size : 0;
        // (one child takes over what the row held)
        for (int64_t i = (children == 1 ? have : 0) + lane; i < a.width; i += kWave) {
            const int32_t page = a.pages[old * a.pages_stride + i];
            if (in_pool(a, page)) atomicAdd(a.refs + page, (i < have ? children : 0) - 1);
        }
    }
}

// 2. What each row needs, summed over a row block, and the free pages of each block of pages.
__global__ __launch_bounds__(kPageThreads) void fork_plan_kernel(Fork f, int64_t row_blocks) {
    const ngpu_kv_fork_t &a = f.a;
    const int64_t R = a.G * a.K;
    if (int64_t(blockIdx.x) < row_blocks) {
        const int64_t row = int64_t(blockIdx.x) * kRowBlock + threadIdx.x;
        int64_t need = 0;
        if (row < R) {
            const int32_t last = f.last[row];
            bool copy = false;
            if (last >= 0) {
                int before = 0;
                for (int64_t r = row / a.K * a.K; r < row; ++r) before += f.last[r] == last ? 1 : 0;
                copy = a.refs[last] - before > 1;
            }
            f.from[row] = copy ? last : -1;
            need = (copy ? 1 : 0) + max(f.more[row], 0);
        }
        int64_t total;
        const int64_t before = scan_threads(need, total);
        if (row < R) f.start[row] = before;
        if (threadIdx.x == 0) f.row_sums[blockIdx.x] = total;
        return;
    }
    const int64_t b = int64_t(blockIdx.x) - row_blocks, p0 = b * f.blocks.per, p1 = min(a.num_pages, p0 + f.blocks.per);
    const int n = over_pages(a.refs, p0, p1, [](int32_t r, int64_t) { return r == 0; },
                             [&](int64_t page, int i) { f.lists[p0 + i] = int32_t(page); });
    if (threadIdx.x == 0) f.counts[b] = n;
}

// The counts' prefix sums in `before`, [blocks + 1].
__device__ __forceinline__ void scan_counts(const int32_t *counts, int blocks, int32_t *before) {
    constexpr int kEach = kMostPageBlocks / kPageThreads;
    int32_t c[kEach];
    int64_t sum = 0, total;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int b = int(threadIdx.x) * kEach + i;
        c[i] = b < blocks ? counts[b] : 0;
        sum += c[i];
    }
    int64_t at = scan_threads(sum, total);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int b = int(threadIdx.x) * kEach + i;
        if (b < blocks) before[b] = int32_t(at);
        at += c[i];
    }
    if (threadIdx.x == 0) before[blocks] = int32_t(total);
    __syncthreads();
}

// 3. A wavefront a row: its fresh pages, or its entries given back.
__global__ __launch_bounds__(kPageThreads) void fork_pages_kernel(Fork f, int64_t row0) {
    const ngpu_kv_fork_t &a = f.a;
    __shared__ int32_t before[kMostPageBlocks + 1];
    scan_counts(f.counts, f.blocks.count, before);
    const int64_t R = a.G * a.K, w0 = row0 + int64_t(blockIdx.x) * kPageWaves, row_block = w0 / kRowBlock;
    int64_t sum = 0, base;
    for (int64_t b = threadIdx.x; b < row_block; b += kPageThreads) sum += f.row_sums[b];
    scan_threads(sum, base);
    const int lane = threadIdx.x % kWave;
    const int64_t row = w0 + threadIdx.x / kWave;
    if (row >= R) return;
    const int32_t parent = a.parents[row];
    const bool live = parent >= 0 && parent < a.W;
    const int32_t from = f.from[row], more = f.more[row];
    const int64_t first = base + f.start[row], need = (from >= 0 ? 1 : 0) + max(more, 0);
    const int64_t n = live ? held_tokens(a, row / a.K * a.W + parent) : 0, have = (n + a.page_size - 1) / a.page_size;
    int32_t *const entries = a.out_pages + row * a.width, *const copy = a.copies + 3 * row;
    if (live && (more < 0 || (need > 0 && first + need > before[f.blocks.count]))) {
        for (int64_t i = lane; i < have; i += kWave) {
            if (const int32_t page = entries[i]; in_pool(a, page)) atomicAdd(a.refs + page, -1);
            entries[i] = -1;
        }
        if (lane == 0) {
            a.out_lengths[row] = -1;
            copy[0] = copy[1] = -1;
            copy[2] = 0;
        }
        return;
    }
    auto fresh = [&](int64_t rank) {   // the free page of this rank
        int lo = 0, hi = f.blocks.count;   // before[lo] <= rank < before[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (before[mid] <= rank)
                lo = mid;
            else
                hi = mid;
        }
        const int32_t page = f.lists[lo * f.blocks.per + (rank - before[lo])];
        a.refs[page] = 1;
        return page;
    };
    if (lane == 0) {
        copy[0] = from;
        copy[1] = -1;
        copy[2] = 0;
        if (from >= 0) {
            const int32_t page = fresh(first);
            copy[1] = entries[have - 1] = page;
            copy[2] = int32_t(n % a.page_size);
            atomicAdd(a.refs + from, -1);
        }
    }
    for (int64_t i = lane; i < more; i += kWave) entries[have + i] = fresh(first + (from >= 0 ? 1 : 0) + i);
}

namespace {

constexpr int64_t kMostGroups = int64_t(1) << 23;   // workgroups a launch

int64_t row_blocks_of(int64_t rows) { return (rows + kRowBlock - 1) / kRowBlock; }

Fork fork_of(const ngpu_kv_fork_t &a, char *ws, size_t *bytes) {
    Fork f{a, page_blocks(a.num_pages)};
    const size_t R = size_t(a.G * a.K);
    char *at = ws;
    auto take = [&](auto *&p, size_t n) {
        p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(at);
        at += (n * sizeof(*p) + 15) / 16 * 16;
    };
    take(f.start, R);
    take(f.row_sums, size_t(row_blocks_of(int64_t(R))));
    take(f.last, R);
    take(f.more, R);
    take(f.from, R);
    take(f.counts, size_t(f.blocks.count));
    take(f.lists, size_t(f.blocks.count) * size_t(f.blocks.per));
    if (bytes) *bytes = size_t(at - ws);
    return f;
}

}  // namespace

size_t kv_fork_workspace(int64_t G, int64_t K, int64_t num_pages) {
    ngpu_kv_fork_t a{};
    a.G = G;
    a.K = K;
    a.num_pages = num_pages;
    size_t bytes;
    fork_of(a, nullptr, &bytes);
    return bytes;
}

hipError_t launch_kv_fork(const ngpu_kv_fork_t &a, void *workspace, hipStream_t stream) {
    const Fork f = fork_of(a, static_cast<char *>(workspace), nullptr);
    const int64_t R = a.G * a.K, rows = R + a.G * a.W;
    for (int64_t r0 = 0; r0 < rows; r0 += kMostGroups * kPageWaves) {
        const int64_t grid = std::min(kMostGroups, (rows - r0 + kPageWaves - 1) / kPageWaves);
        hipLaunchKernelGGL(fork_tables_kernel, dim3(unsigned(grid)), dim3(kPageThreads), 0, stream, f, r0);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (R == 0) return hipSuccess;
    const int64_t row_blocks = row_blocks_of(R);
    hipLaunchKernelGGL(fork_plan_kernel, dim3(unsigned(row_blocks + f.blocks.count)), dim3(kPageThreads), 0, stream, f,
                       row_blocks);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(fork_pages_kernel, dim3(unsigned((R + kPageWaves - 1) / kPageWaves)), dim3(kPageThreads), 0, stream,
                       f, int64_t(0));
    return hipGetLastError();
}

// ---------------------------------------------------------------- compaction

struct Compact {
    int32_t *refs;
    int64_t num_pages;
    int32_t page_size;
    int32_t *copies, *moved;
    PageBlocks blocks;
    int32_t *counts;     // [page blocks] used pages
};

__global__ __launch_bounds__(kPageThreads) void compact_count_kernel(Compact c) {
    const int64_t p0 = int64_t(blockIdx.x) * c.blocks.per, p1 = min(c.num_pages, p0 + c.blocks.per);
    const int n = over_pages(c.refs, p0, p1, [](int32_t r, int64_t) { return r != 0; }, [](int64_t, int) {});
    if (threadIdx.x == 0) c.counts[blockIdx.x] = n;
}

// The two sides of each move: used pages from n on, free ones below.
__global__ __launch_bounds__(kPageThreads) void compact_pairs_kernel(Compact c) {
    __shared__ int32_t before[kMostPageBlocks + 1];
    scan_counts(c.counts, c.blocks.count, before);
    const int64_t n = before[c.blocks.count];   // used pages
    // of them below page n: those of the blocks before its own, and of that block up to it
    const int64_t split = min(n / c.blocks.per, int64_t(c.blocks.count) - 1), s0 = split * c.blocks.per;
    const int64_t low = before[split] + over_pages(c.refs, s0, n, [](int32_t r, int64_t) { return r != 0; }, [](int64_t, int) {});
    __syncthreads();
    const int64_t moves = n - low, half = c.num_pages / 2;
    const int64_t p0 = int64_t(blockIdx.x) * c.blocks.per, p1 = min(c.num_pages, p0 + c.blocks.per);
    const int64_t first = before[blockIdx.x];   // used pages before this block
    over_pages(c.refs, p0, p1, [](int32_t r, int64_t) { return r != 0; },
               [&](int64_t page, int i) {
                   if (page >= n)
                       c.copies[3 * (first + i - low)] = int32_t(page);
                   else
                       c.moved[page] = int32_t(page);
               });
    over_pages(c.refs, p0, p1, [](int32_t r, int64_t) { return r == 0; },
               [&](int64_t page, int i) {
                   c.moved[page] = int32_t(page);
                   if (page < n) c.copies[3 * (p0 - first + i) + 1] = int32_t(page);
               });
    for (int64_t i = p0 / 2 + threadIdx.x; i < min(half, p1 / 2); i += kPageThreads) {
        c.copies[3 * i + 2] = i < moves ? c.page_size : 0;
        if (i >= moves) c.copies[3 * i] = c.copies[3 * i + 1] = -1;
    }
}

__global__ __launch_bounds__(kPageThreads) void compact_move_kernel(Compact c) {
    const int64_t i = int64_t(blockIdx.x) * kPageThreads + threadIdx.x;
    if (i >= c.num_pages / 2) return;
    const int32_t from = c.copies[3 * i], to = c.copies[3 * i + 1];
    if (from < 0) return;
    c.moved[from] = to;
    c.refs[to] = c.refs[from];
    c.refs[from] = 0;
}

__global__ __launch_bounds__(kPageThreads) void move_kernel(int32_t *pages, int64_t rows, int64_t width, int64_t stride,
                                                            const int32_t *moved, int64_t num_pages) {
    const int64_t all = rows * width, step = int64_t(gridDim.x) * kPageThreads;
    for (int64_t i = int64_t(blockIdx.x) * kPageThreads + threadIdx.x; i < all; i += step) {
        int32_t &page = pages[i / width * stride + i % width];
        if (page >= 0 && page < num_pages) page = moved[page];
    }
}

size_t kv_compact_workspace(int64_t num_pages) { return size_t(page_blocks(num_pages).count) * 4; }

hipError_t launch_kv_compact(int32_t *refs, int64_t num_pages, int32_t page_size, int32_t *copies, int32_t *moved,
                             void *workspace, hipStream_t stream) {
    const Compact c{refs, num_pages, page_size, copies, moved, page_blocks(num_pages), static_cast<int32_t *>(workspace)};
    hipLaunchKernelGGL(compact_count_kernel, dim3(unsigned(c.blocks.count)), dim3(kPageThreads), 0, stream, c);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(compact_pairs_kernel, dim3(unsigned(c.blocks.count)), dim3(kPageThreads), 0, stream, c);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int64_t half = num_pages / 2;
    if (half == 0) return hipSuccess;
    hipLaunchKernelGGL(compact_move_kernel, dim3(unsigned((half + kPageThreads - 1) / kPageThreads)), dim3(kPageThreads), 0,
                       stream, c);
    return hipGetLastError();
}

hipError_t launch_kv_move(int32_t *pages, int64_t rows, int64_t width, int64_t stride, const int32_t *moved,
                          int64_t num_pages, hipStream_t stream) {
    const int64_t groups = std::min<int64_t>((rows * width + kPageThreads - 1) / kPageThreads, 4096);
    hipLaunchKernelGGL(move_kernel, dim3(unsigned(groups)), dim3(kPageThreads), 0, stream, pages, rows, width, stride, moved,
                       num_pages);
    return hipGetLastError();
}

}  // namespace ngpu
