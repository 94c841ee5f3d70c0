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
// Three steps, as each needs the one before whole: tables and counts; what every
// row needs and what is free; the pages.  A few rows of a small pool are taken
// by one workgroup in one launch, others by a launch a step; bound by these launches and a few
// dependent round trips each until tables and pool are large: a fork of 64 x 16 rows of 114 entries over 29408 pages takes
// 14.3 us, 8.8 MB of tables and counts, a compaction of 200 pages 2.1 us, of 8000 4.4, of 200000 10.1.  A row that appends into
// a page filled in part looks at the rows before it in its group: 1 x K rows that do take 10 us with K = 16, 31 with 256, 99
// with 1024 and 370 with 4096.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ngpu_lm.h"
#include "reduce.h"

namespace ngpu {

constexpr int kPageThreads = 256;
constexpr int kPageWaves = kPageThreads / kWave;
constexpr int kRowBlock = kPageThreads;        // rows whose needs are summed together
constexpr int kTileSteps = 4;                  // pages a lane takes at a time
constexpr int kTile = kTileSteps * kPageThreads;
constexpr int kOneThreads = 1024;              // of the workgroup that takes a call alone
constexpr int kOneWaves = kOneThreads / kWave;
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
template <int WAVES = kPageWaves>
__device__ __forceinline__ int64_t scan_threads(int64_t x, int64_t &total) {
    __shared__ int64_t sums[WAVES];
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
    for (int w = 0; w < WAVES; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    return before + upto - x;
}

// The pages of a block in ascending order, a tile of coalesced loads at a time: visit(page, whether its count meets `is`, how
// many of the block before it do).  Returns how many do; for the whole workgroup.
template <int WAVES = kPageWaves, class Is, class Visit>
__device__ __forceinline__ int over_pages(const int32_t *refs, int64_t p0, int64_t p1, Is is, Visit visit) {
    constexpr int kSteps = kTileSteps;
    __shared__ int sums[2][WAVES];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int done = 0, turn = 0;
    for (int64_t t0 = p0; t0 < p1; t0 += kSteps * kWave * WAVES, turn ^= 1) {
        const int64_t w0 = t0 + wave * (kSteps * kWave) + lane;
        int r[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) r[i] = w0 + kWave * i < p1 ? refs[w0 + kWave * i] : 0;
        unsigned long long masks[kSteps];
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            masks[i] = __ballot(w0 + kWave * i < p1 && is(r[i]));
            mine += __builtin_popcountll(masks[i]);
        }
        if (lane == 0) sums[turn][wave] = mine;
        __syncthreads();
        int at = done;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            at += w < wave ? sums[turn][w] : 0;
            done += sums[turn][w];
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (w0 + kWave * i < p1) visit(w0 + kWave * i, (masks[i] >> lane & 1) != 0, at + lanes_below(masks[i]));
            at += __builtin_popcountll(masks[i]);
        }
    }
    return done;
}

__device__ __forceinline__ int64_t held_tokens(const ngpu_kv_fork_t &a, int64_t row) {
    return min(max(int64_t(a.lengths[row]), int64_t(0)), a.width * a.page_size);
}
__device__ __forceinline__ bool in_pool(const ngpu_kv_fork_t &a, int32_t page) { return page >= 0 && page < a.num_pages; }

// Counts are changed by many workgroups, or (ONE) by one, which then reads them.
template <bool ONE>
__device__ __forceinline__ void count_page(const ngpu_kv_fork_t &a, int32_t page, int by) {
    if (!in_pool(a, page)) return;
    __hip_atomic_fetch_add(a.refs + page, by, __ATOMIC_RELAXED, ONE ? __HIP_MEMORY_SCOPE_WORKGROUP : __HIP_MEMORY_SCOPE_AGENT);
}

// 1. A wavefront a row, the new ones first: a new row's entries, and an old row's part of the counts (children less one).
template <bool ONE>
__device__ __forceinline__ void fork_tables(const Fork &f, int64_t row, int lane) {
    const ngpu_kv_fork_t &a = f.a;
    const int64_t R = a.G * a.K;
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
        for (int64_t i = (children == 1 ? have : 0) + lane; i < a.width; i += kWave)
            count_page<ONE>(a, a.pages[old * a.pages_stride + i], (i < have ? children : 0) - 1);
    }
}
__global__ __launch_bounds__(kPageThreads) void fork_tables_kernel(Fork f) {
    fork_tables<false>(f, int64_t(blockIdx.x) * kPageWaves + threadIdx.x / kWave, threadIdx.x % kWave);
}

// The fresh pages that a row needs, and the page that it copies.
__device__ __forceinline__ int64_t fork_need(const Fork &f, int64_t row) {
    const ngpu_kv_fork_t &a = f.a;
    const int32_t last = f.last[row];
    bool copy = false;
    if (last >= 0) {
        int before = 0;
        for (int64_t r = row / a.K * a.K; r < row; ++r) before += f.last[r] == last ? 1 : 0;
        copy = a.refs[last] - before > 1;
    }
    f.from[row] = copy ? last : -1;
    return (copy ? 1 : 0) + max(f.more[row], 0);
}

// 2. What each row needs, summed over a row block, and the free pages of each block of pages.
__global__ __launch_bounds__(kPageThreads) void fork_plan_kernel(Fork f, int64_t row_blocks) {
    const ngpu_kv_fork_t &a = f.a;
    const int64_t R = a.G * a.K;
    if (int64_t(blockIdx.x) < row_blocks) {
        const int64_t row = int64_t(blockIdx.x) * kRowBlock + threadIdx.x;
        const int64_t need = row < R ? fork_need(f, row) : 0;
        int64_t total;
        const int64_t before = scan_threads(need, total);
        if (row < R) f.start[row] = before;
        if (threadIdx.x == 0) f.row_sums[blockIdx.x] = total;
        return;
    }
    const int64_t b = int64_t(blockIdx.x) - row_blocks, p0 = b * f.blocks.per, p1 = min(a.num_pages, p0 + f.blocks.per);
    const int n = over_pages(a.refs, p0, p1, [](int32_t r) { return r == 0; }, [&](int64_t page, bool free, int i) {
        if (free) f.lists[p0 + i] = int32_t(page);
    });
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

// 3. A wavefront a row: its fresh pages, from the first-th free one on, or its entries given back.
template <bool ONE>
__device__ __forceinline__ void fork_pages(const Fork &f, int64_t row, int lane, int64_t first, const int32_t *before,
                                           int blocks) {
    const ngpu_kv_fork_t &a = f.a;
    const int32_t parent = a.parents[row];
    const bool live = parent >= 0 && parent < a.W;
    const int32_t from = f.from[row], more = f.more[row];
    const int64_t need = (from >= 0 ? 1 : 0) + max(more, 0);
    const int64_t n = live ? held_tokens(a, row / a.K * a.W + parent) : 0, have = (n + a.page_size - 1) / a.page_size;
    int32_t *const entries = a.out_pages + row * a.width, *const copy = a.copies + 3 * row;
    if (live && (more < 0 || (need > 0 && first + need > before[blocks]))) {
        for (int64_t i = lane; i < have; i += kWave) {
            count_page<ONE>(a, entries[i], -1);
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
        int lo = 0, hi = blocks;   // before[lo] <= rank < before[hi]
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
            count_page<ONE>(a, from, -1);
        }
    }
    for (int64_t i = lane; i < more; i += kWave) entries[have + i] = fresh(first + (from >= 0 ? 1 : 0) + i);
}
__global__ __launch_bounds__(kPageThreads) void fork_pages_kernel(Fork f) {
    __shared__ int32_t before[kMostPageBlocks + 1];
    scan_counts(f.counts, f.blocks.count, before);
    const int64_t w0 = int64_t(blockIdx.x) * kPageWaves, row_block = w0 / kRowBlock;
    int64_t sum = 0, base;
    for (int64_t b = threadIdx.x; b < row_block; b += kPageThreads) sum += f.row_sums[b];
    scan_threads(sum, base);
    const int64_t row = w0 + threadIdx.x / kWave;
    if (row < f.a.G * f.a.K) fork_pages<false>(f, row, threadIdx.x % kWave, base + f.start[row], before, f.blocks.count);
}

// All three, by one workgroup: at most a thread for each new row.
__global__ __launch_bounds__(kOneThreads) void fork_one_kernel(Fork f) {
    const ngpu_kv_fork_t &a = f.a;
    __shared__ int32_t before[2];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int64_t R = a.G * a.K, rows = R + a.G * a.W;
    for (int64_t row = wave; row < rows; row += kOneWaves) fork_tables<true>(f, row, lane);
    __syncthreads();
    int64_t total;
    const int64_t start = scan_threads<kOneWaves>(int64_t(threadIdx.x) < R ? fork_need(f, threadIdx.x) : 0, total);
    if (int64_t(threadIdx.x) < R) f.start[threadIdx.x] = start;
    if (threadIdx.x == 0) before[0] = 0;
    const int n = over_pages<kOneWaves>(a.refs, 0, a.num_pages, [](int32_t r) { return r == 0; },
                                        [&](int64_t page, bool free, int i) {
                                            if (free) f.lists[i] = int32_t(page);
                                        });
    if (threadIdx.x == 0) before[1] = n;
    __syncthreads();
    for (int64_t row = wave; row < R; row += kOneWaves) fork_pages<true>(f, row, lane, f.start[row], before, 1);
}

namespace {

// Old and new rows, a wavefront each, fit a launch (of less than 2^32 work-items).
static_assert(2 * int64_t(NGPU_LM_MAX_SEQUENCES) * kWave <= int64_t(1) << 31, "rows of a launch");

// Most rows (of 64 entries, old and new) and pages that one workgroup takes alone.  us, against three launches: 16 rows and
// 70 pages 4.7 and 6.7, 24 rows 7.8 and 8.3, 48 rows and 416 pages 10.5 and 8.7, 128 rows 18 and 9; 16 rows and 4030 pages 7.5
// and 8.6, 8030 pages 9.1 and 8.8, 16030 pages 13.2 and 9.4.
constexpr int64_t kOneRows = 32, kOnePages = 4096;

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
    const int64_t steps = std::max<int64_t>((a.width + kWave - 1) / kWave, 1);   // of a wavefront over a row
    if (R > 0 && R <= kOneThreads && rows * steps <= kOneRows && a.num_pages <= kOnePages) {
        hipLaunchKernelGGL(fork_one_kernel, dim3(1), dim3(kOneThreads), 0, stream, f);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(fork_tables_kernel, dim3(unsigned((rows + kPageWaves - 1) / kPageWaves)), dim3(kPageThreads), 0, stream,
                       f);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (R == 0) return hipSuccess;
    const int64_t row_blocks = row_blocks_of(R);
    hipLaunchKernelGGL(fork_plan_kernel, dim3(unsigned(row_blocks + f.blocks.count)), dim3(kPageThreads), 0, stream, f,
                       row_blocks);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(fork_pages_kernel, dim3(unsigned((R + kPageWaves - 1) / kPageWaves)), dim3(kPageThreads), 0, stream,
                       f);
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
    const int n = over_pages(c.refs, p0, p1, [](int32_t r) { return r != 0; }, [](int64_t, bool, int) {});
    if (threadIdx.x == 0) c.counts[blockIdx.x] = n;
}

// The two sides of each move: used pages from n on, free ones below.
__global__ __launch_bounds__(kPageThreads) void compact_pairs_kernel(Compact c) {
    __shared__ int32_t before[kMostPageBlocks + 1];
    scan_counts(c.counts, c.blocks.count, before);
    const int64_t n = before[c.blocks.count];   // used pages
    // of them below page n: those of the blocks before its own, and of that block up to it
    const int64_t split = min(n / c.blocks.per, int64_t(c.blocks.count) - 1), s0 = split * c.blocks.per;
    const int64_t low = before[split] + over_pages(c.refs, s0, n, [](int32_t r) { return r != 0; }, [](int64_t, bool, int) {});
    const int64_t moves = n - low, half = c.num_pages / 2;
    const int64_t p0 = int64_t(blockIdx.x) * c.blocks.per, p1 = min(c.num_pages, p0 + c.blocks.per);
    const int64_t first = before[blockIdx.x];   // used pages before this block
    over_pages(c.refs, p0, p1, [](int32_t r) { return r != 0; }, [&](int64_t page, bool used, int i) {
        if (used && page >= n) {
            c.copies[3 * (first + i - low)] = int32_t(page);
            return;
        }
        c.moved[page] = int32_t(page);
        if (!used && page < n) c.copies[3 * (page - first - i) + 1] = int32_t(page);
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

// All of it by one workgroup, E pages a thread: their counts stay in registers.  us, against three launches: 200 pages 2.1
// and 6.4, 2000 2.4 and 8.5, 8000 4.4 and 9.4.
template <int E>
__global__ __launch_bounds__(kOneThreads) void compact_one_kernel(Compact c) {
    extern __shared__ int32_t holes[];   // the free pages below page n, ascending
    __shared__ int used_in[kOneWaves], free_in[kOneWaves];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, P = int(c.num_pages), p0 = wave * E * kWave + lane;
    int r[E];
#pragma unroll
    for (int i = 0; i < E; ++i) r[i] = p0 + kWave * i < P ? c.refs[p0 + kWave * i] : 0;
    int mine = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) mine += __builtin_popcountll(__ballot(r[i] != 0));
    if (lane == 0) used_in[wave] = mine;
    __syncthreads();
    int n = 0, first = 0;   // used pages: all, and those before this wavefront's
#pragma unroll
    for (int w = 0; w < kOneWaves; ++w) {
        first += w < wave ? used_in[w] : 0;
        n += used_in[w];
    }
    int used = first, free = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int page = p0 + kWave * i;
        const unsigned long long mask = __ballot(r[i] != 0), hole = __ballot(r[i] == 0 && page < n);
        if (r[i] == 0 && page < n) holes[page - used - lanes_below(mask)] = page;
        used += __builtin_popcountll(mask);
        free += __builtin_popcountll(hole);
    }
    if (lane == 0) free_in[wave] = free;
    __syncthreads();
    int moves = 0;
#pragma unroll
    for (int w = 0; w < kOneWaves; ++w) moves += free_in[w];
    used = first;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const int page = p0 + kWave * i;
        const unsigned long long mask = __ballot(r[i] != 0);
        if (page < P) {
            int to = page;
            if (r[i] != 0 && page >= n) {
                const int at = used + lanes_below(mask) - (n - moves);
                to = holes[at];
                c.copies[3 * at] = page;
                c.copies[3 * at + 1] = to;
                c.copies[3 * at + 2] = c.page_size;
                c.refs[to] = r[i];
                c.refs[page] = 0;
            }
            c.moved[page] = to;
        }
        used += __builtin_popcountll(mask);
    }
    for (int i = 3 * moves + int(threadIdx.x); i < 3 * (P / 2); i += kOneThreads) c.copies[i] = i % 3 == 2 ? 0 : -1;
}

template <int E>
static hipError_t compact_one(const Compact &c, hipStream_t stream) {
    hipLaunchKernelGGL(compact_one_kernel<E>, dim3(1), dim3(kOneThreads), size_t(c.num_pages / 2) * 4 + 4, stream, c);
    return hipGetLastError();
}

size_t kv_compact_workspace(int64_t num_pages) { return size_t(page_blocks(num_pages).count) * 4; }

hipError_t launch_kv_compact(int32_t *refs, int64_t num_pages, int32_t page_size, int32_t *copies, int32_t *moved,
                             void *workspace, hipStream_t stream) {
    const Compact c{refs, num_pages, page_size, copies, moved, page_blocks(num_pages), static_cast<int32_t *>(workspace)};
    if (num_pages <= 4 * kOneThreads) return compact_one<4>(c, stream);
    if (num_pages <= 8 * kOneThreads) return compact_one<8>(c, stream);
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
