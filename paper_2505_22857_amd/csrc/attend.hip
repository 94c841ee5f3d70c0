// Attention over a paged cache with a prefix that a group of sequences shares:
// the kernels' choice and launches, the kernel for dimensions and strides that
// the matrix kernel (attend_tile.h) does not take, and the join of a row's parts.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>

#include "attend_tile.h"

namespace ngpu {

// One workgroup per row (sequence, query token, head); its wavefronts take every
// fourth key and keep sums of their own, which meet in LDS.  Any dimension and
// stride, an element at a time, and each row reads its keys itself: 8 x 8 sequences,
// 4099 of prefix, 4 x 8 heads of 128 take 3068 us, the matrix kernel 35.
constexpr int kRowWaves = 4;
template <class T>
__global__ __launch_bounds__(kRowWaves * kWave) void attend_row_kernel(Attend p, int64_t row0) {
    const ngpu_attend_t &a = p.a;
    const int64_t row = row0 + blockIdx.x, s = row / a.q_heads / a.T, t = row / a.q_heads % a.T;
    const int head = int(row % a.q_heads), kv = head / (a.q_heads / p.c.heads);
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int64_t nq = query_length(a, s);
    RowPart<T> r;
    r.load(p, s, t, head, lane);
    if (t < nq) {
        if (a.G > 0) {
            const PageTable prefix = prefix_table(p, s / (a.S / a.G));
            for (int64_t j = wave; j < prefix.count; j += kRowWaves) r.take(p, prefix, j, kv, lane);
        }
        if (a.pages) {
            const PageTable own = own_table(p, s);
            for (int64_t j = wave; j < min(own.count, own.count - nq + t + 1); j += kRowWaves) r.take(p, own, j, kv, lane);
        }
    }
    __shared__ float2 stats[kRowWaves];
    __shared__ float sums[kRowWaves][NGPU_LM_MAX_HEAD_DIM];
    if (lane == 0) stats[wave] = make_float2(r.m, r.sum);
#pragma unroll
    for (int i = 0; i < r.kDims; ++i) sums[wave][lane + kWave * i] = r.o[i];
    __syncthreads();
    if (wave != 0) return;
    float top = stats[0].x, total = 0.0f, f[kRowWaves];
    for (int w = 1; w < kRowWaves; ++w) top = stats[w].x > top ? stats[w].x : top;
    for (int w = 0; w < kRowWaves; ++w) {   // (a part without a key: sum 0, whatever the factor)
        f[w] = stats[w].x == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(stats[w].x - top);
        total += stats[w].y * f[w];
    }
    r.m = top;
    r.sum = total;
#pragma unroll
    for (int i = 0; i < r.kDims; ++i) {
        r.o[i] = 0.0f;
        for (int w = 0; w < kRowWaves; ++w) r.o[i] += sums[w][lane + kWave * i] * f[w];
    }
    r.finish(p, row, lane, t < nq);
}

template <class T>
static hipError_t launch_rows(const Attend &p, hipStream_t stream) {
    constexpr int64_t kMost = int64_t(UINT32_MAX) / (kRowWaves * kWave);
    const int64_t rows = p.a.S * p.a.T * p.a.q_heads;
    for (int64_t r0 = 0; r0 < rows; r0 += kMost) {
        hipLaunchKernelGGL((attend_row_kernel<T>), dim3(unsigned(std::min(kMost, rows - r0))),
                           dim3(kRowWaves * kWave), 0, stream, p, r0);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

// A row's parts joined: `lanes` threads take 4 dimensions each, and `groups` such
// sets of threads every groups-th part, eight parts at a time so that their
// loads are in flight together; the sets then meet in LDS.  Bound by reading the
// parts: 12288 rows of 5 or 6 of 128 dimensions (35 MB) 10 us, 160 rows of 33 6 us.
constexpr int kJoinThreads = 256;
template <class T>
__global__ __launch_bounds__(kJoinThreads) void attend_join_kernel(Attend p, AttendPlan plan, int64_t rows, int lanes,
                                                                   int groups, int64_t row0) {
    constexpr int kBatch = 8;
    const ngpu_attend_t &a = p.a;
    const int D = p.c.dim, d = int(threadIdx.x) % lanes * 4, group = int(threadIdx.x) / lanes % groups;
    const int64_t row = row0 + int64_t(blockIdx.x) * (kJoinThreads / (lanes * groups)) + int(threadIdx.x) / (lanes * groups);
    const int64_t token = row / a.q_heads;
    const bool counts = row < rows && token % a.T < query_length(a, token / a.T);
    float top = -__builtin_inff(), sum = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    // the parts of this row: its group's, then its sequence's own
    int first = 0, skip = 0;   // parts of the prefix, and of its room that its group has not
    if (plan.prefix.problems > 0) {
        first = plan.prefix.splits;
        if (plan.prefix.parts > plan.prefix.splits) {
            const int lane = threadIdx.x % kWave;
            const int n = dealt_splits(plan.prefix, int(a.G), lane < a.G ? prefix_table(p, lane).count : 0);
            first = __shfl(n, row < rows ? int(token / a.T / (a.S / a.G)) : 0);
        }
        skip = plan.prefix.parts - first;
    }
    const int parts = first + plan.own.splits;
    auto factor = [](float m, float base) { return m == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m - base); };
    if (counts && d < D) {
        for (int i = group; i < parts; i += groups * kBatch) {
            float2 s[kBatch];
            f32x4 x[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {   // past the last part: the last again, for nothing
                const int n = min(i + u * groups, parts - 1);
                const int64_t at = (n < first ? n : n + skip) * rows + row;
                s[u] = plan.stats[at];
                x[u] = *reinterpret_cast<const f32x4 *>(plan.sums + at * D + d);
            }
            const float before = top;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) top = i + u * groups < parts ? __builtin_fmaxf(top, s[u].x) : top;
            const float base = top == -__builtin_inff() ? 0.0f : top, f0 = factor(before, base);
            sum *= f0;
            o *= f0;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                // a part without a key (sum 0) has written no sums; a NaN sum goes on
                const bool any = i + u * groups < parts && s[u].y != 0.0f;
                const float f = factor(s[u].x, base);
                sum += any ? s[u].y * f : 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] += any ? x[u][e] * f : 0.0f;
            }
        }
    }
    if (groups > 1) {
        __shared__ f32x4 sums[kJoinThreads];
        __shared__ float2 stats[kJoinThreads];
        sums[threadIdx.x] = o;
        stats[threadIdx.x] = make_float2(top, sum);
        __syncthreads();
        if (group != 0) return;
        for (int g = 1; g < groups; ++g) {
            const int at = int(threadIdx.x) + g * lanes;
            const float2 s = stats[at];
            const float now = __builtin_fmaxf(top, s.x), base = now == -__builtin_inff() ? 0.0f : now;
            const float f0 = factor(top, base), f1 = factor(s.x, base);
            sum = sum * f0 + s.y * f1;
            o = o * f0 + sums[at] * f1;
            top = now;
        }
    }
    if (row >= rows || d >= D) return;
    const bool any = sum != 0.0f;
    if (a.lse && d == 0)
        a.lse[row] = any ? (top == -__builtin_inff() ? sum : top * 0.69314718056f + logf(sum)) : -__builtin_inff();
    const float f = 1.0f / sum;
    s16x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = any ? short(from_float<T>(o[i] * f).bits) : short(0);
    *reinterpret_cast<s16x4 *>(static_cast<T *>(a.out) + row * D + d) = y;
}

namespace {

constexpr int kCus = 256;   // of an MI355X

// Which kernel takes a call, and how it is cut.
struct Choice {
    bool tiles;              // the matrix kernel takes it
    int steps;               // 32-dimension steps of a head: 2, 3, 4, 8
    int prefix_tiles, own_tiles;      // 16-row tiles a wavefront
    int prefix_waves, own_waves;      // wavefronts along rows: 1, 2, 4
    AttendPlan plan;
};

// The matrix kernel loads 16 bytes of 8 elements at a time and keeps a row of
// the cache as a 32-bit number of them, and of a query as one of rows: pages that
// span more than 32 GiB of keys or values go by the element kernel.
bool takes_tiles(const ngpu_kv_cache_t &c, const ngpu_attend_t &a) {
    const int64_t strides[] = {c.k_stride_page, c.k_stride_token, c.k_stride_head,
                               c.v_stride_page, c.v_stride_token, c.v_stride_head};
    for (const int64_t s : strides)
        if (s % 8 != 0) return false;
    constexpr int64_t kMost = int64_t(1) << 31;   // 16-byte units: pages and tokens each stay below half the range
    const int64_t pages = std::max<int64_t>(c.num_pages, 1);
    return c.dim % 8 == 0 && reinterpret_cast<uintptr_t>(c.k) % 16 == 0 && reinterpret_cast<uintptr_t>(c.v) % 16 == 0 &&
           reinterpret_cast<uintptr_t>(a.out) % 16 == 0 && c.k_stride_page / 8 <= kMost / pages &&
           c.v_stride_page / 8 <= kMost / pages && c.k_stride_token / 8 <= kMost / c.page_size &&
           c.v_stride_token / 8 <= kMost / c.page_size && a.S * a.T * a.q_heads < kMost / 2;
}

// Rows of a problem to wavefronts.  4 prefixes of 8192 tokens, 8 heads of 128, us: 48 / 64 / 96 / 128 / 384 rows 35 / 38 /
// 38 / 41 / 73; blocks of one wavefront, which read the keys again, 43 / 44 / 50 / 62 / 135; of two for the last three
// 43 / 45 / 97.  Two tiles for up to 16 rows: 30.4, not 29.8; 4 rows of 64 dimensions 11.3, not 10.5.
void cut_rows(int64_t rows, int steps, int &tiles, int &waves, int &blocks) {
    tiles = rows <= 16 || steps > 4 ? 1 : 2;
    waves = rows <= 16 * tiles ? 1 : (rows <= 32 * tiles ? 2 : 4);
    blocks = int((rows + 16 * tiles * waves - 1) / (16 * tiles * waves));
}

Choice choose(const ngpu_kv_cache_t &c, const ngpu_attend_t &a, char *workspace) {
    Choice r{};
    r.tiles = takes_tiles(c, a);
    if (!r.tiles) return r;
    r.steps = c.dim <= 64 ? 2 : (c.dim <= 96 ? 3 : (c.dim <= 128 ? 4 : 8));
    const int64_t rep = a.q_heads / c.heads;
    auto cut = [&](int64_t problems, int64_t rows, int64_t most_keys, int64_t wanted, int &tiles, int &waves) {
        Cut u{problems, 0, 0, 0};
        cut_rows(rows, r.steps, tiles, waves, u.blocks);
        // Two tiles a split at least: 1500 tokens of 8 heads of 64 10.5 us, with one 10.1, with four 11.8; 1000 for 64
        // rows a head 11.9, with one 13.0, with four 12.9.
        const int64_t tile = waves == 4 ? 64 : 32, have = problems * u.blocks;
        const int64_t most = std::max<int64_t>(1, (most_keys + 2 * tile - 1) / (2 * tile));
        u.splits = u.parts = int(std::min<int64_t>(std::min<int64_t>(most, 128), std::max<int64_t>(1, wanted / have)));
        return u;
    };
    // Workgroups a CU: more of them only disturb each other's streams.  One prefix
    // of 100000 tokens for 5 x 4 rows, 8 heads of 128, us: 238 / 205 / 214 / 273 with 2 / 3 /
    // 4 / 5; heads of 64: 67 / 51 / 49 / 52; of 256 (2 fit): 48, 62 with 3.
    const int64_t per_cu = r.steps == 2 ? 4 : (r.steps <= 4 ? 3 : 2);
    const int64_t prefix_rows = a.G > 0 ? a.S / a.G * a.T * rep : 0;
    if (a.pages) {
        // Workgroups: 2 a CU, not 4, where several wavefronts share the keys (us: 4 sequences of 500 tokens that see 3500,
        // 32 / 8 heads of 128 129, not 164; one of 64 that sees 8000 31, not 49), and beside prefixes whose rows
        // take several, where own tokens wait for memory while those compute (64 sequences of one token that see 300, 2048
        // of prefix 60, not 68).
        cut_rows(prefix_rows, r.steps, r.prefix_tiles, r.prefix_waves, r.plan.prefix.blocks);
        cut_rows(a.T * rep, r.steps, r.own_tiles, r.own_waves, r.plan.own.blocks);
        const int64_t keys = a.pages_width * c.page_size, have = a.S * c.heads * r.plan.own.blocks;
        r.plan.own = cut(a.S * c.heads, a.T * rep, keys, (r.prefix_waves > 1 || r.own_waves == 4 ? 2 : 4) * kCus,
                         r.own_tiles, r.own_waves);
        // One workgroup a block of rows would have the last block's be twice as long as the mean: one sequence of
        // 8192 tokens that see each other, 8 heads of 64: 280 us, in two splits 178.
        if (r.own_waves == 4 && 2 * a.T > keys && have <= 2 * kCus) r.plan.own.splits = std::max(r.plan.own.splits, 2);
        r.plan.own.parts = r.plan.own.splits;
    }
    if (a.G > 0) {
        const int64_t left = per_cu * kCus - r.plan.own.works();
        r.plan.prefix = cut(a.G * c.heads, prefix_rows, a.prefix_width * c.page_size,
                            std::max<int64_t>(left, 2 * kCus), r.prefix_tiles, r.prefix_waves);
        if (r.prefix_waves == 4)
            r.plan.prefix = cut(a.G * c.heads, prefix_rows, a.prefix_width * c.page_size, 2 * kCus,
                                r.prefix_tiles, r.prefix_waves);
    }
    if (a.G > 1 && a.G <= kDealt && r.plan.prefix.splits > 1)   // a group may take more than its share
        r.plan.prefix.parts = int(std::min<int64_t>(2 * r.plan.prefix.splits, 1 + a.G * (r.plan.prefix.splits - 1)));
    r.plan.parts = r.plan.prefix.parts + r.plan.own.splits;
    const int64_t rows = a.S * a.T * a.q_heads;
    r.plan.page_magic = c.page_size == 1 ? UINT32_MAX : unsigned((uint64_t(1) << 32) / unsigned(c.page_size));
    r.plan.sums = reinterpret_cast<float *>(workspace);
    r.plan.stats = reinterpret_cast<float2 *>(workspace + size_t(r.plan.parts) * size_t(rows) * c.dim * 4);
    return r;
}

// More LDS than a launch has by default, asked for once a device (bits of `devices`).
template <class K>
hipError_t allow_lds(K *kernel, int bytes, std::atomic<uint64_t> &devices) {
    int device;
    if (const hipError_t e = hipGetDevice(&device); e != hipSuccess) return e;
    const uint64_t bit = uint64_t(1) << device % 64;
    if (device < 64 && (devices.load(std::memory_order_relaxed) & bit)) return hipSuccess;
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess && device < 64) devices.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

template <class T, int DK, int RT, int WR>
hipError_t launch_tile(const Attend &p, const AttendPlan &plan, int64_t w0, int64_t w1, hipStream_t stream) {
    using A = AttendTile<T, DK, RT, WR>;
    constexpr int64_t kMost = int64_t(1) << 23;   // workgroups a launch
    static std::atomic<uint64_t> devices;
    if (const hipError_t e = allow_lds(&attend_tile_kernel<T, DK, RT, WR>, A::kLds, devices); e != hipSuccess) return e;
    for (; w0 < w1; w0 += kMost) {
        hipLaunchKernelGGL((attend_tile_kernel<T, DK, RT, WR>), dim3(unsigned(std::min(kMost, w1 - w0))),
                           dim3(64 * WR), A::kLds, stream, p, plan, unsigned(w0));
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <class T, int DK>
hipError_t launch_tile(const Attend &p, const AttendPlan &plan, int tiles, int waves, int64_t w0, int64_t w1,
                       hipStream_t stream) {
    constexpr int kMost = DK <= 4 ? 2 : 1;   // tiles a wavefront's registers hold
    if (waves == 1 && tiles == 1) return launch_tile<T, DK, 1, 1>(p, plan, w0, w1, stream);
    if (waves == 1) return launch_tile<T, DK, kMost, 1>(p, plan, w0, w1, stream);
    if (waves == 2) return launch_tile<T, DK, kMost, 2>(p, plan, w0, w1, stream);
    return launch_tile<T, DK, kMost, 4>(p, plan, w0, w1, stream);
}
template <class T, int DK, int WR>
hipError_t launch_both(const Attend &p, const AttendPlan &plan, hipStream_t stream) {
    constexpr int RT = DK <= 4 ? 2 : 1;
    using A = AttendTile<T, DK, RT, WR>;
    constexpr int64_t kMost = int64_t(1) << 23;   // workgroups a launch
    static std::atomic<uint64_t> devices;
    if (const hipError_t e = allow_lds(&attend_both_kernel<T, DK, RT, WR>, A::kLds, devices); e != hipSuccess) return e;
    constexpr int kWaves = kOwnWaves<T, DK, RT, WR>;
    const int64_t own = (plan.own.works() + kWaves - 1) / kWaves, all = own + plan.prefix.works();
    for (int64_t b0 = 0; b0 < all; b0 += kMost) {
        hipLaunchKernelGGL((attend_both_kernel<T, DK, RT, WR>), dim3(unsigned(std::min(kMost, all - b0))),
                           dim3(64 * WR), A::kLds, stream, p, plan, unsigned(b0), unsigned(own));
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <class T>
hipError_t launch_both(const Attend &p, const Choice &r, hipStream_t stream) {
    const bool four = r.prefix_waves == 4;
    switch (r.steps) {
        case 2: return four ? launch_both<T, 2, 4>(p, r.plan, stream) : launch_both<T, 2, 2>(p, r.plan, stream);
        case 3: return four ? launch_both<T, 3, 4>(p, r.plan, stream) : launch_both<T, 3, 2>(p, r.plan, stream);
        case 4: return four ? launch_both<T, 4, 4>(p, r.plan, stream) : launch_both<T, 4, 2>(p, r.plan, stream);
        default: return four ? launch_both<T, 8, 4>(p, r.plan, stream) : launch_both<T, 8, 2>(p, r.plan, stream);
    }
}

template <class T>
hipError_t launch_tile(const Attend &p, const Choice &r, int tiles, int waves, int64_t w0, int64_t w1,
                       hipStream_t stream) {
    switch (r.steps) {
        case 2: return launch_tile<T, 2>(p, r.plan, tiles, waves, w0, w1, stream);
        case 3: return launch_tile<T, 3>(p, r.plan, tiles, waves, w0, w1, stream);
        case 4: return launch_tile<T, 4>(p, r.plan, tiles, waves, w0, w1, stream);
        default: return launch_tile<T, 8>(p, r.plan, tiles, waves, w0, w1, stream);
    }
}

template <class T>
hipError_t join(const Attend &p, const Choice &r, hipStream_t stream) {
    const ngpu_attend_t &a = p.a;
    if (r.plan.parts == 1) return hipSuccess;
    int lanes = 2;   // threads a row
    while (4 * lanes < p.c.dim) lanes *= 2;
    int groups = 1;   // sets of them, eight parts each
    while (8 * groups < r.plan.prefix.splits + r.plan.own.splits && 2 * groups * lanes <= kJoinThreads) groups *= 2;
    const int64_t rows = a.S * a.T * a.q_heads, per = kJoinThreads / (lanes * groups), kMost = int64_t(1) << 23;
    for (int64_t r0 = 0; r0 < rows; r0 += kMost * per) {
        const int64_t grid = std::min(kMost, (rows - r0 + per - 1) / per);
        hipLaunchKernelGGL((attend_join_kernel<T>), dim3(unsigned(grid)), dim3(kJoinThreads), 0, stream, p, r.plan,
                           rows, lanes, groups, r0);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T>
hipError_t launch(const Attend &p, void *workspace, hipStream_t stream) {
    const ngpu_attend_t &a = p.a;
    const Choice r = choose(p.c, a, static_cast<char *>(workspace));
    if (!r.tiles) return launch_rows<T>(p, stream);
    const int64_t prefix = r.plan.prefix.works(), all = prefix + r.plan.own.works();
    // Both in one launch.  4 x 16 sequences of 6 tokens with 6000 of prefix and 230 of their own, 8 heads of 128:
    // 79 to 84 us, not 88; 2 x 8 of 4 tokens, 4096 and 100: 37, not 40.
    if (prefix > 0 && all > prefix && (r.prefix_waves == r.own_waves || r.own_waves == 1)) {
        const hipError_t e =
            r.prefix_waves == r.own_waves
                ? launch_tile<T>(p, r, std::max(r.prefix_tiles, r.own_tiles), r.own_waves, 0, all, stream)
                : launch_both<T>(p, r, stream);
        return e != hipSuccess ? e : join<T>(p, r, stream);
    }
    if (prefix > 0)
        if (const hipError_t e = launch_tile<T>(p, r, r.prefix_tiles, r.prefix_waves, 0, prefix, stream);
            e != hipSuccess)
            return e;
    if (all > prefix)
        if (const hipError_t e = launch_tile<T>(p, r, r.own_tiles, r.own_waves, prefix, all, stream); e != hipSuccess)
            return e;
    return join<T>(p, r, stream);
}

}  // namespace

size_t attend_workspace(const ngpu_kv_cache_t &c, const ngpu_attend_t &a) {
    const Choice r = choose(c, a, nullptr);
    return r.tiles && r.plan.parts > 1 ? size_t(r.plan.parts) * size_t(a.S * a.T * a.q_heads) * (size_t(c.dim) * 4 + 8) : 0;
}

hipError_t launch_attend(const ngpu_kv_cache_t &c, const ngpu_attend_t &a, void *workspace, hipStream_t stream) {
    const Attend p{c, a};
    return c.dtype == NGPU_F16 ? launch<F16>(p, workspace, stream) : launch<Bf16>(p, workspace, stream);
}

}  // namespace ngpu
