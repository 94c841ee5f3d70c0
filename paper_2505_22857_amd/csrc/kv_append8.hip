// Appending keys and values to a paged cache in 8 bits.
//
// A wavefront takes the new tokens of one block for one head, keys or values:
// the largest element gives the block's scale, the least power of two that
// holds it, and the elements (keys rotated, in fp32) are divided by that and
// rounded once to e4m3.  A power of two leaves a value its precision wherever
// the type has all its mantissa bits, in this block and when a later token makes
// the scale grow: then the entries before are read, multiplied by the quotient
// of the scales and rounded again, which changes only what falls below the
// type's normal range.
//
// Bound by memory traffic, one read of 16 bits and one write of 8 for each
// element, and, as every block's wavefront waits for a chain of loads (its sequence's
// place, its page, its tokens), by how many of them run beside the queries'
// streaming: 5 x 3500 tokens of 32 + 8 + 8 heads of 128 take 72 us a call among
// others, 299 MB at 4.1 TB/s, and 79 in a graph of calls on the same tokens, as all
// figures below are; in two launches 85.  A few tokens: the launch, 5.4 us.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.h"
#include "reduce.h"
#include "values8.h"

namespace ngpu {

constexpr int kAppendThreads = 256;
constexpr int kAppendWaves = kAppendThreads / kWave;
struct Append8 {
    ngpu_kv_cache8_t c;
    ngpu_kv_append_t a;
    int64_t blocks;      // most blocks a sequence's tokens touch
    int bits;            // 2^bits threads a token's queries
};

typedef short s16x8 __attribute__((ext_vector_type(8)));

// What an element is rotated with: nothing, its like of the other half, or its neighbour.
enum { kAsIs = 0, kHalves = 1, kPairs = 2 };

// N elements of a head's row from dimension d on, rotated by a row of the tables: N is 8, where everything comes in
// eights, or 1.  Everything is loaded first, without a branch that lanes do not share, so that the loads of several pieces
// are in flight together: what a dimension or a position has no use for is read from the row's or the tables' start.
template <class T, int N, int MODE>
struct Piece {
    static constexpr int kWords = MODE == kAsIs ? 0 : (MODE == kHalves || N == 1 ? N : N / 2);   // angles
    T x[N], y[MODE == kHalves || (MODE == kPairs && N == 1) ? N : 1];
    float c[kWords > 0 ? kWords : 1], z[kWords > 0 ? kWords : 1];
    bool turns, known, second;

    template <int M, class U>
    static __device__ __forceinline__ void fetch(const U *from, U (&to)[M]) {   // M: 16 or 32 bytes of eight, or one
        if constexpr (M == 1) {
            to[0] = from[0];
        } else {
            constexpr int kPer = 16 / int(sizeof(U));
#pragma unroll
            for (int i = 0; i < M / kPer; ++i) {
                const i32x4 v = reinterpret_cast<const i32x4 *>(from)[i];
                __builtin_memcpy(to + i * kPer, &v, 16);
            }
        }
    }
    __device__ __forceinline__ void load(const ngpu_kv_append_t &a, const T *row, int d, int64_t position) {
        fetch(row + d, x);
        if constexpr (MODE != kAsIs) {
            const int half = a.rotary / 2;
            turns = d < a.rotary;
            known = position >= 0 && position < a.positions_count;
            second = MODE == kHalves ? d >= half : N == 1 && d % 2 != 0;
            const int at = MODE == kHalves ? (second ? d - half : d) : d / 2;
            if constexpr (MODE == kHalves || N == 1)
                fetch(row + (!turns ? 0 : MODE == kHalves ? (second ? d - half : d + half) : d ^ 1), y);
            if (a.positions_count > 0) {   // (else there are no tables)
                const int64_t from = (known ? position * half : 0) + (turns ? at : 0);
                fetch(a.cos + from, c);
                fetch(a.sin + from, z);
            }
        }
    }
    // the pair's second element, of a piece that holds the first
    __device__ __forceinline__ void other(float (&out)[N]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float f = to_float(x[i]), g = to_float(y[i]);
            out[i] = known ? g * c[i] + f * z[i] : __builtin_nanf("");
        }
    }
    __device__ __forceinline__ void turn(float (&out)[N]) const {
        if constexpr (MODE == kAsIs) {
#pragma unroll
            for (int i = 0; i < N; ++i) out[i] = to_float(x[i]);
        } else if constexpr (MODE == kHalves || N == 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float f = to_float(x[i]), g = to_float(y[i]), t = second ? f * c[i] + g * z[i] : f * c[i] - g * z[i];
                out[i] = !turns ? f : (known ? t : __builtin_nanf(""));
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const float f = to_float(x[i]), g = to_float(x[i + 1]);
                const float t = f * c[i / 2] - g * z[i / 2], u = g * c[i / 2] + f * z[i / 2];
                out[i] = !turns ? f : (known ? t : __builtin_nanf(""));
                out[i + 1] = !turns ? g : (known ? u : __builtin_nanf(""));
            }
        }
    }
};

template <int N>
__device__ __forceinline__ void store8(uint8_t *to, const float (&x)[N]) {
    if constexpr (N == 8) {
        const int2 w = make_int2(pack8(x[0], x[1], x[2], x[3]), pack8(x[4], x[5], x[6], x[7]));
        *reinterpret_cast<int2 *>(to) = w;
    } else {
        *to = uint8_t(pack8(x[0], 0.0f, 0.0f, 0.0f));
    }
}

// n / d for n, d > 0, by a division of 32 bits where they fit it.
__device__ __forceinline__ int64_t divided64(int64_t n, int64_t d) {
    return ((n | d) >> 32) == 0 ? int64_t(unsigned(n) / unsigned(d)) : n / d;
}

// Where the new tokens of one block and head come from and go to.
template <class T>
struct Block {
    const T *from;          // the first new token's row
    uint8_t *to;            // the block's first entry
    float *scale;
    int64_t from_token, to_token, place, n;   // n: the first new token's place in [S, T]
    int lead, tokens;       // entries before the new ones, new ones: 0 where there is nothing to do
    bool values;

    __device__ __forceinline__ Block(const Append8 &p, int64_t unit) {
        const ngpu_kv_append_t &a = p.a;
        const ngpu_kv_cache_t &c = p.c.cache;
        const int block = p.c.block;
        const int64_t sb = divided64(unit / 2, c.heads), s = divided64(sb, p.blocks);
        const int h = int(unit / 2 - sb * c.heads);
        tokens = 0;
        values = unit % 2 != 0;
        // places of the sequence's new tokens, and those of this block
        const int64_t start = a.start[s], count = a.lengths ? min(max(int64_t(a.lengths[s]), int64_t(0)), a.T) : a.T;
        const int64_t first = max(start, int64_t(0)), end = min(start + count, a.pages_width * c.page_size);
        const int64_t b = divided64(first, block) + (sb - s * p.blocks), lo = max(first, b * block), hi = min(end, (b + 1) * block);
        if (lo >= hi) return;
        const int64_t at_page = divided64(b * block, c.page_size);
        const int64_t page = a.pages[s * a.pages_stride + at_page];
        if (page < 0 || page >= c.num_pages) return;
        const int64_t entry = b * block - at_page * c.page_size;   // of the block's first token
        const int64_t which = divided64(entry, block);
        if (values) {
            to = static_cast<uint8_t *>(c.v) + page * c.v_stride_page + entry * c.v_stride_token + h * c.v_stride_head;
            scale = p.c.v_scale + page * p.c.v_scale_stride_page + which * p.c.v_scale_stride_block + h * p.c.v_scale_stride_head;
            from = static_cast<const T *>(a.v) + s * a.v_stride_seq + (lo - start) * a.v_stride_token + h * a.v_stride_head;
            to_token = c.v_stride_token;
            from_token = a.v_stride_token;
        } else {
            to = static_cast<uint8_t *>(c.k) + page * c.k_stride_page + entry * c.k_stride_token + h * c.k_stride_head;
            scale = p.c.k_scale + page * p.c.k_scale_stride_page + which * p.c.k_scale_stride_block + h * p.c.k_scale_stride_head;
            from = static_cast<const T *>(a.k) + s * a.k_stride_seq + (lo - start) * a.k_stride_token + h * a.k_stride_head;
            to_token = c.k_stride_token;
            from_token = a.k_stride_token;
        }
        place = lo;
        n = s * a.T + lo - start;
        lead = int(lo - b * block);
        tokens = int(hi - lo);
    }
};

// The new tokens of a block and head, for WAVES wavefronts.  A lane's items are every kLanes-th: N dimensions of a token each.
template <class T, int N, int MODE, int WAVES, int HELD>
__device__ __forceinline__ void append_block(const Append8 &p, const Block<T> &b) {
    constexpr int kLanes = WAVES * kWave;
    const ngpu_kv_append_t &a = p.a;
    const int lane = threadIdx.x % kLanes, D = p.c.cache.dim, pieces = D / N, items = b.tokens * pieces;
    const int step_t = kLanes / pieces, step_d = kLanes % pieces * N;
    int t = lane / pieces, d = lane % pieces * N;   // of the lane's item
    auto restart = [&]() {
        t = lane / pieces;
        d = lane % pieces * N;
    };
    auto advance = [&]() {
        t += step_t;
        d += step_d;
        if (d >= D) {
            d -= D;
            ++t;
        }
    };
    auto load = [&](Piece<T, N, MODE> &piece) {   // behind the last one: of the last token, for nothing
        const int token = min(t, b.tokens - 1);
        const int64_t position = MODE == kAsIs || !a.positions ? b.place + token : int64_t(a.positions[b.n + token]);
        piece.load(a, b.from + token * b.from_token, d, position);
    };
    // Up to HELD a lane stay in registers, loaded a few at once; those of larger blocks are read again.
    constexpr int kHeld = HELD, kBatch = HELD > 4 && MODE != kHalves ? 4 : (HELD > 2 ? 2 : HELD);
    const bool held = items <= kHeld * kLanes;
    float most = 0.0f, x[kHeld][N];
    auto larger = [&](const float (&y)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float z = __builtin_fabsf(y[e]);
            most = z < __builtin_inff() && z > most ? z : most;
        }
    };
    if (held) {
#pragma unroll
        for (int u = 0; u < kHeld; u += kBatch) {
            if (kLanes * u < items) {
                Piece<T, N, MODE> piece[kBatch];
#pragma unroll
                for (int e = 0; e < kBatch; ++e) {
                    load(piece[e]);
                    advance();
                }
#pragma unroll
                for (int e = 0; e < kBatch; ++e) {
                    piece[e].turn(x[u + e]);
                    if (lane + kLanes * (u + e) < items) larger(x[u + e]);
                }
            }
        }
    } else {
        for (int i = lane; i < items; i += kLanes) {
            Piece<T, N, MODE> piece;
            load(piece);
            advance();
            piece.turn(x[0]);
            larger(x[0]);
        }
    }
    most = wave_max(most);
    if constexpr (WAVES > 1) {
        __shared__ float all[WAVES];
        if (threadIdx.x % kWave == 0) all[threadIdx.x / kWave] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = __builtin_fmaxf(most, all[w]);
    }
    float now = least_scale(most);
    if (b.lead > 0) {
        // (no number above 0 is none: 2^-100; one below that is raised to it, so that its inverse is finite)
        const float had = *b.scale, old = had > 0.0f && had < __builtin_inff() ? had : 0x1p-100f;
        if (most > kMost8 * old || old < 0x1p-100f) {   // it grows: the entries before, again
            const float ratio = old / now;
            for (int i = lane; i < b.lead * pieces; i += kLanes) {
                const int token = i / pieces, from = (i - token * pieces) * N;
                uint8_t *const at = b.to + token * b.to_token + from;
                float y[N];
                if constexpr (N == 8) {
                    const int2 w = *reinterpret_cast<const int2 *>(at);
                    const float2 v[4] = {to_floats8<false>(w.x), to_floats8<true>(w.x), to_floats8<false>(w.y),
                                         to_floats8<true>(w.y)};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y[2 * e] = v[e].x * ratio;
                        y[2 * e + 1] = v[e].y * ratio;
                    }
                } else {
                    y[0] = to_float(E4m3{*at}) * ratio;
                }
                store8<N>(at, y);
            }
        } else {
            now = old;
        }
    }
    const float by = 1.0f / now;
    auto put = [&](float (&y)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = __builtin_fabsf(y[e]) < __builtin_inff() ? y[e] * by : __builtin_nanf("");
        store8<N>(b.to + (b.lead + t) * b.to_token + d, y);
    };
    restart();
    if (held) {
#pragma unroll
        for (int u = 0; u < kHeld; ++u) {
            if (lane + kLanes * u < items) put(x[u]);
            advance();
        }
    } else {
        for (int i = lane; i < items; i += kLanes) {
            Piece<T, N, MODE> piece;
            load(piece);
            piece.turn(x[0]);
            put(x[0]);
            advance();
        }
    }
    if (WAVES > 1 && b.lead > 0) __syncthreads();   // all have read the scale that there was
    if (lane == 0) *b.scale = now;
}

// The queries of 256 >> bits tokens.  Of halves a lane takes both elements of its pairs, else N dimensions at a time; a
// few such items are loaded at once.
template <class T, int N, int MODE>
__device__ __forceinline__ void turn_queries(const Append8 &p, int64_t group) {
    const ngpu_kv_append_t &a = p.a;
    const int64_t n = (group * kAppendThreads + threadIdx.x) >> p.bits;
    if (n >= a.S * a.T) return;
    const int threads = 1 << p.bits, thread = threadIdx.x & (threads - 1);
    const int D = p.c.cache.dim, half = a.rotary / 2, pairs = MODE == kHalves ? half / N : 0, each = D / N - pairs;
    const int64_t s = divided64(n, a.T), t = n - s * a.T;
    T *const to = static_cast<T *>(a.q_out) + n * a.q_heads * D;
    const bool counts = !a.lengths || t < a.lengths[s];
    const int64_t position = a.rotary > 0 && a.positions ? int64_t(a.positions[n]) : int64_t(a.start[s]) + t;
    // a token that does not count reads the sequence's first, for nothing (5 x 3500, a quarter of which do
    // not: 79 us, 80.5 with its own)
    const T *const from = static_cast<const T *>(a.q) + s * a.q_stride_seq + (counts ? t : 0) * a.q_stride_token;
    const int items = a.q_heads * each;
    constexpr int kBatch = N == 1 ? 1 : (MODE == kHalves ? 2 : 4);
    auto put = [&](int at, const float (&x)[N]) {
        T y[N];
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = from_float<T>(counts ? x[e] : 0.0f);
        if constexpr (N == 8)
            *reinterpret_cast<i32x4 *>(to + at) = __builtin_bit_cast(i32x4, y);
        else
            to[at] = y[0];
    };
    for (int i0 = thread; i0 < items; i0 += kBatch * threads) {
        Piece<T, N, MODE> piece[kBatch];
        int head[kBatch], d[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {   // behind the last one: the last, for nothing
            const int i = min(i0 + u * threads, items - 1), in = i - i / each * each;
            head[u] = i / each;
            d[u] = (in < pairs || MODE != kHalves ? in : in + pairs) * N;
            piece[u].load(a, from + head[u] * a.q_stride_head, d[u], position);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i0 + u * threads >= items) break;
            float x[N];
            piece[u].turn(x);
            put(head[u] * D + d[u], x);
            if (MODE == kHalves && piece[u].turns) {
                piece[u].other(x);
                put(head[u] * D + d[u] + half, x);
            }
        }
    }
}

template <class T, int N, int MODE, int WAVES, int HELD>
__global__ __launch_bounds__(kAppendThreads) void append8_kernel(Append8 p, int64_t g0, int64_t block_groups,
                                                                int64_t all_groups) {
    // The blocks' workgroups wait for their loads, one after the other: they are dealt evenly among the queries' (of fewer
    // than 2^31 workgroups: the products fit 64 bits).
    const int64_t at = g0 + blockIdx.x;
    const bool deal = all_groups >> 31 == 0;
    const int64_t group = deal ? divided64(at * block_groups, all_groups) : min(at, block_groups);
    if ((deal ? divided64((at + 1) * block_groups, all_groups) : min(at + 1, block_groups)) == group) {
        turn_queries<T, N, MODE>(p, at - group);
        return;
    }
    constexpr int kUnits = kAppendWaves / WAVES;   // of the workgroup
    const int64_t unit = group * kUnits + (kUnits == 1 ? 0 : __builtin_amdgcn_readfirstlane(int(threadIdx.x) / (WAVES * kWave)));
    if (unit >= p.a.S * p.blocks * p.c.cache.heads * 2) return;
    const Block<T> b(p, unit);
    if (b.tokens == 0) return;
    if (MODE == kAsIs || b.values)
        append_block<T, N, kAsIs, WAVES, HELD>(p, b);
    else
        append_block<T, N, MODE, WAVES, HELD>(p, b);
}

// Whether eight elements can be moved at a time everywhere.
static bool in_eights(const Append8 &p) {
    const ngpu_kv_cache_t &c = p.c.cache;
    const ngpu_kv_append_t &a = p.a;
    auto aligned = [](const void *x, unsigned to) { return reinterpret_cast<uintptr_t>(x) % to == 0; };
    const int64_t strides[] = {c.k_stride_page, c.k_stride_token, c.k_stride_head, c.v_stride_page, c.v_stride_token,
                               c.v_stride_head, a.k_stride_seq, a.k_stride_token, a.k_stride_head, a.v_stride_seq,
                               a.v_stride_token, a.v_stride_head, a.q ? a.q_stride_seq : 0,
                               a.q ? a.q_stride_token : 0, a.q ? a.q_stride_head : 0};
    for (const int64_t s : strides)
        if (s % 8 != 0) return false;
    return c.dim % 8 == 0 && a.rotary % (a.layout == NGPU_ROPE_HALF ? 16 : 8) == 0 && aligned(c.k, 8) && aligned(c.v, 8) &&
           aligned(a.k, 16) && aligned(a.v, 16) && aligned(a.q, 16) && aligned(a.q_out, 16) &&
           (a.rotary == 0 || (aligned(a.cos, 16) && aligned(a.sin, 16)));
}

template <class T, int N, int WAVES, int HELD>
static hipError_t launch(Append8 p, hipStream_t stream) {
    constexpr int64_t kMost = int64_t(1) << 23;
    const ngpu_kv_append_t &a = p.a;
    const int64_t units = a.S * p.blocks * p.c.cache.heads * 2, per_group = kAppendWaves / WAVES;
    const int64_t block_groups = (units + per_group - 1) / per_group;
    const bool halves = a.layout == NGPU_ROPE_HALF;
    const int64_t items = a.q ? int64_t(a.q_heads) * (p.c.cache.dim / N - (halves ? a.rotary / 2 / N : 0)) : 0;
    // Threads a token's queries: one for each item where these are few, else one for eight, or four pairs.  us: 5 x 3500 tokens of
    // 32 + 8 heads of 128, pairs 79, four 86, two 108, one 108; 4 x 2000 of 8 + 4 of 80, halves 14.0, two 16.5, one 19.3.
    const int64_t passes = a.S * a.T * items >= int64_t(1) << 18 ? (halves ? 4 : 8) : 1;
    p.bits = 4;
    while (p.bits < 8 && (passes << p.bits) < items) ++p.bits;
    const int64_t per = kAppendThreads >> p.bits, all = block_groups + (items > 0 ? (a.S * a.T + per - 1) / per : 0);
    const auto kernel = a.rotary == 0 ? &append8_kernel<T, N, kAsIs, WAVES, HELD>
                                      : (halves ? &append8_kernel<T, N, kHalves, WAVES, HELD>
                                                : &append8_kernel<T, N, kPairs, WAVES, HELD>);
    for (int64_t g0 = 0; g0 < all; g0 += kMost) {
        hipLaunchKernelGGL(kernel, dim3(unsigned(std::min(kMost, all - g0))), dim3(kAppendThreads), 0, stream, p, g0,
                           block_groups, all);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Four wavefronts a block where one would have more than eight items a lane (23 x 2000 tokens of 1 head of 128 in blocks of
// 128: 31.5 us, not 74.5; with four from two items a lane on, 5 x 3500 takes 94, not 79); fewer registers where it has two
// (16 x 2000 of 4 heads of 64 in blocks of 16: 46 us, not 50).
template <class T>
static hipError_t launch(const Append8 &p, hipStream_t stream) {
    const int N = in_eights(p) ? 8 : 1;
    const int64_t items = std::min<int64_t>(p.c.block, p.a.T) * (p.c.cache.dim / N);
    if (N == 1) return items > 8 * kWave ? launch<T, 1, 4, 1>(p, stream) : launch<T, 1, 1, 1>(p, stream);
    if (items <= 2 * kWave) return launch<T, 8, 1, 2>(p, stream);
    return items > 8 * kWave ? launch<T, 8, 4, 8>(p, stream) : launch<T, 8, 1, 8>(p, stream);
}

hipError_t launch_kv_append8(const ngpu_kv_cache8_t &c, const ngpu_kv_append_t &a, hipStream_t stream) {
    const Append8 p{c, a, (a.T + c.block - 2) / c.block + 1, 0};
    return c.cache.dtype == NGPU_F16 ? launch<F16>(p, stream) : launch<Bf16>(p, stream);
}

}  // namespace ngpu
