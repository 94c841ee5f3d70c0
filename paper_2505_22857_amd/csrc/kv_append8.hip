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
// element (the second pass finds the tokens in the caches), and for a few
// tokens by the launch.
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

// N elements from dimension d on of a head's row, rotated by the row `position` of the tables: N is 8, where everything
// comes in eights, or 1.
template <class T, int N>
__device__ __forceinline__ void turned(const ngpu_kv_append_t &a, const T *row, int d, bool known, const float *cos,
                                       const float *sin, float (&x)[N]) {
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const int half = a.rotary / 2;
    auto load = [&](int at, float (&y)[N]) {
        if constexpr (N == 8) {
            const s16x8 v = *reinterpret_cast<const s16x8 *>(row + at);
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = to_float(T{uint16_t(v[i])});
        } else {
            y[0] = to_float(row[at]);
        }
    };
    load(d, x);
    if (d >= a.rotary) return;
    if (!known) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __builtin_nanf("");
        return;
    }
    if (a.layout == NGPU_ROPE_HALF) {
        const bool second = d >= half;
        const int at = second ? d - half : d;
        float y[N];
        load(second ? at : d + half, y);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float c = cos[at + i], z = sin[at + i];
            x[i] = second ? x[i] * c + y[i] * z : x[i] * c - y[i] * z;
        }
    } else if constexpr (N == 8) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float c = cos[(d + i) / 2], z = sin[(d + i) / 2], f = x[i], g = x[i + 1];
            x[i] = f * c - g * z;
            x[i + 1] = g * c + f * z;
        }
    } else {
        const float other = to_float(row[d ^ 1]), c = cos[d / 2], z = sin[d / 2];
        x[0] = d & 1 ? x[0] * c + other * z : x[0] * c - other * z;
    }
}

template <int N>
__device__ __forceinline__ void store8(uint8_t *to, const float (&x)[N]) {
    if constexpr (N == 8) {
        const int2 w = make_int2(pack8(x[0], x[1], x[2], x[3]), pack8(x[4], x[5], x[6], x[7]));
        *reinterpret_cast<int2 *>(to) = w;
    } else {
        *to = uint8_t(pack8(x[0], 0.0f, 0.0f, 0.0f));
    }
}

// The new tokens of one block and head, for the whole wavefront.
template <class T, int N>
__device__ __forceinline__ void append_block(const Append8 &p, int64_t unit) {
    const ngpu_kv_append_t &a = p.a;
    const ngpu_kv_cache_t &c = p.c.cache;
    const int lane = threadIdx.x % kWave, D = c.dim, pieces = D / N, block = p.c.block;
    const bool values = unit % 2 != 0;
    const int h = int(unit / 2 % c.heads);
    const int64_t sb = unit / 2 / c.heads, s = sb / p.blocks;
    // places of the sequence's new tokens, and those of this block
    const int64_t start = a.start[s], n = a.lengths ? min(max(int64_t(a.lengths[s]), int64_t(0)), a.T) : a.T;
    const int64_t first = max(start, int64_t(0)), end = min(start + n, a.pages_width * c.page_size);
    const int64_t b = first / block + sb % p.blocks, lo = max(first, b * block), hi = min(end, (b + 1) * block);
    if (lo >= hi) return;
    const int64_t at_page = b * block / c.page_size;
    const int64_t page = a.pages[s * a.pages_stride + at_page];
    if (page < 0 || page >= c.num_pages) return;
    const int64_t entry = b * block - at_page * c.page_size;   // of the block's first token
    uint8_t *const to = static_cast<uint8_t *>(values ? c.v : c.k) +
                        (values ? page * c.v_stride_page + entry * c.v_stride_token + h * c.v_stride_head
                                : page * c.k_stride_page + entry * c.k_stride_token + h * c.k_stride_head);
    const int64_t to_token = values ? c.v_stride_token : c.k_stride_token;
    float *const scale = (values ? p.c.v_scale : p.c.k_scale) +
                         (values ? page * p.c.v_scale_stride_page + entry / block * p.c.v_scale_stride_block + h * p.c.v_scale_stride_head
                                 : page * p.c.k_scale_stride_page + entry / block * p.c.k_scale_stride_block + h * p.c.k_scale_stride_head);
    const int64_t from_token = values ? a.v_stride_token : a.k_stride_token;
    const T *const from = static_cast<const T *>(values ? a.v : a.k) +
                          (values ? s * a.v_stride_seq + h * a.v_stride_head : s * a.k_stride_seq + h * a.k_stride_head) +
                          (lo - start) * from_token;
    const int lead = int(lo - b * block), items = int(hi - lo) * pieces;
    auto element = [&](int i, float (&x)[N]) {   // item i: N dimensions of a token
        const int t = i / pieces, d = (i - t * pieces) * N;
        if (values || a.rotary == 0) {
            ngpu_kv_append_t plain = a;
            plain.rotary = 0;
            turned<T, N>(plain, from + t * from_token, d, true, nullptr, nullptr, x);
        } else {
            const int64_t place = lo + t, position = a.positions ? int64_t(a.positions[s * a.T + place - start]) : place;
            const bool known = position >= 0 && position < a.positions_count;
            turned<T, N>(a, from + t * from_token, d, known, a.cos + position * (a.rotary / 2),
                         a.sin + position * (a.rotary / 2), x);
        }
    };
    float most = 0.0f;
    for (int i = lane; i < items; i += kWave) {
        float x[N];
        element(i, x);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float y = __builtin_fabsf(x[e]);
            most = y < __builtin_inff() && y > most ? y : most;
        }
    }
    most = wave_max(most);
    float now = least_scale(most);
    if (lead > 0) {
        const float had = *scale, old = had >= 0x1p-100f && had < __builtin_inff() ? had : 0x1p-100f;
        if (most > kMost8 * old) {   // it grows: the entries before, again
            const float ratio = old / now;
            for (int i = lane; i < lead * pieces; i += kWave) {
                const int t = i / pieces, d = (i - t * pieces) * N;
                uint8_t *const at = to + t * to_token + d;
                float x[N];
                if constexpr (N == 8) {
                    const int2 w = *reinterpret_cast<const int2 *>(at);
                    const float2 y[4] = {to_floats8<false>(w.x), to_floats8<true>(w.x), to_floats8<false>(w.y),
                                         to_floats8<true>(w.y)};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[2 * e] = y[e].x * ratio;
                        x[2 * e + 1] = y[e].y * ratio;
                    }
                } else {
                    x[0] = to_float(E4m3{*at}) * ratio;
                }
                store8<N>(at, x);
            }
        } else {
            now = old;
        }
    }
    const float by = 1.0f / now;
    for (int i = lane; i < items; i += kWave) {
        float x[N];
        element(i, x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = __builtin_fabsf(x[e]) < __builtin_inff() ? x[e] * by : __builtin_nanf("");
        const int t = i / pieces;
        store8<N>(to + (lead + t) * to_token + (i - t * pieces) * N, x);
    }
    if (lane == 0) *scale = now;
}

// The queries of 256 >> bits tokens, N dimensions at a time.
template <class T, int N>
__device__ __forceinline__ void turn_queries(const Append8 &p, int64_t group) {
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const ngpu_kv_append_t &a = p.a;
    const int64_t n = (group * kAppendThreads + threadIdx.x) >> p.bits;
    if (n >= a.S * a.T) return;
    const int threads = 1 << p.bits, thread = threadIdx.x & (threads - 1);
    const int D = p.c.cache.dim, pieces = D / N;
    const int64_t s = n / a.T, t = n % a.T;
    T *const to = static_cast<T *>(a.q_out) + n * a.q_heads * D;
    const bool counts = !a.lengths || t < a.lengths[s];
    const int64_t position = a.rotary == 0 ? 0 : (a.positions ? int64_t(a.positions[n]) : int64_t(a.start[s]) + t);
    const bool known = position >= 0 && position < a.positions_count;
    const float *const cos = a.cos + position * (a.rotary / 2), *const sin = a.sin + position * (a.rotary / 2);
    const T *const from = static_cast<const T *>(a.q) + s * a.q_stride_seq + t * a.q_stride_token;
    for (int i = thread; i < a.q_heads * pieces; i += threads) {
        const int h = i / pieces, d = (i - h * pieces) * N;
        float x[N] = {};
        if (counts) turned<T, N>(a, from + h * a.q_stride_head, d, known, cos, sin, x);
        if constexpr (N == 8) {
            s16x8 y;
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = short(from_float<T>(x[e]).bits);
            *reinterpret_cast<s16x8 *>(to + i * N) = y;
        } else {
            to[i] = from_float<T>(x[0]);
        }
    }
}

template <class T, int N>
__global__ __launch_bounds__(kAppendThreads) void append8_kernel(Append8 p, int64_t g0, int64_t block_groups) {
    const int64_t group = g0 + blockIdx.x;
    if (group >= block_groups) {
        turn_queries<T, N>(p, group - block_groups);
        return;
    }
    const int64_t unit = group * kAppendWaves + __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
    if (unit < p.a.S * p.blocks * p.c.cache.heads * 2) append_block<T, N>(p, unit);
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
           aligned(a.k, 16) && aligned(a.v, 16) && aligned(a.q, 16) && aligned(a.q_out, 16);
}

template <class T, int N>
static hipError_t launch(Append8 p, hipStream_t stream) {
    constexpr int64_t kMost = int64_t(1) << 23;
    const ngpu_kv_append_t &a = p.a;
    const int64_t units = a.S * p.blocks * p.c.cache.heads * 2, block_groups = (units + kAppendWaves - 1) / kAppendWaves;
    const int64_t items = a.q ? int64_t(a.q_heads) * (p.c.cache.dim / N) : 0;
    p.bits = 4;
    while (p.bits < 8 && (int64_t(1) << p.bits) < items) ++p.bits;
    const int64_t per = kAppendThreads >> p.bits, all = block_groups + (a.q ? (a.S * a.T + per - 1) / per : 0);
    for (int64_t g0 = 0; g0 < all; g0 += kMost) {
        hipLaunchKernelGGL((append8_kernel<T, N>), dim3(unsigned(std::min(kMost, all - g0))), dim3(kAppendThreads), 0, stream,
                           p, g0, block_groups);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_kv_append8(const ngpu_kv_cache8_t &c, const ngpu_kv_append_t &a, hipStream_t stream) {
    const Append8 p{c, a, (a.T + c.block - 2) / c.block + 1, 0};
    const bool half = c.cache.dtype == NGPU_F16;
    if (in_eights(p)) return half ? launch<F16, 8>(p, stream) : launch<Bf16, 8>(p, stream);
    return half ? launch<F16, 1>(p, stream) : launch<Bf16, 1>(p, stream);
}

}  // namespace ngpu
