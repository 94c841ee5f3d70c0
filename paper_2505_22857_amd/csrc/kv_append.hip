// Appending keys and values to a paged cache, with the position rotation of
// keys and queries applied on the way.
//
// A rotated head turns pairs (a, b) of its first R dimensions by the angle of
// its token's position: (a cos - b sin, b cos + a sin), in fp32, rounded once to
// the cache's type; the other dimensions and the values are copied.  Every
// element is read and written once, so the bound is memory traffic, and for a
// few tokens the launch: one token of 8 heads of 64 5.3 us, 4 x 4001 of 32 + 8 + 8
// heads of 128 65 to 72 us, 298 MB at 4.2 to 4.6 TB/s where a large copy reaches 5.0.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.h"
#include "walk.h"

namespace ngpu {

constexpr int kAppendThreads = 256;

struct Append {
    ngpu_kv_cache_t c;
    ngpu_kv_append_t a;
};

// Where a new token goes: its page's number, -1 where it is not stored.
__device__ __forceinline__ int64_t page_of(const Append &p, int64_t s, int64_t place) {
    const int64_t at = place / p.c.page_size;
    if (place < 0 || at >= p.a.pages_width) return -1;
    const int64_t page = p.a.pages[s * p.a.pages_stride + at];
    return page >= 0 && page < p.c.num_pages ? page : -1;
}

// Any dimension, stride and alignment: one workgroup per token; each thread writes
// one element at a time (4 x 4001 tokens as above: 205 us, 16 bytes at a time 68).
template <class T>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(Append p, int64_t n0) {
    const ngpu_kv_append_t &a = p.a;
    const int64_t n = n0 + blockIdx.x, s = n / a.T, t = n % a.T;
    const int D = p.c.dim, half = a.rotary / 2, H = p.c.heads, Hq = a.q ? a.q_heads : 0;
    const bool counts = !a.lengths || t < a.lengths[s];
    T *q_out = static_cast<T *>(a.q_out) + n * Hq * D;
    if (!counts) {
        for (int i = threadIdx.x; i < Hq * D; i += kAppendThreads) q_out[i] = T{};
        return;
    }
    const int64_t place = int64_t(a.start[s]) + t, page = page_of(p, s, place);
    const int64_t slot = page >= 0 ? place % p.c.page_size : 0;
    const int64_t position = a.rotary == 0 ? 0 : (a.positions ? int64_t(a.positions[n]) : place);
    const bool known = position >= 0 && position < a.positions_count;
    const float *cos = a.cos + position * half, *sin = a.sin + position * half;
    auto turned = [&](const T *x, int d) {   // element d of the rotated head x
        if (d >= a.rotary) return x[d];
        const bool halves = a.layout == NGPU_ROPE_HALF;
        const bool second = halves ? d >= half : (d & 1) != 0;
        const int i = halves ? (second ? d - half : d) : d / 2;
        if (!known) return from_float<T>(__builtin_nanf(""));
        const float own = to_float(x[d]), other = to_float(x[halves ? (second ? i : i + half) : (d ^ 1)]);
        return from_float<T>(second ? own * cos[i] + other * sin[i] : own * cos[i] - other * sin[i]);
    };
    for (int e = threadIdx.x; e < (Hq + 2 * H) * D; e += kAppendThreads) {
        const int head = e / D, d = e % D;
        if (head < Hq) {
            const T *x = static_cast<const T *>(a.q) + s * a.q_stride_seq + t * a.q_stride_token +
                         head * a.q_stride_head;
            q_out[head * D + d] = turned(x, d);
        } else if (page < 0) {
            break;
        } else if (head < Hq + H) {
            const int h = head - Hq;
            const T *x = static_cast<const T *>(a.k) + s * a.k_stride_seq + t * a.k_stride_token + h * a.k_stride_head;
            static_cast<T *>(p.c.k)[page * p.c.k_stride_page + slot * p.c.k_stride_token + h * p.c.k_stride_head + d] =
                turned(x, d);
        } else {
            const int h = head - Hq - H;
            const T *x = static_cast<const T *>(a.v) + s * a.v_stride_seq + t * a.v_stride_token + h * a.v_stride_head;
            static_cast<T *>(p.c.v)[page * p.c.v_stride_page + slot * p.c.v_stride_token + h * p.c.v_stride_head + d] =
                x[d];
        }
    }
}

// Dimensions in eights and everything 16-byte aligned: 2^bits threads per token,
// 16 bytes at a time.  An item is 8 dimensions of a head, or with halves the 8
// that it pairs with too.
template <class T, bool HALVES>
__global__ __launch_bounds__(kAppendThreads) void append_vector_kernel(Append p, int64_t n0, int bits) {
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const ngpu_kv_append_t &a = p.a;
    const int64_t n = n0 + ((int64_t(blockIdx.x) * kAppendThreads + threadIdx.x) >> bits);
    if (n >= a.S * a.T) return;
    const unsigned threads = 1u << bits, thread = threadIdx.x & (threads - 1);
    const int64_t s = n / a.T, t = n % a.T;
    const int H = p.c.heads, Hq = a.q ? a.q_heads : 0, half = a.rotary / 2;
    const unsigned pieces = unsigned(p.c.dim) / 8, turned = HALVES ? unsigned(half) / 8 : unsigned(a.rotary) / 8;
    const unsigned items = HALVES ? pieces - turned : pieces;   // of a rotated head
    const unsigned first_v = unsigned(Hq + H) * items, all = first_v + unsigned(H) * pieces;
    T *q_out = static_cast<T *>(a.q_out) + n * Hq * p.c.dim;
    if (a.lengths && t >= a.lengths[s]) {
        for (unsigned e = thread; e < unsigned(Hq) * pieces; e += threads)
            *reinterpret_cast<s16x8 *>(q_out + e * 8) = s16x8{};
        return;
    }
    const int64_t place = int64_t(a.start[s]) + t, page = page_of(p, s, place);
    const int64_t slot = page >= 0 ? place % p.c.page_size : 0;
    const int64_t position = a.rotary == 0 ? 0 : (a.positions ? int64_t(a.positions[n]) : place);
    const bool known = position >= 0 && position < a.positions_count;
    const float *cos = a.cos + position * half, *sin = a.sin + position * half;
    T *const k_to = static_cast<T *>(p.c.k) + page * p.c.k_stride_page + slot * p.c.k_stride_token;
    T *const v_to = static_cast<T *>(p.c.v) + page * p.c.v_stride_page + slot * p.c.v_stride_token;
    const T *const q_from = static_cast<const T *>(a.q) + s * a.q_stride_seq + t * a.q_stride_token;
    const T *const k_from = static_cast<const T *>(a.k) + s * a.k_stride_seq + t * a.k_stride_token;
    const T *const v_from = static_cast<const T *>(a.v) + s * a.v_stride_seq + t * a.v_stride_token;
    auto angle = [&](const float *table, int i) {
        return known ? *reinterpret_cast<const f32x4 *>(table + i) : f32x4{} + __builtin_nanf("");
    };
    for (unsigned e = thread; e < all; e += threads) {
        if (e >= first_v) {
            if (page < 0) break;
            const unsigned h = (e - first_v) / pieces, d = (e - first_v) % pieces * 8;
            *reinterpret_cast<s16x8 *>(v_to + h * p.c.v_stride_head + d) =
                *reinterpret_cast<const s16x8 *>(v_from + h * a.v_stride_head + d);
            continue;
        }
        const unsigned head = e / items, i = e % items;
        const bool query = head < unsigned(Hq);
        if (!query && page < 0) continue;
        const T *from = query ? q_from + head * a.q_stride_head : k_from + (head - Hq) * a.k_stride_head;
        T *to = query ? q_out + head * p.c.dim : k_to + (head - Hq) * p.c.k_stride_head;
        if (HALVES) {
            const unsigned d = i < turned ? i * 8 : (i + turned) * 8;
            s16x8 x = *reinterpret_cast<const s16x8 *>(from + d);
            if (i < turned) {
                s16x8 y = *reinterpret_cast<const s16x8 *>(from + half + d);
#pragma unroll
                for (int u = 0; u < 8; u += 4) {
                    const f32x4 c = angle(cos, d + u), z = angle(sin, d + u);
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float f = to_float(T{uint16_t(x[u + v])}), g = to_float(T{uint16_t(y[u + v])});
                        x[u + v] = short(from_float<T>(f * c[v] - g * z[v]).bits);
                        y[u + v] = short(from_float<T>(g * c[v] + f * z[v]).bits);
                    }
                }
                *reinterpret_cast<s16x8 *>(to + half + d) = y;
            }
            *reinterpret_cast<s16x8 *>(to + d) = x;
        } else {
            s16x8 x = *reinterpret_cast<const s16x8 *>(from + i * 8);
            if (i < turned) {
                const f32x4 c = angle(cos, i * 4), z = angle(sin, i * 4);
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float f = to_float(T{uint16_t(x[2 * v])}), g = to_float(T{uint16_t(x[2 * v + 1])});
                    x[2 * v] = short(from_float<T>(f * c[v] - g * z[v]).bits);
                    x[2 * v + 1] = short(from_float<T>(g * c[v] + f * z[v]).bits);
                }
            }
            *reinterpret_cast<s16x8 *>(to + i * 8) = x;
        }
    }
}

// Whether 16 bytes of 8 elements can be moved everywhere.
static bool in_eights(const Append &p) {
    const ngpu_kv_cache_t &c = p.c;
    const ngpu_kv_append_t &a = p.a;
    auto aligned = [](const void *x) { return reinterpret_cast<uintptr_t>(x) % 16 == 0; };
    const int64_t strides[] = {c.k_stride_page, c.k_stride_token, c.k_stride_head, c.v_stride_page, c.v_stride_token,
                               c.v_stride_head, a.k_stride_seq, a.k_stride_token, a.k_stride_head, a.v_stride_seq,
                               a.v_stride_token, a.v_stride_head, a.q ? a.q_stride_seq : 0,
                               a.q ? a.q_stride_token : 0, a.q ? a.q_stride_head : 0};
    for (const int64_t s : strides)
        if (s % 8 != 0) return false;
    return c.dim % 8 == 0 && a.rotary % (a.layout == NGPU_ROPE_HALF ? 16 : 8) == 0 && aligned(c.k) && aligned(c.v) &&
           aligned(a.k) && aligned(a.v) && aligned(a.q) && aligned(a.q_out) &&
           (a.rotary == 0 || (aligned(a.cos) && aligned(a.sin)));
}

template <class T>
static hipError_t launch(const Append &p, hipStream_t stream) {
    // a grid holds at most 2^32 - 1 work-items
    constexpr int64_t kMost = int64_t(UINT32_MAX) / kAppendThreads;
    const int64_t n = p.a.S * p.a.T;
    if (!in_eights(p)) {
        for (int64_t n0 = 0; n0 < n; n0 += kMost) {
            hipLaunchKernelGGL(append_kernel<T>, dim3(unsigned(std::min(kMost, n - n0))), dim3(kAppendThreads), 0, stream,
                               p, n0);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    const bool halves = p.a.layout == NGPU_ROPE_HALF;
    const int64_t pieces = p.c.dim / 8, items = halves ? pieces - p.a.rotary / 16 : pieces;
    const int64_t all = ((p.a.q ? p.a.q_heads : 0) + p.c.heads) * items + p.c.heads * pieces;
    // Threads a token: one for each item where these are few, else one for four, whose loads are in flight together.  us: 23 x
    // 2554 tokens of 3 + 1 + 1 heads of 128 41, with an item a thread 66, with eight 37, with 256 threads a token
    // 104; 16 x 2000 of 16 + 4 + 4 of 64 39, 67, 35, 74; 3 x 2710 of 4 + 2 + 2 of 96 8.5, 11.3, 9.6, 16.5; 600 of 8 + 1 + 1 of
    // 64 3.7 with an item, 5.5 with four.
    const int64_t passes = n * all >= int64_t(1) << 18 ? 4 : 1;
    int bits = 4;
    while (bits < 8 && (passes << bits) < all) ++bits;
    const auto kernel = halves ? &append_vector_kernel<T, true> : &append_vector_kernel<T, false>;
    const int64_t per = kAppendThreads >> bits;   // tokens a workgroup
    for (int64_t n0 = 0; n0 < n; n0 += kMost * per) {
        hipLaunchKernelGGL(kernel, dim3(unsigned(std::min(kMost, (n - n0 + per - 1) / per))), dim3(kAppendThreads), 0, stream,
                           p, n0, bits);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_kv_append(const ngpu_kv_cache_t &c, const ngpu_kv_append_t &a, hipStream_t stream) {
    const Append p{c, a};
    return c.dtype == NGPU_F16 ? launch<F16>(p, stream) : launch<Bf16>(p, stream);
}

}  // namespace ngpu
