// Appending keys and values to a paged cache, with the position rotation of
// keys and queries applied on the way.
//
// A rotated head turns pairs (a, b) of its first R dimensions by the angle of
// its token's position: (a cos - b sin, b cos + a sin), in fp32, rounded once to
// the cache's type; the other dimensions and the values are copied.  Every
// element is read and written once, so the bound is memory traffic, and for a
// few tokens the launch.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.h"

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

// One workgroup per token; each thread writes one element at a time.
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

template <class T>
static hipError_t launch(const Append &p, hipStream_t stream) {
    // a grid holds at most 2^32 - 1 work-items
    constexpr int64_t kMost = int64_t(UINT32_MAX) / kAppendThreads;
    const int64_t n = p.a.S * p.a.T;
    for (int64_t n0 = 0; n0 < n; n0 += kMost) {
        hipLaunchKernelGGL((append_kernel<T>), dim3(unsigned(std::min(kMost, n - n0))), dim3(kAppendThreads), 0, stream,
                           p, n0);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_kv_append(const ngpu_kv_cache_t &c, const ngpu_kv_append_t &a, hipStream_t stream) {
    const Append p{c, a};
    return c.dtype == NGPU_F16 ? launch<F16>(p, stream) : launch<Bf16>(p, stream);
}

}  // namespace ngpu
