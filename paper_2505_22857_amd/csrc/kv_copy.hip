// Copies of pages within a paged cache: keys and values, the first entries of
// a page to another page.  Every byte is read and written once: bound by memory
// traffic, and for a few pages by the launch.  4800 pages of 16 x 8 x 128 16-bit keys and values: 124 us, 630
// MB at 5.1 TB/s, a plain copy's rate.  A workgroup takes 16 KB of a page (4 x 16 bytes a thread) where it has as many.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.h"
#include "walk.h"

namespace ngpu {

constexpr int kCopyThreads = 256;

struct Copy {
    ngpu_kv_cache_t c;     // dim and strides in units
    ngpu_kv_cache8_t s;    // its scales; block 0: it has none
    const int32_t *copies;
    int64_t n;
    int slices;            // workgroups a page's keys (or values)
};

// A unit is 16 bytes where everything is aligned to them, else an element.
template <class U>
__global__ __launch_bounds__(kCopyThreads) void copy_kernel(Copy p, int64_t w0) {
    const int64_t w = w0 + blockIdx.x, row = w / (2 * p.slices);
    const int part = int(w % (2 * p.slices)), slice = part / 2;
    const bool values = part % 2 != 0;
    const int32_t *copy = p.copies + 3 * row;
    const int32_t from = copy[0], to = copy[1], entries = min(copy[2], p.c.page_size);
    if (from < 0 || from >= p.c.num_pages || to < 0 || to >= p.c.num_pages || from == to || entries <= 0) return;
    if (p.s.block > 0 && slice == 0) {
        float *const scale = values ? p.s.v_scale : p.s.k_scale;
        const int64_t sp = values ? p.s.v_scale_stride_page : p.s.k_scale_stride_page;
        const int64_t sb = values ? p.s.v_scale_stride_block : p.s.k_scale_stride_block;
        const int64_t sh = values ? p.s.v_scale_stride_head : p.s.k_scale_stride_head;
        const int64_t blocks = p.c.page_size / p.s.block;
        for (int64_t i = threadIdx.x; i < blocks * p.c.heads; i += kCopyThreads) {
            const int64_t at = i / p.c.heads * sb + i % p.c.heads * sh;
            scale[to * sp + at] = scale[from * sp + at];
        }
    }
    const int64_t page = values ? p.c.v_stride_page : p.c.k_stride_page;
    const int64_t token = values ? p.c.v_stride_token : p.c.k_stride_token;
    const int64_t head = values ? p.c.v_stride_head : p.c.k_stride_head;
    U *const cache = static_cast<U *>(values ? p.c.v : p.c.k);
    const U *const src = cache + from * page;
    U *const dst = cache + to * page;
    const int64_t dim = p.c.dim, each = dim * p.c.heads, all = each * entries;
    const int64_t step = int64_t(p.slices) * kCopyThreads;
    const bool dense = head == dim && token == each;
    for (int64_t i = int64_t(slice) * kCopyThreads + threadIdx.x; i < all; i += step) {
        int64_t at = i;
        if (!dense) {
            const int64_t t = i / each, rest = i - t * each, h = rest / dim;
            at = t * token + h * head + (rest - h * dim);
        }
        dst[at] = src[at];
    }
}

template <class U>
static hipError_t launch(Copy p, int64_t size, hipStream_t stream) {   // size: bytes of an element
    const int64_t per = int64_t(sizeof(U)) / size;   // elements a unit
    p.c.dim = int32_t(p.c.dim / per);
    for (int64_t *s : {&p.c.k_stride_page, &p.c.k_stride_token, &p.c.k_stride_head, &p.c.v_stride_page,
                       &p.c.v_stride_token, &p.c.v_stride_head})
        *s /= per;
    const int64_t units = int64_t(p.c.page_size) * p.c.heads * p.c.dim;
    p.slices = int(std::min<int64_t>(64, std::max<int64_t>(1, (units + 4 * kCopyThreads - 1) / (4 * kCopyThreads))));
    constexpr int64_t kMost = int64_t(1) << 23;
    const int64_t all = p.n * 2 * p.slices;
    for (int64_t w0 = 0; w0 < all; w0 += kMost) {
        hipLaunchKernelGGL(copy_kernel<U>, dim3(unsigned(std::min(kMost, all - w0))), dim3(kCopyThreads), 0, stream, p, w0);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

// size: bytes of an element
static hipError_t launch_all(const Copy &p, int64_t size, hipStream_t stream) {
    const ngpu_kv_cache_t &c = p.c;
    const int64_t per = 16 / size;
    bool wide = c.dim % per == 0 && reinterpret_cast<uintptr_t>(c.k) % 16 == 0 && reinterpret_cast<uintptr_t>(c.v) % 16 == 0;
    for (const int64_t s : {c.k_stride_page, c.k_stride_token, c.k_stride_head, c.v_stride_page, c.v_stride_token,
                            c.v_stride_head})
        wide = wide && s % per == 0;
    if (wide) return launch<i32x4>(p, size, stream);
    return size == 1 ? launch<uint8_t>(p, size, stream) : launch<uint16_t>(p, size, stream);
}

hipError_t launch_kv_copy(const ngpu_kv_cache_t &c, const int32_t *copies, int64_t n, hipStream_t stream) {
    return launch_all(Copy{c, {}, copies, n, 1}, 2, stream);
}
hipError_t launch_kv_copy8(const ngpu_kv_cache8_t &c, const int32_t *copies, int64_t n, hipStream_t stream) {
    return launch_all(Copy{c.cache, c, copies, n, 1}, 1, stream);
}

}  // namespace ngpu
