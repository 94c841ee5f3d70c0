// Attention over a paged cache with a prefix that a group of sequences shares.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.h"
#include "walk.h"

namespace ngpu {

struct Attend {
    ngpu_kv_cache_t c;
    ngpu_attend_t a;
};

__device__ __forceinline__ int64_t query_length(const ngpu_attend_t &a, int64_t s) {
    return a.q_lengths ? min(max(int64_t(a.q_lengths[s]), int64_t(0)), a.T) : a.T;
}
__device__ __forceinline__ PageTable prefix_of(const Attend &p, int64_t s) {
    if (p.a.G == 0) return {nullptr, 0};
    const int64_t g = s / (p.a.S / p.a.G);
    const int64_t n = max(int64_t(p.a.prefix_lengths[g]), int64_t(0));
    return {p.a.prefix_pages + g * p.a.prefix_stride, min(n, p.a.prefix_width * p.c.page_size)};
}
__device__ __forceinline__ PageTable own_of(const Attend &p, int64_t s) {
    if (!p.a.pages) return {nullptr, 0};
    const int64_t n = max(int64_t(p.a.lengths[s]), int64_t(0));
    return {p.a.pages + s * p.a.pages_stride, min(n, p.a.pages_width * p.c.page_size)};
}

constexpr int kRowWaves = 4;
constexpr int kMostDims = NGPU_LM_MAX_HEAD_DIM / kWave;   // dimensions a lane holds

__device__ __forceinline__ float lanes_sum(float x) {
    for (int d = kWave / 2; d > 0; d /= 2) x += __shfl_xor(x, d);
    return x;
}

// One workgroup per row (sequence, query token, head); its wavefronts take every
// fourth key, a lane every 64th dimension, and keep a running maximum and sum.
template <class T>
__global__ __launch_bounds__(kRowWaves * kWave) void attend_row_kernel(Attend p, int64_t row0) {
    const ngpu_attend_t &a = p.a;
    const int64_t row = row0 + blockIdx.x, s = row / a.q_heads / a.T, t = row / a.q_heads % a.T;
    const int head = int(row % a.q_heads), kv = head / (a.q_heads / p.c.heads), D = p.c.dim;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    T *out = static_cast<T *>(a.out) + row * D;
    const int64_t nq = query_length(a, s);
    float q[kMostDims], o[kMostDims], m = -__builtin_inff(), sum = 0.0f;
    const T *src = static_cast<const T *>(a.q) + s * a.q_stride_seq + t * a.q_stride_token + head * a.q_stride_head;
    for (int i = 0; i < kMostDims; ++i) {
        const int d = lane + kWave * i;
        q[i] = d < D ? to_float(src[d]) : 0.0f;
        o[i] = 0.0f;
    }
    auto attend = [&](const PageTable &table, int64_t seen) {
        for (int64_t j = wave; j < seen; j += kRowWaves) {
            int64_t entry;
            const int64_t page = table.page(p.c, j, entry);
            if (page < 0) continue;
            const T *k = static_cast<const T *>(p.c.k) + page * p.c.k_stride_page + entry * p.c.k_stride_token +
                         kv * p.c.k_stride_head;
            const T *v = static_cast<const T *>(p.c.v) + page * p.c.v_stride_page + entry * p.c.v_stride_token +
                         kv * p.c.v_stride_head;
            float x = 0.0f;
            for (int i = 0; i < kMostDims; ++i)
                if (const int d = lane + kWave * i; d < D) x = __builtin_fmaf(q[i], to_float(k[d]), x);
            x = lanes_sum(x) * a.scale;
            if (!(x <= m)) {   // a NaN score makes the row NaN
                const float f = expf(m - x);
                sum *= f;
                for (int i = 0; i < kMostDims; ++i) o[i] *= f;
                m = x;
            }
            const float w = x == -__builtin_inff() ? 0.0f : expf(x - m);
            sum += w;
            for (int i = 0; i < kMostDims; ++i)
                if (const int d = lane + kWave * i; d < D) o[i] = __builtin_fmaf(w, to_float(v[d]), o[i]);
        }
    };
    if (t < nq) {
        const PageTable prefix = prefix_of(p, s), own = own_of(p, s);
        attend(prefix, prefix.count);
        attend(own, min(own.count, own.count - nq + t + 1));
    }
    __shared__ float part[kRowWaves][2], sums[kRowWaves][NGPU_LM_MAX_HEAD_DIM];
    if (lane == 0) part[wave][0] = m, part[wave][1] = sum;
    for (int i = 0; i < kMostDims; ++i) sums[wave][lane + kWave * i] = o[i];
    __syncthreads();
    float mm = part[0][0], total = 0.0f, f[kRowWaves];
    for (int w = 1; w < kRowWaves; ++w) mm = part[w][0] > mm ? part[w][0] : mm;
    for (int w = 0; w < kRowWaves; ++w) {
        f[w] = part[w][0] == -__builtin_inff() ? 0.0f : expf(part[w][0] - mm);
        total += part[w][1] * f[w];
    }
    for (int d = threadIdx.x; d < D; d += kRowWaves * kWave) {
        float x = 0.0f;
        for (int w = 0; w < kRowWaves; ++w) x += sums[w][d] * f[w];
        out[d] = from_float<T>(mm == -__builtin_inff() ? 0.0f : x / total);
    }
    if (a.lse && threadIdx.x == 0) a.lse[row] = mm == -__builtin_inff() ? mm : mm + logf(total);
}

template <class T>
static hipError_t launch(const Attend &p, hipStream_t stream) {
    constexpr int64_t kMost = int64_t(UINT32_MAX) / (kRowWaves * kWave);
    const int64_t rows = p.a.S * p.a.T * p.a.q_heads;
    for (int64_t r0 = 0; r0 < rows; r0 += kMost) {
        hipLaunchKernelGGL((attend_row_kernel<T>), dim3(unsigned(std::min(kMost, rows - r0))),
                           dim3(kRowWaves * kWave), 0, stream, p, r0);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

size_t attend_workspace(const ngpu_kv_cache_t &, const ngpu_attend_t &) { return 0; }

hipError_t launch_attend(const ngpu_kv_cache_t &c, const ngpu_attend_t &a, void *, hipStream_t stream) {
    const Attend p{c, a};
    return c.dtype == NGPU_F16 ? launch<F16>(p, stream) : launch<Bf16>(p, stream);
}

}  // namespace ngpu
