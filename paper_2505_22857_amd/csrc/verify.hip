// Verification of drafted tokens against the network's logits.
//
// Place k of a sequence scores the vocabulary with p_k = softmax(logits_k /
// temperature).  The drafted token x is kept while every one before it is and
// u_k q_k(x) < p_k(x); at the first place a where it is not, the added token is
// drawn from max(p_a - q_a, 0) as the argmax of that over unit exponential noise.
//
// Two launches: the statistics of every row (maximum and sum of exponentials,
// or the argmax for greedy decoding) over chunks of it, then per sequence the
// kept length and the race over row a, the draft's row and the noise.  Every
// sum is in fp32 and joined in a fixed order.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "group.h"
#include "ngpu_lm.h"
#include "values.h"

namespace ngpu {

constexpr int kStatThreads = 256;
constexpr int kChunk = 8192;          // logits a workgroup of the first launch takes, at least
constexpr int kMostChunks = 64;
constexpr int kChooseThreads = 1024;

struct Verify {
    ngpu_verify_t a;
    float inv_temperature;   // 0: greedy
    int chunks;
    int64_t chunk;           // logits per chunk
    i32x2 *stats;            // [B, K + 1, chunks] {maximum, sum} or {argmax's key, argmax}
};

__device__ __forceinline__ int draft_length(const ngpu_verify_t &a, int64_t b) {
    return a.lengths ? min(max(a.lengths[b], 0), a.K) : a.K;
}

// exp((x - m) / temperature), 1 at the maximum: +inf shares the mass among its like
__device__ __forceinline__ float weight(float x, float m, float inv_temperature) {
    return x == m ? 1.0f : expf((x - m) * inv_temperature);
}

template <class T, bool GREEDY>
__global__ __launch_bounds__(kStatThreads) void verify_stats_kernel(Verify v, int64_t b0) {
    const ngpu_verify_t &a = v.a;
    const int c = int(blockIdx.x) % v.chunks;
    const int64_t row = int64_t(blockIdx.x) / v.chunks;
    const int k = int(row % (a.K + 1));
    const int64_t b = b0 + row / (a.K + 1);
    if (k > draft_length(a, b)) return;   // no place of this sequence
    const T *x = static_cast<const T *>(a.logits) + b * a.logits_stride_b + k * a.logits_stride_k;
    const int64_t lo = c * v.chunk, hi = min(lo + v.chunk, a.V);
    float m = -__builtin_inff(), sum = 0.0f;
    int at = 0;
    for (int64_t i = lo + threadIdx.x; i < hi; i += kStatThreads) {
        const float y = or_lowest(to_float(x[i]));
        if (GREEDY) {
            at = y > m ? int(i) : at;
            m = fmaxf(m, y);
        } else if (y > m) {
            sum = sum * weight(m, y, v.inv_temperature) + 1.0f;
            m = y;
        } else if (y > -__builtin_inff()) {
            sum += weight(y, m, v.inv_temperature);
        }
    }
    __shared__ i32x2 part[kStatThreads];
    part[threadIdx.x] = i32x2{GREEDY ? int(float_key(m)) : __float_as_int(m), GREEDY ? at : __float_as_int(sum)};
    for (int n = kStatThreads / 2; n > 0; n /= 2) {
        __syncthreads();
        if (int(threadIdx.x) < n) {
            const i32x2 p = part[threadIdx.x], q = part[threadIdx.x + n];
            if (GREEDY) {   // equal keys below -inf's do not occur; a tie takes the lower token
                const bool other = unsigned(q.x) > unsigned(p.x) || (q.x == p.x && q.y < p.y);
                part[threadIdx.x] = other ? q : p;
            } else {
                const float mp = __int_as_float(p.x), mq = __int_as_float(q.x), mm = fmaxf(mp, mq);
                const float s = __int_as_float(p.y) * weight(mp, mm, v.inv_temperature) +
                                __int_as_float(q.y) * weight(mq, mm, v.inv_temperature);
                part[threadIdx.x] = i32x2{__float_as_int(mm), __float_as_int(s)};
            }
        }
    }
    if (threadIdx.x == 0) v.stats[(b * (a.K + 1) + k) * v.chunks + c] = part[0];
}

// Sum of a row's exponentials around its maximum, from its chunks.
struct RowSum {
    float m, sum;
};
__device__ __forceinline__ RowSum row_sum(const Verify &v, const i32x2 *stats) {
    float m = -__builtin_inff(), sum = 0.0f;
    for (int c = 0; c < v.chunks; ++c) m = fmaxf(m, __int_as_float(stats[c].x));
    for (int c = 0; c < v.chunks; ++c)
        sum += __int_as_float(stats[c].y) * weight(__int_as_float(stats[c].x), m, v.inv_temperature);
    return {m, sum};
}
// p(x) for a logit; 0 in a row with nothing above -inf
__device__ __forceinline__ float probability(float x, const RowSum &r, float inv_temperature) {
    return x > -__builtin_inff() ? weight(x, r.m, inv_temperature) / r.sum : 0.0f;
}

template <class T, bool GREEDY>
__global__ __launch_bounds__(kChooseThreads) void verify_choose_kernel(Verify v) {
    const ngpu_verify_t &a = v.a;
    const int64_t b = blockIdx.x;
    const int K = a.K, length = draft_length(a, b);
    const i32x2 *stats = v.stats + b * (K + 1) * v.chunks;
    const T *logits = static_cast<const T *>(a.logits) + b * a.logits_stride_b;
    __shared__ int kept_s, end_s, best_s;
    if (threadIdx.x < kWave) {   // lane k: place k
        const int k = threadIdx.x;
        const int token = k < length ? a.tokens[b * K + k] : -1;
        const bool drafted = token >= 0 && token < a.V;
        bool keep = false;
        int best = 0;
        if (GREEDY) {
            unsigned key = 0;
            for (int c = 0; k <= length && c < v.chunks; ++c) {
                const i32x2 p = stats[k * v.chunks + c];
                if (c == 0 || unsigned(p.x) > key) best = p.y, key = unsigned(p.x);
            }
            if (key <= kInfKey) best = 0;   // nothing above -inf
            keep = drafted && best == token && key > kInfKey;
        } else if (drafted) {
            const RowSum r = row_sum(v, stats + k * v.chunks);
            const float p = probability(or_lowest(to_float(logits[k * a.logits_stride_k + token])), r, v.inv_temperature);
            const float q = a.logprobs ? expf(a.logprobs[b * a.logprobs_stride_b + k * a.logprobs_stride_k + token]) : 1.0f;
            keep = a.uniforms[b * K + k] * q < p;
        }
        // the draft ends at its length or at the first token outside the vocabulary
        const int end = min(length, int(__builtin_ctzll(~__ballot(drafted))));
        const int kept = min(end, int(__builtin_ctzll(~__ballot(keep))));
        if (GREEDY) best = __builtin_amdgcn_readlane(best, kept);
        if (k == 0) {
            kept_s = kept;
            end_s = end;
            best_s = best;
        }
    }
    __syncthreads();
    const int kept = kept_s;
    int added = best_s;
    if (!GREEDY) {
        const bool drafted = kept < end_s;
        const RowSum r = row_sum(v, stats + kept * v.chunks);
        const T *x = logits + kept * a.logits_stride_k;
        const float *lq = drafted && a.logprobs ? a.logprobs + b * a.logprobs_stride_b + kept * a.logprobs_stride_k : nullptr;
        const int one = drafted && !a.logprobs ? a.tokens[b * K + kept] : -1;
        const float *noise = a.noise + b * a.noise_stride_b;
        // the race over what the draft leaves of p, and over p for where that is nothing
        unsigned key = 0, key_p = 0;
        int at = 0, at_p = 0;
        for (int64_t i = threadIdx.x; i < a.V; i += kChooseThreads) {
            const float p = probability(or_lowest(to_float(x[i])), r, v.inv_temperature);
            const float q = lq ? expf(lq[i]) : (i == one ? 1.0f : 0.0f);
            const float rest = p - q, e = noise[i];
            if (p > 0.0f) {
                const unsigned n = float_key(or_lowest(p / e));
                if (n > key_p) key_p = n, at_p = int(i);
            }
            if (rest > 0.0f) {
                const unsigned n = float_key(or_lowest(rest / e));
                if (n > key) key = n, at = int(i);
            }
        }
        __shared__ i32x4 part[kChooseThreads];
        part[threadIdx.x] = i32x4{int(key), at, int(key_p), at_p};
        for (int n = kChooseThreads / 2; n > 0; n /= 2) {
            __syncthreads();
            if (int(threadIdx.x) < n) {
                i32x4 p = part[threadIdx.x];
                const i32x4 q = part[threadIdx.x + n];
                if (unsigned(q.x) > unsigned(p.x) || (q.x == p.x && q.y < p.y)) p.x = q.x, p.y = q.y;
                if (unsigned(q.z) > unsigned(p.z) || (q.z == p.z && q.w < p.w)) p.z = q.z, p.w = q.w;
                part[threadIdx.x] = p;
            }
        }
        added = part[0].x != 0 ? part[0].y : (part[0].z != 0 ? part[0].w : 0);
    }
    const int k = threadIdx.x;
    if (k <= K) a.out_tokens[b * (K + 1) + k] = k < kept ? a.tokens[b * K + k] : (k == kept ? added : -1);
    if (k == 0) {
        a.accepted[b] = kept;
        if (a.states) a.states[b] = a.draft_states[b * (K + 1) + kept];
    }
}

static void split_rows(int64_t V, int &chunks, int64_t &chunk) {
    chunk = std::max<int64_t>(kChunk, (V + kMostChunks - 1) / kMostChunks);
    chunks = int((V + chunk - 1) / chunk);
}

size_t verify_workspace(int64_t B, int K, int64_t V) {
    int chunks;
    int64_t chunk;
    split_rows(V, chunks, chunk);
    return size_t(B) * size_t(K + 1) * size_t(chunks) * sizeof(i32x2);
}

template <class T, bool GREEDY>
static hipError_t launch(Verify v, hipStream_t stream) {
    const int64_t per = int64_t(v.a.K + 1) * v.chunks;   // workgroups a sequence
    const int64_t most = int64_t(UINT32_MAX) / kStatThreads / per;
    for (int64_t b0 = 0; b0 < v.a.B; b0 += most) {
        const unsigned grid = unsigned(std::min(most, v.a.B - b0) * per);
        hipLaunchKernelGGL((verify_stats_kernel<T, GREEDY>), dim3(grid), dim3(kStatThreads), 0, stream, v, b0);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((verify_choose_kernel<T, GREEDY>), dim3(unsigned(v.a.B)), dim3(kChooseThreads), 0, stream, v);
    return hipGetLastError();
}
template <class T>
static hipError_t launch(const Verify &v, hipStream_t stream) {
    return v.a.temperature > 0.0f ? launch<T, false>(v, stream) : launch<T, true>(v, stream);
}

hipError_t launch_verify(const ngpu_verify_t &a, void *workspace, hipStream_t stream) {
    Verify v{a, a.temperature > 0.0f ? 1.0f / a.temperature : 0.0f, 0, 0, static_cast<i32x2 *>(workspace)};
    split_rows(a.V, v.chunks, v.chunk);
    switch (a.dtype) {
        case NGPU_F32: return launch<float>(v, stream);
        case NGPU_F16: return launch<F16>(v, stream);
        default: return launch<Bf16>(v, stream);
    }
}

}  // namespace ngpu
