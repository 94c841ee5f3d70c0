// Verification of drafted tokens against the network's logits.
//
// Place k of a sequence scores the vocabulary with p_k = softmax(logits_k /
// temperature).  The drafted token x is kept while every one before it is and
// u_k q_k(x) < p_k(x); at the first place a where it is not, the added token is
// drawn from max(p_a - q_a, 0) as the argmax of that over unit exponential noise.
//
// So every row needs its maximum and sum of exponentials (or its argmax, for
// greedy decoding), and row a once more, with the draft's row and the noise: the
// bound is reading the logits.  A small vocabulary is verified
// in one launch, a workgroup a sequence; a larger one in two, the first over
// chunks of all rows and the second over parts of row a, whose last workgroup
// joins them.  Sums are in fp32 and joined in a fixed order.  Measured: 6.9 us for
// one sequence of 4 + 1 rows of 1024, greedy; 13 us for 64 of 5 + 1 of 8192, fp32 (row after row
// by 16 wavefronts: its latency, at 1.3 TB/s); 69 us for 96 of 7 + 1 of 128001, bf16: 295 MB
// at 4.3 TB/s, where a large copy reaches 5.0.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ngpu_lm.h"
#include "reduce.h"
#include "values.h"

namespace ngpu {

constexpr int64_t kWhole = 8192;      // most tokens of a row that one workgroup takes whole
constexpr int kWholeThreads = 1024;
constexpr int kSegment = 1024;        // of a row, what a wavefront of the one launch takes at a time
constexpr int kStatThreads = 256;
constexpr int kChunk = 8192;          // logits of a row, tokens of a race that a workgroup of the two launches takes
constexpr int kMostChunks = 64;
constexpr int kRaceThreads = 256;
constexpr int kMostParts = 64;

struct Verify {
    ngpu_verify_t a;
    float to_log2;           // log2 e / temperature; 0: greedy
    int chunks, parts;
    int64_t chunk, part;     // logits per chunk, tokens per part
    i32x2 *stats;            // [B, K + 1, chunks] {maximum, sum} or {argmax's key, argmax}
    uint64_t *best;          // [B] best of the parts' races so far: key, then the token's complement
    int *arrived;            // [B] parts that are done
};

__device__ __forceinline__ int draft_length(const ngpu_verify_t &a, int64_t b) {
    return a.lengths ? min(max(a.lengths[b], 0), a.K) : a.K;
}

// exp((x - m) / temperature), 1 at the maximum: +inf shares the mass among its like
__device__ __forceinline__ float weight(float x, float m, float to_log2) {
    return x == m ? 1.0f : __builtin_amdgcn_exp2f((x - m) * to_log2);
}

// Elements [lo, hi) of a row dealt to `threads` threads: f.add(values, n, token of
// the first, stride of the tokens), 16-byte loads where the row's alignment allows, BATCH of them
// in flight.
template <int BATCH, class T, class F>
__device__ __forceinline__ void over_row(const T *row, int64_t lo, int64_t hi, int thread, int threads, F &f) {
    constexpr int N = 16 / sizeof(T);
    struct alignas(16) Pack {
        T v[N];
    };
    const int64_t skip = (16 - int64_t(reinterpret_cast<uintptr_t>(row + lo) % 16)) % 16 / int64_t(sizeof(T));
    const int64_t first = min(lo + skip, hi), packs = (hi - first) / N, tail = first + packs * N;
    const Pack *src = reinterpret_cast<const Pack *>(row + first);
    for (int64_t i = thread; i < packs; i += int64_t(threads) * BATCH) {
        Pack p[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) p[u] = src[min(i + int64_t(u) * threads, packs - 1)];
        float x[BATCH * N];
#pragma unroll
        for (int u = 0; u < BATCH; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e)
                x[u * N + e] = i + int64_t(u) * threads < packs ? or_lowest(to_float(p[u].v[e])) : -__builtin_inff();
        f.template add<BATCH, N>(x, int(first + i * N), threads * N);
    }
    const int64_t edge = thread < first - lo ? lo + thread : tail + (thread - (first - lo));
    if (edge < hi) {   // fewer than 2 N elements, no more than the threads
        float x[1] = {or_lowest(to_float(row[edge]))};
        f.template add<1, 1>(x, int(edge), 0);
    }
}

// The sum of exponentials around the running maximum.
struct SoftSum {
    float to_log2, m = -__builtin_inff(), sum = 0.0f;
    template <int BATCH, int N>
    __device__ __forceinline__ void add(const float (&x)[BATCH * N], int, int) {
        float top = x[0];
#pragma unroll
        for (int e = 1; e < BATCH * N; ++e) top = __builtin_fmaxf(top, x[e]);
        if (top == -__builtin_inff()) return;
        if (top > m) {
            sum *= weight(m, top, to_log2);
            m = top;
        }
        float part = 0.0f;
#pragma unroll
        for (int e = 0; e < BATCH * N; ++e) part += weight(x[e], m, to_log2);
        sum += part;
    }
    __device__ __forceinline__ i32x2 over_wave() const {
        const float top = wave_max(m);
        return {__float_as_int(top), __float_as_int(wave_sum(sum * weight(m, top, to_log2)))};
    }
};
// The largest value and its lowest token.
struct Argmax {
    float to_log2, m = -__builtin_inff();
    int at = 0;
    template <int BATCH, int N>
    __device__ __forceinline__ void add(const float (&x)[BATCH * N], int i, int stride) {
#pragma unroll
        for (int u = 0; u < BATCH; ++u)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float y = x[u * N + e];
                const int token = i + u * stride + e;
                const bool better = y > m || (y == m && token < at);   // (edges come last)
                at = better ? token : at;
                m = better ? y : m;
            }
    }
    __device__ __forceinline__ i32x2 over_wave() const {
        const unsigned key = float_key(m);
        const int who = winner_lane(key, at);
        return {__builtin_amdgcn_readlane(int(key), who), __builtin_amdgcn_readlane(at, who)};
    }
};

// A row's statistics from those of its pieces.
struct RowSum {
    float m, sum;
};
__device__ __forceinline__ RowSum row_sum(const i32x2 *stats, int n, float to_log2) {
    float m = -__builtin_inff(), sum = 0.0f;
#pragma unroll 4
    for (int c = 0; c < n; ++c) m = fmaxf(m, __int_as_float(stats[c].x));
#pragma unroll 4
    for (int c = 0; c < n; ++c) sum += __int_as_float(stats[c].y) * weight(__int_as_float(stats[c].x), m, to_log2);
    return {m, sum};
}
__device__ __forceinline__ i32x2 row_best(const i32x2 *stats, int n) {   // pieces in the tokens' order
    i32x2 r = stats[0];
    for (int c = 1; c < n; ++c)
        if (unsigned(stats[c].x) > unsigned(r.x)) r = stats[c];
    return r;
}
// p(x) for a logit; 0 in a row with nothing above -inf
__device__ __forceinline__ float probability(float x, const RowSum &r, float to_log2) {
    return x > -__builtin_inff() ? weight(x, r.m, to_log2) / r.sum : 0.0f;
}

struct Decision {
    int kept;     // drafted tokens kept
    int end;      // where the draft ends: kept < end says that a drafted token was refused
    int added;    // greedy: the token that is added
    RowSum row;   // of the added token's place
};
// By one wavefront, lane k at place k, from n statistics a row in LDS; uniform.
template <class T, bool GREEDY>
__device__ __forceinline__ Decision decide(const Verify &v, int64_t b, int length, const i32x2 *stats, int n) {
    const ngpu_verify_t &a = v.a;
    const int k = threadIdx.x % kWave;
    const int token = k < length ? a.tokens[b * a.K + k] : -1;
    const bool drafted = token >= 0 && token < a.V;
    bool keep = false;
    int best = 0;
    RowSum row{0.0f, 0.0f};
    if (GREEDY) {
        if (k <= length) {
            const i32x2 r = row_best(stats + k * n, n);
            const bool any = unsigned(r.x) > kInfKey;   // something above -inf
            best = any ? r.y : 0;
            keep = drafted && any && best == token;
        }
    } else if (k <= length) {
        float x = 0.0f, lq = 0.0f, u = 0.0f;   // their loads are in flight while the row is summed
        if (drafted) {
            x = to_float(static_cast<const T *>(a.logits)[b * a.logits_stride_b + k * a.logits_stride_k + token]);
            lq = a.logprobs ? a.logprobs[b * a.logprobs_stride_b + k * a.logprobs_stride_k + token] : 0.0f;
            u = a.uniforms[b * a.K + k];
        }
        row = row_sum(stats + k * n, n, v.to_log2);
        keep = drafted && u * expf(lq) < probability(or_lowest(x), row, v.to_log2);
    }
    // the draft ends at its length or at the first token outside the vocabulary
    const int end = min(length, int(__builtin_ctzll(~__ballot(drafted))));
    const int kept = min(end, int(__builtin_ctzll(~__ballot(keep))));
    return {kept, end, GREEDY ? __builtin_amdgcn_readlane(best, kept) : 0,
            {__int_as_float(__builtin_amdgcn_readlane(__float_as_int(row.m), kept)),
             __int_as_float(__builtin_amdgcn_readlane(__float_as_int(row.sum), kept))}};
}

// The largest weight / noise over tokens lo + thread, ...: of what the draft leaves of p (REST) or of p.
struct Race {
    unsigned key = 0;   // 0: no token with a weight
    int token = 0;
    template <class T, bool REST>
    __device__ __forceinline__ void run(const Verify &v, int64_t b, const Decision &d, int64_t lo, int64_t hi,
                                        int thread, int threads) {
        const ngpu_verify_t &a = v.a;
        const T *x = static_cast<const T *>(a.logits) + b * a.logits_stride_b + d.kept * a.logits_stride_k;
        const float *noise = a.noise + b * a.noise_stride_b;
        const bool drafted = REST && d.kept < d.end;
        const float *lq = drafted && a.logprobs ? a.logprobs + b * a.logprobs_stride_b + d.kept * a.logprobs_stride_k : nullptr;
        const int one = drafted && !a.logprobs ? a.tokens[b * a.K + d.kept] : -1;
        constexpr int kBatch = 8;
        for (int64_t i = lo + thread; i < hi; i += int64_t(threads) * kBatch) {
            float xs[kBatch], es[kBatch], qs[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int64_t j = min(i + int64_t(u) * threads, hi - 1);   // (the last again: no better than itself)
                xs[u] = to_float(x[j]);
                es[u] = noise[j];
            }
            if (lq) {
#pragma unroll
                for (int u = 0; u < kBatch; ++u) qs[u] = lq[min(i + int64_t(u) * threads, hi - 1)];
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int j = int(min(i + int64_t(u) * threads, hi - 1));
                const float p = probability(or_lowest(xs[u]), d.row, v.to_log2);
                const float w = p - (lq ? expf(qs[u]) : (j == one ? 1.0f : 0.0f));
                const unsigned n = float_key(or_lowest(w * __builtin_amdgcn_rcpf(es[u])));
                if (w > 0.0f && n > key) key = n, token = j;   // (tokens rise)
            }
        }
    }
    // the best of the workgroup, uniform; `box` holds an entry per wavefront
    template <int THREADS>
    __device__ __forceinline__ void over_group(i32x2 *box) {
        const int who = winner_lane(key, token);
        __syncthreads();
        if (int(threadIdx.x % kWave) == who) box[threadIdx.x / kWave] = i32x2{int(key), token};
        __syncthreads();
        key = 0;
        for (int w = 0; w < THREADS / kWave; ++w) take(box[w]);
    }
    __device__ __forceinline__ void take(const i32x2 &e) {
        if (unsigned(e.x) > key || (unsigned(e.x) == key && e.y < token)) key = unsigned(e.x), token = e.y;
    }
};

__device__ __forceinline__ void write_result(const ngpu_verify_t &a, int64_t b, const Decision &d, int added) {
    const int k = threadIdx.x;
    if (k <= a.K) a.out_tokens[b * (a.K + 1) + k] = k < d.kept ? a.tokens[b * a.K + k] : (k == d.kept ? added : -1);
    if (k == 0) {
        a.accepted[b] = d.kept;
        if (a.states) a.states[b] = a.draft_states[b * (a.K + 1) + d.kept];
    }
}

// The whole of a sequence in one workgroup.
template <class T, bool GREEDY>
__global__ __launch_bounds__(kWholeThreads) void verify_whole_kernel(Verify v) {
    const ngpu_verify_t &a = v.a;
    const int64_t b = blockIdx.x;
    const int length = draft_length(a, b), V = int(a.V), segments = (V + kSegment - 1) / kSegment;
    constexpr int kWaves = kWholeThreads / kWave;
    __shared__ i32x2 stats[(NGPU_LM_MAX_DRAFT + 1) * int(kWhole / kSegment)];
    __shared__ i32x2 box[kWaves];
    __shared__ Decision decision;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const T *logits = static_cast<const T *>(a.logits) + b * a.logits_stride_b;
    for (int i = wave; i < (length + 1) * segments; i += kWaves) {
        const int k = i / segments, lo = i % segments * kSegment;
        std::conditional_t<GREEDY, Argmax, SoftSum> f{v.to_log2};
        over_row<int(sizeof(T))>(logits + k * a.logits_stride_k, lo, min(lo + kSegment, V), lane, kWave, f);
        const i32x2 r = f.over_wave();
        if (lane == 0) stats[i] = r;
    }
    __syncthreads();
    if (wave == 0) {
        const Decision d = decide<T, GREEDY>(v, b, length, stats, segments);
        if (lane == 0) decision = d;
    }
    __syncthreads();
    const Decision d = decision;
    int added = d.added;
    if (!GREEDY) {
        Race race;
        race.run<T, true>(v, b, d, 0, V, threadIdx.x, kWholeThreads);
        race.over_group<kWholeThreads>(box);
        if (race.key == 0) {   // the draft leaves nothing
            race.run<T, false>(v, b, d, 0, V, threadIdx.x, kWholeThreads);
            race.over_group<kWholeThreads>(box);
        }
        added = race.key != 0 ? race.token : 0;
    }
    write_result(a, b, d, added);
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
    std::conditional_t<GREEDY, Argmax, SoftSum> f{v.to_log2};
    over_row<4>(x, c * v.chunk, min((c + 1) * v.chunk, a.V), threadIdx.x, kStatThreads, f);
    constexpr int kWaves = kStatThreads / kWave;
    __shared__ i32x2 part[kWaves];
    const i32x2 r = f.over_wave();
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = r;
    __syncthreads();
    if (threadIdx.x != 0) return;
    if (k == 0 && c == 0) {
        v.arrived[b] = 0;
        v.best[b] = 0;
    }
    i32x2 all;
    if (GREEDY) {   // a thread's tokens are not in the wavefronts' order
        all = part[0];
        for (int w = 1; w < kWaves; ++w)
            if (unsigned(part[w].x) > unsigned(all.x) || (part[w].x == all.x && part[w].y < all.y)) all = part[w];
    } else {
        const RowSum s = row_sum(part, kWaves, v.to_log2);
        all = i32x2{__float_as_int(s.m), __float_as_int(s.sum)};
    }
    v.stats[(b * (a.K + 1) + k) * v.chunks + c] = all;
}

template <class T, bool GREEDY>
__global__ __launch_bounds__(kRaceThreads) void verify_race_kernel(Verify v, int64_t b0) {
    const ngpu_verify_t &a = v.a;
    const int64_t b = b0 + int64_t(blockIdx.x) / v.parts;
    const int part = int(int64_t(blockIdx.x) % v.parts);
    extern __shared__ i32x4 lds4[];
    i32x2 *stats = reinterpret_cast<i32x2 *>(lds4);   // all loaded at once: one by one a row's would wait for each
    __shared__ Decision decision;
    __shared__ i32x2 box[kRaceThreads / kWave];
    __shared__ int last;
    const int length = draft_length(a, b);
    for (int i = threadIdx.x; i < (length + 1) * v.chunks; i += kRaceThreads)
        stats[i] = v.stats[b * (a.K + 1) * v.chunks + i];
    __syncthreads();
    if (threadIdx.x < kWave) {
        const Decision d = decide<T, GREEDY>(v, b, length, stats, v.chunks);
        if (threadIdx.x == 0) decision = d;
    }
    __syncthreads();
    const Decision d = decision;
    if (GREEDY) return write_result(a, b, d, d.added);   // (one part)
    Race race;
    race.run<T, true>(v, b, d, part * v.part, min((part + 1) * v.part, a.V), threadIdx.x, kRaceThreads);
    race.over_group<kRaceThreads>(box);
    if (v.parts > 1) {   // the last part to arrive has the best of all
        if (threadIdx.x == 0) {
            // The maximum has been taken when its old value is back: no fence, which would write back the whole
            // L2 for each of the parts (96 sequences, 16 parts: 97 us instead of 37).
            const uint64_t mine = uint64_t(race.key) << 32 | unsigned(~race.token);
            uint64_t old = __hip_atomic_fetch_max(&v.best[b], mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" : "+v"(old)::"memory");
            last = __hip_atomic_fetch_add(&v.arrived[b], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == v.parts - 1;
        }
        __syncthreads();
        if (!last) return;
        const uint64_t e = __hip_atomic_load(&v.best[b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        race.key = unsigned(e >> 32);
        race.token = int(~unsigned(e));
    }
    if (race.key == 0) {   // the draft leaves nothing
        race.run<T, false>(v, b, d, 0, a.V, threadIdx.x, kRaceThreads);
        race.over_group<kRaceThreads>(box);
    }
    write_result(a, b, d, race.key != 0 ? race.token : 0);
}

static void split_row(int64_t V, int64_t least, int most, int &n, int64_t &size) {
    size = std::max<int64_t>(least, (V + most - 1) / most);
    n = int((V + size - 1) / size);
}

static Verify plan(const ngpu_verify_t &a, char *workspace, size_t *bytes) {
    Verify v{};
    v.a = a;
    v.to_log2 = a.temperature > 0.0f ? 1.44269504088896f / a.temperature : 0.0f;
    *bytes = 0;
    // One launch takes 8.5 / 9.4 / 19 us for 1 / 64 / 512 sequences of 5 rows of 4096 (fp32, 5 or 6 rows), two with
    // the chunks below 8.7 / 10.2 / 20; of 8192 10.6 / 12.6 / 26.8, two 8.8 / 12.3 / 30.2; of 16384 one 18.7 / 22 / 47,
    // two 9.5 / 14.4 / 51.  So up to 8192 tokens no batch needs a workspace, though a few sequences of 8192 would be 2 us
    // faster by two.
    if (a.V <= kWhole) return v;
    // Smaller chunks while they fill the chip at most twice: 9.7 us, not 13.2, for one sequence of 5 rows of
    // 32768, 14.4, not 16.3, for 64 of 6 of 16384.  More of them only repeat what each does first: 96 sequences of 128001
    // 81 us with halves for the second launch, not 74.
    auto least = [&](int64_t rows) {
        const int64_t full = rows * ((a.V + kChunk - 1) / kChunk);
        return full <= 512 ? kChunk / 4 : (full < 1024 ? kChunk / 2 : kChunk);
    };
    split_row(a.V, least(a.B * (a.K + 1)), kMostChunks, v.chunks, v.chunk);
    split_row(a.V, least(a.B), kMostParts, v.parts, v.part);
    const size_t stats = size_t(a.B) * size_t(a.K + 1) * size_t(v.chunks) * sizeof(i32x2);
    const size_t best = size_t(a.B) * sizeof(uint64_t);
    if (a.temperature == 0.0f) v.parts = 1, v.part = a.V;   // nothing is drawn
    v.stats = reinterpret_cast<i32x2 *>(workspace);
    v.best = reinterpret_cast<uint64_t *>(workspace + stats);
    v.arrived = reinterpret_cast<int *>(workspace + stats + best);
    *bytes = stats + best + size_t(a.B) * sizeof(int);
    return v;
}

size_t verify_workspace(int64_t B, int K, int64_t V) {
    ngpu_verify_t a{};
    a.B = B, a.K = K, a.V = V;
    size_t bytes;
    plan(a, nullptr, &bytes);
    return bytes;
}

template <class T, bool GREEDY>
static hipError_t launch(const Verify &v, hipStream_t stream) {
    if (v.chunks == 0) {
        hipLaunchKernelGGL((verify_whole_kernel<T, GREEDY>), dim3(unsigned(v.a.B)), dim3(kWholeThreads), 0, stream, v);
        return hipGetLastError();
    }
    // a grid holds at most 2^32 - 1 work-items
    const auto each = [&](int64_t per, int threads, auto go) {
        const int64_t most = int64_t(UINT32_MAX) / threads / per;
        for (int64_t b0 = 0; b0 < v.a.B; b0 += most) {
            go(dim3(unsigned(std::min(most, v.a.B - b0) * per)), b0);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    const hipError_t e = each(int64_t(v.a.K + 1) * v.chunks, kStatThreads, [&](dim3 grid, int64_t b0) {
        hipLaunchKernelGGL((verify_stats_kernel<T, GREEDY>), grid, dim3(kStatThreads), 0, stream, v, b0);
    });
    if (e != hipSuccess) return e;
    const size_t lds = size_t(v.a.K + 1) * v.chunks * sizeof(i32x2);
    return each(v.parts, kRaceThreads, [&](dim3 grid, int64_t b0) {
        hipLaunchKernelGGL((verify_race_kernel<T, GREEDY>), grid, dim3(kRaceThreads), lds, stream, v, b0);
    });
}
template <class T>
static hipError_t launch(const Verify &v, hipStream_t stream) {
    return v.a.temperature > 0.0f ? launch<T, false>(v, stream) : launch<T, true>(v, stream);
}

hipError_t launch_verify(const ngpu_verify_t &a, void *workspace, hipStream_t stream) {
    size_t bytes;
    const Verify v = plan(a, static_cast<char *>(workspace), &bytes);
    switch (a.dtype) {
        case NGPU_F32: return launch<float>(v, stream);
        case NGPU_F16: return launch<F16>(v, stream);
        default: return launch<Bf16>(v, stream);
    }
}

}  // namespace ngpu
