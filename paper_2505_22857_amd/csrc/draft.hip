// Drafting from the n-gram model: K tokens for each sequence in one launch, one
// workgroup a sequence, its tokens dealt to W wavefronts (group.h).
//
// A step scores the vocabulary as the query does, x[v] = lm[v], and draws a
// token: with m = max x and w[v] = exp((x[v] - m) / temperature), the argmax of
// w[v] / e[v] over unit exponential noise e is v with probability w[v] / sum w.
// Its log-probability row is (x[v] - m) / temperature - log sum w, all in fp32.
// The wavefronts take m, sum w and the best ratio over their own tokens and
// meet once a step: the ratios and sums are then rescaled by exp of the
// difference of the maxima, as the parts of a split softmax are joined.
//
// A step is a chain of dependent accesses (chain record, dense row and arcs,
// exchange, next record), so small batches are bound by latency; the noise rows
// do not depend on the chain and are loaded a step ahead.  Large ones are bound
// by reading the noise and writing the rows (8 bytes a token).  Measured, n-grams of a corpus of 5000 tokens (the first)
// or 200,000: 5.8 us for 4 greedy tokens of 4 sequences (trigram, 128 tokens), 28 us for 8 sampled ones of 256 (6-gram,
// 1024 tokens: 3.5 us a step, of which the noise and the rows would take 0.4), 52 us for 5 of 301 (4-gram, 8192 tokens:
// 99 MB, 1.9 TB/s, and as much again of the model's dense rows).
#include <hip/hip_runtime.h>

#include "reduce.h"

namespace ngpu {

constexpr int kStream = 2;   // aux bits of a buffer load: non-temporal (noise is read once)

struct Draft {
    DevTrie t;
    int uni_base;   // dense row of the state entered by token w: uni_base + w, or -1: the row's head says it
    const int32_t *states, *last;
    const float *noise;
    int64_t noise_b, noise_k;
    int K;
    float to_log2;   // log2 e / temperature
    float inverse;   // 1 / temperature
    int32_t *tokens, *draft_states;
    float *logprobs;
    bool streams;
};

// STREAM: the rows go past the caches.
template <int W, int NT, bool FULL, bool SAMPLE, bool STREAM>
__global__ __launch_bounds__(W * kWave) void draft_kernel(Draft d) {
    extern __shared__ i32x4 lds4[];
    const DevTrie &t = d.t;
    const int64_t b = blockIdx.x;
    const int V = t.vocab_size, K = d.K;
    Meet *meet = reinterpret_cast<Meet *>(lds4);
    const Group<W, NT, FULL> g(V, reinterpret_cast<i32x2 *>(meet + 1));
    const int wave = g.wave, lane = g.lane;
    int32_t *tokens = d.tokens + b * K, *states = d.draft_states + b * (K + 1);
    float *rows = SAMPLE && d.logprobs ? d.logprobs + b * K * V : nullptr;

    int s = __builtin_amdgcn_readfirstlane(d.states[b]);
    const int last = d.last ? __builtin_amdgcn_readfirstlane(d.last[b]) : -1;
    if (s < 0 || s >= t.num_states || last < -1 || last >= V) {
        if (wave == 0 && lane == 0) atomicAdd(&t.status[0], 1);
        for (int k = threadIdx.x; k <= K; k += W * kWave) {
            if (k < K) tokens[k] = -1;
            states[k] = -1;
        }
        if (rows)
            for (int64_t i = threadIdx.x; i < int64_t(K) * V; i += W * kWave) rows[i] = __builtin_nanf("");
        return;
    }
    const RecordIndex ri = record_index(t, lane);
    Words<NT> noise, noise_next, dw, dt;
    const float *noise_row = SAMPLE ? d.noise + b * d.noise_b : nullptr;
    if (SAMPLE) g.template load_row<kStream>(noise_row, noise);
    int4 rec = load_record(ri, s, lane);
    g.clear_slots();
    bool dirty = false;
    int turn = 0;   // of the meeting point's two buffers
    // The record of the state entered by `token` and, where the token alone names it, the dense row.
    auto enter = [&](int token) {
        rec = load_record(ri, s, lane);
        if (dirty) g.clear_slots();
        dirty = false;
        g.load_dense(t, d.uni_base >= 0 ? unsigned(d.uni_base + token) : unsigned(__builtin_amdgcn_readlane(rec.x, 0)), dw,
                     dt);
    };

    if (last >= 0) {   // the state after `last`, whose wavefront finds it
        const ChainHead h = head_of(rec);
        dirty = g.put_levels(t, rec, h);
        int to = 0;
        const int at = last - g.t0;
        const bool mine = at >= 0 && at < g.own;
        if (mine) {
            const int put = g.slots[at].y;
            to = (put != 0 ? put : t.dense_to[int64_t(h.dense_row) * V + last]) & kStateMask;
        }
        if (W > 1) {
            if (mine && lane == 0) meet->b[turn][0] = to;
            lds_barrier();
            to = meet->b[turn][0];
            turn ^= 1;
        }
        s = __builtin_amdgcn_readfirstlane(to);
        enter(last);
    } else {
        g.load_dense(t, unsigned(__builtin_amdgcn_readlane(rec.x, 0)), dw, dt);
    }
    if (threadIdx.x == 0) states[0] = s;

    float x[NT], m = 0.0f, log_total = 0.0f;
    // The row of step k: what its wavefronts have found of it since.
    auto write_row = [&](int k) {
        if (!rows) return;
        float *row = rows + int64_t(k) * V + g.t0;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            if (FULL || kWave * i + lane < g.own) {
                const float y = (x[i] - m) * d.inverse - log_total;
                if (STREAM)
                    __builtin_nontemporal_store(y, &row[kWave * i + lane]);
                else
                    row[kWave * i + lane] = y;
            }
        }
    };
    for (int k = 0; k < K; ++k) {
        const ChainHead h = head_of(rec);
        dirty |= g.put_levels(t, rec, h);
        // What is not on the chain goes out here, behind the arcs: the wait for the next record is the next that
        // it delays, and that has the rest of the step.
        if (SAMPLE && k > 0) write_row(k - 1);
        if (SAMPLE) {   // (on every path, or the compiler would wait for all loads: at the end the last row again)
            noise_row += k + 1 < K ? d.noise_k : 0;
            g.template load_row<kStream>(noise_row, noise_next);
        }
        float r[NT], bx;
        int nx[NT], bi;
        g.lm_values(h, dw, dt, dirty, x, nx);
        float total = 0.0f;   // this and m: of this wavefront's tokens, then of all
        if (!FULL) {
#pragma unroll
            for (int i = 0; i < NT; ++i) x[i] = kWave * i + lane < g.own ? x[i] : -__builtin_inff();
        }
        if (SAMPLE) {
            float lm = x[0];
#pragma unroll
            for (int i = 1; i < NT; ++i) lm = __builtin_fmaxf(lm, x[i]);
            // a wavefront without tokens takes the lowest finite value: its terms are exp(-inf) = 0
            m = __builtin_fmaxf(wave_max(lm), -3.4e38f);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const float w = __builtin_amdgcn_exp2f((x[i] - m) * d.to_log2);
                total += w;
                // the noise of tokens past V reads as 0: 0 * inf is NaN and loses
                r[i] = w * __builtin_amdgcn_rcpf(noise.f(i));
            }
            total = wave_sum(total);
            if (!FULL) {
#pragma unroll
                for (int i = 0; i < NT; ++i) r[i] = kWave * i + lane < g.own ? r[i] : -__builtin_inff();
            }
            g.lane_best(r, bx, bi);
        } else {
            g.lane_best(x, bx, bi);
        }
        int to = nx[0];
#pragma unroll
        for (int i = 1; i < NT; ++i) to = bi == kWave * i ? nx[i] : to;
        to &= kStateMask;
        unsigned key = float_key(bx);
        int token = g.t0 + bi + lane;
        const int who = winner_lane(key, token);
        if (W > 1) {
            if (lane == who) {
                const i32x4 e = {SAMPLE ? __float_as_int(bx) : int(key), token, to, __float_as_int(m)};
                meet->a[turn][wave] = e;
                meet->b[turn][wave] = __float_as_int(total);
            }
            lds_barrier();
            const i32x4 e = meet->a[turn][lane & (W - 1)];
            key = unsigned(e.x);
            if (SAMPLE) {
                const float part = __int_as_float(meet->b[turn][lane & (W - 1)]);
                const float mw = __int_as_float(e.w);
                m = key_float(max_over_waves<W>(float_key(mw)));
                const float f = __builtin_amdgcn_exp2f((mw - m) * d.to_log2);
                total = sum_over_waves<W>(part * f);
                // a wavefront without tokens keeps its -inf; inf * 0 (no noise, no weight) is NaN and loses
                const float best = __int_as_float(e.x);
                key = float_key(best > 0.0f ? or_lowest(best * f) : best);
            }
            turn ^= 1;
            const int w = winner_entry<W>(key, e.y);
            token = __builtin_amdgcn_readlane(e.y, w);
            to = __builtin_amdgcn_readlane(e.z, w);
        } else {
            token = __builtin_amdgcn_readlane(token, who);
            to = __builtin_amdgcn_readlane(to, who);
        }
        s = to;
        enter(token);
        if (SAMPLE) log_total = __builtin_amdgcn_logf(total) * 0.693147180559945f;   // (v_log_f32 is log2)
        if (threadIdx.x == 0) {
            tokens[k] = token;
            states[k + 1] = s;
        }
        if (SAMPLE) noise = noise_next;
    }
    if (SAMPLE) write_row(K - 1);
}

template <int W, int NT, bool FULL, bool SAMPLE, bool STREAM>
static hipError_t launch_group(Draft d, int64_t B, hipStream_t stream) {
    // a grid holds at most 2^32 - 1 work-items: larger batches go in several launches
    constexpr int64_t kMost = int64_t(UINT32_MAX) / (W * kWave);
    const size_t lds = sizeof(Meet) + size_t(W) * kWave * NT * sizeof(i32x2);
    for (int64_t b0 = 0; b0 < B; b0 += kMost) {
        Draft p = d;
        p.states += b0;
        if (p.last) p.last += b0;
        if (SAMPLE) p.noise += b0 * d.noise_b;
        p.tokens += b0 * d.K;
        p.draft_states += b0 * (d.K + 1);
        if (p.logprobs) p.logprobs += b0 * d.K * d.t.vocab_size;
        hipLaunchKernelGGL((draft_kernel<W, NT, FULL, SAMPLE, STREAM>), dim3(unsigned(B - b0 < kMost ? B - b0 : kMost)),
                           dim3(W * kWave), lds, stream, p);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <int W, int NT, bool FULL>
static hipError_t launch_group(const Draft &d, int64_t B, hipStream_t stream) {
    if (!d.noise) return launch_group<W, NT, FULL, false, false>(d, B, stream);
    return d.streams ? launch_group<W, NT, FULL, true, true>(d, B, stream)
                     : launch_group<W, NT, FULL, true, false>(d, B, stream);
}
template <int W, int NT>
static hipError_t launch_group(const Draft &d, int64_t B, hipStream_t stream) {
    return d.t.vocab_size == W * kWave * NT ? launch_group<W, NT, true>(d, B, stream)
                                            : launch_group<W, NT, false>(d, B, stream);
}

hipError_t launch_draft(const DevTrie &t, const int32_t *states, const int32_t *last, int64_t B, int K,
                        float temperature, const float *noise, int64_t noise_b, int64_t noise_k, int32_t *tokens,
                        int32_t *draft_states, float *logprobs, hipStream_t stream) {
    const bool sample = temperature > 0.0f;
    // as the whole decode: order-1 states are numbered by token when every token has a unigram
    const int n1 = (t.max_order > 2 ? t.first[2] : t.num_states) - 1;
    const int uni = t.max_order > 1 && n1 == t.vocab_size + (t.final_w ? 1 : 0) ? 1 : -1;
    // Rows larger together than the L2 caches (8 x 4 MB) would drive the model out of them: 301 x 5 rows of 8192
    // 51.5 us instead of 58.5; 16 x 8 rows 33 instead of 30.
    const bool streams = B * K * t.vocab_size * 4 > (int64_t(32) << 20);
    const Draft d{t, uni, states, last, sample ? noise : nullptr, noise_b, noise_k, K, sample ? 1.44269504088896f / temperature : 0.0f,
                  sample ? 1.0f / temperature : 0.0f, tokens, draft_states, sample ? logprobs : nullptr, streams};
    const int V = t.vocab_size;
    // Wavefronts a sequence: one exchange more against fewer tokens a lane.  us for 8 steps of 4 / 256 / 1024
    // sequences from states of their own, 6-grams (above 1024 tokens 4-grams) of a corpus of 200,000: 256 tokens 17 / 19 /
    // 27 by one wavefront, 20 / 22 / 36 by four; 512 20 / 22 / 31 by one, 20 / 23 / 37 by four; 1024 21 / 29 / 39 by four,
    // 23 / 30 / 39 by two, 22 / 31 / 67 by eight; 2048 18 / 27 / 63 by eight, 20 / 28 / 43 by four; 4096 22 / 33 / 89 by
    // eight, 24 / 34 / 125 by 16.
    if (V <= 256) return launch_group<1, 4>(d, B, stream);
    if (V <= 512) return launch_group<1, 8>(d, B, stream);
    if (V <= 1024) return launch_group<4, 4>(d, B, stream);
    if (V <= 2048) return B > 512 ? launch_group<4, 8>(d, B, stream) : launch_group<8, 4>(d, B, stream);
    if (V <= 4096) return launch_group<8, 8>(d, B, stream);
    return launch_group<16, 8>(d, B, stream);
}

}  // namespace ngpu
