// One step of a beam search with the n-gram model fused in: the k best
// continuations over all hypotheses of an utterance and the whole vocabulary.
//
// A hypothesis is expanded by a group of wavefronts: the query's walk and the
// fused scores stay in its registers (group.h), as in the top-k, and the
// hypothesis's score is added (the sums are what is ordered, since adding
// rounds).  A continuation's key is the sum's order-preserving bits above the
// complement of its place in (hypothesis, class) order, so that larger keys
// come first and all differ.  Selection: a lower bound of the k-th largest sum
// from the maxima of disjoint parts, halvings of the interval while too many
// reach it, then a short list in LDS whose entries find their ranks by
// counting; where more continuations share the last sum than the list holds,
// the first of them by place.
//
// Two ways.  Few hypotheses of small vocabularies: one launch, a workgroup an
// utterance with a selection over all of it.  Else two: the first lists the k
// best of a hypothesis, a workgroup each, the second the k largest of these.
//
// What has to be read is each class's score once and the dense rows of the
// states (8 bytes a token, from L2 where hypotheses share them): the smallest
// calls are bound by the latency of the chain state, record, arcs, selection
// (1 x 4 hypotheses of 128 tokens: 4.7 us, an empty launch 3.9), the largest by
// the same chain with two workgroups a CU, whose slots fill LDS: 592 hypotheses
// of 8192 tokens take 16.5 + 3.5 us and fetch 52 MB, 19 of scores and the rest of
// dense rows (10 us at a copy's rate), while their wavefronts wait for 53 % of
// their cycles and issue 450 vector and 440 scalar instructions each.  The
// selection's bound matters too: with the smallest of enough parts' maxima instead
// of the k-th largest of 64, two or three more halvings, it was 19.6 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "launch.h"
#include "reduce.h"

namespace ngpu {

typedef unsigned long long u64;

struct Beam {
    ngpu_beam_step_t a;
    int classes;         // of a row: V, or V + 1
    u64 *keys;           // [B, W, k + 1] the hypothesis's best, descending, and that of class V; 0: none
    int32_t *next;       // [B, W, k + 1] their states
};

// Sum over 16 lanes, in each of them.
__device__ __forceinline__ int row_sum(int x) {
    auto moved = [](int v, auto ctrl) { return __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, 0xf, 0xf, true); };
    x += moved(x, std::integral_constant<int, 0xB1>{});    // lane ^ 1
    x += moved(x, std::integral_constant<int, 0x4E>{});    // lane ^ 2
    x += moved(x, std::integral_constant<int, 0x141>{});   // other half of 8
    x += moved(x, std::integral_constant<int, 0x140>{});   // other half of 16
    return x;
}
// What a hypothesis's wavefronts exchange.
struct alignas(16) BeamMeet {
    unsigned parts[kWave];   // keys of their largest
    int ranks[kWave];
    unsigned bound;
    int b[2][16];
};
template <int W>
constexpr int beam_list() { return W * kWave > NGPU_LM_MAX_BEAMS ? W * kWave : NGPU_LM_MAX_BEAMS; }

template <int W, int NT, bool FULL>
__global__ __launch_bounds__(W * kWave) void beam_expand_kernel(DevTrie t, Beam p, int64_t n0) {
    extern __shared__ i32x4 lds4[];
    load_trie_args(t);
    load_args(p.a.asr, p.a.states, p.a.scores, p.a.last, p.keys, p.next, p.a.W, p.a.k, p.a.lambda);
    constexpr int kList = beam_list<W>();
    const int64_t n = n0 + blockIdx.x, b = n / p.a.W;
    const int V = t.vocab_size, hyp = int(n - b * p.a.W), k = p.a.k;
    BeamMeet *meet = reinterpret_cast<BeamMeet *>(lds4);
    const Group<W, NT, FULL> g(V, reinterpret_cast<i32x2 *>(meet + 1));
    // the list takes the slots' place: every wavefront has read its slots before the barrier of the first exchange
    u64 *lkey = reinterpret_cast<u64 *>(meet + 1);       // kList: key of the sum, ~token
    int *lnext = reinterpret_cast<int *>(lkey + kList);  // kList: next state
    const int wave = g.wave, lane = g.lane, tid = threadIdx.x;
    u64 *const keys = p.keys + n * (k + 1);
    int32_t *const next = p.next + n * (k + 1);
    const unsigned place0 = unsigned(hyp) * unsigned(p.classes);

    const int s_l = p.a.states[n];   // issued before the row, so its wait leaves the row in flight
    const float score_l = p.a.scores[n];
    const int last_l = p.a.last ? p.a.last[n] : -1;
    Words<NT> row, dw, dt;
    const float *const asr = p.a.asr + b * p.a.asr_stride_b + hyp * p.a.asr_stride_w;
    g.load_row(asr, row);
    const RecordIndex ri = record_index(t, lane);
    g.clear_slots();
    const int s = __builtin_amdgcn_readfirstlane(s_l), last = __builtin_amdgcn_readfirstlane(last_l);
    const float score = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(score_l)));
    const bool is = score > -__builtin_inff(), ended = last == V;
    if (!is || ended || s < 0 || s >= t.num_states) {
        if (tid == 0 && is && !ended) atomicAdd(&t.status[0], 1);
        for (int j = tid; j < k; j += W * kWave) keys[j] = 0;
        if (tid == 0) {
            keys[k] = is && ended ? u64(float_key(score)) << 32 | ~(place0 + unsigned(V)) : 0;
            next[k] = s;
        }
        return;
    }
    const int4 rec = load_record(ri, s, lane);
    if (tid == 0) {   // class V keeps the state
        u64 key = 0;
        if (p.classes > V) {
            const float lm = p.a.mode == kAed ? t.final_w[s] : 0.0f;
            const float total = score + __builtin_fmaf(p.a.lambda, lm, asr[V]);
            if (total > -__builtin_inff()) key = u64(float_key(total)) << 32 | ~(place0 + unsigned(V));
        }
        keys[k] = key;
        next[k] = s;
    }
    const ChainHead h = head_of(rec);
    g.load_dense(t, unsigned(h.dense_row), dw, dt);
    const bool any = g.template put_levels<true>(t, rec, h);
    float x[NT];
    int nx[NT];
    unsigned key[NT];
    g.lm_values(h, dw, dt, any, x, nx);
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        x[i] = score + __builtin_fmaf(p.a.lambda, x[i], row.f(i));
        // a token's key lies from -inf's (also a NaN's) to +inf's, below ~0; past V: below every token's
        key[i] = FULL || kWave * i + lane < g.own ? float_key(or_lowest(x[i])) : 0u;
        m = max(m, key[i]);
    }

    int xi = 0;
    // value of every wavefront, entry l mod W in lane l
    auto gather = [&](unsigned a) -> unsigned {
        if (W == 1) return a;
        const int buf = xi & 1;
        ++xi;
        if (lane == 0) meet->b[buf][wave] = int(a);
        lds_barrier();
        return unsigned(meet->b[buf][lane & (W - 1)]);
    };
    // 1. the bound, and the largest key
    const int wanted = min(k, V);
    unsigned lo, top;
    if constexpr (W >= 4) {
        // the wanted-th largest of 64 disjoint parts' maxima: fewer are above it and at least as many no smaller (none
        // where fewer parts hold tokens); each wavefront looks whether it is one of its parts
        constexpr int kParts = kWave / W, kLanes = kWave / kParts;
        static_assert(kLanes <= 16, "parts within a row");
        const unsigned part = max_over_waves<kLanes>(m);
        if (lane % kLanes == 0) meet->parts[wave * kParts + lane / kLanes] = part;
        if (wave == 0) meet->ranks[lane] = 0;
        if (tid == 0) meet->bound = 0;
        lds_barrier();
        const unsigned mine = meet->parts[lane];
        top = wave_max_u32(mine);
#pragma unroll
        for (int l = 0; l < kParts; ++l) {
            const unsigned o = unsigned(__builtin_amdgcn_readlane(int(mine), wave * kParts + l));
            if (__builtin_popcountll(__ballot(mine > o)) < wanted && __builtin_popcountll(__ballot(mine >= o)) >= wanted &&
                lane == 0)
                meet->bound = o;
        }
        lds_barrier();
        lo = __builtin_amdgcn_readfirstlane(int(meet->bound));
    } else {
        // the smallest of the maxima of at least as many parts
        const int full = ((V >> 6) * kWave + g.range - 1) / g.range;   // wavefronts whose lanes all hold tokens
        unsigned part = m;
        if (wanted <= 16 * full) {
            part = max_over_waves<4>(part);
            if (wanted <= 4 * full) part = max_over_waves<16>(part);
        }
        const unsigned wtop = wave_max_u32(m);
        if (wanted <= full) part = wtop;
        const unsigned wlow = wave < full ? wave_max_u32(~part) : 0u;   // complement of the smallest part
        top = __builtin_amdgcn_readfirstlane(max_over_waves<W>(gather(wtop)));
        lo = wanted <= kWave * full ? ~unsigned(__builtin_amdgcn_readfirstlane(max_over_waves<W>(gather(wlow)))) : 0u;
    }
    if (lo == 0) lo = 1;   // every token's key is above 0

    // keys >= x in this wavefront, and in the group: total, and of the wavefronts before this one
    int total = 0, before = 0;
    auto count = [&](unsigned at) {
        int c = 0;
#pragma unroll
        for (int i = 0; i < NT; ++i) c += __builtin_popcountll(__ballot(key[i] >= at));
        if constexpr (W == 1) {
            total = c;
        } else {
            const int of = int(gather(unsigned(c))), e = lane < W ? of : 0;
            static_assert(NT * kWave * W < 65536, "two sums in a word");
            const unsigned sums = __builtin_amdgcn_readfirstlane(row_sum(lane < wave ? e << 16 | e : e));
            before = int(sums >> 16);
            total = int(sums & 0xffffu);
        }
    };
    // 2. at least `wanted` keys reach lo, fewer reach hi (hi - lo modulo 2^32)
    const int most = min(kList, max(kWave, wanted + wanted / 4));
    unsigned hi = top + 1;
    count(lo);
    for (int halvings = 0; total > most && hi - lo > 1 && (halvings < 6 || total > kList); ++halvings) {
        const unsigned mid = lo + (hi - lo) / 2;
        const int t0 = total, b0 = before;
        count(mid);
        if (total >= wanted) {
            lo = mid;
        } else {
            hi = mid;
            total = t0;
            before = b0;
        }
    }
    // 3. the list
    int listed = total;
    auto put = [&](bool take, int at, int i) {
        if (take) {
            lkey[at] = (u64(key[i]) << 32) | ~unsigned(g.token(i));
            lnext[at] = nx[i] & kStateMask;
        }
    };
    if (listed <= kList) {
        int at = before;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const bool take = key[i] >= lo;
            const u64 mask = __ballot(take);
            put(take, at + lanes_below(mask), i);
            at += __builtin_popcountll(mask);
        }
    } else {   // hi = lo + 1: the last key is lo, shared by more tokens than the list holds
        const int all_before = before;
        count(hi);
        const int above = total;
        int at = before, tie = above + all_before - before;
        listed = wanted;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const bool over = key[i] >= hi, same = key[i] == lo;
            const u64 mo = __ballot(over), ms = __ballot(same);
            put(over, at + lanes_below(mo), i);
            put(same && tie + lanes_below(ms) < wanted, tie + lanes_below(ms), i);
            at += __builtin_popcountll(mo);
            tie += __builtin_popcountll(ms);
        }
    }
    if (W > 1) lds_barrier();
    // entry tid of the list (which has no more than the group has threads, as k is at most 64)
    static_assert(kList <= W * kWave, "an entry a thread");
    auto write = [&](int i, u64 one, int rank) {
        if (rank >= wanted) return;
        const unsigned sum = unsigned(one >> 32);   // -inf is not selected
        keys[rank] = sum > kInfKey ? u64(sum) << 32 | ~(place0 + ~unsigned(one)) : 0;
        next[rank] = lnext[i];
    };
    if (W >= 4 && listed <= kWave) {   // the wavefronts share the comparisons
        const u64 mine = lane < listed ? lkey[lane] : ~0ull;
        int rank = 0;
#pragma unroll 4
        for (int q = wave; q < listed; q += W) rank += lkey[q] > mine ? 1 : 0;
        if (rank > 0) atomicAdd(&meet->ranks[lane], rank);
        lds_barrier();
        if (tid < listed) write(tid, mine, meet->ranks[tid]);
    } else if (wave * kWave < listed) {
        const u64 mine = tid < listed ? lkey[tid] : ~0ull;
        int rank = 0;
#pragma unroll 8
        for (int q = 0; q < listed; ++q) rank += lkey[q] > mine ? 1 : 0;
        if (tid < listed) write(tid, mine, rank);
    }
    for (int j = wanted + tid; j < k; j += W * kWave) keys[j] = 0;
}

// An utterance's k largest of its hypotheses' keys, E a thread.
constexpr int kSelectThreads = 256, kSelectWaves = kSelectThreads / kWave;
template <int E>
__global__ __launch_bounds__(kSelectThreads) void beam_select_kernel(Beam p, int64_t b0) {
    __shared__ u64 list[E * kSelectThreads];
    __shared__ int from[E * kSelectThreads];
    __shared__ int counts[2][kSelectWaves];
    __shared__ unsigned bounds[2][kSelectWaves];
    __shared__ int ranks[kWave];
    const int64_t b = b0 + blockIdx.x;
    const int k = p.a.k, n = p.a.W * (k + 1), tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const u64 *const keys = p.keys + b * n;
    u64 x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = e * kSelectThreads + tid < n ? keys[e * kSelectThreads + tid] : 0;
    int turn = 0, total = 0, before = 0;
    auto count = [&](unsigned at) {   // keys whose sum's bits reach `at`: all, and those of the wavefronts before
        int c = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) c += __builtin_popcountll(__ballot(unsigned(x[e] >> 32) >= at));
        if (lane == 0) counts[turn][wave] = c;
        __syncthreads();
        total = before = 0;
#pragma unroll
        for (int w = 0; w < kSelectWaves; ++w) {
            before += w < wave ? counts[turn][w] : 0;
            total += counts[turn][w];
        }
        turn ^= 1;
    };
    // a hypothesis's keys but that of class V descend, so the k-th largest of all is no less than any hypothesis's k-th
    unsigned lo = 0, top = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const unsigned of = unsigned(x[e] >> 32);
        top = max(top, of);
        if (unsigned(e * kSelectThreads + tid) % unsigned(k + 1) == unsigned(k - 1)) lo = max(lo, of);
    }
    lo = wave_max_u32(lo);
    top = wave_max_u32(top);
    if (lane == 0) {
        bounds[0][wave] = lo;
        bounds[1][wave] = top;
    }
    if (wave == 0) ranks[lane] = 0;
    __syncthreads();
    lo = max(unsigned(__builtin_amdgcn_readfirstlane(int(max_over_waves<kSelectWaves>(bounds[0][lane % kSelectWaves])))), 1u);
    top = __builtin_amdgcn_readfirstlane(int(max_over_waves<kSelectWaves>(bounds[1][lane % kSelectWaves])));
    // at least min(k, keys that there are) reach lo; fewer than k reach hi
    unsigned hi = top + 1;
    count(lo);
    const int there = total;   // (with fewer than k, lo is 1)
    while (total > max(kWave, 2 * k) && hi - lo > 1) {
        const unsigned mid = lo + (hi - lo) / 2;
        const int t0 = total, c0 = before;
        count(mid);
        if (total >= k) {
            lo = mid;
        } else {
            hi = mid;
            total = t0;
            before = c0;
        }
    }
    int at = before;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const bool take = unsigned(x[e] >> 32) >= lo;
        const u64 mask = __ballot(take);
        if (take) {
            list[at + lanes_below(mask)] = x[e];
            from[at + lanes_below(mask)] = e * kSelectThreads + tid;
        }
        at += __builtin_popcountll(mask);
    }
    __syncthreads();
    auto write = [&](int i, u64 one, int rank) {
        if (rank >= k) return;
        const unsigned place = ~unsigned(one), parent = place / unsigned(p.classes);
        const int64_t out = b * k + rank;
        p.a.out_tokens[out] = int32_t(place - parent * unsigned(p.classes));
        p.a.out_parents[out] = int32_t(parent);
        p.a.out_scores[out] = key_float(unsigned(one >> 32));
        p.a.out_states[out] = p.next[b * n + from[i]];
    };
    if (total <= kWave) {   // the wavefronts share the comparisons
        const u64 one = lane < total ? list[lane] : ~0ull;
        int rank = 0;
#pragma unroll 4
        for (int q = wave; q < total; q += kSelectWaves) rank += list[q] > one ? 1 : 0;
        if (rank > 0) atomicAdd(&ranks[lane], rank);
        __syncthreads();
        if (tid < total) write(tid, one, ranks[tid]);
    } else {
        for (int i = tid; i < total; i += kSelectThreads) {
            const u64 one = list[i];
            int rank = 0;
#pragma unroll 8
            for (int q = 0; q < total; ++q) rank += list[q] > one ? 1 : 0;
            write(i, one, rank);
        }
    }
    for (int j = there + tid; j < k; j += kSelectThreads) {   // left over
        const int64_t out = b * k + j;
        p.a.out_tokens[out] = p.a.out_parents[out] = -1;
        p.a.out_scores[out] = -__builtin_inff();
        p.a.out_states[out] = 0;
    }
}

// A whole utterance in one launch, where its hypotheses' rows fit a workgroup's registers and LDS: HW wavefronts a
// hypothesis, each with the walk of its part of the row, and one selection over all of them, so that no hypothesis lists its
// own best.  The bound is the k-th largest of 64 disjoint parts' maxima, four a wavefront (in a small workgroup some are
// none, and the bound may be none too).
constexpr int kWholeWaves = 16;
constexpr int kWholeList = 512;   // continuations that are listed
struct alignas(16) WholeMeet {
    unsigned parts[4 * kWholeWaves];   // keys of their largest
    int ranks[kWave];
    int counts[2][kWholeWaves];
    unsigned bound;
};
template <int HW, int NT, bool FULL>
__global__ __launch_bounds__(kWholeWaves * kWave) void beam_whole_kernel(DevTrie t, Beam p, int64_t b0) {
    extern __shared__ i32x4 lds4[];
    load_trie_args(t);
    load_args(p.a.asr, p.a.states, p.a.scores, p.a.last, p.a.W, p.a.k, p.a.lambda);
    WholeMeet *const sh = reinterpret_cast<WholeMeet *>(lds4);
    // the list takes the slots' place: every wavefront has read its slots before the first barrier
    u64 *const list = reinterpret_cast<u64 *>(sh + 1);        // kWholeList
    int *const list_next = reinterpret_cast<int *>(list + kWholeList);
    const int V = t.vocab_size, W = p.a.W, k = p.a.k, waves = W * HW, tid = threadIdx.x;
    const int64_t b = b0 + blockIdx.x;
    const int in = __builtin_amdgcn_readfirstlane(tid / kWave), hyp = in / HW;
    Group<HW, NT, FULL> g(V, in % HW);
    g.slots = reinterpret_cast<i32x2 *>(list) + in * (kWave * NT);
    const int lane = g.lane;
    const int64_t n = b * W + hyp;

    const int s_l = p.a.states[n];
    const float score_l = p.a.scores[n];
    const int last_l = p.a.last ? p.a.last[n] : -1;
    const float *const asr = p.a.asr + b * p.a.asr_stride_b + hyp * p.a.asr_stride_w;
    Words<NT> row, dw, dt;
    g.load_row(asr, row);
    const RecordIndex ri = record_index(t, lane);
    g.clear_slots();
    const int s = __builtin_amdgcn_readfirstlane(s_l), last = __builtin_amdgcn_readfirstlane(last_l);
    const float score = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(score_l)));
    const bool closes = g.wave == HW - 1 && lane == 0;   // its class V comes behind all tokens
    const bool is = score > -__builtin_inff(), ended = last == V, walks = is && !ended && s >= 0 && s < t.num_states;
    if (is && !ended && !walks && closes) atomicAdd(&t.status[0], 1);
    // the lane's keys, of its tokens and, in one lane of a hypothesis, of class V; 0: no continuation
    unsigned key[NT + 1];
    int nx[NT];
#pragma unroll
    for (int i = 0; i <= NT; ++i) key[i] = 0;
    if (walks) {
        const int4 rec = load_record(ri, s, lane);
        float class_v = -__builtin_inff();
        if (closes && p.classes > V) {
            const float lm = p.a.mode == kAed ? t.final_w[s] : 0.0f;
            class_v = score + __builtin_fmaf(p.a.lambda, lm, asr[V]);
        }
        const ChainHead h = head_of(rec);
        g.load_dense(t, unsigned(h.dense_row), dw, dt);
        const bool any = g.template put_levels<true>(t, rec, h);
        float x[NT];
        g.lm_values(h, dw, dt, any, x, nx);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            x[i] = score + __builtin_fmaf(p.a.lambda, x[i], row.f(i));
            const unsigned of = float_key(or_lowest(x[i]));
            key[i] = (FULL || kWave * i + lane < g.own) && of > kInfKey ? of : 0u;
        }
        if (class_v > -__builtin_inff()) key[NT] = float_key(class_v);
    } else if (is && ended && closes) {
        key[NT] = float_key(score);
    }
    unsigned m = key[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) m = max(m, key[i]);
    const unsigned part = max_over_waves<16>(m);   // of each row of 16 lanes
    if (lane % 16 == 0) sh->parts[in * 4 + lane / 16] = part;
    if (in == 0) sh->ranks[lane] = 0;
    if (tid == 0) sh->bound = 0;
    lds_barrier();
    const unsigned mine = lane < 4 * waves ? sh->parts[lane] : 0u;
    const unsigned top = wave_max_u32(mine);
    // a wavefront looks whether one of its parts is the k-th largest: fewer than k are above it and at least k no smaller
#pragma unroll
    for (int l = 0; l < 4; ++l) {
        const unsigned o = unsigned(__builtin_amdgcn_readlane(int(mine), in * 4 + l));
        if (__builtin_popcountll(__ballot(mine > o)) < k && __builtin_popcountll(__ballot(mine >= o)) >= k && lane == 0)
            sh->bound = o;
    }
    lds_barrier();
    // with fewer than k parts: every continuation
    unsigned lo = max(unsigned(__builtin_amdgcn_readfirstlane(int(sh->bound))), 1u);

    int turn = 0, total = 0, before = 0;
    auto count = [&](unsigned at) {   // keys that reach `at`: of all, and of the wavefronts before this one
        int c = 0;
#pragma unroll
        for (int i = 0; i <= NT; ++i) c += __builtin_popcountll(__ballot(key[i] >= at));
        if (lane == 0) sh->counts[turn][in] = c;
        lds_barrier();
        const int e = lane < waves ? sh->counts[turn][lane % kWholeWaves] : 0;
        static_assert((NT + 1) * kWave * kWholeWaves < 65536, "two sums in a word");
        const unsigned sums = __builtin_amdgcn_readfirstlane(row_sum(lane < in ? e << 16 | e : e));
        before = int(sums >> 16);
        total = int(sums & 0xffffu);
        turn ^= 1;
    };
    // at least min(k, all) keys reach lo; fewer than k reach hi, where that is not 0 (hi - lo modulo 2^32)
    count(lo);
    unsigned hi = top + 1;
    const int wanted = total < k ? total : k;   // (lo is 1 then)
    const int want = max(kWave, 2 * k);
    for (int halvings = 0; total > want && hi - lo > 1 && (halvings < 6 || total > kWholeList); ++halvings) {
        const unsigned mid = lo + (hi - lo) / 2;
        const int t0 = total, c0 = before;
        count(mid);
        if (total >= k) {
            lo = mid;
        } else {
            hi = mid;
            total = t0;
            before = c0;
        }
    }
    const unsigned place0 = unsigned(hyp) * unsigned(p.classes);
    auto put = [&](bool take, int at, int i) {
        if (!take) return;
        const int token = i < NT ? g.token(i) : V;
        list[at] = u64(key[i]) << 32 | ~(place0 + unsigned(token));
        list_next[at] = i < NT ? nx[i < NT ? i : 0] & kStateMask : s;
    };
    int listed = total;
    if (listed <= kWholeList) {
        int at = before;
#pragma unroll
        for (int i = 0; i <= NT; ++i) {
            const bool take = key[i] >= lo;
            const u64 mask = __ballot(take);
            put(take, at + lanes_below(mask), i);
            at += __builtin_popcountll(mask);
        }
    } else {   // hi = lo + 1: the last sum is lo, shared by more continuations than the list holds, which come in order
        const int all_before = before;
        count(hi);
        const int over_all = total;
        int at = before, tie = over_all + all_before - before;
        listed = k;
#pragma unroll
        for (int i = 0; i <= NT; ++i) {
            const bool over = key[i] >= hi, even = key[i] == lo;
            const u64 mo = __ballot(over), ms = __ballot(even);
            put(over, at + lanes_below(mo), i);
            put(even && tie + lanes_below(ms) < k, tie + lanes_below(ms), i);
            at += __builtin_popcountll(mo);
            tie += __builtin_popcountll(ms);
        }
    }
    lds_barrier();
    auto write = [&](int i, u64 one, int rank) {
        if (rank >= k) return;
        const unsigned place = ~unsigned(one), parent = place / unsigned(p.classes);
        const int64_t out = b * k + rank;
        p.a.out_tokens[out] = int32_t(place - parent * unsigned(p.classes));
        p.a.out_parents[out] = int32_t(parent);
        p.a.out_scores[out] = key_float(unsigned(one >> 32));
        p.a.out_states[out] = list_next[i];
    };
    if (listed <= kWave) {   // the wavefronts share the comparisons
        const u64 one = lane < listed ? list[lane] : ~0ull;
        int rank = 0;
#pragma unroll 4
        for (int q = in; q < listed; q += waves) rank += list[q] > one ? 1 : 0;
        if (rank > 0) atomicAdd(&sh->ranks[lane], rank);
        lds_barrier();
        if (tid < listed) write(tid, one, sh->ranks[tid]);
    } else {
        for (int i = tid; i < listed; i += waves * kWave) {
            const u64 one = list[i];
            int rank = 0;
#pragma unroll 8
            for (int q = 0; q < listed; ++q) rank += list[q] > one ? 1 : 0;
            write(i, one, rank);
        }
    }
    for (int j = wanted + tid; j < k; j += waves * kWave) {   // left over
        const int64_t out = b * k + j;
        p.a.out_tokens[out] = p.a.out_parents[out] = -1;
        p.a.out_scores[out] = -__builtin_inff();
        p.a.out_states[out] = 0;
    }
}

template <int HW, int NT>
static hipError_t whole(const DevTrie &t, const Beam &p, hipStream_t stream) {
    constexpr int64_t kMost = int64_t(1) << 22;
    const int waves = p.a.W * HW;
    const size_t lds = sizeof(WholeMeet) + std::max(size_t(kWholeList) * 12, size_t(waves) * kWave * NT * sizeof(i32x2));
    constexpr int kMostLds = sizeof(WholeMeet) + kWholeWaves * kWave * NT * sizeof(i32x2);
    const bool full = t.vocab_size == HW * kWave * NT;
    if (lds > 65536) {
        static std::atomic<uint64_t> devices[2];
        const hipError_t e = full ? allow_lds(&beam_whole_kernel<HW, NT, true>, kMostLds, devices[1])
                                  : allow_lds(&beam_whole_kernel<HW, NT, false>, kMostLds, devices[0]);
        if (e != hipSuccess) return e;
    }
    for (int64_t b0 = 0; b0 < p.a.B; b0 += kMost) {
        const dim3 grid(unsigned(std::min(kMost, p.a.B - b0))), block(waves * kWave);
        if (full)
            hipLaunchKernelGGL((beam_whole_kernel<HW, NT, true>), grid, block, lds, stream, t, p, b0);
        else
            hipLaunchKernelGGL((beam_whole_kernel<HW, NT, false>), grid, block, lds, stream, t, p, b0);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int W, int NT>
static hipError_t expand(const DevTrie &t, const Beam &p, hipStream_t stream) {
    constexpr int64_t kMost = int64_t(1) << 22;   // workgroups a launch
    constexpr size_t lds = sizeof(BeamMeet) + std::max(size_t(beam_list<W>()) * 12, size_t(W) * kWave * NT * sizeof(i32x2));
    const int64_t all = p.a.B * p.a.W;
    const bool full = t.vocab_size == W * kWave * NT;
    if constexpr (lds > 65536) {
        static std::atomic<uint64_t> devices[2];
        const hipError_t e = full ? allow_lds(&beam_expand_kernel<W, NT, true>, int(lds), devices[1])
                                  : allow_lds(&beam_expand_kernel<W, NT, false>, int(lds), devices[0]);
        if (e != hipSuccess) return e;
    }
    for (int64_t n0 = 0; n0 < all; n0 += kMost) {
        const dim3 grid(unsigned(std::min(kMost, all - n0))), block(W * kWave);
        if (full)
            hipLaunchKernelGGL((beam_expand_kernel<W, NT, true>), grid, block, lds, stream, t, p, n0);
        else
            hipLaunchKernelGGL((beam_expand_kernel<W, NT, false>), grid, block, lds, stream, t, p, n0);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int E>
static hipError_t select(const Beam &p, hipStream_t stream) {
    constexpr int64_t kMost = int64_t(1) << 22;
    for (int64_t b0 = 0; b0 < p.a.B; b0 += kMost) {
        hipLaunchKernelGGL(beam_select_kernel<E>, dim3(unsigned(std::min(kMost, p.a.B - b0))), dim3(kSelectThreads), 0, stream,
                           p, b0);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Whether one launch takes the call: where each lane has four tokens of at most 16 wavefronts.  64 utterances take 5.0
// against 7.4 us in two launches (4 hypotheses, 128 tokens), 6.4 against 8.6 (8, 512) and 6.3 against 8.0 (4, 1024); with
// eight tokens a lane, 16 hypotheses of 512 gain nothing (11.3 against 9.5), while 5 to 8 of 513 to 1024 do: of 1024, 6-grams,
// calls in a graph, 1 / 64 / 256 utterances take 6.5 / 6.8 / 7.1 us with 5 hypotheses (two launches 7.9 / 9.1 / 10.5) and
// 7.1 / 7.8 / 8.1 with 8 (7.9 / 9.4 / 11.5), and calls that the host paces 8.1, not 10.9.  Past a workgroup a CU
// small ones still gain, 600 utterances of 4 hypotheses 6.0 against 8.9 (128 tokens) and 7.8 against 9.5 (512), larger
// ones do not: 8 hypotheses of 512 tokens 17.8 against 12.0.
static bool takes_whole(int64_t B, int W, int V) {
    const int range = V <= 256 ? 1 : V <= 512 ? 2 : V <= 1024 ? 4 : 8;   // wavefronts a hypothesis, of 256 tokens
    return V <= 2048 && (W * range <= (B <= 256 ? kWholeWaves : 8) || (B <= 256 && W <= 8 && V <= 1024));
}
static hipError_t whole(const DevTrie &t, const Beam &p, int V, hipStream_t stream) {
    if (V <= 256) return whole<1, 4>(t, p, stream);
    if (V <= 512) return whole<2, 4>(t, p, stream);
    if (V <= 1024) return p.a.W <= 4 ? whole<4, 4>(t, p, stream) : whole<2, 8>(t, p, stream);
    return whole<8, 4>(t, p, stream);
}

// Wavefronts and tokens per lane of a hypothesis: the top-k kernel's rules for k up to 64.
static hipError_t expand(const DevTrie &t, const Beam &p, int V, hipStream_t stream) {
    const int64_t n = p.a.B * p.a.W;
    if (V <= 256) return expand<1, 4>(t, p, stream);
    if (V <= 512) return p.a.k > 32 && n <= 1024 ? expand<2, 4>(t, p, stream) : expand<1, 8>(t, p, stream);
    if (V <= 768 && n > 1024) return expand<1, 12>(t, p, stream);
    if (V <= 1024) return n > 1024 ? expand<2, 8>(t, p, stream) : expand<4, 4>(t, p, stream);
    if (V <= 1536 && n > 768) return V <= 1280 ? expand<2, 10>(t, p, stream) : expand<2, 12>(t, p, stream);
    if (V <= 2048) return expand<4, 8>(t, p, stream);
    if (V <= 4096) return n <= 128 ? expand<8, 8>(t, p, stream) : expand<4, 16>(t, p, stream);
    if (V <= 6144) return expand<8, 12>(t, p, stream);
    return expand<8, 16>(t, p, stream);
}

size_t beam_step_workspace(int64_t B, int W, int k) {
    return (size_t(B) * size_t(W) * size_t(k + 1) * 12 + 15) / 16 * 16;
}

hipError_t launch_beam_step(const DevTrie &t, const ngpu_beam_step_t &a, void *workspace, hipStream_t stream) {
    const size_t n = size_t(a.B) * size_t(a.W) * size_t(a.k + 1);
    u64 *const keys = static_cast<u64 *>(workspace);
    const Beam p{a, t.vocab_size + (a.mode == kPlain ? 0 : 1), keys, reinterpret_cast<int32_t *>(keys + n)};
    if (takes_whole(a.B, a.W, t.vocab_size)) return whole(t, p, t.vocab_size, stream);
    if (const hipError_t e = expand(t, p, t.vocab_size, stream); e != hipSuccess) return e;
    const int each = a.W * (a.k + 1);
    if (each <= kSelectThreads) return select<1>(p, stream);
    if (each <= 4 * kSelectThreads) return select<4>(p, stream);
    static_assert(NGPU_LM_MAX_BEAMS * (NGPU_LM_MAX_BEAMS + 1) <= 17 * kSelectThreads, "the largest beams' keys");
    return select<17>(p, stream);
}

}  // namespace ngpu
