// Shared-prefix attention on the matrix cores.
//
// A problem is the keys of one cache head (of a group's prefix, or of a
// sequence's own tokens) against every query row that reads them: the rows of
// all sequences of the group, of all their query tokens and of the heads that
// share the cache head, stacked.  So a prefix is read once for its group, and
// the rows fill the matrix instructions' columns.
//
// Per tile of 32 keys a wavefront computes the scores transposed, S^T = K Q^T
// (16x16x32: lane l holds 4 keys of row l mod 16), so that a row's maximum and sum
// run over a lane's own registers and four lanes, and the weights are already
// laid out as the second operand of O^T += V^T P^T: lane l holds the keys 16 u + 4
// (l / 16) + i, and the transposing LDS load fetches V's 4 x 16 blocks in that
// order.  K and V go from memory straight to LDS, double-buffered; 16-byte
// chunks of a row are stored at their place XOR the row, which leaves neither
// load a bank conflict.
//
// The running maximum of a row is raised only when a score exceeds it by more
// than 2^8 (the weights then stay below 2^8, and their sum's rounding is the
// same): otherwise the accumulators need no rescaling.  Scores, sums and
// accumulators are fp32; the weights are rounded to the cache's type, which the
// matrix instructions need, before they multiply V.
#pragma once

#include <hip/hip_runtime.h>

#include "cache.h"
#include "walk.h"

namespace ngpu {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

struct Attend {
    ngpu_kv_cache_t c;
    ngpu_attend_t a;
};

__device__ __forceinline__ int64_t query_length(const ngpu_attend_t &a, int64_t s) {
    return a.q_lengths ? min(max(int64_t(a.q_lengths[s]), int64_t(0)), a.T) : a.T;
}
__device__ __forceinline__ PageTable prefix_table(const Attend &p, int64_t g) {
    const int64_t n = max(int64_t(p.a.prefix_lengths[g]), int64_t(0));
    return {p.a.prefix_pages + g * p.a.prefix_stride, min(n, p.a.prefix_width * p.c.page_size)};
}
__device__ __forceinline__ PageTable own_table(const Attend &p, int64_t s) {
    const int64_t n = max(int64_t(p.a.lengths[s]), int64_t(0));
    return {p.a.pages + s * p.a.pages_stride, min(n, p.a.pages_width * p.c.page_size)};
}

// How a call is cut into workgroups: problems of a group's prefix and of a
// sequence's own tokens, each in blocks of rows and splits of keys.
struct Cut {
    int64_t problems;    // groups (or sequences) times cache heads
    int blocks, splits;
    __host__ __device__ int64_t works() const { return problems * blocks * splits; }
};
struct AttendPlan {
    Cut prefix, own;
    int parts;           // splits of both: partial results a row
    float *sums;         // [parts, rows, dim] sums of weight times v around the part's maximum
    float2 *stats;       // [parts, rows] {maximum in log2, sum of weights}
};

// 16 bytes of zeros, which stand for keys and dimensions that do not exist.
static __device__ __attribute__((aligned(16))) unsigned kNoData[4];

template <class T>
using LdsPtr = __attribute__((address_space(3))) T *;

template <class T>
struct Matrix;
template <>
struct Matrix<Bf16> {
    static constexpr short kExponent = 0x7f80;
    static __device__ __forceinline__ f32x4 mul(s16x8 a, s16x8 b, f32x4 c) {
        typedef __bf16 v8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};
template <>
struct Matrix<F16> {
    static constexpr short kExponent = 0x7c00;
    static __device__ __forceinline__ f32x4 mul(s16x8 a, s16x8 b, f32x4 c) {
        typedef _Float16 v8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};

// Maximum over the four lanes that hold a row (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float row_max(float x) {
    auto both = [](float v, auto r) { return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])); };
    x = both(x, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return both(x, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
}
__device__ __forceinline__ float row_sum4(float x) {
    auto both = [](float v, auto r) { return __uint_as_float(r[0]) + __uint_as_float(r[1]); };
    x = both(x, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return both(x, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
}

// Waits for everything this wavefront has loaded (registers and LDS).
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void wait_loads_all() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// 16 bytes a lane from memory to LDS at `at` + 16 lane (uniform `at`).  As asm, since
// the compiler would wait for it before any later LDS load.  (m0 is a reserved register, which
// nothing else in these kernels uses: a clobber would only be warned about.)
__device__ __forceinline__ void load_to_lds(const void *p, unsigned at) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(p) : "memory");
}

// DK: 32-dimension steps of a head; RT: tiles of 16 rows a wavefront; WR, WK:
// wavefronts along rows and along keys.
template <class T, int DK, int RT, int WR, int WK>
struct AttendTile {
    static constexpr int kWaves = WR * WK;
    static constexpr int kChunks = WK > 1 ? 1 : 2;              // of 32 keys, a wavefront and tile
    static constexpr int kKeys = 32 * kChunks * WK;             // a tile
    static constexpr int kLoad = kKeys / kWaves;                // keys a wavefront loads
    static constexpr int kRows = 16 * RT * WR;                  // a workgroup
    static constexpr int kPitch = DK <= 2 ? 128 : (DK <= 4 ? 256 : 512);   // bytes of a row in LDS
    static constexpr int kPieces = kPitch / 16;                 // 16-byte chunks of it
    static constexpr int kStage = 2 * kKeys * kPitch;           // keys, then values
    static constexpr int kLds = 2 * kStage;
    static constexpr int kPerLoad = kWave / kPieces;            // rows a load instruction brings
    static constexpr int kLoads = kLoad / kPerLoad;
    static constexpr int kTiles = 2 * DK;                       // of 16 dimensions
    static constexpr int kDims = 32 * DK;
    static_assert(WK == 1 || kWaves * 16 * RT * kDims * 4 <= kLds, "the wavefronts' sums meet in the tiles' LDS");
    static_assert(kLoad == 16 || kLoad == 32, "a wavefront's lanes hold its keys' pages");

    static __device__ __forceinline__ int key_swizzle(int row) { return kPieces == 8 ? (row >> 1) & 7 : row & 15; }
    static __device__ __forceinline__ int value_swizzle(int row) {
        return kPieces == 8 ? ((row >> 1) & 3) << 1 : (row & 7) << 1;
    }
};

template <class T, int DK, int RT, int WR, int WK>
__global__ __launch_bounds__(64 * WR * WK) void attend_tile_kernel(Attend p, AttendPlan plan, int64_t work0) {
    using A = AttendTile<T, DK, RT, WR, WK>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ unsigned masks[2][4];   // per stage, the keys of each loading wavefront that exist (WR > 1)
    const unsigned lds0 = unsigned(reinterpret_cast<uintptr_t>((LdsPtr<char>)lds));
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wk = wave / WR, wr = wave % WR, col = lane % 16, quad = lane / 16;
    const ngpu_attend_t &a = p.a;
    const int H = p.c.heads, rep = a.q_heads / H, D = p.c.dim, T_ = int(a.T);

    // Workgroups go to the 8 XCDs in turn; those of one problem follow each
    // other on one XCD, whose L2 then serves the row blocks' common keys.
    int64_t w = work0 + (gridDim.x % 8 == 0 ? blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8 : blockIdx.x);
    const bool own = w >= plan.prefix.works();
    const Cut &cut = own ? plan.own : plan.prefix;
    if (own) w -= plan.prefix.works();
    const int block = int(w % cut.blocks), split = int(w / cut.blocks % cut.splits);
    const int64_t problem = w / cut.blocks / cut.splits;
    const int h = int(problem % H);
    const int64_t g = problem / H;
    const int64_t beam = own ? 1 : a.S / a.G, s0 = g * beam;
    const int64_t rows = beam * T_ * rep;
    const PageTable table = own ? own_table(p, s0) : prefix_table(p, g);
    const int count = int(table.count);

    // this wavefront's query rows: operand registers, and the keys each row sees
    s16x8 q[RT][DK];
    int limit[RT];
    int64_t out_row[RT];   // -1: no row
    bool counts[RT];       // a query token that counts
    const int64_t row0 = int64_t(block) * A::kRows + wr * 16 * RT;
    const bool aligned = (reinterpret_cast<uintptr_t>(a.q) % 16 == 0) && a.q_stride_seq % 8 == 0 &&
                         a.q_stride_token % 8 == 0 && a.q_stride_head % 8 == 0;
    int least = count;   // keys that every row of the workgroup's sequences sees
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int64_t row = row0 + 16 * r + col;
        const bool is = row < rows;
        const int64_t i = is ? row : 0, s = s0 + i / (int64_t(T_) * rep);
        const int t = int(i / rep % T_), head = h * rep + int(i % rep);
        out_row[r] = is ? (s * T_ + t) * a.q_heads + head : -1;
        const int nq = int(query_length(a, s));
        counts[r] = t < nq;
        limit[r] = count;
        if (own) {
            limit[r] = min(count, max(0, count - nq + t + 1));
            least = min(least, max(0, count - nq + 1));
        }
        const T *src = static_cast<const T *>(a.q) + s * a.q_stride_seq + t * a.q_stride_token + head * a.q_stride_head;
#pragma unroll
        for (int k = 0; k < DK; ++k) {
            const int d = 32 * k + 8 * quad;
            s16x8 x = {};
            if (is && d < D) {   // D is a multiple of 8
                if (aligned) {
                    x = *reinterpret_cast<const s16x8 *>(src + d);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = short(src[d + e].bits);
                }
            }
            q[r][k] = x;
        }
    }
    least = __builtin_amdgcn_readfirstlane(least);

    // this split's keys
    const int tiles = (count + A::kKeys - 1) / A::kKeys, per = (tiles + cut.splits - 1) / cut.splits;
    const int tile0 = min(tiles, split * per), tile1 = min(tiles, tile0 + per);

    // A lane's key of a tile: its row of the cache in 16-byte units, all ones where there is none.
    const unsigned page_size = unsigned(p.c.page_size);
    const int my_key = wave * A::kLoad + lane % A::kLoad;
    auto page_of = [&](int tile) {
        const int j = tile * A::kKeys + my_key;
        return tile < tile1 && j < count ? table.pages[unsigned(j) / page_size] : -1;
    };
    const uint64_t k_page = uint64_t(p.c.k_stride_page) / 8, v_page = uint64_t(p.c.v_stride_page) / 8;
    const unsigned k_token = unsigned(p.c.k_stride_token / 8), v_token = unsigned(p.c.v_stride_token / 8);
    const char *k_head = static_cast<const char *>(p.c.k) + int64_t(h) * p.c.k_stride_head * 2;
    const char *v_head = static_cast<const char *>(p.c.v) + int64_t(h) * p.c.v_stride_head * 2;
    const int piece = lane % A::kPieces, in_load = lane / A::kPieces;
    const int pieces = D / 8;
    unsigned valid = 0;   // keys that exist among those this wavefront loaded last
    auto fetch = [&](int tile, int stage, int page) {
        const int j = tile * A::kKeys + my_key;
        const bool is = page >= 0 && page < p.c.num_pages;   // (-1 past the end)
        const unsigned entry = unsigned(j) % page_size;
        const unsigned k_at = is ? unsigned(uint64_t(unsigned(page)) * k_page) + entry * k_token : 0u;
        const unsigned v_at = is ? unsigned(uint64_t(unsigned(page)) * v_page) + entry * v_token : 0u;
        const unsigned long long mask = __ballot(is);
        valid = unsigned(mask) & (A::kLoad == 32 ? 0xffffffffu : 0xffffu);
        if (WR > 1 && lane == 0) masks[stage][wave] = valid;
        const unsigned at = lds0 + unsigned(stage * A::kStage + wave * A::kLoad * A::kPitch);
#pragma unroll
        for (int u = 0; u < A::kLoads; ++u) {
            const int row = u * A::kPerLoad + in_load;   // of this wavefront's keys
            const int full = wave * A::kLoad + row;      // of the tile
            const unsigned k_row = __shfl(k_at, row), v_row = __shfl(v_at, row);
            const bool there = (valid >> row) & 1u;
            const int kp = piece ^ A::key_swizzle(full), vp = piece ^ A::value_swizzle(full);
            const char *ks = there && kp < pieces ? k_head + (uint64_t(k_row) + unsigned(kp)) * 16
                                                  : reinterpret_cast<const char *>(kNoData);
            const char *vs = there && vp < pieces ? v_head + (uint64_t(v_row) + unsigned(vp)) * 16
                                                  : reinterpret_cast<const char *>(kNoData);
            load_to_lds(ks, at + u * kWave * 16);
            load_to_lds(vs, at + A::kKeys * A::kPitch + u * kWave * 16);
        }
    };

    f32x4 o[RT][A::kTiles];
    float m[RT], sum[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -__builtin_inff();
        sum[r] = 0.0f;
#pragma unroll
        for (int d = 0; d < A::kTiles; ++d) o[r][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const float to_log2 = a.scale * 1.44269504088896f;

    int next_page = -1;
    if (tile0 < tile1) {
        fetch(tile0, 0, page_of(tile0));
        next_page = page_of(tile0 + 1);
    }
    for (int tile = tile0; tile < tile1; ++tile) {
        const int stage = (tile - tile0) & 1;
        const unsigned mine = valid;
        if (WR > 1)
            wait_loads_all();
        else
            wait_loads();
        if (tile + 1 < tile1) {
            fetch(tile + 1, stage ^ 1, next_page);
            next_page = page_of(tile + 2);
        }
        const char *keys = lds + stage * A::kStage + wk * 32 * A::kChunks * A::kPitch;
        const char *values = keys + A::kKeys * A::kPitch;
#pragma unroll
        for (int c = 0; c < A::kChunks; ++c) {
            const int key0 = tile * A::kKeys + (wk * A::kChunks + c) * 32;
            unsigned exists = mine;
            if (WR > 1) {
                const int first = (wk * A::kChunks + c) * 32 / A::kLoad;
                exists = masks[stage][first] | (A::kLoad == 16 ? masks[stage][first + 1] << 16 : 0u);
            }
            exists = __builtin_amdgcn_readfirstlane(exists);
            if (exists == 0) continue;
            // scores
            f32x4 x[RT][2];
#pragma unroll
            for (int r = 0; r < RT; ++r) x[r][0] = x[r][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int row = c * 32 + u * 16 + col;   // of this key group
                const int full = wk * 32 * A::kChunks + row;
#pragma unroll
                for (int k = 0; k < DK; ++k) {
                    const s16x8 kx = *reinterpret_cast<const s16x8 *>(
                        keys + row * A::kPitch + 16 * ((4 * k + quad) ^ A::key_swizzle(full)));
#pragma unroll
                    for (int r = 0; r < RT; ++r) x[r][u] = Matrix<T>::mul(kx, q[r][k], x[r][u]);
                }
            }
            const bool partial = exists != 0xffffffffu || (own && key0 + 32 > least);   // uniform
            s16x8 weights[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = x[r][e / 4][e % 4] * to_log2;
                if (partial) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int key = 16 * (e / 4) + 4 * quad + e % 4;
                        const bool sees = ((exists >> key) & 1u) && key0 + key < limit[r];
                        y[e] = sees ? y[e] : -__builtin_inff();
                    }
                }
                float top = y[0];
#pragma unroll
                for (int e = 1; e < 8; ++e) top = __builtin_fmaxf(top, y[e]);
                top = row_max(top);
                if (__ballot(top > m[r] + 8.0f)) {   // (also while m is -inf)
                    const float now = __builtin_fmaxf(m[r], top);
                    const float f = now == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m[r] - now);
                    m[r] = now;
                    sum[r] *= f;
#pragma unroll
                    for (int d = 0; d < A::kTiles; ++d) o[r][d] *= f;
                }
                const float base = m[r] == -__builtin_inff() ? 0.0f : m[r];
                float part = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = __builtin_amdgcn_exp2f(y[e] - base);
                    part += z;
                    weights[r][e] = short(from_float<T>(z).bits);
                }
                sum[r] += part;
            }
            // values
            const bool some_rows = own && key0 + 32 > least;   // a key that only some rows see
#pragma unroll
            for (int d = 0; d < A::kTiles; ++d) {
                s16x8 vx;
                bool odd = false;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int row = c * 32 + u * 16 + 4 * quad + col / 4;
                    const int full = wk * 32 * A::kChunks + row;
                    const char *at = values + row * A::kPitch + 16 * ((2 * d + ((col & 3) >> 1)) ^ A::value_swizzle(full)) +
                                     8 * (col & 1);
                    const s16x4 part = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr<s16x4>)(const_cast<char *>(at)));
#pragma unroll
                    for (int e = 0; e < 4; ++e) vx[4 * u + e] = part[e];
                }
                if (some_rows) {
                    // A value that is not finite must not reach the rows that do not see its key (0 * inf): it
                    // is left out here and added below to the rows that do.
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const bool bad = (vx[e] & Matrix<T>::kExponent) == Matrix<T>::kExponent;
                        odd |= bad;
                        vx[e] = bad ? short(0) : vx[e];
                    }
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) o[r][d] = Matrix<T>::mul(vx, weights[r], o[r][d]);
                if (some_rows && __ballot(odd)) {
                    for (int key = 0; key < 32; ++key) {
                        const int row = c * 32 + key, full = wk * 32 * A::kChunks + row;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int dim = 16 * d + 4 * quad + i;
                            const T v = *reinterpret_cast<const T *>(
                                values + row * A::kPitch + 16 * ((dim / 8) ^ A::value_swizzle(full)) + 2 * (dim % 8));
                            const bool bad = (short(v.bits) & Matrix<T>::kExponent) == Matrix<T>::kExponent;
#pragma unroll
                            for (int r = 0; r < RT; ++r) {
                                int z = 0;   // the row's weight of this key
#pragma unroll
                                for (int e = 0; e < 8; ++e) z = key / 16 * 4 + key % 4 == e ? weights[r][e] : z;
                                z = __shfl(z, key % 16 / 4 * 16 + col);
                                if (bad && key0 + key < limit[r])
                                    o[r][d][i] += to_float(T{uint16_t(z)}) * to_float(v);
                            }
                        }
                    }
                }
            }
        }
    }

#pragma unroll
    for (int r = 0; r < RT; ++r) sum[r] = row_sum4(sum[r]);

    // The wavefronts that share rows join their parts.
    if (WK > 1) {
        wait_loads_all();   // nothing reads or loads a tile any more
        float *box = reinterpret_cast<float *>(lds);             // [WR][RT * 16][kDims], one key group's turn
        __shared__ float join[2][WK][WR * RT * 16];
#pragma unroll
        for (int r = 0; r < RT; ++r)
            if (quad == 0) {
                join[0][wk][(wr * RT + r) * 16 + col] = m[r];
                join[1][wk][(wr * RT + r) * 16 + col] = sum[r];
            }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int at = (wr * RT + r) * 16 + col;
            float top = join[0][0][at], total = 0.0f;
#pragma unroll
            for (int k = 1; k < WK; ++k) top = __builtin_fmaxf(top, join[0][k][at]);
            const float base = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
            for (int k = 0; k < WK; ++k) total += join[1][k][at] * __builtin_amdgcn_exp2f(join[0][k][at] - base);
            const float f = __builtin_amdgcn_exp2f(m[r] - base);
#pragma unroll
            for (int d = 0; d < A::kTiles; ++d) o[r][d] *= f;
            m[r] = top;
            sum[r] = total;
        }
        // key group 0 collects: the others write, group after group of dimensions is summed by all
        constexpr int kGroup = WR * RT * 16 * A::kDims;   // floats of one key group
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int d = 0; d < A::kTiles; ++d)
                *reinterpret_cast<f32x4 *>(box + wk * kGroup + ((wr * RT + r) * A::kTiles + d) * 256 + lane * 4) = o[r][d];
        __syncthreads();
        if (wk == 0) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int d = 0; d < A::kTiles; ++d)
#pragma unroll
                    for (int k = 1; k < WK; ++k)
                        o[r][d] += *reinterpret_cast<const f32x4 *>(
                            box + k * kGroup + ((wr * RT + r) * A::kTiles + d) * 256 + lane * 4);
        }
        if (wk != 0) return;
    }

    const int64_t all_rows = a.S * a.T * a.q_heads;
    const int part = (own ? plan.prefix.splits : 0) + split;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (out_row[r] < 0) continue;
        if (plan.parts > 1) {
            if (quad == 0) plan.stats[part * all_rows + out_row[r]] = make_float2(m[r], sum[r]);
            if (sum[r] == 0.0f) continue;
            float *dst = plan.sums + (part * all_rows + out_row[r]) * D;
#pragma unroll
            for (int d = 0; d < A::kTiles; ++d)
                if (const int at = 16 * d + 4 * quad; at < D) *reinterpret_cast<f32x4 *>(dst + at) = o[r][d];
        } else {
            const bool any = counts[r] && sum[r] != 0.0f;   // (a NaN sum too)
            if (a.lse && quad == 0)
                a.lse[out_row[r]] = any ? (m[r] == -__builtin_inff() ? sum[r] : m[r] * 0.69314718056f + logf(sum[r]))
                                        : -__builtin_inff();
            T *dst = static_cast<T *>(a.out) + out_row[r] * D;
            const float f = 1.0f / sum[r];
#pragma unroll
            for (int d = 0; d < A::kTiles; ++d) {
                if (const int at = 16 * d + 4 * quad; at < D) {
                    s16x4 y;
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = any ? short(from_float<T>(o[r][d][i] * f).bits) : short(0);
                    *reinterpret_cast<s16x4 *>(dst + at) = y;
                }
            }
        }
    }
}

}  // namespace ngpu
