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
    static __device__ __forceinline__ s16x8 round(const float (&x)[8]) {
        typedef __bf16 v8 __attribute__((ext_vector_type(8)));
        typedef float f8 __attribute__((ext_vector_type(8)));
        return __builtin_bit_cast(s16x8, __builtin_convertvector(f8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]}, v8));
    }
};
template <>
struct Matrix<F16> {
    static constexpr short kExponent = 0x7c00;
    static __device__ __forceinline__ f32x4 mul(s16x8 a, s16x8 b, f32x4 c) {
        typedef _Float16 v8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ s16x8 round(const float (&x)[8]) {
        typedef _Float16 v8 __attribute__((ext_vector_type(8)));
        typedef float f8 __attribute__((ext_vector_type(8)));
        return __builtin_bit_cast(s16x8, __builtin_convertvector(f8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]}, v8));
    }
};

// Maximum over the four lanes that hold a row (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float row_max(float x) {
    auto both = [](auto r) { return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])); };
    x = both(__builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return both(__builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
}

// The sum of the four, alike in each.
__device__ __forceinline__ float row_sum(float x) {
    auto both = [](auto r) { return __uint_as_float(r[0]) + __uint_as_float(r[1]); };
    x = both(__builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return both(__builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
}

// Waits for everything this wavefront has loaded (registers and LDS).
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void wait_loads_all() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// 16 bytes a lane from memory to LDS at `at` + 16 lane (uniform `at`).  As asm, since
// the compiler would wait for it before any later LDS load.  (m0 is a reserved register, which
// nothing else in these kernels uses: a clobber would only be warned about.)
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const void *p, unsigned at) {
    if (ONCE)
        asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(at), "v"(p) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(p) : "memory");
}

// The same from a uniform address and a lane's offset.
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const void *base, unsigned offset, unsigned at) {
    if (ONCE)
        asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(at), "v"(offset), "s"(base) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(offset), "s"(base) : "memory");
}

// DK: 32-dimension steps of a head; RT: tiles of 16 rows a wavefront; WR:
// wavefronts, each with rows of its own, that share the tiles of keys.
template <class T, int DK, int RT, int WR>
struct AttendTile {
    static constexpr int kChunks = WR > 2 ? 2 : 1;              // of 32 keys, a tile
    static constexpr int kKeys = 32 * kChunks;                  // a tile
    static constexpr int kLoad = kKeys / WR;                // keys a wavefront loads
    static constexpr int kRows = 16 * RT * WR;                  // a workgroup
    static constexpr int kPitch = DK <= 2 ? 128 : (DK <= 4 ? 256 : 512);   // bytes of a row in LDS
    static constexpr int kPieces = kPitch / 16;                 // 16-byte chunks of it
    static constexpr int kStage = 2 * kKeys * kPitch;           // keys, then values
    static constexpr int kLds = 2 * kStage;
    static constexpr int kPerLoad = kWave / kPieces;            // rows a load instruction brings
    static constexpr int kLoads = kLoad / kPerLoad;
    static constexpr bool kOnce = WR == 1;                      // no other workgroup reads these keys
    static constexpr int kTiles = 2 * DK;                       // of 16 dimensions
    static_assert(kLoad == 16 || kLoad == 32, "a wavefront's lanes hold its keys' pages");

    static __device__ __forceinline__ int key_swizzle(int row) { return kPieces == 8 ? (row >> 1) & 7 : row & 15; }
    static __device__ __forceinline__ int value_swizzle(int row) {
        return kPieces == 8 ? ((row >> 1) & 3) << 1 : (row & 7) << 1;
    }
};

// Registers are held to what two workgroups of four wavefronts a CU leave each where that spills nothing.
template <class T, int DK, int RT, int WR>
__global__ __launch_bounds__(64 * WR, DK <= 4 ? 2 : 1) void attend_tile_kernel(Attend p, AttendPlan plan,
                                                                                   unsigned work0) {
    using A = AttendTile<T, DK, RT, WR>;
    using M = Matrix<T>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    unsigned (*masks)[4] = nullptr;   // per stage, the keys of each loading wavefront that exist
    if constexpr (WR > 1) {
        __shared__ unsigned shared_masks[2][4];
        masks = shared_masks;
    }
    const unsigned lds0 = unsigned(reinterpret_cast<uintptr_t>((LdsPtr<char>)lds));
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane % 16, quad = lane / 16;
    const ngpu_attend_t &a = p.a;
    const int H = p.c.heads, rep = a.q_heads / H, D = p.c.dim, T_ = int(a.T);

    // Workgroups go to the 8 XCDs in turn.  Each XCD takes a run of the prefixes'
    // works, which share keys (row blocks) or rows of pages (heads) in its L2.
    const unsigned prefix_works = unsigned(plan.prefix.works());
    unsigned w = work0 + blockIdx.x;
    const bool own = w >= prefix_works;
    const Cut &cut = own ? plan.own : plan.prefix;
    if (own)
        w -= prefix_works;
    else
        w = w % 8 * (prefix_works / 8) + min(w % 8, prefix_works % 8) + w / 8;
    const int block = int(w % unsigned(cut.blocks));
    w /= unsigned(cut.blocks);
    const int h = int(w % unsigned(H));
    w /= unsigned(H);
    const int split = int(w % unsigned(cut.splits)), g = int(w / unsigned(cut.splits));
    const int beam = own ? 1 : int(a.S / a.G), s0 = g * beam;
    const unsigned rows = unsigned(beam) * T_ * rep;   // (all rows of a call are below 2^31)
    const PageTable table = own ? own_table(p, s0) : prefix_table(p, g);
    const int count = int(table.count);

    // this split's keys
    const int tiles = (count + A::kKeys - 1) / A::kKeys, per = (tiles + cut.splits - 1) / cut.splits;
    const int tile0 = min(tiles, split * per), tile1 = min(tiles, tile0 + per);

    // A lane's key of a tile: its row of the cache in 16-byte units.
    const unsigned page_size = unsigned(p.c.page_size);
    const int my_key = wave * A::kLoad + lane % A::kLoad;
    auto page_of = [&](int tile) {
        const int j = tile * A::kKeys + my_key;
        return tile < tile1 && j < count ? table.pages[unsigned(j) / page_size] : -1;
    };
    int page = page_of(tile0), next_page = page_of(tile0 + 1);

    // this wavefront's query rows: operand registers, and the keys each row sees
    s16x8 q[RT][DK];
    int limit[RT];
    int out_row[RT];   // -1: no row
    bool counts[RT];   // a query token that counts
    const bool aligned = (reinterpret_cast<uintptr_t>(a.q) % 16 == 0) && a.q_stride_seq % 8 == 0 &&
                         a.q_stride_token % 8 == 0 && a.q_stride_head % 8 == 0;
    const short flip = a.scale < 0.0f ? short(0x8000) : short(0);   // the scores' sign, so that the factor is not negative
    int least = count;   // keys that every row of the workgroup's sequences sees
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const unsigned row = unsigned(block) * A::kRows + (wave * RT + r) * 16 + col;
        const bool is = row < rows;
        const unsigned i = is ? row : 0, token = i / unsigned(rep);
        const int s = s0 + int(token / unsigned(T_)), t = int(token % unsigned(T_));
        const int head = h * rep + int(i - token * unsigned(rep));
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
            q[r][k] = x ^ flip;
        }
    }
    least = __builtin_amdgcn_readfirstlane(least);

    const uint64_t k_page = uint64_t(p.c.k_stride_page) / 8, v_page = uint64_t(p.c.v_stride_page) / 8;
    const unsigned k_token = unsigned(p.c.k_stride_token / 8), v_token = unsigned(p.c.v_stride_token / 8);
    const char *k_head = static_cast<const char *>(p.c.k) + int64_t(h) * p.c.k_stride_head * 2;
    const char *v_head = static_cast<const char *>(p.c.v) + int64_t(h) * p.c.v_stride_head * 2;
    const int piece = lane % A::kPieces, in_load = lane / A::kPieces;
    // Where a wavefront's keys lie in one page and a row has no missing
    // dimensions, a lane's offsets are the same for every tile.
    const bool in_page = page_size % A::kLoad == 0 && D == 32 * DK && k_token < (1u << 21) && v_token < (1u << 21);
    unsigned k_off[A::kLoads], v_off[A::kLoads];
#pragma unroll
    for (int u = 0; u < A::kLoads; ++u) {
        const int row = u * A::kPerLoad + in_load, full = wave * A::kLoad + row;
        k_off[u] = (unsigned(row) * k_token + unsigned(piece ^ A::key_swizzle(full))) * 16;
        v_off[u] = (unsigned(row) * v_token + unsigned(piece ^ A::value_swizzle(full))) * 16;
    }
    unsigned valid = 0;   // keys that exist among those this wavefront loaded last
    auto fetch = [&](int tile, int stage) {
        const bool is = page >= 0 && page < p.c.num_pages;   // (-1 past the end)
        const unsigned long long mask = __ballot(is);
        constexpr unsigned kAll = A::kLoad == 32 ? 0xffffffffu : 0xffffu;
        valid = unsigned(mask) & kAll;
        if (WR > 1 && lane == 0) masks[stage][wave] = valid;
        const unsigned at = __builtin_amdgcn_readfirstlane(lds0 + unsigned(stage * A::kStage + wave * A::kLoad * A::kPitch));
        const unsigned entry = unsigned(tile * A::kKeys + my_key) % page_size;
        if (in_page && valid == kAll) {
            const unsigned e0 = __builtin_amdgcn_readfirstlane(entry), p0 = __builtin_amdgcn_readfirstlane(page);
            const char *kb = k_head + (p0 * k_page + e0 * uint64_t(k_token)) * 16;
            const char *vb = v_head + (p0 * v_page + e0 * uint64_t(v_token)) * 16;
#pragma unroll
            for (int u = 0; u < A::kLoads; ++u) {
                const int full = wave * A::kLoad + u * A::kPerLoad + in_load;
                if (4 * DK == A::kPieces || (piece ^ A::key_swizzle(full)) < 4 * DK)
                    load_to_lds<A::kOnce>(kb, k_off[u], at + u * kWave * 16);
                if (4 * DK == A::kPieces || (piece ^ A::value_swizzle(full)) < 4 * DK)
                    load_to_lds<A::kOnce>(vb, v_off[u], at + A::kKeys * A::kPitch + u * kWave * 16);
            }
            return;
        }
        const unsigned k_at = is ? unsigned(unsigned(page) * k_page) + entry * k_token : 0u;
        const unsigned v_at = is ? unsigned(unsigned(page) * v_page) + entry * v_token : 0u;
        const int pieces = D / 8;
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
            load_to_lds<A::kOnce>(ks, at + u * kWave * 16);
            load_to_lds<A::kOnce>(vs, at + A::kKeys * A::kPitch + u * kWave * 16);
        }
    };

    // this lane's places in a tile: the operand rows of K and the blocks of V
    unsigned k_at[DK], v_at[A::kTiles];
#pragma unroll
    for (int k = 0; k < DK; ++k) k_at[k] = unsigned(col * A::kPitch + 16 * ((4 * k + quad) ^ A::key_swizzle(col)));
#pragma unroll
    for (int d = 0; d < A::kTiles; ++d) {
        const int row = 4 * quad + col / 4;
        v_at[d] = unsigned(row * A::kPitch + 16 * ((2 * d + (col % 4) / 2) ^ A::value_swizzle(row)) + 8 * (col & 1));
    }

    f32x4 o[RT][A::kTiles];
    float m[RT], sum[RT];   // sum: of the weights of this lane's keys, before they are rounded
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -__builtin_inff();
        sum[r] = 0.0f;
#pragma unroll
        for (int d = 0; d < A::kTiles; ++d) o[r][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const float to_log2 = __builtin_fabsf(a.scale) * 1.44269504088896f;

    if (tile0 < tile1) fetch(tile0, 0);
    for (int tile = tile0; tile < tile1; ++tile) {
        const int stage = (tile - tile0) & 1;
        const unsigned mine = valid;
        if (WR > 1)
            wait_loads_all();
        else
            wait_loads();
        if (tile + 1 < tile1) {
            page = next_page;
            next_page = page_of(tile + 2);
            fetch(tile + 1, stage ^ 1);
        }
        const char *keys = lds + stage * A::kStage;
        const char *values = keys + A::kKeys * A::kPitch;
        const int key0 = tile * A::kKeys;
        // which of the keys exist
        unsigned exists[A::kChunks];
        bool partial = own && key0 + 32 * A::kChunks > least;   // some rows do not see some of them
        const bool some_rows = partial;
#pragma unroll
        for (int c = 0; c < A::kChunks; ++c) {
            exists[c] = mine;
            if (WR > 1) {
                const int first = c * 32 / A::kLoad;
                exists[c] = masks[stage][first] | (A::kLoad == 16 ? masks[stage][first + 1] << 16 : 0u);
            }
            exists[c] = __builtin_amdgcn_readfirstlane(exists[c]);
            partial |= exists[c] != 0xffffffffu;
        }

        f32x4 x[RT][2 * A::kChunks];
#pragma unroll
        for (int k = 0; k < DK; ++k)
#pragma unroll
            for (int u = 0; u < 2 * A::kChunks; ++u) {
                const s16x8 kx = *reinterpret_cast<const s16x8 *>(keys + u * 16 * A::kPitch + k_at[k]);
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    x[r][u] = M::mul(kx, q[r][k], k == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : x[r][u]);
            }
        s16x8 weights[RT][A::kChunks];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if (partial) {
#pragma unroll
                for (int e = 0; e < 8 * A::kChunks; ++e) {
                    const int key = 16 * (e / 4 % 2) + 4 * quad + e % 4;
                    const bool sees = ((exists[e / 8] >> key) & 1u) && key0 + e / 8 * 32 + key < limit[r];
                    x[r][e / 4][e % 4] = sees ? x[r][e / 4][e % 4] : -__builtin_inff();
                }
            }
            float top = x[r][0][0];
#pragma unroll
            for (int e = 1; e < 8 * A::kChunks; ++e) top = __builtin_fmaxf(top, x[r][e / 4][e % 4]);
            top *= to_log2;
            if (__ballot(top > m[r] + 8.0f)) {   // (also while m is -inf)
                const float now = __builtin_fmaxf(m[r], row_max(top));
                const float f = now == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m[r] - now);
                m[r] = now;
                sum[r] *= f;
#pragma unroll
                for (int d = 0; d < A::kTiles; ++d) o[r][d] *= f;
            }
            const float base = m[r] == -__builtin_inff() ? 0.0f : m[r];
#pragma unroll
            for (int c = 0; c < A::kChunks; ++c) {
                float z[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    z[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r][2 * c + e / 4][e % 4], to_log2, -base));
                if (partial) {   // (a score of -inf times a factor of 0 is NaN)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int key = 16 * (e / 4) + 4 * quad + e % 4;
                        z[e] = ((exists[c] >> key) & 1u) && key0 + c * 32 + key < limit[r] ? z[e] : 0.0f;
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[r] += z[e];
                weights[r][c] = M::round(z);
            }
        }
#pragma unroll
        for (int c = 0; c < A::kChunks; ++c) {
#pragma unroll
            for (int d = 0; d < A::kTiles; ++d) {
                s16x8 vx;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const s16x4 part = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (LdsPtr<s16x4>)(const_cast<char *>(values + (c * 32 + u * 16) * A::kPitch + v_at[d])));
#pragma unroll
                    for (int e = 0; e < 4; ++e) vx[4 * u + e] = part[e];
                }
                if (some_rows) {
                    // A value that is not finite must not reach the rows that do not see its key (0 * inf): it
                    // is left out here and added below to the rows that do.
                    bool odd = false;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const bool bad = (vx[e] & M::kExponent) == M::kExponent;
                        odd |= bad;
                        vx[e] = bad ? short(0) : vx[e];
                    }
                    if (__ballot(odd)) {
                        for (int key = 0; key < 32; ++key) {
                            const int row = c * 32 + key;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int dim = 16 * d + 4 * quad + i;
                                const T v = *reinterpret_cast<const T *>(
                                    values + row * A::kPitch + 16 * ((dim / 8) ^ A::value_swizzle(row)) + 2 * (dim % 8));
                                const bool bad = (short(v.bits) & M::kExponent) == M::kExponent;
#pragma unroll
                                for (int r = 0; r < RT; ++r) {
                                    int z = 0;   // the row's weight of this key
#pragma unroll
                                    for (int e = 0; e < 8; ++e) z = key / 16 * 4 + key % 4 == e ? weights[r][c][e] : z;
                                    z = __shfl(z, key % 16 / 4 * 16 + col);
                                    if (bad && key0 + row < limit[r])
                                        o[r][d][i] += to_float(T{uint16_t(z)}) * to_float(v);
                                }
                            }
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) o[r][d] = M::mul(vx, weights[r][c], o[r][d]);
            }
        }
    }

    float total[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) total[r] = row_sum(sum[r]);
    const int64_t all_rows = a.S * a.T * a.q_heads;
    const int part = (own ? plan.prefix.splits : 0) + split;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (out_row[r] < 0) continue;
        if (plan.parts > 1) {
            if (quad == 0) plan.stats[part * all_rows + out_row[r]] = make_float2(m[r], total[r]);
            if (total[r] == 0.0f) continue;
            float *dst = plan.sums + (part * all_rows + out_row[r]) * D;
#pragma unroll
            for (int d = 0; d < A::kTiles; ++d)
                if (const int at = 16 * d + 4 * quad; at < D) *reinterpret_cast<f32x4 *>(dst + at) = o[r][d];
        } else {
            const bool any = counts[r] && total[r] != 0.0f;   // (a NaN sum too)
            if (a.lse && quad == 0)
                a.lse[out_row[r]] = any ? (m[r] == -__builtin_inff() ? total[r] : m[r] * 0.69314718056f + logf(total[r]))
                                        : -__builtin_inff();
            T *dst = static_cast<T *>(a.out) + int64_t(out_row[r]) * D;
            const float f = 1.0f / total[r];
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
