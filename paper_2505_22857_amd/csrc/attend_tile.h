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
// order.  K and V go from memory straight to LDS, two tiles in turn; 16-byte
// chunks of a row are stored at their place XOR the row, which leaves neither
// load a bank conflict.
//
// The running maximum of a row is raised only when a score exceeds it by more
// than 2^8 (the weights then stay below 2^8, and their sum's rounding is the
// same): otherwise the accumulators need no rescaling.  Scores, sums and
// accumulators are fp32; the weights are rounded to the cache's type, which the
// matrix instructions need, before they multiply V, which makes the result's error 1.3
// (half) to 1.4 (bfloat16) times that of fp32 weights.  A half rounds what is below
// 2^-25 to zero, which many keys far below one would miss: its weights are
// taken 2^7 higher, up to 2^15, so that one counts down to 2^-32 of the row's largest.
//
// What bounds it depends on the rows.  Few: reading the cache, once (3 prefixes of
// 100000 tokens for 5 x 4 rows, 8 heads of 128, bf16: 197 to 204 us, 1.24 GB at 6.1
// to 6.3 TB/s, 0.9 of a fill's rate).  Many: the matrix instructions, the exponentials between
// them and LDS's reads, which take about as long as the first, share a SIMD's two
// wavefronts (4 x 384 rows: 7.4 us per 1024 tokens of prefix, 870 TFLOP/s, behind 24 us
// for launches, first loads, partial sums and their join; 32768 tokens ran at 630 to 710 in
// all).  Short ones: the chain of page table, first tile and join.
//
// A cache in 8 bits (Attend8).  An element stands for e s, s the scale of its block of tokens and its head, so
// that S = (q . e_k) s_k and O = sum_k (w_k s_k) e_v: the scales are numbers of a key, which a lane has four
// of, and no product of theirs reaches the elements.  These go to LDS as they are; a key's 16 bytes are a lane's
// dimensions of two steps and are widened after the load, which is exact, values by the transposing load of
// bytes.  Scales go to LDS beside their tile, one a key.  w s is split into two bfloat16 (2^-17 of it is lost):
// with one the result's error was 1.35 to 1.58 times that of fp32 weights, which it now equals, for 4 %
// of the time of many rows; halves would need one, but not every s leaves w s in their range.
// Reading is bound as above at half the bytes (4 prefixes of 120000 tokens for 2 x 4 rows, 8 heads of 128: 170 us, 988 MB at
// 5.8 TB/s); many rows by vector instructions, 620 a tile of 64 keys and 32 rows beside 96 of the matrix
// cores, with two wavefronts a SIMD (4 groups of 60 tokens that see up to 7000 of prefix and 300, 32 / 8 heads of 128:
// 65 to 68 us a call among others, 72 to 73 in a graph; 585 TFLOP/s behind 17 us for launches, first tiles, partial sums and join; one group of 128 that sees
// 20000: 480 in all).
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "cache.h"
#include "values8.h"
#include "walk.h"

namespace ngpu {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));

typedef int i32x2 __attribute__((ext_vector_type(2)));

struct Attend {
    ngpu_kv_cache_t c;
    ngpu_attend_t a;
};
// The same over a cache in 8 bits.
struct Attend8 : Attend {
    const float *k_scale, *v_scale;
    int64_t k_scale_page, k_scale_block, k_scale_head, v_scale_page, v_scale_block, v_scale_head;
    unsigned block, block_magic;   // tokens a scale; floor(2^32 / that), 2^32 - 1 for 1
};
// Of a call whose cache holds elements of type C, queries and output of type T.
template <class C>
using AttendOf = std::conditional_t<std::is_same_v<C, E4m3>, Attend8, Attend>;

// n / d, by floor(2^32 / d) (2^32 - 1 for d = 1): the product is up to one too low.
__device__ __forceinline__ unsigned divided(unsigned n, unsigned d, unsigned magic) {
    const unsigned i = __umulhi(n, magic);
    return n - i * d >= d ? i + 1 : i;
}

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
    int parts;           // most splits of a problem: splits, or more where they are dealt by length
    __host__ __device__ int64_t works() const { return problems * blocks * splits; }
};

// Most groups whose splits are dealt by their lengths: a lane holds one.
constexpr int kDealt = kWave;

// The splits of the group in this lane, of those the call has for all groups
// together: one each, and the rest by length, so that a workgroup's share of the
// keys hardly depends on its group.  For the whole wavefront; G <= kDealt.
__device__ __forceinline__ int dealt_splits(const Cut &cut, int G, int64_t length) {
    unsigned units = unsigned(length + 63) / 64;
    unsigned total = units;
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) total += __shfl_xor(total, d);
    const int lane = threadIdx.x % kWave, spare = G * (cut.splits - 1);
    const int coarse = max(0, 14 - int(__builtin_clz(total | 1)));   // so that the product fits 32 bits
    const int share = total > 0 ? int(unsigned(spare) * (units >> coarse) / (total >> coarse)) : cut.splits - 1;
    return lane < G ? min(1 + share, cut.parts) : 0;
}

struct AttendPlan {
    Cut prefix, own;
    int parts;           // of both: most partial results a row
    unsigned page_magic; // floor(2^32 / page size), 2^32 - 1 for 1: a key's page up to one too low
    float *sums;         // [parts, rows, dim] sums of weight times v around the part's maximum
    float2 *stats;       // [parts, rows] {maximum in log2, sum of weights}
};

// 16 bytes of zeros, which stand for keys and dimensions that do not exist, and for such keys' scales.
static __device__ __attribute__((aligned(16))) unsigned kNoData[4];

// One row's running maximum (in log2) and sums, a wavefront's lanes holding every
// 64th dimension: for what the matrix instructions do not take.
template <class T, class C>
struct RowPart {
    static constexpr int kDims = NGPU_LM_MAX_HEAD_DIM / kWave;
    float q[kDims], o[kDims], m = -__builtin_inff(), sum = 0.0f;
    __device__ __forceinline__ void load(const Attend &p, int64_t s, int64_t t, int head, int lane) {
        const T *src = static_cast<const T *>(p.a.q) + s * p.a.q_stride_seq + t * p.a.q_stride_token +
                       head * p.a.q_stride_head;
#pragma unroll
        for (int i = 0; i < kDims; ++i) {
            q[i] = lane + kWave * i < p.c.dim ? to_float(src[lane + kWave * i]) : 0.0f;
            o[i] = 0.0f;
        }
    }
    __device__ __forceinline__ void take(const AttendOf<C> &p, const PageTable &table, int64_t j, int kv, int lane) {
        int64_t entry;
        const int64_t page = table.page(p.c, j, entry);
        if (page < 0) return;
        const C *k = static_cast<const C *>(p.c.k) + page * p.c.k_stride_page + entry * p.c.k_stride_token +
                     kv * p.c.k_stride_head;
        const C *v = static_cast<const C *>(p.c.v) + page * p.c.v_stride_page + entry * p.c.v_stride_token +
                     kv * p.c.v_stride_head;
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < kDims; ++i)
            if (const int d = lane + kWave * i; d < p.c.dim) x = __builtin_fmaf(q[i], to_float(k[d]), x);
        for (int d = kWave / 2; d > 0; d /= 2) x += __shfl_xor(x, d);
        x *= p.a.scale * 1.44269504088896f;
        float vs = 1.0f;
        if constexpr (std::is_same_v<C, E4m3>) {
            const int64_t block = entry / p.block;
            x *= p.k_scale[page * p.k_scale_page + block * p.k_scale_block + kv * p.k_scale_head];
            vs = p.v_scale[page * p.v_scale_page + block * p.v_scale_block + kv * p.v_scale_head];
        }
        if (!(x <= m)) {   // a NaN score makes the row NaN
            const float f = __builtin_amdgcn_exp2f(m - x);
            sum *= f;
#pragma unroll
            for (int i = 0; i < kDims; ++i) o[i] *= f;
            m = x;
        }
        const float w = x == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(x - m);
        sum += w;
        const float by = w * vs;
#pragma unroll
        for (int i = 0; i < kDims; ++i)
            if (const int d = lane + kWave * i; d < p.c.dim) o[i] = __builtin_fmaf(by, to_float(v[d]), o[i]);
    }
    // the finished row; `counts`: of a query token that counts
    __device__ __forceinline__ void finish(const Attend &p, int64_t row, int lane, bool counts) const {
        const bool any = counts && sum != 0.0f;   // (a NaN sum too)
        if (p.a.lse && lane == 0) p.a.lse[row] = any ? m * 0.69314718056f + logf(sum) : -__builtin_inff();
        T *dst = static_cast<T *>(p.a.out) + row * p.c.dim;
#pragma unroll
        for (int i = 0; i < kDims; ++i)
            if (const int d = lane + kWave * i; d < p.c.dim) dst[d] = from_float<T>(any ? o[i] / sum : 0.0f);
    }
};

template <class T>
using LdsPtr = __attribute__((address_space(3))) T *;

template <class T>
struct Matrix;
template <>
struct Matrix<Bf16> {
    static constexpr unsigned short kInfinity = 0x7f80;   // its bits
    static constexpr float kRoom = 0.0f;                  // of its exponents above the weights', see above
    static __device__ __forceinline__ f32x4 mul(s16x8 a, s16x8 b, f32x4 c) {
        typedef __bf16 v8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned round(float a, float b) {
        typedef __bf16 v2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(unsigned, v2{__bf16(a), __bf16(b)});
    }
    // eight e4m3 values, which bfloat16 and half hold exactly
    static __device__ __forceinline__ s16x8 widen(int a, int b) {
        return __builtin_bit_cast(s16x8, u32x4{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false)),
                                               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true)),
                                               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false)),
                                               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true))});
    }
};
template <>
struct Matrix<F16> {
    static constexpr unsigned short kInfinity = 0x7c00;
    static constexpr float kRoom = 7.0f;
    static __device__ __forceinline__ f32x4 mul(s16x8 a, s16x8 b, f32x4 c) {
        typedef _Float16 v8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned round(float a, float b) {
        typedef _Float16 v2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(unsigned, v2{_Float16(a), _Float16(b)});
    }
    static __device__ __forceinline__ s16x8 widen(int a, int b) {
        return __builtin_bit_cast(s16x8, u32x4{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false)),
                                               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true)),
                                               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false)),
                                               __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true))});
    }
};

template <class T>
__device__ __forceinline__ LdsPtr<T> lds_at(unsigned at) {
    return (LdsPtr<T>)(uintptr_t)at;
}

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

// Waits for this wavefront's loads from memory and its LDS loads and stores.
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
// 16 bytes a lane from memory to LDS at `at` + 16 lane (uniform `at`).  As asm, since
// the compiler would wait for it before any later LDS load.  (m0 is a reserved register, which
// nothing else in these kernels uses: a clobber would only be warned about.)  The load has to come a
// wait state after the write of m0, and the compiler adds none inside the asm.
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const void *p, unsigned at) {
    if (ONCE)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(at), "v"(p) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(p) : "memory");
}

// A uniform address in scalar registers (the compiler may hold it in vector ones).
__device__ __forceinline__ uint64_t uniform_address(const void *p) {
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return uint64_t(unsigned(__builtin_amdgcn_readfirstlane(int(a >> 32)))) << 32 |
           unsigned(__builtin_amdgcn_readfirstlane(int(a)));
}
// The same from a uniform address and a lane's offset.  Where the address was read from vector registers the load
// has to come five wait states after that: the move and four of the s_nop.
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const void *from, unsigned offset, unsigned at) {
    const uint64_t base = uniform_address(from);
    if (ONCE)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(at), "v"(offset), "s"(base) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(offset), "s"(base) : "memory");
}
// Two of these, which share the wait: 3 prefixes of 100000 tokens as above 202 us, 210 one by one.
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const void *from0, unsigned offset0, unsigned at0, const void *from1,
                                            unsigned offset1, unsigned at1) {
    const uint64_t base0 = uniform_address(from0), base1 = uniform_address(from1);
    if (ONCE)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2 nt\n\t"
                     "s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %5 nt"
                     ::"s"(at0), "v"(offset0), "s"(base0), "s"(at1), "v"(offset1), "s"(base1) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2\n\t"
                     "s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %5"
                     ::"s"(at0), "v"(offset0), "s"(base0), "s"(at1), "v"(offset1), "s"(base1) : "memory");
}

// 4 bytes a lane from memory to LDS at `at` + 4 lane, as above.
__device__ __forceinline__ void load_word_to_lds(const void *p, unsigned at) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(at), "v"(p) : "memory");
}

// Steps that operands are loaded from LDS before the matrix instructions that take them.
constexpr int kKeysAhead = 2, kValuesAhead = 3;

// DK: 32-dimension steps of a head; RT: tiles of 16 rows a wavefront; WR:
// wavefronts, each with rows of its own, that share the tiles of keys.  Two stages: three and four,
// or tiles of 32 keys for four wavefronts, were no faster.
template <class T, class C, int DK, int RT, int WR>
struct AttendTile {
    static constexpr bool kEight = std::is_same_v<C, E4m3>;
    static constexpr int kPer = 16 / int(sizeof(C));            // elements of a 16-byte chunk
    static constexpr int kChunks = WR > 2 ? 2 : 1;              // of 32 keys, a tile
    static constexpr int kKeys = 32 * kChunks;                  // a tile
    static constexpr int kLoad = kKeys / WR;                // keys a wavefront loads
    static constexpr int kRows = 16 * RT * WR;                  // a workgroup
    static constexpr int kPitch = (DK <= 2 ? 64 : (DK <= 4 ? 128 : 256)) * int(sizeof(C));   // bytes of a row in LDS
    static constexpr int kPieces = kPitch / 16;                 // 16-byte chunks of it
    static constexpr int kUsed = 32 * DK / kPer;                // of which DK steps read
    static constexpr int kStage = 2 * kKeys * kPitch + (kEight ? 8 * kKeys : 0);   // keys, values, and their scales
    static constexpr int kStages = 2;                           // tiles in LDS: one in use, the other on its way
    static constexpr int kLds = kStages * kStage;
    static constexpr int kPerLoad = kWave / kPieces;            // rows a load instruction brings
    static constexpr int kLoads = kLoad / kPerLoad;
    static constexpr bool kOnce = WR == 1;                      // its problem's only block of rows: keys are read once
    static constexpr int kTiles = 2 * DK;                       // of 16 dimensions
    static_assert(kKeysAhead <= DK && kValuesAhead <= kTiles, "the first steps lie in the first chunk");
    static_assert(kLoad == (WR == 1 ? 32 : 16), "a wavefront's keys are half of a mask where several share it");

    static __device__ __forceinline__ int key_swizzle(int row) {
        return kPieces == 4 ? (row >> 2) & 3 : (kPieces == 8 ? (row >> 1) & 7 : row & 15);
    }
    static __device__ __forceinline__ int value_swizzle(int row) {
        if (kEight)   // a transposing load of 8 bits reads rows 0 to 3 and 16 to 19 of its 32 with a quarter of the lanes
            return kPieces == 4 ? ((row >> 2) & 1) | ((row >> 3) & 2)
                                : (kPieces == 8 ? ((row >> 1) & 3) | ((row >> 2) & 4) : (row & 7) | ((row >> 1) & 8));
        return kPieces == 8 ? ((row >> 1) & 3) << 1 : (row & 7) << 1;
    }
};

// The kernel's arguments for what follows its loop.  Of a cache in 8 bits they are read again: beside what the loop needs
// they do not fit the scalar registers.
template <class C>
struct LastArgs {
    const AttendOf<C> &p;
    const AttendPlan &plan;
    __device__ __forceinline__ LastArgs(const AttendOf<C> &p, const AttendPlan &plan) : p(p), plan(plan) {}
};
template <>
struct LastArgs<E4m3> {
    struct Args {   // as they lie in memory
        Attend8 p;
        AttendPlan plan;
    };
    const Attend8 &p;
    const AttendPlan &plan;
    __device__ __forceinline__ LastArgs(const Attend8 &, const AttendPlan &) : LastArgs(*read()) {}

private:
    __device__ __forceinline__ explicit LastArgs(const Args &a) : p(a.p), plan(a.plan) {}
    static __device__ __forceinline__ const Args *read() {
        const Args *args = (const Args *)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(args));
        return args;
    }
};

// Work `w` of the plan, for WR wavefronts with LDS from `lds0` on.
template <class T, class C, int DK, int RT, int WR>
__device__ __forceinline__ void attend_tiles(const AttendOf<C> &p, const AttendPlan &plan, unsigned w, unsigned lds0) {
    using A = AttendTile<T, C, DK, RT, WR>;
    using M = Matrix<T>;
    unsigned (*masks)[A::kChunks] = nullptr;   // per stage, a bit for each key that exists
    if constexpr (WR > 1) {
        __shared__ unsigned shared_masks[A::kStages][A::kChunks];
        masks = shared_masks;
    }
    const int lane = threadIdx.x % kWave, wave = WR == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane % 16, quad = lane / 16;
    const ngpu_attend_t &a = p.a;
    const int H = p.c.heads, rep = a.q_heads / H, D = p.c.dim, T_ = int(a.T);

    // Workgroups go to the 8 XCDs in turn.  Each XCD takes a run of the prefixes'
    // works, which share keys (row blocks) or rows of pages (heads) in its L2.
    const unsigned prefix_works = unsigned(plan.prefix.works());
    const bool own = w >= prefix_works;
    const Cut &cut = own ? plan.own : plan.prefix;
    if (own)
        w -= prefix_works;
    else
        w = w % 8 * (prefix_works / 8) + min(w % 8, prefix_works % 8) + w / 8;
    // Of own tokens the last blocks of rows see most keys: they come first, of all problems, a head to an XCD.  A
    // prompt of 8192 tokens, 8 heads of 64: 178 us, 301 block by block; of 4 x 4001, 32 / 8 heads of 128: 1010, 1160.
    const unsigned each = unsigned(cut.problems) * unsigned(cut.splits);
    const int block = own ? cut.blocks - 1 - int(w / each) : int(w % unsigned(cut.blocks));
    w = own ? w % each : w / unsigned(cut.blocks);
    const int h = int(w % unsigned(H));
    w /= unsigned(H);
    int split = int(w % unsigned(cut.splits)), splits = cut.splits, g = int(w / unsigned(cut.splits));
    if (!own && plan.prefix.parts > splits) {
        const int n = dealt_splits(cut, int(a.G), lane < a.G ? prefix_table(p, lane).count : 0);
        int end = n;   // of the splits of the groups up to this lane's
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const int below = __shfl_up(end, d);   // (of all lanes: a lane that does not take part gives nothing)
            end += lane >= d ? below : 0;
        }
        const int before = __builtin_popcountll(__ballot(lane < a.G && end <= int(w)));
        if (before >= a.G) return;   // one that rounding left over
        g = before;
        splits = __builtin_amdgcn_readlane(n, before);
        split = int(w) - (__builtin_amdgcn_readlane(end, before) - splits);
    }
    const int beam = own ? 1 : int(a.S / a.G), s0 = g * beam;
    const unsigned rows = unsigned(beam) * T_ * rep;   // (all rows of a call are below 2^31)
    const PageTable table = own ? own_table(p, s0) : prefix_table(p, g);
    const int count = int(table.count);

    // this split's keys, of those that the last row of the block sees (4 x 4001 tokens: 1160 us, 1900 with all keys)
    int sees = count;
    if (own) {
        const unsigned last = min(rows, unsigned(block + 1) * A::kRows) - 1;
        sees = min(count, max(0, count - int(query_length(a, s0)) + int(last / unsigned(rep)) + 1));
    }
    const int tiles = int((unsigned(sees) + A::kKeys - 1) / A::kKeys), per = (tiles + splits - 1) / splits;
    const int tile0 = min(tiles, split * per), tile1 = min(tiles, tile0 + per);

    // The keys that this wavefront loads of each tile.  Where pages hold whole
    // multiples of them they lie in one page, which is found once for all lanes;
    // else each lane finds its own key's, and the loads may go in page by page.
    const unsigned page_size = unsigned(p.c.page_size);
    const bool in_page = page_size % A::kLoad == 0;
    auto first_key = [&](int tile) { return unsigned(tile) * A::kKeys + unsigned(wave * A::kLoad); };
    auto page_index = [&](unsigned j) { return divided(j, page_size, plan.page_magic); };
    // in_page: lane l has the page of tile base + l, so that no load is waited for between tiles; else the
    // page of its key of the next tile
    int base_tile = tile0, pages = -1;
    auto load_pages = [&]() {
        const unsigned j = first_key(base_tile + lane);
        pages = base_tile + lane < tile1 && int(j) < count ? table.pages[page_index(j)] : -1;
    };
    auto page_of = [&](int tile) {   // of this lane's key
        const unsigned j = first_key(tile) + unsigned(lane % A::kLoad);
        return tile < tile1 && int(j) < count ? table.pages[page_index(j)] : -1;
    };
    if (in_page)
        load_pages();
    else
        pages = page_of(tile0);

    // this wavefront's query rows: operand registers, and the keys each row sees
    s16x8 q[RT][DK];
    int limit[RT];
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
        const int nq = int(query_length(a, s));
        limit[r] = count;
        if (own) {
            limit[r] = min(count, max(0, count - nq + t + 1));
            least = min(least, max(0, count - nq + 1));
        }
        const T *src = static_cast<const T *>(a.q) + s * a.q_stride_seq + t * a.q_stride_token + head * a.q_stride_head;
#pragma unroll
        for (int k = 0; k < DK; ++k) {
            // (16 bytes of a key in 8 bits are a lane's dimensions of two steps)
            const int d = A::kEight ? 64 * (k / 2) + 16 * quad + 8 * (k % 2) : 32 * k + 8 * quad;
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

    const uint64_t k_page = uint64_t(p.c.k_stride_page) / A::kPer, v_page = uint64_t(p.c.v_stride_page) / A::kPer;
    const unsigned k_token = unsigned(p.c.k_stride_token / A::kPer), v_token = unsigned(p.c.v_stride_token / A::kPer);
    const char *k_head = static_cast<const char *>(p.c.k) + int64_t(h) * p.c.k_stride_head * int(sizeof(C));
    const char *v_head = static_cast<const char *>(p.c.v) + int64_t(h) * p.c.v_stride_head * int(sizeof(C));
    const int piece = lane % A::kPieces, in_load = lane / A::kPieces, pieces = D / A::kPer;
    auto key_piece = [&](int u) { return piece ^ A::key_swizzle(wave * A::kLoad + u * A::kPerLoad + in_load); };
    auto value_piece = [&](int u) { return piece ^ A::value_swizzle(wave * A::kLoad + u * A::kPerLoad + in_load); };
    // A lane's offsets from the first of its keys in one page, kept where several
    // wavefronts share the loads; one that streams alone has too many, and time to compute them.
    unsigned k_off[A::kLoads], v_off[A::kLoads];
#pragma unroll
    for (int u = 0; u < A::kLoads; ++u) {
        k_off[u] = (unsigned(u * A::kPerLoad + in_load) * k_token + unsigned(key_piece(u))) * 16;
        v_off[u] = (unsigned(u * A::kPerLoad + in_load) * v_token + unsigned(value_piece(u))) * 16;
        if (WR > 1) asm volatile("" : "+v"(k_off[u]), "+v"(v_off[u]));
    }
    // In 8 bits, the chunks that a head does not have are zeros from here on: no load writes them otherwise.
    const bool whole_head = D == 32 * DK;
    if (A::kEight && !whole_head) {
        for (int i = WR == 1 ? lane : int(threadIdx.x); i < A::kLds / 16; i += 64 * WR)
            *lds_at<u32x4>(lds0 + 16 * unsigned(i)) = u32x4{0, 0, 0, 0};
        wait_loads();
        if (WR > 1) asm volatile("s_barrier" ::: "memory");
    }
    const bool whole_rows = (A::kEight || whole_head) && k_token < (1u << 21) && v_token < (1u << 21);
    // (in 8 bits) the scales that this lane loads: its key's, or that key's value's; strides in vector registers
    const float *scales = nullptr;
    uint64_t scales_page = 0, scales_block = 0;
    if constexpr (A::kEight) {
        const bool values = lane >= A::kLoad;
        scales = values ? p.v_scale + h * p.v_scale_head : p.k_scale + h * p.k_scale_head;
        scales_page = uint64_t(values ? p.v_scale_page : p.k_scale_page);
        scales_block = uint64_t(values ? p.v_scale_block : p.k_scale_block);
        asm volatile("" : "+v"(scales), "+v"(scales_page), "+v"(scales_block));
    }
    const char *no_data = reinterpret_cast<const char *>(kNoData);
    asm volatile("" : "+s"(no_data));   // its address is loaded once
    unsigned valid = 0;   // keys that exist among those this wavefront loaded last
    auto fetch = [&](int tile, int stage) {
        constexpr unsigned kAll = A::kLoad == 32 ? 0xffffffffu : 0xffffu;
        const unsigned at = __builtin_amdgcn_readfirstlane(lds0 + unsigned(stage * A::kStage + wave * A::kLoad * A::kPitch));
        const unsigned values_at = at + A::kKeys * A::kPitch;
        const unsigned j = first_key(tile);
        auto put_mask = [&]() {
            if (WR > 1 && lane == 0) reinterpret_cast<uint16_t *>(masks[stage])[wave] = uint16_t(valid);
        };
        // the u-th rows of a whole tile, all of whose dimensions exist
        auto load_whole = [&](int u, const char *kb, const char *vb) {
            const unsigned k_to = at + unsigned(u * kWave * 16), v_to = values_at + unsigned(u * kWave * 16);
            if (A::kUsed == A::kPieces && (!A::kEight || whole_head)) {
                load_to_lds<A::kOnce>(kb, k_off[u], k_to, vb, v_off[u], v_to);
            } else {
                const int used = A::kEight ? pieces : A::kUsed;
                if (key_piece(u) < used) load_to_lds<A::kOnce>(kb, k_off[u], k_to);
                if (value_piece(u) < used) load_to_lds<A::kOnce>(vb, v_off[u], v_to);
            }
        };
        // the scales of this wavefront's keys, then values, a lane each; 0 where there is no key
        auto load_scales = [&](unsigned page, unsigned entry, bool there) {
            if constexpr (A::kEight) {
                const float *from = scales + uint64_t(page) * scales_page + uint64_t(divided(entry, p.block, p.block_magic)) * scales_block;
                if (lane < 2 * A::kLoad)
                    load_word_to_lds(there ? static_cast<const void *>(from) : no_data, lds0 + unsigned(stage * A::kStage + 2 * A::kKeys * A::kPitch +
                                                                              wave * 8 * A::kLoad));
            }
        };
        if (in_page) {
            if (tile == base_tile + kWave) {
                base_tile = tile;
                load_pages();
            }
            const int p0 = __builtin_amdgcn_readlane(pages, tile - base_tile);
            const int left = count - int(j);   // keys from the first on
            const bool is = p0 >= 0 && p0 < p.c.num_pages && left > 0;
            valid = !is ? 0u : (left >= A::kLoad ? kAll : (1u << left) - 1u);
            put_mask();
            const uint64_t entry = is ? j - page_index(j) * page_size : 0u, pg = is ? unsigned(p0) : 0u;
            const char *kb = k_head + (pg * k_page + entry * k_token) * 16;
            const char *vb = v_head + (pg * v_page + entry * v_token) * 16;
            load_scales(unsigned(pg), unsigned(entry) + unsigned(lane % A::kLoad), is && lane % A::kLoad < left);
            if (valid == kAll && whole_rows) {
#pragma unroll
                for (int u = 0; u < A::kLoads; ++u) load_whole(u, kb, vb);
                return;
            }
#pragma unroll
            for (int u = 0; u < A::kLoads; ++u) {
                const unsigned row = unsigned(u * A::kPerLoad + in_load);
                const int kp = key_piece(u), vp = value_piece(u);
                const bool there = int(row) < left && is;
                load_to_lds<A::kOnce>(
                    there && kp < pieces ? kb + (row * uint64_t(k_token) + unsigned(kp)) * 16 : no_data,
                    at + u * kWave * 16);
                load_to_lds<A::kOnce>(
                    there && vp < pieces ? vb + (row * uint64_t(v_token) + unsigned(vp)) * 16 : no_data,
                    values_at + u * kWave * 16);
                __builtin_amdgcn_sched_barrier(0);   // (addresses of all loads at once would not fit the registers)
            }
            return;
        }
        // the lane's key: its row of the cache in 16-byte units
        const unsigned mine = j + unsigned(lane % A::kLoad), entry = mine - page_index(mine) * page_size;
        asm volatile("" : "+v"(pages));   // (what follows from them stays behind the wait for this tile)
        const int page = pages;
        pages = page_of(tile + 1);
        const bool is = page >= 0 && page < p.c.num_pages;
        valid = unsigned(__ballot(is)) & kAll;
        put_mask();
        load_scales(is ? unsigned(page) : 0u, entry, is);
        if (valid == kAll && whole_rows && page_size % A::kPerLoad == 0) {   // a load's keys lie in one page
            unsigned e = j - page_index(j) * page_size;
            const char *kb = nullptr, *vb = nullptr;   // of the page's entry 0, for this load's offsets
#pragma unroll
            for (int u = 0; u < A::kLoads; ++u) {
                if (u == 0 || e == 0) {
                    const uint64_t pg = unsigned(__builtin_amdgcn_readlane(page, u * A::kPerLoad));
                    const int64_t back = int64_t(e) - u * A::kPerLoad;
                    kb = k_head + (int64_t(pg * k_page) + back * k_token) * 16;
                    vb = v_head + (int64_t(pg * v_page) + back * v_token) * 16;
                }
                load_whole(u, kb, vb);
                e = e + A::kPerLoad == page_size ? 0 : e + A::kPerLoad;
            }
            return;
        }
        const unsigned k_at = is ? unsigned(unsigned(page) * k_page) + entry * k_token : 0u;
        const unsigned v_at = is ? unsigned(unsigned(page) * v_page) + entry * v_token : 0u;
#pragma unroll
        for (int u = 0; u < A::kLoads; ++u) {
            const int row = u * A::kPerLoad + in_load;   // of this wavefront's keys
            const unsigned k_row = __shfl(k_at, row), v_row = __shfl(v_at, row);
            const bool there = (valid >> row) & 1u;
            const int kp = key_piece(u), vp = value_piece(u);
            load_to_lds<A::kOnce>(there && kp < pieces ? k_head + (uint64_t(k_row) + unsigned(kp)) * 16 : no_data,
                                  at + u * kWave * 16);
            load_to_lds<A::kOnce>(there && vp < pieces ? v_head + (uint64_t(v_row) + unsigned(vp)) * 16 : no_data,
                                  values_at + u * kWave * 16);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // This lane's places in a tile: step 0 of its operand row of K, dimensions 0 of its blocks of V; step k
    // is at the first XOR 64 k, dimensions 16 d at the second XOR 32 d.
    // (In 8 bits a step is of 64 dimensions, and a transposing load brings 8 keys, which come as two blocks of 4 do.)
    const int v_in = A::kEight ? 4 * quad + col / 2 % 4 + 16 * (col / 8) : 4 * quad + col / 4;
    const unsigned k_first = unsigned(col * A::kPitch + 16 * (quad ^ A::key_swizzle(col)));
    const unsigned v_first = unsigned(v_in * A::kPitch +
                                      16 * ((A::kEight ? 0 : (col % 4) / 2) ^ A::value_swizzle(v_in)) + 8 * (col & 1));
    // the scales of this lane's keys of chunk c, block u
    auto scales_at = [&](unsigned tile_at, int c, int u, bool values) {
        const unsigned at = tile_at + 2 * A::kKeys * A::kPitch;
        return *lds_at<f32x4>(at + unsigned(A::kLoad == 32 ? 64 * u + (values ? 128 : 0) : 128 * (2 * c + u) + (values ? 64 : 0)) +
                              16 * unsigned(quad));
    };

    f32x4 o[RT][A::kTiles];
    float m[RT], sum[RT];   // m: what weights are relative to; sum: of this lane's keys', before they are rounded
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -__builtin_inff();
        sum[r] = 0.0f;
#pragma unroll
        for (int d = 0; d < A::kTiles; ++d) o[r][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // (a factor of 0 would make NaN of the -inf of a key that is not seen)
    const float to_log2 = __builtin_fmaxf(__builtin_fabsf(a.scale) * 1.44269504088896f, 1e-30f);
    constexpr float kRoom = A::kEight ? 0.0f : M::kRoom;   // (weights of values in 8 bits are bfloat16 always)

    // A value that is not finite would reach the rows that do not see its key (0 *
    // inf): where a tile holds such keys and values, the rows are computed one by one at the end.
    bool one_by_one = false;
    // A tile's keys into every row's sums: those whose bit of `exists` is set.
    auto take = [&](int stage, int key0, const unsigned (&exists)[A::kChunks]) {
        constexpr int N = A::kChunks;
        const unsigned tile_at = lds0 + unsigned(stage * A::kStage);
        unsigned k_at = tile_at + k_first, v_at = tile_at + A::kKeys * A::kPitch + v_first;
        asm volatile("" : "+v"(k_at), "+v"(v_at));   // their steps are computed below, not kept in registers
        // Operands are loaded a few steps ahead of the matrix instructions, which hides LDS's latency, and no
        // further: hoisted loads would not fit the registers.
        f32x4 x[RT][2 * N];
        s16x8 kx[kKeysAhead + 1][2], vx[kValuesAhead + 1];   // as they are multiplied, or
        i32x4 kx8[2][2];                                     // in 8 bits
        i32x2 vx8[kValuesAhead + 1];
        auto load_keys8 = [&](int i) {   // 32 keys of steps 2 i mod DK and the one behind
#pragma unroll
            for (int u = 0; u < 2; ++u)
                kx8[i % 2][u] = *lds_at<i32x4>((k_at ^ unsigned(64 * (i % (DK / 2)))) + (i / (DK / 2) * 2 + u) * 16 * A::kPitch);
        };
        auto load_keys = [&](int i) {   // 32 keys of step i mod DK
#pragma unroll
            for (int u = 0; u < 2; ++u)
                kx[i % (kKeysAhead + 1)][u] = *lds_at<s16x8>((k_at ^ unsigned(64 * (i % DK))) + (i / DK * 2 + u) * 16 * A::kPitch);
        };
        auto load_values = [&](int i) {   // 32 keys, dimensions 16 (i mod kTiles) on
            if constexpr (A::kEight) {
                vx8[i % (kValuesAhead + 1)] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    lds_at<i32x2>((v_at ^ unsigned(16 * (i % A::kTiles))) + i / A::kTiles * 32 * A::kPitch));
                return;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const s16x4 part = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4>(
                    (v_at ^ unsigned(32 * (i % A::kTiles))) + (i / A::kTiles * 2 + u) * 16 * A::kPitch));
#pragma unroll
                for (int e = 0; e < 4; ++e) vx[i % (kValuesAhead + 1)][4 * u + e] = part[e];
            }
        };
        if constexpr (A::kEight) {
            constexpr int kSteps = N * DK / 2;
            load_keys8(0);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                if (i + 1 < kSteps) load_keys8(i + 1);
                if (i + 1 == kSteps) {
#pragma unroll
                    for (int j = 0; j < kValuesAhead; ++j) load_values(j);
                }
                const int c = i / (DK / 2), k = i % (DK / 2) * 2;
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const i32x4 raw = kx8[i % 2][u];
                        const s16x8 key = e == 0 ? M::widen(raw[0], raw[1]) : M::widen(raw[2], raw[3]);
#pragma unroll
                        for (int r = 0; r < RT; ++r)
                            x[r][2 * c + u] = M::mul(key, q[r][k + e], k + e == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : x[r][2 * c + u]);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
            // the scores in log2, from here on
#pragma unroll
            for (int c = 0; c < N; ++c)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const f32x4 by = scales_at(tile_at, c, u, false) * to_log2;
#pragma unroll
                    for (int r = 0; r < RT; ++r) x[r][2 * c + u] *= by;
                }
        } else {
#pragma unroll
            for (int i = 0; i < kKeysAhead; ++i) load_keys(i);
#pragma unroll
            for (int i = 0; i < N * DK; ++i) {
                if (i + kKeysAhead < N * DK) load_keys(i + kKeysAhead);
                if (i + 1 == N * DK) {
#pragma unroll
                    for (int j = 0; j < kValuesAhead; ++j) load_values(j);
                }
                const int c = i / DK, k = i % DK;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        x[r][2 * c + u] = M::mul(kx[i % (kKeysAhead + 1)][u], q[r][k], k == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : x[r][2 * c + u]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        const bool some_rows = own && key0 > least - A::kKeys;   // some rows do not see some of the keys
        bool all = !some_rows;
#pragma unroll
        for (int c = 0; c < N; ++c) all = all && exists[c] == 0xffffffffu;
        if (!all) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    // the row's view of this lane's keys: bit 16 u + i is key 16 u + 4 quad + i
                    const int below = limit[r] - key0 - 32 * c - 4 * quad;
                    const unsigned sees = exists[c] >> (4 * quad) &
                                          (below >= 32 ? 0xffffffffu : (below > 0 ? (1u << below) - 1u : 0u));
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[r][2 * c + e / 4][e % 4] = sees >> (16 * (e / 4) + e % 4) & 1u ? x[r][2 * c + e / 4][e % 4]
                                                                                       : -__builtin_inff();
                    __builtin_amdgcn_sched_barrier(0);
                }
            if (some_rows) {
                if constexpr (A::kEight) {
                    unsigned nan = 0;   // a byte whose lower bits are all set
                    for (int i = lane; i < A::kKeys * A::kPieces; i += kWave) {
                        const u32x4 v = *lds_at<u32x4>(tile_at + A::kKeys * A::kPitch + 16 * i) & 0x7f7f7f7fu;
#pragma unroll
                        for (int e = 0; e < 4; ++e) nan |= (v[e] + 0x01010101u) & 0x80808080u;
                    }
                    bool odd = nan != 0;
#pragma unroll
                    for (int c = 0; c < N; ++c)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const f32x4 vs = scales_at(tile_at, c, u, true);
#pragma unroll
                            for (int e = 0; e < 4; ++e) odd |= !(__builtin_fabsf(vs[e]) < __builtin_inff());
                        }
                    if (__ballot(odd)) one_by_one = true;
                } else {
                    u16x8 most = {};   // the largest bits of a value: from those of infinity on, one is not finite
                    for (int i = lane; i < A::kKeys * A::kPieces; i += kWave) {
                        // (the places of pieces that a head does not have hold what was in LDS before)
                        if (A::kUsed != A::kPieces && (i % A::kPieces ^ A::value_swizzle(i / A::kPieces)) >= A::kUsed) continue;
                        most = __builtin_elementwise_max(
                            most, *lds_at<u16x8>(tile_at + A::kKeys * A::kPitch + 16 * i) & (unsigned short)(0x7fff));
                    }
                    bool odd = false;
#pragma unroll
                    for (int e = 0; e < 8; ++e) odd |= most[e] >= M::kInfinity;
                    if (__ballot(odd)) one_by_one = true;
                }
            }
        }
        float top[RT];
        bool rises = false;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            top[r] = x[r][0][0];
#pragma unroll
            for (int e = 1; e < 8 * N; ++e) top[r] = __builtin_fmaxf(top[r], x[r][e / 4][e % 4]);
            if (!A::kEight) top[r] *= to_log2;
            rises |= top[r] > m[r] + (8.0f + kRoom);   // (also while m is -inf)
        }
        if (__ballot(rises)) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float now = __builtin_fmaxf(m[r], row_max(top[r]) - kRoom);
                const float f = now == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m[r] - now);
                m[r] = now;
                sum[r] *= f;
#pragma unroll
                for (int d = 0; d < A::kTiles; ++d) o[r][d] *= f;
            }
        }
        float base[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) base[r] = m[r] == -__builtin_inff() ? 0.0f : m[r];
        u32x4 weights[RT][N];   // of chunk c: pairs of rounded ones
        // In 8 bits a weight takes its value's scale along, in bfloat16, whose exponents have room for both, and in two
        // parts, the second what the first's rounding has left.
        u32x4 rests[RT][N];
        f32x4 v_scales[N][2];
        if constexpr (A::kEight) {
#pragma unroll
            for (int c = 0; c < N; ++c)
#pragma unroll
                for (int u = 0; u < 2; ++u) v_scales[c][u] = scales_at(tile_at, c, u, true);
        }
        auto weigh = [&](int c, int pair) {   // the pair-th of the chunk's 4 RT
            const int r = pair / 4, e = pair % 4 * 2;
            if constexpr (A::kEight) {
                const float z0 = __builtin_amdgcn_exp2f(x[r][2 * c + e / 4][e % 4] - base[r]);
                const float z1 = __builtin_amdgcn_exp2f(x[r][2 * c + e / 4][e % 4 + 1] - base[r]);
                sum[r] += z0;
                sum[r] += z1;
                const float y0 = z0 * v_scales[c][e / 4][e % 4], y1 = z1 * v_scales[c][e / 4][e % 4 + 1];
                const unsigned both = Matrix<Bf16>::round(y0, y1);
                weights[r][c][pair % 4] = both;
                rests[r][c][pair % 4] =
                    Matrix<Bf16>::round(y0 - __uint_as_float(both << 16), y1 - __uint_as_float(both & 0xffff0000u));
                return;
            }
            const float z0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r][2 * c + e / 4][e % 4], to_log2, -base[r]));
            const float z1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r][2 * c + e / 4][e % 4 + 1], to_log2, -base[r]));
            sum[r] += z0;
            sum[r] += z1;
            weights[r][c][pair % 4] = M::round(z0, z1);
        };
#pragma unroll
        for (int i = 0; i < 4 * RT; ++i) weigh(0, i);
        __builtin_amdgcn_sched_barrier(0);
        // A wavefront here goes before one that computes weights: 69 us instead of 72 for the prefix of 4 x 16 x 6
        // rows over 6144 tokens.
        __builtin_amdgcn_s_setprio(1);
        // the next chunk's weights are computed between the matrix instructions of this one
        constexpr int kPairs = (4 * RT + A::kTiles - 1) / A::kTiles;
#pragma unroll
        for (int i = 0; i < N * A::kTiles; ++i) {
            const int c = i / A::kTiles, d = i % A::kTiles;
            if (i + kValuesAhead < N * A::kTiles) load_values(i + kValuesAhead);
            if constexpr (A::kEight) {
                const i32x2 raw = vx8[i % (kValuesAhead + 1)];
                const s16x8 value = Matrix<Bf16>::widen(raw[0], raw[1]);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    o[r][d] = Matrix<Bf16>::mul(value, __builtin_bit_cast(s16x8, weights[r][c]), o[r][d]);
                    o[r][d] = Matrix<Bf16>::mul(value, __builtin_bit_cast(s16x8, rests[r][c]), o[r][d]);
                }
            } else {
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    o[r][d] = M::mul(vx[i % (kValuesAhead + 1)], __builtin_bit_cast(s16x8, weights[r][c]), o[r][d]);
            }
            if (c + 1 < N) {
#pragma unroll
                for (int j = 0; j < kPairs; ++j)
                    if (d * kPairs + j < 4 * RT) weigh(c + 1, d * kPairs + j);
                __builtin_amdgcn_sched_barrier(0);
            } else if (d % 2) {
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
    };

    // Tiles are fetched one ahead.
    int stage = 0;
    if (tile0 < tile1) fetch(tile0, 0);
    for (int tile = tile0; tile < tile1; ++tile) {
        const unsigned mine = valid;   // of this tile's keys
        wait_loads();
        if (WR > 1) asm volatile("s_barrier" ::: "memory");
        if (tile + 1 < tile1) fetch(tile + 1, 1 - stage);
        unsigned exists[A::kChunks];
#pragma unroll
        for (int c = 0; c < A::kChunks; ++c)
            exists[c] = __builtin_amdgcn_readfirstlane(WR > 1 ? masks[stage][c] : mine);
        take(stage, tile * A::kKeys, exists);
        stage = 1 - stage;
    }

    const LastArgs<C> last(p, plan);
    float total[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) total[r] = row_sum(sum[r]);
    const int64_t all_rows = last.p.a.S * last.p.a.T * last.p.a.q_heads;
    const int part = (own ? last.plan.prefix.parts : 0) + split;
    if (one_by_one) {
        for (unsigned i = 0; i < 16 * RT; ++i) {
            const unsigned row = unsigned(block) * A::kRows + unsigned(wave) * 16 * RT + i;
            if (row >= rows) break;
            const int t = int(row / unsigned(rep)), head = h * rep + int(row % unsigned(rep));   // (own: one sequence)
            const int nq = int(query_length(last.p.a, s0)), seen = max(0, min(count, count - nq + t + 1));
            RowPart<T, C> r;
            r.load(last.p, s0, t, head, lane);
            const unsigned end = min(unsigned(tile1) * A::kKeys, unsigned(seen));
            for (unsigned j = unsigned(tile0) * A::kKeys; j < end; ++j) r.take(last.p, table, j, h, lane);
            const int64_t out = (int64_t(s0) * T_ + t) * last.p.a.q_heads + head;
            if (last.plan.parts > 1) {
                if (lane == 0) last.plan.stats[part * all_rows + out] = make_float2(r.m, r.sum);
#pragma unroll
                for (int e = 0; e < r.kDims; ++e)
                    if (const int d = lane + kWave * e; d < D) last.plan.sums[(part * all_rows + out) * D + d] = r.o[e];
            } else {
                r.finish(last.p, out, lane, t < nq);
            }
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const unsigned i = unsigned(block) * A::kRows + (wave * RT + r) * 16 + col, token = i / unsigned(rep);
        if (i >= rows) continue;
        const int s = s0 + int(token / unsigned(T_)), t = int(token % unsigned(T_));
        const int64_t row = int64_t(s * T_ + t) * last.p.a.q_heads + h * rep + int(i - token * unsigned(rep));
        if (last.plan.parts > 1) {
            if (quad == 0) last.plan.stats[part * all_rows + row] = make_float2(m[r], total[r]);
            if (total[r] == 0.0f) continue;
            float *dst = last.plan.sums + (part * all_rows + row) * D;
#pragma unroll
            for (int d = 0; d < A::kTiles; ++d)
                if (const int at = 16 * d + 4 * quad; at < D) *reinterpret_cast<f32x4 *>(dst + at) = o[r][d];
        } else {
            const bool any = t < query_length(last.p.a, s) && total[r] != 0.0f;   // (a NaN sum too)
            if (last.p.a.lse && quad == 0)
                last.p.a.lse[row] = any ? (m[r] == -__builtin_inff() ? total[r] : m[r] * 0.69314718056f + logf(total[r]))
                                        : -__builtin_inff();
            T *dst = static_cast<T *>(last.p.a.out) + row * D;
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

// The first byte of the launch's LDS (a row's pieces are found by exclusive or).
__device__ __forceinline__ unsigned tile_lds() {
    extern __shared__ __attribute__((aligned(512))) char lds[];
    return unsigned(reinterpret_cast<uintptr_t>((LdsPtr<char>)lds));
}

// Registers are held to what two workgroups of four wavefronts a CU leave each where that spills nothing.
template <class T, class C, int DK, int RT, int WR>
__global__ __launch_bounds__(64 * WR, DK <= 4 ? 2 : 1) void attend_tile_kernel(AttendOf<C> p, AttendPlan plan,
                                                                              unsigned work0) {
    attend_tiles<T, C, DK, RT, WR>(p, plan, work0 + blockIdx.x, tile_lds());
}

// Prefixes whose rows take WR wavefronts, and own tokens whose rows take one, in
// one launch: the second wait for memory while the first compute.  A workgroup
// is either WR wavefronts at one work of a prefix or, first, as many as have
// room in the same LDS at a work of own tokens each.  In 8 bits all WR are (there
// is LDS for it), and own tokens come last behind prefixes of four wavefronts, whose works are the longer ones: 4
// x 12 sequences of 5 tokens that see up to 7000 of prefix and 300, 32 / 8 heads of 128, calls in a graph: 72 to 73 us, with own
// tokens first 78, without either and with half the splits of own tokens 81.  With prefixes of two wavefronts it depends: 16 x 16
// of one token that see 100 gain (49.5, not 51.8), 4 x 12 of one that see 3000 lose (181, not 157).
template <class T, class C, int DK, int RT, int WR>
constexpr int kOwnWaves = AttendTile<T, C, DK, RT, WR>::kEight
                              ? WR
                              : AttendTile<T, C, DK, RT, WR>::kLds / AttendTile<T, C, DK, RT, 1>::kLds;
template <class T, class C, int DK, int RT, int WR>
constexpr int kBothLds = AttendTile<T, C, DK, RT, WR>::kEight && WR * AttendTile<T, C, DK, RT, 1>::kLds > AttendTile<T, C, DK, RT, WR>::kLds
                             ? WR * AttendTile<T, C, DK, RT, 1>::kLds
                             : AttendTile<T, C, DK, RT, WR>::kLds;
template <class T, class C, int DK, int RT, int WR>
__global__ __launch_bounds__(64 * WR, DK <= 4 ? 2 : 1) void attend_both_kernel(AttendOf<C> p, AttendPlan plan,
                                                                              unsigned block0, unsigned own_blocks) {
    constexpr int kWaves = kOwnWaves<T, C, DK, RT, WR>;
    constexpr bool kOwnLast = AttendTile<T, C, DK, RT, WR>::kEight && WR == 4;
    const unsigned lds0 = tile_lds(), at = block0 + blockIdx.x;
    const unsigned own0 = kOwnLast ? unsigned(plan.prefix.works()) : 0u, block = at - own0;   // among those of own tokens
    if (kOwnLast ? at < own0 : at >= own_blocks) {
        attend_tiles<T, C, DK, RT, WR>(p, plan, kOwnLast ? at : at - own_blocks, lds0);
        return;
    }
    const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), w = block * kWaves + wave;
    if (wave < kWaves && w < unsigned(plan.own.works()))
        attend_tiles<T, C, DK, RT, 1>(p, plan, unsigned(plan.prefix.works()) + w, lds0 + wave * AttendTile<T, C, DK, RT, 1>::kLds);
}

}  // namespace ngpu
