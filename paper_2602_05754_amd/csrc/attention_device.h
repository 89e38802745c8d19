// What the attention kernels share: 32 x 32 tiles on the matrix cores, their operands in LDS, the softmax between the products, and
// what is done again where a result is not finite.  The layout of a tile and why it is so: attention.hip.
#pragma once
#include "gemm_device.h"

#include <algorithm>
#include <cmath>

namespace tf {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kOwn = 32 * kWaves;          // rows that a block owns: queries, or keys for dk and dv
constexpr int kStageRows = 64;             // rows of a stage: keys, or queries for dk and dv
constexpr int kUnits = 256;                 // compute units of the GPU that this is for
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// kD: elements of a head, a multiple of 16.  A row has room for 64 or 128 in a stage, so that its pieces can be swizzled; what is
// there past its end (its first piece again) is multiplied with nothing but columns of a result that are not stored.
template <typename T_, int kD_>
struct Head {
    typedef T_ T;
    static constexpr int kD = kD_;
    static constexpr bool kBf16 = sizeof(T) == 2;
    static constexpr int kPitch = (kD > 64 ? 128 : 64) * int(sizeof(T));       // bytes of a stage's row
    static constexpr int kRoom = kPitch / 16;                      // 16-byte pieces there is room for
    static constexpr int kChunks = kD * int(sizeof(T)) / 16;       // and those there are
    static constexpr int kSteps = kChunks / 2;                     // a step contracts two of them, one a half wave
    static constexpr int kBlocks = (kD + 31) / 32;                 // blocks of 32 columns
    static constexpr int kStage = kStageRows * kPitch;
    // Whether there are kernels of 128 rows.  With more than 64 elements of fp32 those of 32 take all calls: the matrix units, which
    // both keep one wave each on, bound them, and four waves to a tile come to their diagonal and their end sooner.  us, 4096
    // tokens, 32 / 8 heads of 128, forward and backward: one sequence 1558 4886 (32 rows 1319 4400), 16 sequences 183 670 (192 579).
    static constexpr bool kHasWide = kBf16 || kD <= 64;
};

// Which physical piece of row R holds logical piece c: c ^ swizzle(R).  LDS gives 256 bytes a cycle.  Rows are read 16 lanes a cycle, one piece of
// 16 rows in a row, and the transpose reads take 64 bytes of 4 rows: with more than 64 elements of bf16 both touch every bank once.  With
// others 8 rows' pieces are apart, and rows are read at half of that: a column's rows 8 apart are the same way then and want no
// second address, which is worth more there (us, backward, heads of 128, 4096 tokens: 16 rows apart 492, 8 rows 508; heads of 64, 8192
// tokens in 11 sequences: 277, 271; fp32's matrix instructions leave LDS idle).
template <class H>
__device__ __forceinline__ int swizzle(int row) {
    if constexpr (H::kBf16 && H::kPitch == 256) return ((row & 3) << 2) | ((row >> 2) & 3);
    else if constexpr (H::kPitch >= 256) return ((row & 3) << 2) | ((row >> 1) & 2);
    else return ((row & 2) << 1) | ((row >> 1) & 2);
}
template <class H> constexpr uint32_t kRow8 = H::kPitch == 256 ? 32 : 0;        // bf16: what row + 8 changes in a piece's byte

__device__ __forceinline__ uint32_t lds_address(const void* p) { return uint32_t(uintptr_t(TF_LPTR(const_cast<void*>(p)))); }
template <typename V> __device__ __forceinline__ V lds_read(uint32_t at) {
    return *(__attribute__((address_space(3))) const V*)(uintptr_t(at));
}

// The other half's value beside one's own: f(lane's, that of lane ^ 32), the same in both.
template <class F>
__device__ __forceinline__ float with_other_half(float x, F&& f) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Rows [first, first + 64) of the `rows` that exist, at least one, `pitch` elements apart -> stage.
template <class H, int kFilling = kWaves>
__device__ __forceinline__ void fill_stage(const typename H::T* base, int64_t pitch, int first, int rows, uint32_t stage) {
    int thread = threadIdx.x;
    if constexpr (kFilling > kWaves) asm volatile("" : "+v"(thread));          // offsets formed anew, not kept: that kernel's registers are all in use
    const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int kRowsPerLoad = 1024 / H::kPitch, kStep = kRowsPerLoad * kFilling, kLoads = kStageRows / kStep;
    static_assert(kStep % (H::kBf16 && H::kPitch == 256 ? 16 : 8) == 0, "the swizzle is the same in all of a lane's rows");
    const int last = rows - 1 - first;                             // the last row that exists, counted from the stage's first (>= 0)
    const uint64_t at = reinterpret_cast<uint64_t>(base + int64_t(first) * pitch);     // the same in all lanes, as the loads want it said
    const uint32_t high = __builtin_amdgcn_readfirstlane(uint32_t(at >> 32)), low = __builtin_amdgcn_readfirstlane(uint32_t(at));      // (it gives an int)
    const char* from = reinterpret_cast<const char*>(uint64_t(high) << 32 | low);
    const uint32_t row_bytes = uint32_t(pitch) * uint32_t(sizeof(typename H::T));
    const int r = wave * kRowsPerLoad + lane / H::kRoom;
    int c = (lane % H::kRoom) ^ swizzle<H>(r);
    if constexpr (H::kChunks < H::kRoom) c = c < H::kChunks ? c : 0;
    const uint32_t to = __builtin_amdgcn_readfirstlane(stage + uint32_t(wave) * 1024);
    if (last >= kStageRows - 1) {
        const uint32_t off = uint32_t(r) * row_bytes + uint32_t(c) * 16;
        static_for<kLoads>([&](auto i) __attribute__((always_inline)) { direct_load_16B<i * kFilling * 1024>(from + uint64_t(i * kStep) * row_bytes, off, to); });
    } else {
        static_for<kLoads>([&](auto i) __attribute__((always_inline)) {
            direct_load_16B<i * kFilling * 1024>(from, uint32_t(min(r + i * kStep, last)) * row_bytes + uint32_t(c) * 16, to);
        });
    }
}

// Where a lane reads a stage's rows and columns, from the stage's first byte on: what is added to these is the same for all lanes.
template <class H>
struct Lane {
    uint32_t row[H::kSteps];                           // piece 2 s + lane / 32 of row lane % 32
    uint32_t col[H::kBf16 ? H::kBlocks : 4 * H::kBlocks];          // see add_product()
    __device__ __forceinline__ explicit Lane(uint32_t lds) {
        const int lane = threadIdx.x & 63, r = lane & 31, half = lane >> 5;
#pragma unroll
        for (int s = 0; s < H::kSteps; ++s) row[s] = lds + uint32_t(r) * H::kPitch + (uint32_t((2 * s + half) ^ swizzle<H>(r)) << 4);
        if constexpr (H::kBf16) {
            const int x = 4 * half + ((lane & 15) >> 2);           // the row of eight that this lane fetches for a transpose read
#pragma unroll
            for (int b = 0; b < H::kBlocks; ++b) {
                const int c = 4 * b + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
                col[b] = lds + uint32_t(x) * H::kPitch + (uint32_t(c ^ swizzle<H>(x)) << 4) + (lane & 1) * 8;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int b = 0; b < H::kBlocks; ++b)
                    col[4 * b + e] = lds + uint32_t(4 * half + e) * H::kPitch + (uint32_t((8 * b + (r >> 2)) ^ swizzle<H>(4 * half + e)) << 4) + (r & 3) * 4;
        }
    }
};

// A lane's share of a row as an operand: pieces 2 s + lane / 32, in registers.
template <class H>
__device__ __forceinline__ void load_own(const typename H::T* row, U4 (&x)[H::kSteps]) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int s = 0; s < H::kSteps; ++s) x[s] = *reinterpret_cast<const U4*>(reinterpret_cast<const char*>(row) + (2 * s + half) * 16);
}

// One step of a product over the head's elements.
template <class H>
__device__ __forceinline__ f32x16 multiply_rows(const U4& a, const U4& b, f32x16 c) {
    if constexpr (H::kBf16) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
        return c;
    }
}

// (32 rows from byte `at` of the stages) x (own rows, 32): lane l has column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4.
template <class H, bool kAhead = H::kBf16>          // (fp32, 256 tokens, 4 heads of 64: dk and dv 26 us, 30 with the reads ahead)
__device__ __forceinline__ f32x16 scores(const Lane<H>& lane, uint32_t at, const U4 (&own)[H::kSteps], f32x16 c = {}) {
    U4 x[H::kSteps];
#pragma unroll
    for (int s = 0; s < H::kSteps; ++s) x[s] = lds_read<U4>(lane.row[s] + at);
    if constexpr (kAhead) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < H::kSteps; ++s) c = multiply_rows<H>(x[s], own[s], c);
    return c;
}

// The same, own rows those from byte `own` of the stages.
template <class H>
__device__ __forceinline__ f32x16 scores(const Lane<H>& lane, uint32_t at, uint32_t own, f32x16 c = {}) {
#pragma unroll
    for (int s = 0; s < H::kSteps; ++s) c = multiply_rows<H>(lds_read<U4>(lane.row[s] + at), lds_read<U4>(lane.row[s] + own), c);
    return c;
}

// acc^T += X^T w: X the 32 rows from byte `at` (columns in blocks of 32), w their weights for 32 columns as scores() lays
// them out.
template <class H>
__device__ __forceinline__ void add_product(const Lane<H>& lane, uint32_t at, const f32x16& w, f32x16 (&acc)[H::kBlocks]) {
    if constexpr (H::kBf16) {
#pragma unroll
        for (int sl = 0; sl < 2; ++sl) {
            U4 packed;
#pragma unroll
            for (int i = 0; i < 4; ++i) packed[i] = f32x2_to_bf16x2(w[8 * sl + 2 * i], w[8 * sl + 2 * i + 1]);
#pragma unroll
            for (int b = 0; b < H::kBlocks; ++b) {
                const uint32_t p = lane.col[b] + (at + sl * 16 * H::kPitch);
                uint32_t p8 = p + 8 * H::kPitch;
                if constexpr (kRow8<H> != 0) p8 = (lane.col[b] ^ kRow8<H>) + (at + (sl * 16 + 8) * H::kPitch);
                typedef __attribute__((address_space(3))) char* P3;
                const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsBf16x4Ptr)(P3)(uintptr_t)p);
                const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsBf16x4Ptr)(P3)(uintptr_t)p8);
                acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7),
                                                                 __builtin_bit_cast(bf16x8, packed), acc[b], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int b = 0; b < H::kBlocks; ++b)
                acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(lds_read<float>(lane.col[4 * b + i % 4] + (at + i / 4 * 8 * H::kPitch)), w[i], acc[b], 0, 0, 0);
    }
}

// acc^T += X^T (what rounding to bf16 has taken from w).  For the gradients of sequences of one tile, on all kernels: what a sequence gets does not
// depend on those that it is packed with.  Root mean square error, heads of 64 and 128, over that of 32-bit products rounded once: dq and dk 1.42,
// dv 1.25 to 1.39 at any length from 4 to 256; with this 1.00.  us, backward, 100 sequences of 20 tokens, 32 / 8 heads of 64 and 128:
// 53 92, with this 56 101; calls without such sequences take no longer.  In sequences of more tiles it would be three more products to the seven.
template <class H>
__device__ __forceinline__ void add_rest(const Lane<H>& lane, uint32_t at, const f32x16& w, f32x16 (&acc)[H::kBlocks]) {
    if constexpr (H::kBf16) {
        f32x16 rest;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const uint32_t rounded = f32x2_to_bf16x2(w[i], w[i + 1]);
            rest[i] = w[i] - __uint_as_float(rounded << 16);
            rest[i + 1] = w[i + 1] - __uint_as_float(rounded & 0xffff0000u);
        }
        add_product<H>(lane, at, rest, acc);
    }
}
constexpr int kShort = 32;                 // rows of such a sequence, at most

// One block of 32 columns of such a product, each element of X multiplied only where keep(row of the tile, column of w) holds.
template <class H, class F>
__device__ __forceinline__ void add_block_where(uint32_t rows_at, const f32x16& w, f32x16& acc, int block, F&& keep) {
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
#pragma unroll 1
    for (int r = 0; r < 32; ++r) {
        float mine = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) mine = i == 4 * (r >> 3) + (r & 3) ? w[i] : mine;
        const float weight = __shfl(mine, col + 32 * ((r >> 2) & 1), 64);
        const bool here = keep(r, col);
        const uint32_t at = rows_at + uint32_t(r) * H::kPitch;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t byte = uint32_t(32 * block + 8 * (i / 4) + 4 * half + i % 4) * uint32_t(sizeof(typename H::T));
            const uint32_t p = at + (((byte >> 4) ^ uint32_t(swizzle<H>(r))) << 4) + (byte & 15);
            float x;
            if constexpr (H::kBf16) x = __uint_as_float(uint32_t(lds_read<uint16_t>(p)) << 16);
            else x = lds_read<float>(p);
            acc[i] += here ? weight * x : 0.f;
        }
    }
}

template <int kN>
__device__ __forceinline__ bool all_finite(const f32x16 (&x)[kN]) {
    float zero = 0.f;
#pragma unroll
    for (int b = 0; b < kN; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) zero += 0.f * x[b][i];
    return zero == 0.f;
}

// acc^T -> rows: lane l writes columns 32 b + 8 g + 4 (l / 32) + 0..3 of its row.
template <class H>
__device__ __forceinline__ void store_block(typename H::T* row, const f32x16& acc, int block, float scale) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int c = 32 * block + 8 * g + 4 * half;
        if (H::kD % 32 != 0 && c >= H::kD) continue;
        const float x0 = acc[4 * g] * scale, x1 = acc[4 * g + 1] * scale, x2 = acc[4 * g + 2] * scale, x3 = acc[4 * g + 3] * scale;
        if constexpr (H::kBf16) *reinterpret_cast<U2*>(row + c) = U2{f32x2_to_bf16x2(x0, x1), f32x2_to_bf16x2(x2, x3)};
        else *reinterpret_cast<F4*>(row + c) = F4{x0, x1, x2, x3};
    }
}
// Of such a block, the values that are not finite where it stands.
template <class H>
__device__ __forceinline__ void mend_block(typename H::T* row, const f32x16& acc, int block, float scale) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int c = 32 * block + 8 * (i / 4) + 4 * half + i % 4;
        if (H::kD % 32 != 0 && c >= H::kD) continue;
        if constexpr (H::kBf16) {
            if ((row[c] & 0x7f80) == 0x7f80) row[c] = uint16_t(f32x2_to_bf16x2(acc[i] * scale, 0.f));
        } else {
            if ((__float_as_uint(row[c]) & 0x7f800000u) == 0x7f800000u) row[c] = acc[i] * scale;
        }
    }
}
template <class H>
__device__ __forceinline__ void store_row(typename H::T* row, const f32x16 (&acc)[H::kBlocks], float scale) {
#pragma unroll
    for (int b = 0; b < H::kBlocks; ++b) store_block<H>(row, acc[b], b, scale);
}

// Between the products and the first other instruction that reads the sums (see wait_for_sums()), which are left where the
// matrix instructions have them: with fp32 that is the accumulation registers, and a copy out of them would be such a reader.
template <class H>
__device__ __forceinline__ void settle(f32x16 (&x)[H::kBlocks]) {
    auto tie = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < H::kBlocks; ++b) {
            if constexpr (H::kBf16) asm volatile("" : "+v"(x[b]));
            else asm volatile("" : "+a"(x[b]));
        }
    };
    tie();
    asm volatile("s_nop 15\n\ts_nop 15");
    tie();
}

// The compiler's own wait for two tiles, and a little more: it may have counted an s_waitcnt among the wait states.
__device__ __forceinline__ void settle(f32x16& x, f32x16& y) {
    asm volatile("" : "+v"(x), "+v"(y));
    asm volatile("s_nop 1");
    asm volatile("" : "+v"(x), "+v"(y));
}

// Whether x holds in any thread of the block.  Once in a kernel.
__device__ __forceinline__ bool any_in_block(bool x) {
    __shared__ int of_wave[8];
    const bool here = __any(x);
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = here;
    __syncthreads();
    int found = 0;
    for (int i = 0; i < int(blockDim.x) / 64; ++i) found |= of_wave[i];
    return __builtin_amdgcn_readfirstlane(found) != 0;
}

// Keys after the query.
__device__ __forceinline__ void mask_later(f32x16& s) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 8 * (i / 4) + 4 * (lane >> 5) + i % 4 <= (lane & 31) ? s[i] : -INFINITY;
}

// Keys -> queries, 32 of each: softmax with a running reference m (of the exponents of 2), sum l and result o.  The reference begins finite, below
// all scores: of a query that has seen nothing but scores of -infinity the weights are 0, exp2(-infinity - m), and what comes counts in full.
constexpr float kNoReference = -3.402823466e+38f;
template <class H>
__device__ __forceinline__ void attend(const Lane<H>& at, uint32_t keys, uint32_t values, const U4 (&q)[H::kSteps], float c, bool diagonal,
                                       float& m, float& l, f32x16 (&o)[H::kBlocks]) {
    f32x16 s = scores<H>(at, keys, q);
    if (diagonal) mask_later(s);
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    top = with_other_half(top, [](float x, float y) { return fmaxf(x, y); }) * c;
    // The reference of the exponentials follows the maximum only when it has grown by 2^8 or more: sums and
    // products stay within 2^8 of those with the maximum itself, and their quotient is the same.  A query's follows by its own scores, those
    // of other queries in the tile leave its bits as they are.
    if (__any(top > m + 8.f)) {
        const float next = top > m + 8.f ? top : m, shrink = __builtin_amdgcn_exp2f(m - next);
        m = next;
        l *= shrink;
#pragma unroll
        for (int b = 0; b < H::kBlocks; ++b) o[b] *= shrink;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -m));
        l += s[i];
    }
    add_product<H>(at, values, s, o);
}

// dP - D: with bf16 the matrix instructions start from -D, with fp32, where they and not the others are what takes time, it is added.
__device__ __forceinline__ f32x16 all(float x) {
    f32x16 r;
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = x;
    return r;
}

// dS^T of 32 keys and the lanes' queries.  lse: times log2 e.
template <class H>
__device__ __forceinline__ f32x16 score_gradients(const Lane<H>& at, uint32_t keys, uint32_t values, const U4 (&q)[H::kSteps], const U4 (&go)[H::kSteps],
                                                  float c, float lse, float minus_d, bool diagonal) {
    f32x16 s = scores<H>(at, keys, q), dp = scores<H>(at, values, go, all(H::kBf16 ? minus_d : 0.f));
    settle(s, dp);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -lse)) * (H::kBf16 ? dp[i] : dp[i] + minus_d);
    const int lane = threadIdx.x & 63;
    if (diagonal)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 8 * (i / 4) + 4 * (lane >> 5) + i % 4 <= (lane & 31) ? s[i] : 0.f;
    return s;
}

// -D of 32 queries by rows, from byte `at` of this half wave on.
__device__ __forceinline__ f32x16 by_rows(uint32_t at) {
    f32x16 r;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const F4 x = lds_read<F4>(at + g * 32);
#pragma unroll
        for (int e = 0; e < 4; ++e) r[4 * g + e] = x[e];
    }
    return r;
}

// Scores -> P and dP (bf16: - D) -> dS, queries by rows; their lse (`lse_scale` makes it one of powers of 2) and -D are in LDS, from byte `stats` of
// this half wave on and `apart` bytes behind it.
template <class H>
__device__ __forceinline__ void weigh(f32x16& p, f32x16& ds, uint32_t stats, uint32_t apart, float c, float lse_scale = 1.f) {
    settle(p, ds);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const F4 lse = lds_read<F4>(stats + g * 32);
        [[maybe_unused]] F4 minus_d;
        if constexpr (!H::kBf16) minus_d = lds_read<F4>(stats + g * 32 + apart);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 4 * g + e;
            p[i] = __builtin_amdgcn_exp2f(fmaf(p[i], c, -(lse[e] * lse_scale)));
            if constexpr (H::kBf16) ds[i] *= p[i];
            else ds[i] = p[i] * (ds[i] + minus_d[e]);
        }
    }
}

// Of such a tile, only its queries [from, to) see the key.
__device__ __forceinline__ void mask_unseen(f32x16& p, f32x16& ds, int from, int to) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int r = 8 * (i / 4) + 4 * half + i % 4;
        const bool seen = r >= from && r < to;
        p[i] = seen ? p[i] : 0.f;
        ds[i] = seen ? ds[i] : 0.f;
    }
}

// The tiles once more for each of `jobs` blocks of 32 columns: fill(tile), add(tile, its part, job, acc), store(job, acc).
template <class H, class Fill, class Add, class Store>
__device__ __forceinline__ void repair(int tiles, Fill&& fill, int jobs, Add&& add, Store&& store) {
#pragma unroll 1
    for (int job = 0; job < jobs; ++job) {
        f32x16 acc = {};
#pragma unroll 1
        for (int t = 0; t < tiles; ++t) {
            __syncthreads();                                       // the tile before has been read
            fill(t);
            wait_direct_loads();
            __syncthreads();
#pragma unroll 1
            for (int part = 0; part < kStageRows; part += 32) add(t, part, job, acc);
        }
        store(job, acc);
    }
}

// do o of this lane's row, of which it has its share of do.
template <class H>
__device__ __forceinline__ float row_product(const typename H::T* row, const U4 (&go)[H::kSteps]) {
    U4 o[H::kSteps];
    load_own<H>(row, o);
    float sum = 0.f;
#pragma unroll
    for (int s = 0; s < H::kSteps; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (H::kBf16) {
                sum += __uint_as_float(o[s][j] << 16) * __uint_as_float(go[s][j] << 16);
                sum += __uint_as_float(o[s][j] & 0xffff0000u) * __uint_as_float(go[s][j] & 0xffff0000u);
            } else {
                sum += __uint_as_float(o[s][j]) * __uint_as_float(go[s][j]);
            }
        }
    return with_other_half(sum, [](float x, float y) { return x + y; });
}

// Tokens of no sequence, block `number` of a.pad_blocks: zeros, and no logarithm.
template <typename T>
__device__ __forceinline__ void clear_padding(const AttentionCall& a, int number) {
    const int wide = a.hq * a.d, narrow = wide / a.group;
    for (int64_t t = a.pad_first + number; t < a.T; t += a.pad_blocks) {
        auto clear = [&](void* p, int64_t stride, int n) __attribute__((always_inline)) {
            for (int c = threadIdx.x; c < n; c += kThreads) static_cast<T*>(p)[t * stride + c] = T(0);
        };
        if (a.dq) {
            clear(a.dq, a.q_stride, wide);
            clear(a.dk, a.k_stride, narrow);
            clear(a.dv, a.v_stride, narrow);
        } else {
            clear(a.o, a.o_stride, wide);
            for (int h = threadIdx.x; h < a.hq; h += kThreads) a.lse[t * a.hq + h] = -INFINITY;
        }
    }
}

// What a block works on: a head and a tile of a sequence.
struct Work {
    int head, first, rows, begin;          // of `heads`; first own row in the sequence; its rows; the sequence's first token
};

// Blocks run head by head within a tile, tiles in the launch's order, so that those with most to do come first.  Block b runs on XCD
// b % 8: where the heads divide by 8, consecutive heads, which share keys and values, stay on one.
template <int kRows>
__device__ __forceinline__ Work find_work(const AttentionCall& a, int number, int heads, bool last_first) {
    const int tile = number / heads, slot = number % heads;
    int lo = 0, hi = a.n_seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (tile >= a.seq[mid].tile_start) lo = mid;
        else hi = mid - 1;
    }
    Work w;
    w.head = heads % kXcds == 0 ? slot % kXcds * (heads / kXcds) + slot / kXcds : slot;
    w.begin = a.seq[lo].begin;
    w.rows = a.seq[lo].rows;
    const int tiles = (w.rows + kRows - 1) / kRows, t = tile - a.seq[lo].tile_start;
    w.first = (last_first ? tiles - 1 - t : t) * kRows;
    return w;
}

template <class F>
void with_head(Dtype dtype, int d, F&& f) {
    static_for<8>([&](auto i) {
        constexpr int kD = 16 * (i + 1);
        if (d != kD) return;
        if (dtype == Dtype::BF16) f(Head<uint16_t, kD>{});
        else f(Head<float, kD>{});
    });
}

template <auto kernel>
hipError_t launch_tiles(hipStream_t stream, const AttentionCall& a, int lds, int blocks, int threads = kThreads) {
    if (lds > 65536) {                                 // allowed once per kernel and device
        constexpr int kMaxDevices = 64;
        static bool lds_allowed[kMaxDevices] = {false};
        int dev = -1;
        if (hipGetDevice(&dev) != hipSuccess || dev >= kMaxDevices) dev = -1;
        if (dev < 0 || !lds_allowed[dev]) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            if (e != hipSuccess) return e;
            if (dev >= 0) lds_allowed[dev] = true;
        }
    }
    hipLaunchKernelGGL(kernel, dim3(uint32_t(blocks)), dim3(threads), lds, stream, a);
    return hipGetLastError();
}

}  // namespace
}  // namespace tf
