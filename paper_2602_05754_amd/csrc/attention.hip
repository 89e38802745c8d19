// Causal attention over packed sequences with grouped heads, forward and backward.
//
//   S_ij = scale q_i k_j (j <= i, same sequence), P = softmax(S) by rows, lse = log sum exp S, o = P v
//   D_i = do_i o_i,  dP = do v^T,  dS = P (dP - D),  dq = scale dS k,  dk = scale dS^T q,  dv = P^T do
//
// Everything is a product of 32 x 32 tiles on the matrix cores (bf16: 32x32x16, fp32: 32x32x2).  The first
// product of a pair is laid out so that its result is the second one's operand as it stands: a lane of
// S^T = K Q^T holds 16 keys of one query, keys 8 (i / 4) + 4 (lane / 32) + i % 4, and contracted over keys in that
// order it is the right operand of o^T = V^T P^T; V^T is read in the same order (bf16: LDS transpose reads).
// Softmax statistics of a query are in its lane and the one 32 further on.
//
//   forward     a wave has 32 queries (their rows in registers, o^T in the accumulators), a block 128; keys and
//               values pass by in LDS stages of 64
//   dq          the same with dP^T = V dO^T beside S^T and dq^T = K^T dS^T; also D
//   dk, dv      a wave has 32 keys, queries pass by: S = Q K^T and dP = dO V^T, then dv^T = dO^T P and
//               dk^T = Q^T dS.  A block takes one or more query heads of a group; where they are not all, their sums
//               are added by a kernel of their own, in order: no atomics, and the same call gives the same bits.
//
// P and dS are rounded to bf16 for the second products (bf16 inputs), the type that the matrix cores take at sixteen times the rate of fp32;
// sums, statistics and the factors in between are 32-bit.  The results' error, root mean square, is 1.25 to 1.42 times that of 32-bit products.
// What the rounding takes away as a product of its own makes it 1.00, and costs 28 to 34 % of the time (forward, 4096 tokens, heads of 128 and 64:
// 152 196, 90 121; backward, heads of 64: 281 373) and registers that dk and dv of heads of 128 do not have; the gradients of short sequences
// have it (add_rest()).
//
// Stages are filled by direct loads, rows past a sequence's end by its last row again: their scores are masked.
// A masked score is a select, but a zero weight times an infinite or NaN row is NaN: a block whose results are not
// all finite works those again, 32 columns at a time, the products element by element (`repair`).
//
// Bound by waiting: two waves are what a matrix unit's registers hold, and one tile's product, exponentials and next product follow on each
// other.  Of the cycles the matrix cores are busy 40 to 50 % (heads of 128; 30 to 36 with 64), vector instructions 30 to 40, LDS 30.
// us, and TFLOP/s of the 2 (forward) or 5 products that the result needs, of which the backward does 7 (large library products: 1180):
//   bf16, 4096 tokens, 32 / 8 heads of 128       forward 151, 910      backward 492, 699 (dk and dv 310, dq 170 to 200, parts 14)
//   bf16, 8192 tokens in 11 sequences, 32 / 8 heads of 64              backward 271, 478
// Two tiles of queries to a wave, heads of 64: 116 for 88 (4096 tokens, forward).
#include "attention_device.h"

namespace tf {
namespace {

// The keys that a block's queries see, a stage of 64 at a time and the next one on its way: fill(stage number, byte of the
// stages) and add(byte of 32 rows, whether they are the wave's diagonal tile).  All keys before the block's first query, an even
// number of stages, are every wave's; of the last two a wave takes what its queries see.
template <class H, class Fill, class Add>
__device__ __forceinline__ void walk_keys(const Work& w, int tiles, int own0, bool live, Fill&& fill, Add&& add) {
    fill(0, 0);
    const int whole = w.first / kStageRows;
    static_assert(kOwn / kStageRows == 2, "stages in pairs");
    for (int t = 0; t < whole; t += 2)
        static_for<2>([&](auto odd) __attribute__((always_inline)) {
            wait_direct_loads();
            __syncthreads();
            fill(t + odd + 1, (1 - odd) * H::kStage);
            add(odd * H::kStage, false);
            add(odd * H::kStage + 32 * H::kPitch, false);
        });
    for (int t = whole; t < tiles; ++t) {
        wait_direct_loads();
        __syncthreads();
        const uint32_t now = (t & 1) * H::kStage;
        if (t + 1 < tiles) fill(t + 1, H::kStage - now);
#pragma unroll 1
        for (int part = 0; part < kStageRows; part += 32) {
            const int key0 = t * kStageRows + part;
            if (live && key0 <= own0) add(now + part * H::kPitch, key0 == own0);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------
template <class H>
__global__ __launch_bounds__(kThreads, H::kBf16 ? 2 : 1) void attention_forward_kernel(AttentionCall a) {
    typedef typename H::T T;
    if (int(blockIdx.x) >= a.tiles * a.hq) return clear_padding<T>(a, blockIdx.x - a.tiles * a.hq);
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t stages = lds_address(lds);
    constexpr uint32_t kValues = 2 * H::kStage;                    // bytes to the values' stages
    const Lane<H> at(stages);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const Work w = find_work<kOwn>(a, blockIdx.x, a.hq, true);
    const int kv = w.head / a.group;
    const T* k = static_cast<const T*>(a.k) + int64_t(w.begin) * a.k_stride + kv * H::kD;
    const T* v = static_cast<const T*>(a.v) + int64_t(w.begin) * a.v_stride + kv * H::kD;
    const int own0 = w.first + 32 * wave, row = own0 + (lane & 31);          // this lane's query
    const bool live = own0 < w.rows;
    const int64_t token = int64_t(w.begin) + min(row, w.rows - 1);
    U4 q[H::kSteps];
    load_own<H>(static_cast<const T*>(a.q) + token * a.q_stride + w.head * H::kD, q);
    const int tiles = (min(w.first + kOwn, w.rows) + kStageRows - 1) / kStageRows;
    const float c = a.scale * kLog2e;

    f32x16 o[H::kBlocks];
#pragma unroll
    for (int b = 0; b < H::kBlocks; ++b) o[b] = f32x16{};
    float m = kNoReference, l = 0.f;
    auto add_keys = [&](uint32_t rows, bool diagonal) __attribute__((always_inline)) {
        attend<H>(at, rows, kValues + rows, q, c, diagonal, m, l, o);
    };
    walk_keys<H>(w, tiles, own0, live, [&](int t, uint32_t stage) __attribute__((always_inline)) {
        fill_stage<H>(k, a.k_stride, t * kStageRows, w.rows, stages + stage);
        fill_stage<H>(v, a.v_stride, t * kStageRows, w.rows, stages + kValues + stage);
    }, add_keys);
    settle<H>(o);
    l = with_other_half(l, [](float x, float y) { return x + y; });
    T* out = static_cast<T*>(a.o) + token * a.o_stride + w.head * H::kD;
    const float inverse = 1.f / l;
    const bool mine = row < w.rows;
    if (mine) {
        store_row<H>(out, o, inverse);
        if (half == 0) a.lse[token * a.hq + w.head] = (m + __builtin_amdgcn_logf(l)) * kLn2;
    }
    if (!any_in_block(live && !all_finite(o))) return;
    repair<H>(tiles, [&](int t) __attribute__((always_inline)) {
        fill_stage<H>(k, a.k_stride, t * kStageRows, w.rows, stages);
        fill_stage<H>(v, a.v_stride, t * kStageRows, w.rows, stages + kValues);
    }, H::kBlocks, [&](int t, int part, int block, f32x16& acc) __attribute__((always_inline)) {
        const int key0 = t * kStageRows + part;
        if (!live || key0 > own0) return;
        f32x16 s = scores<H>(at, part * H::kPitch, q);
        if (key0 == own0) mask_later(s);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -m));
        add_block_where<H>(stages + kValues + part * H::kPitch, s, acc, block, [&](int key, int query) __attribute__((always_inline)) { return key0 + key <= own0 + query; });
    }, [&](int block, const f32x16& acc) __attribute__((always_inline)) {
        if (mine) mend_block<H>(out, acc, block, inverse);
    });
}

// ---------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------
// D = do o by rows, 16 lanes each, for the kernels of 32 rows, which have blocks for dk and dv beside those for dq: `blocks` blocks; then tokens of
// no sequence.
template <typename T>
__global__ __launch_bounds__(kThreads) void attention_delta_kernel(AttentionCall a, int64_t first, int64_t rows, int blocks) {
    if (int(blockIdx.x) >= blocks) return clear_padding<T>(a, blockIdx.x - blocks);
    constexpr int kPiece = 16 / int(sizeof(T));
    const int64_t i = first + (int64_t(blockIdx.x) * kThreads + threadIdx.x) / 16;
    const int lane = threadIdx.x & 15;
    float sum = 0.f;
    if (i < rows) {
        const int64_t token = i / a.hq, head = i % a.hq;
        const T* o = static_cast<const T*>(a.o) + token * a.o_stride + head * a.d;
        const T* g = static_cast<const T*>(a.go) + token * a.o_stride + head * a.d;
        for (int c = lane * kPiece; c < a.d; c += 16 * kPiece) {
            const U4 x = *reinterpret_cast<const U4*>(o + c), y = *reinterpret_cast<const U4*>(g + c);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 4) sum += __uint_as_float(x[j]) * __uint_as_float(y[j]);
                else sum += __uint_as_float(x[j] << 16) * __uint_as_float(y[j] << 16) + __uint_as_float(x[j] & 0xffff0000u) * __uint_as_float(y[j] & 0xffff0000u);
            }
        }
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 16);
    if (i < rows && lane == 0) a.minus_d[i] = -sum;
}

template <class H>
__global__ __launch_bounds__(kThreads, H::kBf16 ? 2 : 1) void attention_dq_kernel(AttentionCall a) {
    typedef typename H::T T;
    if (int(blockIdx.x) >= a.tiles * a.hq) return clear_padding<T>(a, blockIdx.x - a.tiles * a.hq);
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t stages = lds_address(lds);
    constexpr uint32_t kValues = 2 * H::kStage;                    // bytes to the values' stages
    const Lane<H> at(stages);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Work w = find_work<kOwn>(a, blockIdx.x, a.hq, true);
    const int kv = w.head / a.group;
    const T* k = static_cast<const T*>(a.k) + int64_t(w.begin) * a.k_stride + kv * H::kD;
    const T* v = static_cast<const T*>(a.v) + int64_t(w.begin) * a.v_stride + kv * H::kD;
    const int own0 = w.first + 32 * wave, row = own0 + (lane & 31);
    const bool live = own0 < w.rows;
    const int64_t token = int64_t(w.begin) + min(row, w.rows - 1);
    U4 q[H::kSteps], go[H::kSteps];
    load_own<H>(static_cast<const T*>(a.q) + token * a.q_stride + w.head * H::kD, q);
    load_own<H>(static_cast<const T*>(a.go) + token * a.o_stride + w.head * H::kD, go);
    const float lse = a.lse[token * a.hq + w.head] * kLog2e;
    // D = do o of the lane's row, which the kernel for dk and dv reads after this one
    const float minus_d = -row_product<H>(static_cast<const T*>(a.o) + token * a.o_stride + w.head * H::kD, go);
    const bool mine = row < w.rows;
    if (mine && lane < 32) a.minus_d[token * a.hq + w.head] = minus_d;
    const int tiles = (min(w.first + kOwn, w.rows) + kStageRows - 1) / kStageRows;
    const float c = a.scale * kLog2e;

    auto gradient = [&](uint32_t rows, bool diagonal) __attribute__((always_inline)) {
        return score_gradients<H>(at, rows, kValues + rows, q, go, c, lse, minus_d, diagonal);
    };

    f32x16 dq[H::kBlocks];
#pragma unroll
    for (int b = 0; b < H::kBlocks; ++b) dq[b] = f32x16{};
    walk_keys<H>(w, tiles, own0, live, [&](int t, uint32_t stage) __attribute__((always_inline)) {
        fill_stage<H>(k, a.k_stride, t * kStageRows, w.rows, stages + stage);
        fill_stage<H>(v, a.v_stride, t * kStageRows, w.rows, stages + kValues + stage);
    }, [&](uint32_t rows, bool diagonal) __attribute__((always_inline)) {
        const f32x16 ds = gradient(rows, diagonal);
        add_product<H>(at, rows, ds, dq);
        if (diagonal && w.rows <= kShort) add_rest<H>(at, rows, ds, dq);
    });
    settle<H>(dq);
    T* out = static_cast<T*>(a.dq) + token * a.q_stride + w.head * H::kD;
    if (mine) store_row<H>(out, dq, a.scale);
    if (!any_in_block(live && !all_finite(dq))) return;
    repair<H>(tiles, [&](int t) __attribute__((always_inline)) {
        fill_stage<H>(k, a.k_stride, t * kStageRows, w.rows, stages);
        fill_stage<H>(v, a.v_stride, t * kStageRows, w.rows, stages + kValues);
    }, H::kBlocks, [&](int t, int part, int block, f32x16& acc) __attribute__((always_inline)) {
        const int key0 = t * kStageRows + part;
        if (!live || key0 > own0) return;
        add_block_where<H>(stages + part * H::kPitch, gradient(part * H::kPitch, key0 == own0), acc, block, [&](int key, int query) __attribute__((always_inline)) { return key0 + key <= own0 + query; });
    }, [&](int block, const f32x16& acc) __attribute__((always_inline)) {
        if (mine) mend_block<H>(out, acc, block, a.scale);
    });
}

// Shape of the kernel for dk and dv.  For 128 elements of bf16 the sums and the own rows leave four waves of a block, each
// alone on its matrix unit (registers for one), with nothing to do while they wait: there a block has eight, two for each 32 keys,
// which take the two halves of a stage's queries and add up their sums at the end, and the values come from LDS.
// us, 4096 tokens, 32 / 8 heads of 128: four waves 372, eight 322.
template <class H>
struct KeyBlock {
    static constexpr bool kPairs = H::kBf16 && (H::kD > 96);
    static constexpr int kThreads = kPairs ? 512 : 256, kFilling = kThreads / 64;
    static constexpr int kPerUnit = H::kBf16 && !kPairs ? 2 : 1;   // blocks of a compute unit
    static constexpr uint32_t kGrads = 2 * H::kStage, kValues = 4 * H::kStage, kStats = kPairs ? 6 * H::kStage : 4 * H::kStage;   // bytes into LDS
    static constexpr int kLds = kStats + 2 * 128 * 4;
};

// dk and dv of one key head, from a.per of its query heads: the gradients themselves where that is the whole group, otherwise sums
// in 32 bits, in [token][key head][part of the group][d].
template <class H>
__global__ __launch_bounds__(KeyBlock<H>::kThreads, KeyBlock<H>::kPairs ? 2 : KeyBlock<H>::kPerUnit) void attention_dkv_kernel(AttentionCall a) {
    typedef typename H::T T;
    typedef KeyBlock<H> B;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t stages = lds_address(lds);
    constexpr uint32_t kGrads = B::kGrads;                         // bytes to the stages of the gradients of o
    float* stats = reinterpret_cast<float*>(lds + B::kStats);      // [stage][lse, -D][64]
    const Lane<H> at(stages);
    const int lane = threadIdx.x & 63, all_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int wave = all_wave & 3, second = all_wave >> 2;         // second of a pair
    const Work w = find_work<kOwn>(a, blockIdx.x, a.hq / a.per, false);
    const int kv = w.head * a.per / a.group;
    const T* q0 = static_cast<const T*>(a.q) + int64_t(w.begin) * a.q_stride + w.head * a.per * H::kD;
    const T* go0 = static_cast<const T*>(a.go) + int64_t(w.begin) * a.o_stride + w.head * a.per * H::kD;
    const int own0 = w.first + 32 * wave, row = own0 + (lane & 31);          // this lane's key
    const bool live = own0 < w.rows;
    U4 k[H::kSteps], v[B::kPairs ? 1 : H::kSteps];
    {
        const int64_t token = int64_t(w.begin) + min(row, w.rows - 1);
        load_own<H>(static_cast<const T*>(a.k) + token * a.k_stride + kv * H::kD, k);
        if constexpr (!B::kPairs) load_own<H>(static_cast<const T*>(a.v) + token * a.v_stride + kv * H::kD, v);
    }
    const int first_tile = w.first / kStageRows, tiles = (w.rows + kStageRows - 1) / kStageRows;
    const float c = a.scale * kLog2e;
    // lse (times log2 e) and -D of a stage's queries: one value a thread of the first two waves
    float next = 0.f;
    auto fetch_stats = [&](int t, int head) __attribute__((always_inline)) {
        if (threadIdx.x >= 128) return;
        const uint32_t i = uint32_t(min(t * kStageRows + int(threadIdx.x & 63), w.rows - 1)) * uint32_t(a.hq);     // (below 2^29)
        const int64_t first = int64_t(w.begin) * a.hq + w.head * a.per + head;
        next = threadIdx.x < 64 ? (a.lse + first)[i] * kLog2e : (a.minus_d + first)[i];
    };
    auto put_stats = [&](int stage) __attribute__((always_inline)) {
        if (threadIdx.x < 128) stats[stage * 128 + threadIdx.x] = next;
    };
    auto fill_queries = [&](int t, int head, int stage) __attribute__((always_inline)) {
        fill_stage<H, B::kFilling>(q0 + head * H::kD, a.q_stride, t * kStageRows, w.rows, stages + stage * H::kStage);
        fill_stage<H, B::kFilling>(go0 + head * H::kD, a.o_stride, t * kStageRows, w.rows, stages + kGrads + stage * H::kStage);
        fetch_stats(t, head);
    };
    if constexpr (B::kPairs) {
        const T* values = static_cast<const T*>(a.v) + int64_t(w.begin) * a.v_stride + kv * H::kD;
        fill_stage<H, B::kFilling>(values, a.v_stride, w.first, w.rows, stages + B::kValues);
        if (w.first + kStageRows < w.rows) fill_stage<H, B::kFilling>(values, a.v_stride, w.first + kStageRows, w.rows, stages + B::kValues + H::kStage);
    }
    // P and dS of a tile: rows `part` on of stage `stage`, queries from query0 on
    const uint32_t stats_lane = stages + B::kStats + half * 16, own_values = B::kValues + wave * 32 * H::kPitch;
    auto weights = [&](int stage, int part, int query0, bool masked, f32x16& p, f32x16& ds) __attribute__((always_inline)) {
        const uint32_t rows = stage * H::kStage + part * H::kPitch;
        const uint32_t stats_at = stats_lane + (stage * 512 + part * 4);
        p = scores<H, H::kBf16 && !B::kPairs>(at, rows, k);
        const f32x16 from = H::kBf16 ? by_rows(stats_at + 256) : f32x16{};
        if constexpr (B::kPairs) ds = scores<H>(at, kGrads + rows, own_values, from);
        else ds = scores<H>(at, kGrads + rows, v, from);
        weigh<H>(p, ds, stats_at, 256, c);
        if (masked) mask_unseen(p, ds, query0 == own0 ? (lane & 31) : 0, w.rows - query0);
    };

    f32x16 dk[H::kBlocks], dv[H::kBlocks];
#pragma unroll
    for (int b = 0; b < H::kBlocks; ++b) dk[b] = dv[b] = f32x16{};
    auto add_queries = [&](int stage, int part, int query0, bool masked) __attribute__((always_inline)) {
        f32x16 p, ds;
        weights(stage, part, query0, masked, p, ds);
        const uint32_t rows = stage * H::kStage + part * H::kPitch;
        add_product<H>(at, kGrads + rows, p, dv);
        if (masked && w.rows <= kShort) add_rest<H>(at, kGrads + rows, p, dv);
        add_product<H>(at, rows, ds, dk);
        if (masked && w.rows <= kShort) add_rest<H>(at, rows, ds, dk);
    };
    // Stages of queries: of all heads the masked ones (the two of the block's own rows and the last one, if it is not whole), then
    // of all heads the others, of which every wave takes all.  (Both kinds in one loop cost the compiler copies of the sums.)
    const int count = tiles - first_tile, odd = w.rows % kStageRows != 0 && count > 2, broken = min(2 + odd, count);
    const int masked = broken * a.per, all = count * a.per;
    int head = 0, local = 0, now = 0;                  // of the next stage: its head and its place there; the tile of this one
    bool rest = false;                                 // it is one of the others
    auto fill_next = [&](int stage) __attribute__((always_inline)) {
        const int t = !rest && local == 2 ? tiles - 1 : first_tile + local;
        fill_queries(t, head, stage);
        if (++local == (rest ? count - odd : broken)) {
            if (++head == a.per) { head = 0; rest = true; }
            local = rest ? 2 : 0;
        }
        return t;
    };
    constexpr int kStep = B::kPairs ? kStageRows : 32;
    now = fill_next(masked & 1);
    for (int i = 0; i < masked; ++i) {
        const int stage = (i + masked) & 1, t = now;   // those after begin with stage 0
        put_stats(stage);
        wait_direct_loads();
        __syncthreads();
        if (i + 1 < all) now = fill_next(stage ^ 1);
#pragma unroll 1
        for (int part = 32 * second; part < kStageRows; part += kStep) {
            const int query0 = t * kStageRows + part;
            if (live && query0 >= own0 && query0 < w.rows) add_queries(stage, part, query0, query0 == own0 || query0 + 32 > w.rows);
        }
    }
    for (int i = masked; i < all; ++i) {
        const int stage = (i + masked) & 1;
        put_stats(stage);
        wait_direct_loads();
        __syncthreads();
        if (i + 1 < all) fill_next(stage ^ 1);
#pragma unroll
        for (int part = 0; part < kStageRows; part += kStep) add_queries(stage, part + 32 * second, 0, false);
    }
    settle<H>(dk);
    settle<H>(dv);
    int thread = threadIdx.x;                          // what follows from it is worked out anew rather than kept
    asm volatile("" : "+v"(thread));
    if constexpr (B::kPairs) {                         // the second halves' sums, through the stages, to the first
        static_assert(kWaves * H::kBlocks * 16 * 256 <= 4 * H::kStage, "one gradient's sums fit");
        float* mine = reinterpret_cast<float*>(lds) + wave * H::kBlocks * 16 * 64 + (thread & 63);
        auto join = [&](f32x16 (&x)[H::kBlocks]) __attribute__((always_inline)) {
            __syncthreads();
#pragma unroll
            for (int b = 0; b < H::kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (second) mine[(b * 16 + i) * 64] = x[b][i];
            __syncthreads();
#pragma unroll
            for (int b = 0; b < H::kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!second) x[b][i] += mine[(b * 16 + i) * 64];
        };
        join(dk);
        join(dv);
    }
    const int last_row = own0 + (thread & 31);
    const int64_t token = int64_t(w.begin) + min(last_row, w.rows - 1);
    const bool first_of_pair = second == 0, mine = first_of_pair && last_row < w.rows;
    T* dk_out = static_cast<T*>(a.dk) + token * a.k_stride + kv * H::kD;
    T* dv_out = static_cast<T*>(a.dv) + token * a.v_stride + kv * H::kD;
    typedef Head<float, H::kD> Sums;
    const int parts = a.hq / a.per;
    float* dk_part = a.parts + (token * parts + w.head) * H::kD;
    float* dv_part = dk_part + a.T * parts * H::kD;
    auto store = [&](T* out, float* part, int block, const f32x16& acc, float scale) __attribute__((always_inline)) {
        if (!mine) return;
        if (a.group == a.per) store_block<H>(out, acc, block, scale);
        else store_block<Sums>(part, acc, block, scale);
    };
    auto mend = [&](T* out, float* part, int block, const f32x16& acc, float scale) __attribute__((always_inline)) {
        if (!mine) return;
        if (a.group == a.per) mend_block<H>(out, acc, block, scale);
        else mend_block<Sums>(part, acc, block, scale);
    };
#pragma unroll
    for (int b = 0; b < H::kBlocks; ++b) {
        store(dk_out, dk_part, b, dk[b], a.scale);
        store(dv_out, dv_part, b, dv[b], 1.f);
    }
    if (!any_in_block(live && first_of_pair && !(all_finite(dk) && all_finite(dv)))) return;
    repair<H>(tiles * a.per, [&](int i) __attribute__((always_inline)) {
        fill_queries(i % tiles, i / tiles, 0);
        put_stats(0);
    }, 2 * H::kBlocks, [&](int i, int part, int job, f32x16& acc) __attribute__((always_inline)) {
        const int query0 = i % tiles * kStageRows + part, block = job >> 1;
        if (!live || !first_of_pair || query0 < own0 || query0 >= w.rows) return;
        f32x16 p, ds;
        weights(0, part, query0, query0 == own0 || query0 + 32 > w.rows, p, ds);
        const bool values = job & 1;
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = values ? p[i] : ds[i];
        add_block_where<H>(stages + (values ? kGrads : 0) + part * H::kPitch, p, acc, block,
                           [&](int query, int key) __attribute__((always_inline)) { return query0 + query >= own0 + key && query0 + query < w.rows; });
    }, [&](int job, const f32x16& acc) __attribute__((always_inline)) {
        if (job & 1) mend(dv_out, dv_part, job >> 1, acc, 1.f);
        else mend(dk_out, dk_part, job >> 1, acc, a.scale);
    });
}

// The parts of a group added up, in their order: four elements a thread.
template <typename T>
__global__ __launch_bounds__(kThreads) void attention_group_kernel(AttentionCall a, int64_t first, int64_t n) {
    const int64_t i = first + (int64_t(blockIdx.x) * kThreads + threadIdx.x) * 4;
    if (i >= n) return;
    const int hkv = a.hq / a.group;
    const int64_t row = i / a.d, token = row / hkv;                // of dk and dv
    const int column = int(i % a.d), head = int(row % hkv);
    const int parts = a.group / a.per;
    const float* part = a.parts + (blockIdx.y ? a.T * hkv * parts * a.d : 0) + row * parts * a.d + column;
    F4 sum = *reinterpret_cast<const F4*>(part);
    for (int g = 1; g < parts; ++g) sum += *reinterpret_cast<const F4*>(part + int64_t(g) * a.d);
    T* out = (blockIdx.y ? static_cast<T*>(a.dv) + token * a.v_stride : static_cast<T*>(a.dk) + token * a.k_stride) + head * a.d + column;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<F4*>(out) = sum;
    else *reinterpret_cast<U2*>(out) = U2{f32x2_to_bf16x2(sum.x, sum.y), f32x2_to_bf16x2(sum.z, sum.w)};
}

}  // namespace

int attention_tile_rows(bool narrow) { return narrow ? 32 : kOwn; }

bool attention_has_wide(int d, Dtype dtype) {
    bool has = false;
    with_head(dtype, d, [&](auto head) { has = decltype(head)::kHasWide; });
    return has;
}

// Query heads of a group that one block adds up for dk and dv: as many as leave two blocks or more for each that can run at a time,
// so that the short ones (a causal block's work is that of the rows behind it) fill in behind the long ones.  Parts are written and
// read again in 32 bits.
int attention_heads_per_block(int64_t tiles, int hq, int group, int d, Dtype dtype) {
    int per_unit = 1;
    with_head(dtype, d, [&](auto head) { per_unit = KeyBlock<decltype(head)>::kPerUnit; });
    for (int per = group; per > 1; --per)
        if (group % per == 0 && tiles * (hq / per) >= 2 * per_unit * int64_t(kUnits)) return per;
    return 1;
}

hipError_t launch_attention_forward(hipStream_t stream, const AttentionCall& a, Dtype dtype) {
    hipError_t e = hipSuccess;
    with_head(dtype, a.d, [&](auto head) {
        typedef decltype(head) H;
        if constexpr (H::kHasWide) e = launch_tiles<attention_forward_kernel<H>>(stream, a, 4 * H::kStage, a.tiles * a.hq + a.pad_blocks);
        else e = hipErrorInvalidValue;
    });
    return e;
}

hipError_t launch_attention_delta(hipStream_t stream, const AttentionCall& a, int64_t tokens, Dtype dtype) {
    const int64_t rows = tokens * a.hq, per = kThreads / 16;
    int64_t first = 0;
    do {
        const int blocks = int((std::min(rows - first, kMaxRowBlocks * per) + per - 1) / per);
        const bool last = first + kMaxRowBlocks * per >= rows;
        const dim3 grid(uint32_t(blocks + (last ? a.pad_blocks : 0)));
        if (dtype == Dtype::BF16) hipLaunchKernelGGL((attention_delta_kernel<uint16_t>), grid, dim3(kThreads), 0, stream, a, first, rows, blocks);
        else hipLaunchKernelGGL((attention_delta_kernel<float>), grid, dim3(kThreads), 0, stream, a, first, rows, blocks);
        first += kMaxRowBlocks * per;
    } while (first < rows);
    return hipGetLastError();
}

hipError_t launch_attention_backward(hipStream_t stream, const AttentionCall& a, Dtype dtype) {
    hipError_t e = hipSuccess;
    with_head(dtype, a.d, [&](auto head) {
        typedef decltype(head) H;
        if constexpr (H::kHasWide) {
            e = launch_tiles<attention_dq_kernel<H>>(stream, a, 4 * H::kStage, a.tiles * a.hq + a.pad_blocks);
            if (e == hipSuccess && a.tiles > 0) e = launch_tiles<attention_dkv_kernel<H>>(stream, a, KeyBlock<H>::kLds, a.tiles * (a.hq / a.per), KeyBlock<H>::kThreads);
        } else {
            e = hipErrorInvalidValue;
        }
    });
    return e;
}

hipError_t launch_attention_group(hipStream_t stream, const AttentionCall& a, int64_t tokens, Dtype dtype) {
    const int64_t n = tokens * (a.hq / a.group) * a.d, per = int64_t(kThreads) * 4;
    for (int64_t first = 0; first < n; first += kMaxRowBlocks * per) {
        const dim3 grid(uint32_t((std::min(n - first, kMaxRowBlocks * per) + per - 1) / per), 2);
        if (dtype == Dtype::BF16) hipLaunchKernelGGL((attention_group_kernel<uint16_t>), grid, dim3(kThreads), 0, stream, a, first, n);
        else hipLaunchKernelGGL((attention_group_kernel<float>), grid, dim3(kThreads), 0, stream, a, first, n);
    }
    return hipGetLastError();
}

}  // namespace tf
