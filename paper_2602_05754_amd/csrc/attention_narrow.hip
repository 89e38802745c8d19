// Attention for calls with few tiles: a block owns 32 rows instead of 128, and its four waves share out what passes by.
//
// The formulas, tiles and operands are those of attention.hip.  There a wave walks all the keys of its queries (or queries of its
// keys): with few tokens and heads most units have nothing to do, and the call takes as long as the longest walk.  Here each wave
// takes every fourth tile of 32 rows, through stages of its own (no barrier until the end), and the waves' parts are
// joined in LDS: results of the forward pass by their references and sums, gradients by adding up, wave by wave in their order.
// The blocks for dk and dv and those for dq are one launch, but for fp32 heads of more than 96 elements, whose two
// kinds of sums and own rows do not fit one kernel's registers.
#include "attention_device.h"

namespace tf {
namespace {

template <class H>
struct Narrow {
    static constexpr int kTile = 32 * H::kPitch;                   // bytes of 32 rows of one tensor
    static constexpr int kBuffers = kWaves * 4 * kTile <= 128 * 1024 ? 2 : 1;
    static constexpr int kStats = kBuffers * 2 * kTile;            // bytes to a wave's [buffer][lse, -D][32], or its m and l
    static constexpr int kWave = kStats + 512;
    static constexpr int kLds = kWaves * kWave;
    static constexpr bool kOwnInLds = !H::kBf16 && H::kD > 96;     // the block's own values, for dk and dv: registers are short
    static constexpr int kKeysLds = kLds + (kOwnInLds ? kTile : 0);
    static constexpr int kLoads = 2 * kTile / 1024;                // of a tile of two tensors
    static constexpr int kPerUnit = H::kBf16 && kLds <= 80 * 1024 ? 2 : 1;
    static_assert(2 * H::kBlocks * 4096 <= kStats, "the sums of two gradients fit");
};

// Rows [first, first + 32) of the `rows` that exist, at least one -> this wave's LDS.
template <class H>
__device__ __forceinline__ void fill_tile(const typename H::T* base, int64_t pitch, int first, int rows, uint32_t to) {
    const int lane = threadIdx.x & 63;
    constexpr int kRowsPerLoad = 1024 / H::kPitch;
    const int last = rows - 1 - first;
    const uint64_t at = reinterpret_cast<uint64_t>(base + int64_t(first) * pitch);
    const uint32_t high = __builtin_amdgcn_readfirstlane(uint32_t(at >> 32)), low = __builtin_amdgcn_readfirstlane(uint32_t(at));      // (it gives an int)
    const char* from = reinterpret_cast<const char*>(uint64_t(high) << 32 | low);
    const uint32_t row_bytes = uint32_t(pitch) * uint32_t(sizeof(typename H::T)), lds = __builtin_amdgcn_readfirstlane(to);
    static_for<32 / kRowsPerLoad>([&](auto i) __attribute__((always_inline)) {
        const int r = i * kRowsPerLoad + lane / H::kRoom;
        int c = (lane % H::kRoom) ^ swizzle<H>(r);
        if constexpr (H::kChunks < H::kRoom) c = c < H::kChunks ? c : 0;
        direct_load_16B<i * 1024>(from, uint32_t(min(r, last)) * row_bytes + uint32_t(c) * 16, lds);
    });
}

// Four bytes a lane, from anywhere, to the wave's 256 bytes at `to` (see direct_load_16B()).
__device__ __forceinline__ void direct_load_4B(const float* from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from)
                 : "memory", "m0");
}

template <typename V> __device__ __forceinline__ void lds_write(uint32_t at, V v) {
    *(__attribute__((address_space(3))) V*)(uintptr_t(at)) = v;
}

// This wave's tiles, `wave`, wave + 4, ... of `tiles`: fill(tile, buffer), of kLoads direct loads, ahead of add(tile, buffer).
template <class H, int kLoads, class Fill, class Add>
__device__ __forceinline__ void walk_tiles(int wave, int tiles, Fill&& fill, Add&& add) {
    typedef Narrow<H> N;
    int buffer = 0;
    if (wave < tiles) fill(wave, 0);
#pragma unroll 1
    for (int t = wave; t < tiles; t += kWaves) {
        if (N::kBuffers == 2 && t + kWaves < tiles) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the tile before has been read
            fill(t + kWaves, buffer ^ 1);
            wait_loads<kLoads>();
        } else {
            wait_direct_loads();
        }
        asm volatile("" ::: "memory");
        add(t, buffer);
        if (N::kBuffers == 1) {
            if (t + kWaves < tiles) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                fill(t + kWaves, 0);
            }
        } else {
            buffer ^= 1;
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// acc^T of this wave -> its LDS, and a block of 32 columns of all waves' added up, each times its factor.
template <class H>
__device__ __forceinline__ void put_sums(uint32_t to, const f32x16 (&x)[H::kBlocks]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int b = 0; b < H::kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) lds_write<float>(to + uint32_t((b * 16 + i) * 256 + lane * 4), x[b][i]);
}
template <class H>
__device__ __forceinline__ f32x16 take_sums(uint32_t stages, int block, const float (&factor)[kWaves]) {
    const int lane = threadIdx.x & 63;
    f32x16 sum = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] += factor[w] * lds_read<float>(stages + uint32_t(w * Narrow<H>::kWave + (block * 16 + i) * 256 + lane * 4));
    return sum;
}
__device__ __forceinline__ bool is_finite(const f32x16& x) {
    float zero = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) zero += 0.f * x[i];
    return zero == 0.f;
}

template <class H>
__global__ __launch_bounds__(kThreads, Narrow<H>::kPerUnit) void attention_forward_narrow_kernel(AttentionCall a) {
    typedef typename H::T T;
    typedef Narrow<H> N;
    if (int(blockIdx.x) >= a.tiles * a.hq) return clear_padding<T>(a, blockIdx.x - a.tiles * a.hq);
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const uint32_t stages = lds_address(lds), own_stage = stages + wave * N::kWave;
    const Lane<H> at(own_stage);
    const Work w = find_work<32>(a, blockIdx.x, a.hq, true);
    const int kv = w.head / a.group, row = w.first + (lane & 31);
    const T* k = static_cast<const T*>(a.k) + int64_t(w.begin) * a.k_stride + kv * H::kD;
    const T* v = static_cast<const T*>(a.v) + int64_t(w.begin) * a.v_stride + kv * H::kD;
    const int64_t token = int64_t(w.begin) + min(row, w.rows - 1);
    U4 q[H::kSteps];
    load_own<H>(static_cast<const T*>(a.q) + token * a.q_stride + w.head * H::kD, q);
    const float c = a.scale * kLog2e;
    const int tiles = w.first / 32 + 1;
    f32x16 o[H::kBlocks];
#pragma unroll
    for (int b = 0; b < H::kBlocks; ++b) o[b] = f32x16{};
    float m = kNoReference, l = 0.f;
    auto fill = [&](int t, int buffer) __attribute__((always_inline)) {
        fill_tile<H>(k, a.k_stride, t * 32, w.rows, own_stage + buffer * 2 * N::kTile);
        fill_tile<H>(v, a.v_stride, t * 32, w.rows, own_stage + buffer * 2 * N::kTile + N::kTile);
    };
    walk_tiles<H, N::kLoads>(wave, tiles, fill, [&](int t, int buffer) __attribute__((always_inline)) {
        const uint32_t rows = buffer * 2 * N::kTile;
        attend<H>(at, rows, rows + N::kTile, q, c, t == tiles - 1, m, l, o);
    });
    settle<H>(o);
    l = with_other_half(l, [](float x, float y) { return x + y; });
    put_sums<H>(own_stage, o);
    lds_write<float>(own_stage + N::kStats + lane * 4, m);
    lds_write<float>(own_stage + N::kStats + 256 + lane * 4, l);
    __syncthreads();
    float of_wave[kWaves], factor[kWaves], top = kNoReference, sum = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        of_wave[i] = lds_read<float>(stages + uint32_t(i * N::kWave + N::kStats + lane * 4));
        top = fmaxf(top, of_wave[i]);
    }
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        factor[i] = __builtin_amdgcn_exp2f(of_wave[i] - top);
        sum += factor[i] * lds_read<float>(stages + uint32_t(i * N::kWave + N::kStats + 256 + lane * 4));
    }
    const bool taking = wave < H::kBlocks;             // a block of 32 columns
    const int block = taking ? wave : 0;
    const f32x16 mine = take_sums<H>(stages, block, factor);
    const float inverse = 1.f / sum;
    T* out = static_cast<T*>(a.o) + token * a.o_stride + w.head * H::kD;
    const bool writes = taking && row < w.rows;
    if (writes) {
        store_block<H>(out, mine, block, inverse);
        if (wave == 0 && half == 0) a.lse[token * a.hq + w.head] = (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
    if (!any_in_block(!is_finite(mine)) || !taking) return;
    f32x16 again = {};                                 // (see repair())
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        fill(t, 0);
        wait_direct_loads();
        asm volatile("" ::: "memory");
        f32x16 s = scores<H>(at, 0, q);
        if (t == tiles - 1) mask_later(s);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -top));
        add_block_where<H>(own_stage + N::kTile, s, again, block,
                           [&](int key, int query) __attribute__((always_inline)) { return t * 32 + key <= w.first + query; });
    }
    if (writes) mend_block<H>(out, again, block, inverse);
}

template <class H>
__device__ __forceinline__ void narrow_dq(const AttentionCall& a, int number, char* lds) {
    typedef typename H::T T;
    typedef Narrow<H> N;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t stages = lds_address(lds), own_stage = stages + wave * N::kWave;
    const Lane<H> at(own_stage);
    const Work w = find_work<32>(a, number, a.hq, true);
    const int kv = w.head / a.group, row = w.first + (lane & 31);
    const T* k = static_cast<const T*>(a.k) + int64_t(w.begin) * a.k_stride + kv * H::kD;
    const T* v = static_cast<const T*>(a.v) + int64_t(w.begin) * a.v_stride + kv * H::kD;
    const int64_t token = int64_t(w.begin) + min(row, w.rows - 1);
    U4 q[H::kSteps], go[H::kSteps];
    load_own<H>(static_cast<const T*>(a.q) + token * a.q_stride + w.head * H::kD, q);
    load_own<H>(static_cast<const T*>(a.go) + token * a.o_stride + w.head * H::kD, go);
    const float lse = a.lse[token * a.hq + w.head] * kLog2e, minus_d = a.minus_d[token * a.hq + w.head], c = a.scale * kLog2e;
    const int tiles = w.first / 32 + 1;
    f32x16 dq[H::kBlocks];
#pragma unroll
    for (int b = 0; b < H::kBlocks; ++b) dq[b] = f32x16{};
    auto fill = [&](int t, int buffer) __attribute__((always_inline)) {
        fill_tile<H>(k, a.k_stride, t * 32, w.rows, own_stage + buffer * 2 * N::kTile);
        fill_tile<H>(v, a.v_stride, t * 32, w.rows, own_stage + buffer * 2 * N::kTile + N::kTile);
    };
    walk_tiles<H, N::kLoads>(wave, tiles, fill, [&](int t, int buffer) __attribute__((always_inline)) {
        const uint32_t rows = buffer * 2 * N::kTile;
        const f32x16 ds = score_gradients<H>(at, rows, rows + N::kTile, q, go, c, lse, minus_d, t == tiles - 1);
        add_product<H>(at, rows, ds, dq);
        if (w.rows <= kShort) add_rest<H>(at, rows, ds, dq);
    });
    settle<H>(dq);
    put_sums<H>(own_stage, dq);
    __syncthreads();
    const float ones[kWaves] = {1.f, 1.f, 1.f, 1.f};
    const bool taking = wave < H::kBlocks;
    const int block = taking ? wave : 0;
    const f32x16 mine = take_sums<H>(stages, block, ones);
    T* out = static_cast<T*>(a.dq) + token * a.q_stride + w.head * H::kD;
    const bool writes = taking && row < w.rows;
    if (writes) store_block<H>(out, mine, block, a.scale);
    if (!any_in_block(!is_finite(mine)) || !taking) return;
    f32x16 again = {};
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        fill(t, 0);
        wait_direct_loads();
        asm volatile("" ::: "memory");
        add_block_where<H>(own_stage, score_gradients<H>(at, 0, N::kTile, q, go, c, lse, minus_d, t == tiles - 1), again, block,
                           [&](int key, int query) __attribute__((always_inline)) { return t * 32 + key <= w.first + query; });
    }
    if (writes) mend_block<H>(out, again, block, a.scale);
}

template <class H>
__device__ __forceinline__ void narrow_dkv(const AttentionCall& a, int number, char* lds) {
    typedef typename H::T T;
    typedef Narrow<H> N;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const uint32_t stages = lds_address(lds), own_stage = stages + wave * N::kWave;
    const Lane<H> at(own_stage);
    const Work w = find_work<32>(a, number, a.hq / a.per, false);
    const int kv = w.head * a.per / a.group, row = w.first + (lane & 31);
    const T* q0 = static_cast<const T*>(a.q) + int64_t(w.begin) * a.q_stride + w.head * a.per * H::kD;
    const T* go0 = static_cast<const T*>(a.go) + int64_t(w.begin) * a.o_stride + w.head * a.per * H::kD;
    const int64_t token = int64_t(w.begin) + min(row, w.rows - 1);
    U4 k[H::kSteps];
    [[maybe_unused]] U4 v[H::kSteps];
    load_own<H>(static_cast<const T*>(a.k) + token * a.k_stride + kv * H::kD, k);
    if constexpr (N::kOwnInLds) {
        if (wave == 0) {
            fill_tile<H>(static_cast<const T*>(a.v) + int64_t(w.begin) * a.v_stride + kv * H::kD, a.v_stride, w.first, w.rows, stages + kWaves * N::kWave);
            wait_direct_loads();
        }
        __syncthreads();
    } else {
        load_own<H>(static_cast<const T*>(a.v) + token * a.v_stride + kv * H::kD, v);
    }
    const float c = a.scale * kLog2e;
    const int of_head = (w.rows - w.first + 31) / 32, tiles = of_head * a.per;         // of queries, from the block's own rows on
    f32x16 dk[H::kBlocks], dv[H::kBlocks];
#pragma unroll
    for (int b = 0; b < H::kBlocks; ++b) dk[b] = dv[b] = f32x16{};
    auto fill = [&](int i, int buffer) __attribute__((always_inline)) {
        const int head = i / of_head, first = w.first + (i - head * of_head) * 32;
        fill_tile<H>(q0 + head * H::kD, a.q_stride, first, w.rows, own_stage + buffer * 2 * N::kTile);
        fill_tile<H>(go0 + head * H::kD, a.o_stride, first, w.rows, own_stage + buffer * 2 * N::kTile + N::kTile);
        const int64_t of = int64_t(w.begin + min(first + (lane & 31), w.rows - 1)) * a.hq + w.head * a.per + head;
        direct_load_4B((half == 0 ? a.lse : a.minus_d) + of, own_stage + N::kStats + buffer * 256);
    };
    auto weights = [&](int i, int buffer, f32x16& p, f32x16& ds) __attribute__((always_inline)) {
        const uint32_t rows = buffer * 2 * N::kTile;
        p = scores<H>(at, rows, k);
        const uint32_t stats_at = own_stage + N::kStats + buffer * 256 + half * 16;
        if constexpr (N::kOwnInLds) ds = scores<H>(at, rows + N::kTile, uint32_t((kWaves - wave) * N::kWave));
        else ds = scores<H>(at, rows + N::kTile, v, H::kBf16 ? by_rows(stats_at + 128) : f32x16{});
        weigh<H>(p, ds, stats_at, 128, c, kLog2e);
        const int tile = i % of_head, left = w.rows - (w.first + tile * 32);
        if (tile == 0 || left < 32) mask_unseen(p, ds, tile == 0 ? (lane & 31) : 0, left);
    };
    walk_tiles<H, N::kLoads + 1>(wave, tiles, fill, [&](int i, int buffer) __attribute__((always_inline)) {
        const uint32_t rows = buffer * 2 * N::kTile;
        f32x16 p, ds;
        weights(i, buffer, p, ds);
        add_product<H>(at, rows + N::kTile, p, dv);
        add_product<H>(at, rows, ds, dk);
        if (w.rows <= kShort) {
            add_rest<H>(at, rows + N::kTile, p, dv);
            add_rest<H>(at, rows, ds, dk);
        }
    });
    settle<H>(dk);
    settle<H>(dv);
    put_sums<H>(own_stage, dk);
    put_sums<H>(own_stage + H::kBlocks * 4096, dv);
    __syncthreads();
    typedef Head<float, H::kD> Sums;
    const int parts = a.hq / a.per;
    T* dk_out = static_cast<T*>(a.dk) + token * a.k_stride + kv * H::kD;
    T* dv_out = static_cast<T*>(a.dv) + token * a.v_stride + kv * H::kD;
    float* dk_part = a.parts + (token * parts + w.head) * H::kD;
    float* dv_part = dk_part + a.T * parts * H::kD;
    const float ones[kWaves] = {1.f, 1.f, 1.f, 1.f};
    const bool inside = row < w.rows, whole = a.group == a.per;
    bool bad = false;
    // 2 kBlocks blocks of 32 columns, those of dk first, in turn to the waves
#pragma unroll 1
    for (int job = wave; job < 2 * H::kBlocks; job += kWaves) {
        const f32x16 mine = take_sums<H>(stages, job, ones);
        bad = bad || !is_finite(mine);
        if (!inside) continue;
        if (job < H::kBlocks) {
            if (whole) store_block<H>(dk_out, mine, job, a.scale);
            else store_block<Sums>(dk_part, mine, job, a.scale);
        } else {
            if (whole) store_block<H>(dv_out, mine, job - H::kBlocks, 1.f);
            else store_block<Sums>(dv_part, mine, job - H::kBlocks, 1.f);
        }
    }
    if (!any_in_block(bad)) return;
#pragma unroll 1
    for (int job = wave; job < 2 * H::kBlocks; job += kWaves) {
        const bool values = job >= H::kBlocks;
        const int block = values ? job - H::kBlocks : job;
        f32x16 again = {};
#pragma unroll 1
        for (int i = 0; i < tiles; ++i) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            fill(i, 0);
            wait_direct_loads();
            asm volatile("" ::: "memory");
            f32x16 p, ds;
            weights(i, 0, p, ds);
#pragma unroll
            for (int e = 0; e < 16; ++e) p[e] = values ? p[e] : ds[e];
            const int from = i % of_head * 32, left = w.rows - w.first - from;
            add_block_where<H>(own_stage + (values ? N::kTile : 0), p, again, block,
                               [&](int query, int key) __attribute__((always_inline)) { return from + query >= key && query < left; });
        }
        if (!inside) continue;
        if (values) {
            if (whole) mend_block<H>(dv_out, again, block, 1.f);
            else mend_block<Sums>(dv_part, again, block, 1.f);
        } else {
            if (whole) mend_block<H>(dk_out, again, block, a.scale);
            else mend_block<Sums>(dk_part, again, block, a.scale);
        }
    }
}

enum class Half { kBoth, kKeys, kQueries };
template <class H, Half kHalf>
__global__ __launch_bounds__(kThreads, Narrow<H>::kPerUnit) void attention_backward_narrow_kernel(AttentionCall a) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    if constexpr (kHalf == Half::kKeys) {
        narrow_dkv<H>(a, blockIdx.x, lds);
    } else if constexpr (kHalf == Half::kQueries) {
        narrow_dq<H>(a, blockIdx.x, lds);
    } else {
        const int keys = a.tiles * (a.hq / a.per);
        if (int(blockIdx.x) < keys) narrow_dkv<H>(a, blockIdx.x, lds);
        else narrow_dq<H>(a, int(blockIdx.x) - keys, lds);
    }
}

}  // namespace

hipError_t launch_attention_forward_narrow(hipStream_t stream, const AttentionCall& a, Dtype dtype) {
    hipError_t e = hipSuccess;
    with_head(dtype, a.d, [&](auto head) {
        typedef decltype(head) H;
        e = launch_tiles<attention_forward_narrow_kernel<H>>(stream, a, Narrow<H>::kLds, a.tiles * a.hq + a.pad_blocks);
    });
    return e;
}

hipError_t launch_attention_backward_narrow(hipStream_t stream, const AttentionCall& a, Dtype dtype) {
    hipError_t e = hipSuccess;
    with_head(dtype, a.d, [&](auto head) {
        typedef decltype(head) H;
        constexpr int kLds = Narrow<H>::kLds;
        const int keys = a.tiles * (a.hq / a.per), queries = a.tiles * a.hq;
        if constexpr (!Narrow<H>::kOwnInLds) {
            e = launch_tiles<attention_backward_narrow_kernel<H, Half::kBoth>>(stream, a, kLds, keys + queries);
        } else {
            e = launch_tiles<attention_backward_narrow_kernel<H, Half::kKeys>>(stream, a, Narrow<H>::kKeysLds, keys);
            if (e == hipSuccess) e = launch_tiles<attention_backward_narrow_kernel<H, Half::kQueries>>(stream, a, kLds, queries);
        }
    });
    return e;
}

}  // namespace tf
