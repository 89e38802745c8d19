// Embedding lookup with scaling and its gradient.
//
//   forward   out_t = scale table[id_t]
//   backward  dtable_v (+)= scale sum of dout_t over the tokens with id_t = v, t ascending
// An id outside [0, rows) stands for no row: zeros, and nothing added.
//
// Bound by memory.  The gradient sums in a fixed order without atomics: the tokens are sorted by id (radix sort of chunks in LDS,
// which keeps the order of equal ids, and a merge where there are several chunks), and the sorted places are shared out in windows of
// kWindow, so that a frequent id is no more work to one block than rare ones.  An id whose tokens are within a window is
// done there; the sums of one that goes on in others are added up, window by window, by a kernel after it.
// Rows without tokens are zeros: the blocks that do not sort fill the whole gradient meanwhile, at the rate of
// a fill, and the rows that have tokens are written again.
//
// us, 4096 tokens of 65536 ids, 4096 columns of bf16 (537 MB, which a fill alone writes in 80): sort and fill 85, windows 19 to 21 (67 MB), join 5
// to 7; 8192 tokens, 2048 columns, forward: 10.2 (34 MB written, as much or less read).
// Added to fp32 sums no fill hides the sort, which has one workgroup for 8192 tokens.  us and those of the bytes alone, 32000 ids, 2048
// columns: 1024 tokens 22, 3; 4096 33, 10; 8192 52, 18; 16384 86, 31; 65536 ids, 4096 columns, 4096 tokens 46, 20.  The merge searches every
// other chunk for each token, tokens times chunks: 131072 tokens of 64 columns 105, 2^20 1080.
#include "row_device.h"

#include <algorithm>

namespace tf {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = kEmbeddingChunk, kWindow = kEmbeddingWindow;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kPerThread = kChunk / kSortThreads;
constexpr int kJoinThreads = 512, kJoinWaves = kJoinThreads / 64;
constexpr int kFewTokens = kSortThreads / 2;           // sorted by counting.  us, 64 tokens of 30000 ids: radix 11, counting 4

// Lanes of a row: a power of two, each with pieces kLanes apart.
int lanes_of(int d, int per, int most) {
    int lanes = 1;
    while (lanes < most && lanes * per < d) lanes *= 2;
    return lanes;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void lookup_kernel(EmbeddingCall e, int lanes, int64_t first) {
    const int64_t t = first + int64_t(blockIdx.x) * (kThreads / lanes) + threadIdx.x / lanes;
    if (t >= e.T) return;
    const int id = e.ids[t];
    const bool there = id >= 0 && id < e.rows;
    const T* row = static_cast<const T*>(e.table) + int64_t(there ? id : 0) * e.d;
    T* out = static_cast<T*>(e.out) + t * e.d;
    for (int c = threadIdx.x % lanes * kPer<T>; c < e.d; c += lanes * kPer<T>) {
        float x[kPer<T>];
        unpack<T>(there ? load_piece(row + c, e.d - c) : U4{0, 0, 0, 0}, x);
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j) x[j] = there ? x[j] * e.scale : 0.f;
        store_piece(out + c, e.d - c, x);
    }
}

// Blocks [0, chunks): sort a chunk.  The other blocks: zeros to the gradient, `n` pieces of 16 bytes and `rest` bytes.
__global__ __launch_bounds__(kSortThreads) void sort_kernel(EmbeddingCall e, int bits, int64_t n, int rest) {
    if (int(blockIdx.x) >= e.chunks) {
        U4* out = static_cast<U4*>(e.dtable);
        const int64_t blocks = gridDim.x - e.chunks, each = (n + blocks - 1) / blocks, begin = each * (blockIdx.x - e.chunks), end = min(n, begin + each);
        for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads) out[i] = U4{0, 0, 0, 0};
        if (int(blockIdx.x) == e.chunks && int(threadIdx.x) * 2 < rest) reinterpret_cast<uint16_t*>(out + n)[threadIdx.x] = 0;
        return;
    }
    __shared__ __attribute__((aligned(16))) uint32_t key[kChunk];
    __shared__ uint16_t token[kChunk];
    __shared__ int count[kSortWaves][64];              // of a digit in a wave's keys, then where they go
    __shared__ int wave_sum[kSortWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = int64_t(blockIdx.x) * kChunk;
    const int here = int(min(int64_t(kChunk), e.T - first));
    auto put = [&](int place, uint32_t k, int from) __attribute__((always_inline)) {
        const bool there = k < uint32_t(e.rows);
        e.sorted_id[first + place] = there ? int(k) : -1;
        e.sorted_token[first + place] = there ? int(first) + from : 0;
    };
    auto key_of = [&](int i) __attribute__((always_inline)) {
        const int id = i < here ? e.ids[first + i] : -1;
        return i < here ? id >= 0 && id < e.rows ? uint32_t(id) : uint32_t(e.rows) : ~0u;
    };
    if (e.T <= kFewTokens) {                           // a key's place: the keys before it, counted by `sharing` threads
        int sharing = kSortThreads / kFewTokens;
        while (sharing < 16 && 2 * sharing * here <= kSortThreads) sharing *= 2;
        if (threadIdx.x < kFewTokens) key[threadIdx.x] = key_of(threadIdx.x);
        __syncthreads();
        const int i = int(threadIdx.x) / sharing, pieces = (here + 3) / 4, each = (pieces + sharing - 1) / sharing;
        const int begin = int(threadIdx.x) % sharing * each, end = min(begin + each, pieces);
        const uint32_t mine = key[i];
        int place = 0;
        for (int j = begin; j < end; ++j) {
            const U4 x = *reinterpret_cast<const U4*>(key + 4 * j);
#pragma unroll
            for (int q = 0; q < 4; ++q) place += x[q] < mine + (4 * j + q < i);
        }
        for (int o = sharing / 2; o > 0; o /= 2) place += __shfl_xor(place, o, 64);
        if (threadIdx.x % sharing == 0) put(i < here ? place : i, mine, i);            // (the last window to its end)
        return;
    }
    const int rounds = (here + kSortThreads - 1) / kSortThreads, mine = wave * rounds * 64 + lane;     // a wave's keys are neighbours
    for (int r = 0; r < rounds; ++r) {
        const int i = mine + r * 64;
        key[i] = min(key_of(i), uint32_t(e.rows));
        token[i] = uint16_t(i);
    }
    for (int shift = 0; shift < bits; shift += 6) {
        __syncthreads();
        uint32_t k[kPerThread];
        int from[kPerThread], rank[kPerThread], seen = 0;              // seen: of digit `lane` so far
#pragma unroll
        for (int r = 0; r < kPerThread; ++r) {
            if (r >= rounds) continue;
            k[r] = key[mine + r * 64];
            from[r] = token[mine + r * 64];
            const int digit = int(k[r] >> shift) & 63;
            uint64_t same = ~uint64_t(0), of_lane = ~uint64_t(0);
#pragma unroll
            for (int b = 0; b < 6; ++b) {
                const uint64_t set = __ballot(digit >> b & 1);
                same &= digit >> b & 1 ? set : ~set;
                of_lane &= lane >> b & 1 ? set : ~set;
            }
            rank[r] = __shfl(seen, digit, 64) + __popcll(same & ((uint64_t(1) << lane) - 1));
            seen += __popcll(of_lane);
        }
        count[wave][lane] = seen;
        __syncthreads();
        // the 64 x 16 counts in the order (digit, wave): their sums so far
        const int digit = threadIdx.x / kSortWaves, w = threadIdx.x % kSortWaves;
        const int mine_count = count[w][digit];
        int sum = mine_count;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int other = __shfl_up(sum, o, 64);
            if (lane >= o) sum += other;
        }
        if (lane == 63) wave_sum[wave] = sum;
        __syncthreads();
        for (int i = 0; i < wave; ++i) sum += wave_sum[i];
        count[w][digit] = sum - mine_count;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kPerThread; ++r) {
            if (r >= rounds) continue;
            const int to = count[wave][int(k[r] >> shift) & 63] + rank[r];
            key[to] = k[r];
            token[to] = uint16_t(from[r]);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kChunk; i += kSortThreads) put(i, i < here ? key[i] : ~0u, token[i]);
}

// The chunks' orders made one: a place moves behind those of smaller ids in all other chunks, and of the same id in those before.
__global__ __launch_bounds__(kThreads) void merge_kernel(EmbeddingCall e, int64_t first) {
    const int64_t place = first + int64_t(blockIdx.x) * kThreads + threadIdx.x;
    if (place >= int64_t(e.chunks) * kChunk) return;
    const int own = int(place / kChunk);
    const uint32_t id = uint32_t(e.sorted_id[place]);              // (no row, -1, comes last)
    int64_t to = place;
    if (place < e.T) {
        to = place % kChunk;
        for (int k = 0; k < e.chunks; ++k) {
            if (k == own) continue;
            const int32_t* ids = e.sorted_id + int64_t(k) * kChunk;
            int lo = 0, hi = int(min(int64_t(kChunk), e.T - int64_t(k) * kChunk));
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                const uint32_t x = uint32_t(ids[mid]);
                if (k < own ? x <= id : x < id) lo = mid + 1;
                else hi = mid;
            }
            to += lo;
        }
    }
    e.merged_id[to] = int(id);
    e.merged_token[to] = e.sorted_token[place];
}

// Eight or four columns of a row of the gradient.
template <typename T, typename TOut, bool kAdd>
__device__ __forceinline__ void put_row(const EmbeddingCall& e, int id, int c, const float (&acc)[kPer<T>], const float (&old)[kPer<T>]) {
    TOut* out = static_cast<TOut*>(e.dtable) + int64_t(id) * e.d + c;
#pragma unroll
    for (int j = 0; j < kPer<T>; j += kPer<TOut>) {
        float part[kPer<TOut>];
#pragma unroll
        for (int q = 0; q < kPer<TOut>; ++q) part[q] = fmaf(acc[j + q], e.scale, kAdd ? old[j + q] : 0.f);
        if (c + j < e.d) store_piece(out + j, e.d - c - j, part);
    }
}
template <typename T, typename TOut, bool kAdd>
__device__ __forceinline__ void old_row(const EmbeddingCall& e, int id, int c, float (&old)[kPer<T>]) {
    if constexpr (kAdd) {
        const TOut* out = static_cast<const TOut*>(e.dtable) + int64_t(id) * e.d + c;
#pragma unroll
        for (int j = 0; j < kPer<T>; j += kPer<TOut>) {
            float part[kPer<TOut>];
            unpack<TOut>(c + j < e.d ? load_piece(out + j, e.d - c - j) : U4{0, 0, 0, 0}, part);
#pragma unroll
            for (int q = 0; q < kPer<TOut>; ++q) old[j + q] = part[q];
        }
    }
}

// A window: `lanes` threads, kPer<T> columns each, and as many blocks beside each other as its columns take.  What an id gets
// from it is the row, or goes to windows[w][0] where earlier windows have the id too and to windows[w][1] where later ones only.
template <typename T, typename TOut, bool kAdd>
__global__ __launch_bounds__(kThreads) void window_kernel(EmbeddingCall e, int lanes, int64_t first) {
    const int64_t from = (first + int64_t(blockIdx.x) * (kThreads / lanes) + threadIdx.x / lanes) * kWindow;
    const int c = (blockIdx.y * kThreads + threadIdx.x % lanes) * kPer<T>;
    if (from >= e.T || c >= e.d) return;
    int id[kWindow + 1], token[kWindow];
#pragma unroll
    for (int j = 0; j < kWindow; j += 4) {
        const U4 x = *reinterpret_cast<const U4*>(e.merged_id + from + j), y = *reinterpret_cast<const U4*>(e.merged_token + from + j);
#pragma unroll
        for (int q = 0; q < 4; ++q) { id[j + q] = int(x[q]); token[j + q] = int(y[q]); }
    }
    id[kWindow] = from + kWindow < e.T ? e.merged_id[from + kWindow] : -1;
    const int before = from > 0 ? e.merged_id[from - 1] : -1;
    const T* dout = static_cast<const T*>(e.dout) + c;
    float* sums = e.windows + from / kWindow * 2 * e.pitch + c;
    constexpr int kAhead = kAdd ? 8 : 16;              // rows on their way
    float acc[kPer<T>] = {};
    bool begins = id[0] != before;
#pragma unroll
    for (int part = 0; part < kWindow; part += kAhead) {
        U4 x[kAhead];
        [[maybe_unused]] float old[kAhead][kPer<T>];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            x[j] = load_piece(dout + int64_t(token[part + j]) * e.d, e.d - c);         // (of no row: some token's)
            if constexpr (kAdd)
                if (id[part + j] >= 0 && id[part + j + 1] != id[part + j]) old_row<T, TOut, kAdd>(e, id[part + j], c, old[j]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int here = id[part + j];
            const bool last = part + j == kWindow - 1, ends = id[part + j + 1] != here;
            float v[kPer<T>];
            unpack<T>(x[j], v);
#pragma unroll
            for (int q = 0; q < kPer<T>; ++q) acc[q] += v[q];
            if (!ends && !last) continue;
            if (here >= 0) {
                if (begins && ends) {
                    put_row<T, TOut, kAdd>(e, here, c, acc, old[j]);
                } else {
                    float* to = sums + (begins ? e.pitch : 0);
#pragma unroll
                    for (int q = 0; q < kPer<T>; q += 4) *reinterpret_cast<F4*>(to + q) = F4{acc[q], acc[q + 1], acc[q + 2], acc[q + 3]};
                }
            }
#pragma unroll
            for (int q = 0; q < kPer<T>; ++q) acc[q] = 0.f;
            begins = true;
        }
    }
}

// The ids of several windows, by the block of the window that they begin in: its waves take every kJoinWaves-th window, 512 columns.
template <typename TOut, bool kAdd>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(EmbeddingCall e, int64_t first) {
    const int64_t w = first + blockIdx.x, from = w * kWindow, windows = (e.T + kWindow - 1) / kWindow;
    const int id = e.merged_id[from + kWindow];
    if (id < 0 || e.merged_id[from + kWindow - 1] != id || (from > 0 && e.merged_id[from - 1] == id)) return;
    __shared__ float part[kJoinThreads][8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t end = w + 1;                               // behind the windows that have the id
    for (bool more = true; more;) {
        int found = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t k = end + 64 * i + lane;
            found += __popcll(__ballot(k < windows && e.merged_id[min(k, windows - 1) * kWindow] == id));
        }
        end += found;
        more = found == 256;
    }
    const int c = blockIdx.y * 512 + lane * 8;
    const float* sums = e.windows + min(c, e.pitch - 8);           // (a lane without columns: the last ones, for nothing)
    float acc[8] = {};
    constexpr int kAhead = 8;
    for (int64_t k = w + 1 + wave; k < end; k += kAhead * kJoinWaves) {
        F4 x[kAhead][2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) x[i][h] = *reinterpret_cast<const F4*>(sums + 2 * min(k + i * kJoinWaves, end - 1) * e.pitch + 4 * h);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int q = 0; q < 8; ++q) acc[q] += k + i * kJoinWaves < end ? x[i][q / 4][q % 4] : 0.f;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) part[threadIdx.x][q] = acc[q];
    __syncthreads();
    if (wave > 0 || c >= e.d) return;
    float old[8] = {};
    old_row<uint16_t, TOut, kAdd>(e, id, c, old);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        acc[q] = sums[(2 * w + 1) * e.pitch + q];
#pragma unroll
        for (int i = 0; i < kJoinWaves; ++i) acc[q] += part[i * 64 + lane][q];
    }
    put_row<uint16_t, TOut, kAdd>(e, id, c, acc, old);
}

// Launches of up to kMaxRowBlocks blocks over n rows: f(blocks, first row).
template <class F>
void row_launches(int64_t n, int rows, F&& f) {
    for (int64_t first = 0; first < n; first += kMaxRowBlocks * rows)
        f(dim3(uint32_t((std::min(n - first, kMaxRowBlocks * rows) + rows - 1) / rows)), first);
}

template <typename T, typename TOut, bool kAdd>
void gradient(hipStream_t stream, const EmbeddingCall& e) {
    const int lanes = lanes_of(e.d, kPer<T>, kThreads), columns = kThreads * kPer<T>, slices = lanes == kThreads ? (e.d + columns - 1) / columns : 1;
    row_launches((e.T + kWindow - 1) / kWindow, kThreads / lanes, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL((window_kernel<T, TOut, kAdd>), dim3(grid.x, slices), dim3(kThreads), 0, stream, e, lanes, first);
    });
    if (e.T > kWindow)
        row_launches((e.T - 1) / kWindow, 1, [&](dim3 grid, int64_t first) {
            hipLaunchKernelGGL((join_kernel<TOut, kAdd>), dim3(grid.x, (e.d + 511) / 512), dim3(kJoinThreads), 0, stream, e, first);
        });
}

}  // namespace

hipError_t launch_embedding_forward(hipStream_t stream, const EmbeddingCall& e, Dtype dtype) {
    const int lanes = lanes_of(e.d, dtype == Dtype::BF16 ? kPer<uint16_t> : kPer<float>, kThreads);
    row_launches(e.T, kThreads / lanes, [&](dim3 grid, int64_t first) {
        if (dtype == Dtype::BF16) hipLaunchKernelGGL((lookup_kernel<uint16_t>), grid, dim3(kThreads), 0, stream, e, lanes, first);
        else hipLaunchKernelGGL((lookup_kernel<float>), grid, dim3(kThreads), 0, stream, e, lanes, first);
    });
    return hipGetLastError();
}

hipError_t launch_embedding_backward(hipStream_t stream, const EmbeddingCall& e, Dtype dtype, Dtype dw_dtype, bool accumulate) {
    constexpr int kFillBlocks = 2048;                  // us, 537 MB and the gradient of 4096 tokens: 512 131, 1024 136, 2048 122, 8192 127
    const int64_t bytes = accumulate ? 0 : int64_t(e.rows) * e.d * (dw_dtype == Dtype::BF16 ? 2 : 4);
    const int64_t fill = std::min<int64_t>(kFillBlocks, (bytes + 16 * kSortThreads - 1) / (16 * kSortThreads));
    int bits = 1;
    while (bits < 31 && e.rows >> bits) ++bits;        // of the ids and of one past them
    hipLaunchKernelGGL(sort_kernel, dim3(uint32_t(e.chunks + fill)), dim3(kSortThreads), 0, stream, e, bits, bytes / 16, int(bytes % 16));
    if (e.chunks > 1)
        row_launches(int64_t(e.chunks) * kChunk, kThreads, [&](dim3 grid, int64_t first) {
            hipLaunchKernelGGL(merge_kernel, grid, dim3(kThreads), 0, stream, e, first);
        });
    if (dtype == Dtype::F32) accumulate ? gradient<float, float, true>(stream, e) : gradient<float, float, false>(stream, e);
    else if (dw_dtype == Dtype::BF16) gradient<uint16_t, uint16_t, false>(stream, e);
    else accumulate ? gradient<uint16_t, float, true>(stream, e) : gradient<uint16_t, float, false>(stream, e);
    return hipGetLastError();
}

}  // namespace tf
