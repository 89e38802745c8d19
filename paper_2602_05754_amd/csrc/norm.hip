// Layer norm and root-mean-square norm over the rows of [T x d], forward and backward.
//
//   forward   mean = sum x / d (0 without centring), rstd = 1 / sqrt(sum (x - mean)^2 / d + eps),
//             y = (x - mean) rstd w + b
//   backward  xh = (x - mean) rstd, g = dy w,
//             dx = rstd (g - [sum g / d] - xh sum (g xh) / d),  dw = sum_t dy xh,  db = sum_t dy
//
// Bound by memory: x is read once and y written once, backward x and dy read and dx written.  A row is
// held in the registers of kWaves waves (up to 32 elements a lane), so that the variance is taken of the
// centred values and nothing is read twice.  Sums are 32-bit, over at most 32 elements in a lane and
// then a tree.  The weight gradients sum over rows: a block of the backward walks every gridDim.x-th
// group of rows, a lane keeps the sums of its columns, and the blocks' partial sums are added by a second
// kernel in the order of the blocks, so that the same call gives the same bits.
//
// us and GB/s of what has to move (copies run at 5000), forward | backward with the sums: bf16, 4096 columns, 4096 rows 13.5, 4970 |
// 25.6, 3930 (of which the sums 4), 8192 rows 26.6, 5050 | 43.7, 4600; fp32, 2048 columns, 16384 rows 51.5, 5210 | 79.3, 5080.
// Rows of an odd number of bf16 start at odd addresses, where a wide load takes longer: 2731 columns, 8192 rows 25.4, 3530 | 66.2, 2030.
#include "row_device.h"

#include <algorithm>

namespace tf {
namespace {

constexpr int kMaxElems = 32;                          // of a row in one lane

// Waves of a row, rows of a block, pieces of a lane.
template <typename T, int kElems, int kWaves_, int kThreads_>
struct RowShape {
    static constexpr int kWaves = kWaves_, kThreads = kThreads_, kRows = kThreads_ / 64 / kWaves_;
    static constexpr int kPieces = kElems / kPer<T>;
    static constexpr int kSpan = 64 * kWaves;          // pieces apart are a lane's
};

// Sums of two values over the waves of each row; every thread of the block takes part.
template <class S>
__device__ __forceinline__ void row_sums(float& a, float& b, float (&lds)[2][S::kThreads / 64]) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (S::kWaves > 1) {
        const int wave = threadIdx.x >> 6, first = wave / S::kWaves * S::kWaves;
        __syncthreads();                               // the sums before these have been read
        if ((threadIdx.x & 63) == 0) { lds[0][wave] = a; lds[1][wave] = b; }
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int i = 0; i < S::kWaves; ++i) { a += lds[0][first + i]; b += lds[1][first + i]; }
    }
}

template <typename T, class S>
__global__ __launch_bounds__(S::kThreads) void norm_forward_kernel(NormRows r) {
    __shared__ float lds[2][S::kThreads / 64];
    const int in_row = threadIdx.x % S::kSpan;
    const int64_t row = int64_t(blockIdx.x) * S::kRows + threadIdx.x / S::kSpan;
    const bool live = row < r.T;
    const T* x = static_cast<const T*>(r.x) + row * r.d;
    float v[S::kPieces][kPer<T>];
    float sum = 0.f, none = 0.f;
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i) {
        const int c = (i * S::kSpan + in_row) * kPer<T>;
        unpack<T>(live && c < r.d ? load_piece(x + c, r.d - c) : U4{0, 0, 0, 0}, v[i]);
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j) sum += v[i][j];
    }
    float mean = 0.f;
    if (r.center) {
        row_sums<S>(sum, none, lds);
        mean = sum / float(r.d);
    }
    float square = 0.f;
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i) {
        const int c = (i * S::kSpan + in_row) * kPer<T>;
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j) {
            v[i][j] -= mean;
            if (c + j < r.d) square += v[i][j] * v[i][j];
        }
    }
    row_sums<S>(square, none, lds);
    if (!live) return;
    const float rstd = 1.f / sqrtf(square / float(r.d) + r.eps);
    T* y = static_cast<T*>(r.y) + row * r.d;
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i) {
        const int c = (i * S::kSpan + in_row) * kPer<T>;
        if (c >= r.d) continue;
        float w[kPer<T>], b[kPer<T>];
        unpack<T>(load_piece(static_cast<const T*>(r.w) + c, r.d - c), w);
        if (r.b) unpack<T>(load_piece(static_cast<const T*>(r.b) + c, r.d - c), b);
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j) v[i][j] = r.b ? v[i][j] * rstd * w[j] + b[j] : v[i][j] * rstd * w[j];
        store_piece(y + c, r.d - c, v[i]);
    }
    if (in_row == 0) {
        r.rstd[row] = rstd;
        if (r.center) r.mean[row] = mean;
    }
}

template <typename T, class S>
__global__ __launch_bounds__(S::kThreads) void norm_backward_kernel(NormRows r) {
    constexpr int kElems = S::kPieces * kPer<T>;
    constexpr bool kAhead = kElems < kMaxElems;
    __shared__ float lds[2][S::kThreads / 64];
    __shared__ float add[S::kRows > 1 ? S::kThreads * kElems : 1];
    const int in_row = threadIdx.x % S::kSpan, slot = threadIdx.x / S::kSpan;
    float w[S::kPieces][kPer<T>], dw[S::kPieces][kPer<T>], db[S::kPieces][kPer<T>];
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i) {
        const int c = (i * S::kSpan + in_row) * kPer<T>;
        unpack<T>(c < r.d ? load_piece(static_cast<const T*>(r.w) + c, r.d - c) : U4{0, 0, 0, 0}, w[i]);
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j) dw[i][j] = db[i][j] = 0.f;
    }
    U4 xn[S::kPieces], dyn[S::kPieces];                // the next row, on its way while this one is worked on
    float mean_n = 0.f, rstd_n = 0.f;
    auto fetch = [&](int64_t row) __attribute__((always_inline)) {
        const bool live = row < r.T;
        const T* x = static_cast<const T*>(r.x) + row * r.d;
        const T* dy = static_cast<const T*>(r.dy) + row * r.d;
#pragma unroll
        for (int i = 0; i < S::kPieces; ++i) {
            const int c = (i * S::kSpan + in_row) * kPer<T>;
            const bool there = live && c < r.d;
            xn[i] = there ? load_piece(x + c, r.d - c) : U4{0, 0, 0, 0};
            dyn[i] = there ? load_piece(dy + c, r.d - c) : U4{0, 0, 0, 0};
        }
        mean_n = live && r.center ? r.mean[row] : 0.f;
        rstd_n = live ? r.rstd[row] : 0.f;
    };
    const int64_t groups = (r.T + S::kRows - 1) / S::kRows;
    if constexpr (kAhead) fetch(int64_t(blockIdx.x) * S::kRows + slot);
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t row = g * S::kRows + slot;
        if constexpr (!kAhead) fetch(row);
        float xh[S::kPieces][kPer<T>], dy[S::kPieces][kPer<T>];
        const float mean = mean_n, rstd = rstd_n;
#pragma unroll
        for (int i = 0; i < S::kPieces; ++i) {
            unpack<T>(xn[i], xh[i]);
            unpack<T>(dyn[i], dy[i]);
        }
        if constexpr (kAhead) fetch(row + int64_t(gridDim.x) * S::kRows);
        float sg = 0.f, sgx = 0.f;
#pragma unroll
        for (int i = 0; i < S::kPieces; ++i)
#pragma unroll
            for (int j = 0; j < kPer<T>; ++j) {
                // (past the row's end dy is 0: nothing is added there)
                xh[i][j] = (xh[i][j] - mean) * rstd;
                dw[i][j] += dy[i][j] * xh[i][j];
                db[i][j] += dy[i][j];
                dy[i][j] *= w[i][j];
                sg += dy[i][j];
                sgx += dy[i][j] * xh[i][j];
            }
        row_sums<S>(sg, sgx, lds);
        const float a = r.center ? sg / float(r.d) : 0.f, b = sgx / float(r.d);
        if (row < r.T) {
            T* dx = static_cast<T*>(r.dx) + row * r.d;
#pragma unroll
            for (int i = 0; i < S::kPieces; ++i) {
                const int c = (i * S::kSpan + in_row) * kPer<T>;
                if (c >= r.d) continue;
#pragma unroll
                for (int j = 0; j < kPer<T>; ++j) xh[i][j] = rstd * (dy[i][j] - a - xh[i][j] * b);
                store_piece(dx + c, r.d - c, xh[i]);
            }
        }
    }
    // the block's sums, row slot by row slot, into its row of the workspace
    auto put = [&](float (&v)[S::kPieces][kPer<T>], float* out) __attribute__((always_inline)) {
        if constexpr (S::kRows > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kElems; ++i) add[(slot * kElems + i) * S::kSpan + in_row] = v[i / kPer<T>][i % kPer<T>];
            __syncthreads();
            if (slot != 0) return;
#pragma unroll
            for (int i = 0; i < kElems; ++i)
                for (int s = 1; s < S::kRows; ++s) v[i / kPer<T>][i % kPer<T>] += add[(s * kElems + i) * S::kSpan + in_row];
        }
#pragma unroll
        for (int i = 0; i < S::kPieces; ++i) {
            const int c = (i * S::kSpan + in_row) * kPer<T>;
#pragma unroll
            for (int j = 0; j < kPer<T>; ++j)
                if (c + j < r.d) out[c + j] = v[i][j];
        }
    };
    if (r.dw) put(dw, r.partials + int64_t(blockIdx.x) * r.d);
    if (r.db) put(db, r.partials + (int64_t(gridDim.x) + blockIdx.x) * r.d);
}

constexpr int kSumWaves = 16;

// Block (columns of 64, 0: dw / 1: db): the sum of `n` partial rows.
__global__ __launch_bounds__(64 * kSumWaves) void norm_sum_kernel(NormRows r, int n, int dw_bf16, int accumulate) {
    __shared__ float lds[kSumWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    void* out = blockIdx.y == 0 ? r.dw : r.db;
    if (!out) return;
    const float* p = r.partials + int64_t(blockIdx.y) * n * r.d;
    const int per = (n + kSumWaves - 1) / kSumWaves;
    float s = 0.f;
    if (c < r.d)
#pragma unroll 8
        for (int i = wave * per; i < min(n, (wave + 1) * per); ++i) s += p[int64_t(i) * r.d + c];
    lds[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= r.d) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < kSumWaves; ++i) s += lds[i][lane];
    if (dw_bf16) static_cast<uint16_t*>(out)[c] = from_f32<uint16_t>(s);
    else static_cast<float*>(out)[c] = accumulate ? static_cast<float*>(out)[c] + s : s;
}

// Calls f(RowShape) with the shape for rows of d elements: 16 elements a lane but for the widest rows, whose
// backward then has too few registers to fetch a row ahead.
template <typename T, int kThreads, class F>
void with_shape(int d, F&& f) {
    if (d <= 64 * 8) f(RowShape<T, 8, 1, kThreads>{});
    else if (d <= 64 * 16) f(RowShape<T, 16, 1, kThreads>{});
    else if (d <= 64 * 16 * 2) f(RowShape<T, 16, 2, kThreads>{});
    else if (d <= 64 * 16 * 4) f(RowShape<T, 16, 4, kThreads>{});
    else if (d <= 64 * 16 * 8) f(RowShape<T, 16, 8, 512>{});
    else f(RowShape<T, 32, 8, 512>{});
}
constexpr int kForwardThreads = 256, kBackwardThreads = 512;
static_assert(kNormMaxWidth == 64 * kMaxElems * 8, "the widest row: 32 elements in the lanes of eight waves");

template <typename T>
void forward(hipStream_t stream, const NormRows& r) {
    with_shape<T, kForwardThreads>(r.d, [&](auto shape) {
        typedef decltype(shape) S;
        for (int64_t done = 0; done < r.T; done += kMaxRowBlocks * S::kRows) {
            NormRows part = r;
            part.T = std::min(r.T - done, kMaxRowBlocks * S::kRows);
            part.x = static_cast<const T*>(r.x) + done * r.d;
            part.y = static_cast<T*>(r.y) + done * r.d;
            if (r.mean) part.mean = r.mean + done;
            part.rstd = r.rstd + done;
            hipLaunchKernelGGL((norm_forward_kernel<T, S>), dim3(uint32_t((part.T + S::kRows - 1) / S::kRows)), dim3(S::kThreads), 0, stream, part);
        }
    });
}
template <typename T>
void backward(hipStream_t stream, const NormRows& r, int blocks) {
    with_shape<T, kBackwardThreads>(r.d, [&](auto shape) {
        typedef decltype(shape) S;
        hipLaunchKernelGGL((norm_backward_kernel<T, S>), dim3(blocks), dim3(S::kThreads), 0, stream, r);
    });
}

}  // namespace

// Groups of rows that the blocks of a backward take one after the other.
static int64_t backward_groups(int64_t T, int d) {
    int rows = 1;
    with_shape<float, kBackwardThreads>(d, [&](auto shape) { rows = decltype(shape)::kRows; });
    return (T + rows - 1) / rows;
}

// As few blocks as take the same number of rounds: each leaves two rows of sums.
static int backward_blocks(int64_t T, int d) {
    const int64_t groups = backward_groups(T, d), rounds = (groups + kNormBlocks - 1) / kNormBlocks;
    return int((groups + rounds - 1) / rounds);
}

// The most blocks of any call with up to T rows: 300 rows take fewer than 256 do, and a workspace for the one has to do for the other.
int norm_backward_most_blocks(int64_t T, int d) { return int(std::min<int64_t>(backward_groups(T, d), kNormBlocks)); }

hipError_t launch_norm_forward(hipStream_t stream, const NormRows& r, Dtype dtype) {
    dtype == Dtype::BF16 ? forward<uint16_t>(stream, r) : forward<float>(stream, r);
    return hipGetLastError();
}

hipError_t launch_norm_backward(hipStream_t stream, const NormRows& r, Dtype dtype, Dtype dw_dtype, bool accumulate) {
    const int blocks = backward_blocks(r.T, r.d);
    dtype == Dtype::BF16 ? backward<uint16_t>(stream, r, blocks) : backward<float>(stream, r, blocks);
    if (r.dw || r.db)
        hipLaunchKernelGGL(norm_sum_kernel, dim3((r.d + 63) / 64, 2), dim3(64 * kSumWaves), 0, stream, r, blocks, dw_dtype == Dtype::BF16, accumulate);
    return hipGetLastError();
}

}  // namespace tf
