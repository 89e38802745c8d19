// Distillation loss from a teacher's top logits, with the gradient of the student's logits.
//
//   p = softmax(teacher / tau) over the row's K entries,  log q = z / tau - log sum exp (z / tau)
//   loss_t = w_t tau^2 sum_k p_k (log p_k - log q[id_k])
//   dz     = grad_scale w_t tau (q - p put at its ids)
//
// Bound by memory: z is read once and dz written once.  A block has one row, held in its
// registers as it came (up to 16 pieces of 16 bytes a thread) from the sum to the gradient; of longer rows
// the rest is read twice.  Each thread takes the running maximum and sum of its pieces as they arrive, so that the exponentials of
// the sum are done by the time the row is there, as those of the gradient are while it is written; what is to be done for
// the K entries is done while the row is on its way.  The K entries of p are put in by writing those elements again, behind a barrier.
// us and logical GB/s (copies run at 5000), bf16, K = 32: 4096 rows of 65536 207, 5180 (two blocks to a compute unit); 2048 of 131072 236,
// 4540 (one: a row fills the registers, and nothing is read while it is written); 2048 of 160000 289, 4530.  The loss alone: 92, 129 (4160: one
// block to a unit, as with the gradient).  fp32, 2048 rows of 32000: 106, alone 46.  Each entry is compared with all of its row, for words
// that are named twice: 2048 rows of 32000 with K = 32, 256 and 1024 take 62, 93 and 580.
// Exponentials are of (z - maximum) / tau, the difference first: z / tau of a word masked with the type's lowest value
// need not be finite, and where q is large the difference is exact.  The loss adds up tau log p and tau log q for the same reason: log q of such
// a word is not finite at a temperature below 1, tau^2 log q is.
#include "row_device.h"

#include <algorithm>

namespace tf {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

template <int kThreads>
__device__ __forceinline__ float block_max(float x, float* lds) {
    x = wave_max(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int i = 1; i < kThreads / 64; ++i) x = fmaxf(x, lds[i]);
    return x;
}
template <int kThreads>
__device__ __forceinline__ float block_sum(float x, float* lds) {
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) x += lds[i];
    return x;
}

// kPieces: of a thread, the whole row or (kMore) its beginning, the rest being read twice.
template <typename T, int kThreads, int kPieces, bool kMore>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillCall a) {
    __shared__ int ids[kDistillMaxK];
    __shared__ float p[kDistillMaxK];
    __shared__ float z_of[kDistillMaxK], at_id[kDistillMaxK];
    __shared__ float red[kThreads / 64];
    const int64_t t = blockIdx.x;
    const int V = a.V, K = a.K;
    const T* z = static_cast<const T*>(a.logits) + t * V;
    T* dz = a.dlogits ? static_cast<T*>(a.dlogits) + t * V : nullptr;
    const float weight = a.weight ? a.weight[t] : 1.f;
    const float inv_tau = 1.f / a.temperature, to2 = inv_tau * kLog2e;

    // the teacher's entry of each thread and then the row, all on their way before any is used
    int first_id = -1;
    float first_teacher = -INFINITY;
    if (int(threadIdx.x) < K) {
        first_id = a.ids[t * K + threadIdx.x];
        first_teacher = a.teacher[t * K + threadIdx.x];
    }
    auto clear = [&]() __attribute__((always_inline)) {                // nothing to learn here
        if (threadIdx.x == 0) a.loss[t] = 0.f;
        if (!dz) return;
        const float zero[kPer<T>] = {};
        for (int64_t c = threadIdx.x * kPer<T>; c < V; c += kThreads * kPer<T>) store_piece(dz + c, V - c, zero);
    };
    if (weight == 0.f) return clear();
    const T minus_infinity = from_f32<T>(-INFINITY);
    U4 row[kPieces];
    auto each = [&](auto&& f) __attribute__((always_inline)) {          // f(piece, column)
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int c = (i * kThreads + int(threadIdx.x)) * kPer<T>;
            if (c < V) f(row[i], c);
        }
        if constexpr (kMore)
            for (int64_t c = (kPieces * kThreads + int(threadIdx.x)) * kPer<T>; c < V; c += kThreads * kPer<T>) f(load_piece(z + c, V - c, minus_infinity), int(c));
    };
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int c = (i * kThreads + int(threadIdx.x)) * kPer<T>;
        if (c < V) row[i] = load_piece(z + c, V - c, minus_infinity);
    }
    for (int k = threadIdx.x; k < K; k += kThreads) {
        const bool first = k < kThreads;
        const int id = first ? first_id : a.ids[t * K + k];
        const bool there = id >= 0 && id < V;
        ids[k] = there ? id : -1;
        p[k] = !there ? -INFINITY : first ? first_teacher : a.teacher[t * K + k];
    }
    __syncthreads();
    const int first_there = int(threadIdx.x) < K ? max(ids[threadIdx.x], 0) : 0;
    const T first_z = z[first_there];                  // the student's logit of the thread's entry
    float tmax = -INFINITY;
    bool nan = false;                                  // a NaN among the teacher's logits is passed on
    for (int k = threadIdx.x & 63; k < K; k += 64) {
        tmax = fmaxf(tmax, p[k]);
        nan = nan || p[k] != p[k];
    }
    tmax = wave_max(tmax);
    if (__any(nan)) tmax = NAN;
    if (tmax == -INFINITY) return clear();
    float tsum = 0.f;
    for (int k = threadIdx.x & 63; k < K; k += 64) tsum += expf((p[k] - tmax) * inv_tau);
    tsum = wave_sum(tsum);
    const float log_tsum = logf(tsum), inv_tsum = 1.f / tsum;
    // what p puts at an id: all its entries', at the first of them; -1 at the others and where there is no word
    if (dz) {
        for (int k = threadIdx.x; k < K; k += kThreads) {
            const int id = ids[k];
            float sum_p = 0.f;
            bool first = id >= 0;
            for (int i = 0; i < K; ++i)
                if (ids[i] == id) {
                    first = first && i >= k;
                    sum_p += expf((p[i] - tmax) * inv_tau);
                }
            at_id[k] = first ? sum_p * inv_tsum : -1.f;
        }
    }

    float mine = -INFINITY, sum = 0.f;                 // of this thread: the maximum, and the sum of 2^((z - maximum) to2)
    each([&](const U4& x, int) __attribute__((always_inline)) {
        float v[kPer<T>];
        unpack<T>(x, v);
        float top = v[0];
#pragma unroll
        for (int j = 1; j < kPer<T>; ++j) top = fmaxf(top, v[j]);
        const float next = fmaxf(mine, top);
        const float base = next == -INFINITY ? 0.f : next;             // nothing but -infinity so far
        sum *= __builtin_amdgcn_exp2f((mine - base) * to2);
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j) sum += __builtin_amdgcn_exp2f((v[j] - base) * to2);
        mine = next;
    });
    for (int k = threadIdx.x; k < K; k += kThreads) z_of[k] = to_f32(k < kThreads ? first_z : z[max(ids[k], 0)]);
    const float top = block_max<kThreads>(mine, red);
    sum *= mine == -INFINITY ? (sum != sum ? NAN : 0.f) : __builtin_amdgcn_exp2f((mine - top) * to2);
    sum = block_sum<kThreads>(sum, red);
    const float log_sum = logf(sum), inv_sum = 1.f / sum;

    if (threadIdx.x < 64) {
        const float factor = weight * a.temperature;
        float l = 0.f;
        for (int k = threadIdx.x; k < K; k += 64) {
            const float pk = expf((p[k] - tmax) * inv_tau - log_tsum);
            if (pk == 0.f) continue;                   // nothing of an absent or hopeless entry, whatever log q is
            const float tau_logp = (p[k] - tmax) - a.temperature * log_tsum, tau_logq = (z_of[k] - top) - a.temperature * log_sum;
            l += pk * factor * (tau_logp - tau_logq);
        }
        l = wave_sum(l);
        if (threadIdx.x == 0) a.loss[t] = l;
    }
    if (!dz) return;
    const float scale = a.grad_scale * weight * a.temperature;
    const float cq = scale * inv_sum;
    each([&](const U4& x, int c) __attribute__((always_inline)) {
        float v[kPer<T>];
        unpack<T>(x, v);
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j) v[j] = __builtin_amdgcn_exp2f((v[j] - top) * to2) * cq;
        store_piece(dz + c, V - c, v);
    });
    __syncthreads();                                   // those elements' first values are written
    for (int k = threadIdx.x; k < K; k += kThreads) {
        if (at_id[k] < 0.f) continue;
        const float q = __builtin_amdgcn_exp2f((z_of[k] - top) * to2) * inv_sum;
        dz[ids[k]] = from_f32<T>(scale * (q - at_id[k]));
    }
}

template <typename T>
void launch(hipStream_t stream, const DistillCall& a) {
    auto go = [&](auto threads, auto pieces, auto more) {
        for (int64_t done = 0; done < a.T; done += kMaxRowBlocks) {
            DistillCall part = a;
            part.T = std::min(a.T - done, kMaxRowBlocks);
            part.logits = static_cast<const T*>(a.logits) + done * a.V;
            part.ids = a.ids + done * a.K;
            part.teacher = a.teacher + done * a.K;
            if (a.weight) part.weight = a.weight + done;
            part.loss = a.loss + done;
            if (a.dlogits) part.dlogits = static_cast<T*>(a.dlogits) + done * a.V;
            hipLaunchKernelGGL((distill_kernel<T, threads, pieces, more>), dim3(uint32_t(part.T)), dim3(threads), 0, stream, part);
        }
    };
    auto fits = [&](int threads, int pieces) { return a.V <= threads * pieces * kPer<T>; };
    using std::integral_constant;
    constexpr std::false_type whole;
    if (fits(256, 4)) go(integral_constant<int, 256>{}, integral_constant<int, 4>{}, whole);
    else if (fits(256, 8)) go(integral_constant<int, 256>{}, integral_constant<int, 8>{}, whole);
    else if (fits(256, 16)) go(integral_constant<int, 256>{}, integral_constant<int, 16>{}, whole);
    else if (fits(512, 16)) go(integral_constant<int, 512>{}, integral_constant<int, 16>{}, whole);
    else if (fits(1024, 16)) go(integral_constant<int, 1024>{}, integral_constant<int, 16>{}, whole);
    else go(integral_constant<int, 1024>{}, integral_constant<int, 16>{}, std::true_type{});
}

}  // namespace

hipError_t launch_distill(hipStream_t stream, const DistillCall& a, Dtype dtype) {
    dtype == Dtype::BF16 ? launch<uint16_t>(stream, a) : launch<float>(stream, a);
    return hipGetLastError();
}

}  // namespace tf
