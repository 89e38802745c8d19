// C ABI of the operators around a stage's linear layers: argument checks and launches.
// Declarations and contracts: include/tf.h.
#include "tf_context.h"

#include <cfloat>
#include <cmath>
#include <new>

namespace {

using namespace tf;

inline uintptr_t address(const void* p) { return reinterpret_cast<uintptr_t>(p); }
constexpr int64_t kMaxTokens = (int64_t(1) << 31) - 4096;

// The tensors of a call: each required or not, its bytes, read or written.  Takes no memory: nothing here can throw.
struct Tensors {
    ByteRange ranges[10];
    int n = 0, status = TF_OK;
    void add(const void* p, int64_t bytes, bool output, bool required = true) {
        if (status != TF_OK) return;
        if (!p) { if (required) status = TF_ERR_INVALID_ARG; return; }
        if (!aligned16(p)) { status = TF_ERR_ALIGN; return; }
        ranges[n++] = {address(p), address(p) + uintptr_t(bytes), output};
    }
    void in(const void* p, int64_t bytes, bool required = true) { add(p, bytes, false, required); }
    void out(const void* p, int64_t bytes, bool required = true) { add(p, bytes, true, required); }
    int check() {
        for (int i = 0; i < n; ++i)
            for (int j = 0; j < i; ++j)
                if (status == TF_OK && (ranges[i].output || ranges[j].output) && ranges[i].lo < ranges[j].hi && ranges[j].lo < ranges[i].hi)
                    status = TF_ERR_ALIAS;
        return status;
    }
};

inline int64_t size_of(tf_dtype d) { return d == TF_BF16 ? 2 : 4; }

int finish(tf_ctx* ctx, hipError_t e) { return e == hipSuccess ? TF_OK : hip_fail(ctx, e); }

// Types of the gradient of a parameter of a call in io_dtype.
int check_gradient_type(tf_dtype io_dtype, tf_dtype dw_dtype, int accumulate) {
    if (accumulate != 0 && accumulate != 1) return TF_ERR_INVALID_ARG;
    if (!valid_dtype(io_dtype) || !valid_dtype(dw_dtype)) return TF_ERR_DTYPE;
    if ((io_dtype == TF_F32 || accumulate) && dw_dtype != TF_F32) return TF_ERR_DTYPE;
    return TF_OK;
}

int check_norm(int64_t T, int64_t d, int center) {
    if (center != 0 && center != 1) return TF_ERR_INVALID_ARG;
    if (T <= 0 || T > kMaxTokens || d <= 0 || d > kNormMaxWidth) return TF_ERR_SHAPE;
    return TF_OK;
}

struct EmbeddingPlan {
    int64_t chunks, tokens, pitch, merged, windows, bytes;      // byte offsets of the parts of the workspace; the ids are the first
};
EmbeddingPlan embedding_plan(int64_t T, int64_t d) {
    EmbeddingPlan p;
    p.chunks = (T + kEmbeddingChunk - 1) / kEmbeddingChunk;
    p.tokens = p.chunks * kEmbeddingChunk * 4;
    p.pitch = (d + 7) / 8 * 8;
    p.merged = p.chunks > 1 ? 2 * p.tokens : 0;
    p.windows = p.merged + 2 * p.tokens;
    p.bytes = p.windows + (T + kEmbeddingWindow - 1) / kEmbeddingWindow * 2 * p.pitch * 4;
    return p;
}
int check_embedding(int64_t T, int64_t rows, int64_t d, float scale) {
    if (T <= 0 || T > kMaxTokens || rows <= 0 || rows > kMaxTokens || d <= 0 || d > (1 << 20)) return TF_ERR_SHAPE;
    return std::isfinite(scale) ? TF_OK : TF_ERR_INVALID_ARG;
}

// What an attention call names: rows of a matrix, `stride` elements apart.
struct Rows {
    const void* p;
    int64_t stride, width;
    bool output;
};
// Two tensors of T rows share memory; views of one buffer beside each other do not.
bool rows_overlap(const Rows& x, const Rows& y, int64_t T, int64_t e) {
    const Rows &a = address(x.p) <= address(y.p) ? x : y, &b = address(x.p) <= address(y.p) ? y : x;
    const uintptr_t apart = address(b.p) - address(a.p);
    if (apart >= uintptr_t(((T - 1) * a.stride + a.width) * e)) return false;
    if (a.stride != b.stride) return true;
    const int64_t column = int64_t(apart % uintptr_t(a.stride * e));
    return column < a.width * e || column + b.width * e > a.stride * e;
}

constexpr int64_t kMaxStride = int64_t(1) << 24;
// Blocks of 128 rows and a head in a sequence, and in a launch: four times as many of 32 rows, twice for a backward pass, stay a grid.
constexpr int64_t kMaxAttentionBlocks = int64_t(1) << 20;

int check_attention_sizes(int64_t T, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim, tf_dtype io_dtype) {
    if (!valid_dtype(io_dtype)) return TF_ERR_DTYPE;
    if (T <= 0 || T > kMaxTokens || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads != 0) return TF_ERR_SHAPE;
    if (head_dim <= 0 || head_dim > 128 || head_dim % 16 != 0 || n_heads * head_dim > kMaxStride) return TF_ERR_SHAPE;
    return TF_OK;
}

int64_t attention_tiles(int64_t rows, bool narrow = false) { return (rows + attention_tile_rows(narrow) - 1) / attention_tile_rows(narrow); }
int64_t attention_tiles(int32_t n_seqs, const int64_t* starts, bool narrow) {
    int64_t tiles = 0;
    for (int32_t s = 0; s < n_seqs; ++s) tiles += attention_tiles(starts[s + 1] - starts[s], narrow);
    return tiles;
}

// tf_internal_attention_route: by the rule, the kernels of 128 rows, those of 32.
enum { kAttentionByRule = 0, kAttentionWide = 1, kAttentionNarrow = 2 };
// Whether the kernels of 32 rows take a call: where blocks of 128 rows and a head are few.  Their blocks cost the more to start
// and to join the less there is to do in one, and with wide heads only one fits a compute unit.  us, kernels of 128 rows and of 32,
// forward | backward; tokens in equal sequences, blocks of 128 rows with 32 query heads:
//   bf16, heads of 64    2 x 128 tokens,  64 blocks  5.9 5.1 | 19.9 14.7    1 x 1000, 256  18.7 16.6 | 58.0 48.1    3 x 334, 288  9.6 12.6 | 36.7 37.1
//                        1 x 2048, 512  34.5 37.7 | 104 104    1 x 4096, 1024  88 124 | 274 331
//   bf16, heads of 128   2 x 128,  64  7.6 6.9 | 30 24    1 x 512, 128  14.4 14.3 | 51 49    1 x 1000, 256  24 34 | 76 98    3 x 334, 288  14 27 | 54 66
//   fp32, heads of 64    1 x 512, 128  43 26 | 169 81    1 x 1000, 256  78 73 | 318 225    3 x 334, 288  36 44 | 138 122    1 x 2048, 512  200 248 | 727 784
// Of sequences up to 64 tokens there is nothing to share out in a forward pass (bf16, heads of 64 and 128, 64 tokens: 4.6 4.7, 5.4 6.1).
// The blocks of all sequences are counted, and 256 is where equal ones part on the whole, not everywhere (fp32 backward, 3 x 334).  Nor does it
// see uneven ones: of 934, 54 and 13 tokens (320 blocks, bf16, heads of 64) the kernels of 128 rows take 18.2 | 55.8, those of 32 16.2 | 47.6.
bool attention_narrow(const tf_ctx* ctx, Dtype dtype, int d, bool backward, int32_t n_seqs, const int64_t* starts, int64_t heads) {
    if (!attention_has_wide(d, dtype)) return true;
    if (ctx->attention_route != kAttentionByRule) return ctx->attention_route == kAttentionNarrow;
    int64_t longest = 0;
    for (int32_t s = 0; s < n_seqs; ++s) longest = std::max(longest, starts[s + 1] - starts[s]);
    if (dtype == Dtype::BF16 && !backward && longest <= 64) return false;
    return attention_tiles(n_seqs, starts, false) * heads <= (dtype == Dtype::BF16 && d > 64 ? 128 : 256);
}

// Everything about a call but its other tensors (`more`), the workspace among them.
int check_attention(int32_t n_seqs, const int64_t* starts, int64_t T, int64_t hq, int64_t hkv, int64_t d, tf_dtype io_dtype, float scale,
                    const std::vector<Rows>& tensors, std::vector<ByteRange>& dense) {
    if (const int bad = check_attention_sizes(T, hq, hkv, d, io_dtype)) return bad;
    if (n_seqs < 0 || !starts || !(scale > 0.f) || !std::isfinite(scale)) return TF_ERR_INVALID_ARG;
    if (starts[0] != 0) return TF_ERR_INVALID_ARG;
    for (int32_t s = 0; s < n_seqs; ++s) {
        if (starts[s + 1] < starts[s] || starts[s + 1] > T) return TF_ERR_INVALID_ARG;
        if (attention_tiles(starts[s + 1] - starts[s]) * hq > kMaxAttentionBlocks) return TF_ERR_SHAPE;
    }
    const int64_t e = size_of(io_dtype), per = 16 / e;
    for (const Rows& r : tensors) {
        if (!r.p) return TF_ERR_INVALID_ARG;
        if (r.stride < r.width || r.stride > kMaxStride) return TF_ERR_SHAPE;
        if (!aligned16(r.p) || r.stride % per != 0) return TF_ERR_ALIGN;
    }
    for (const ByteRange& r : dense) {
        if (!r.lo) return TF_ERR_INVALID_ARG;
        if (r.lo % 16 != 0) return TF_ERR_ALIGN;
    }
    for (size_t i = 0; i < tensors.size(); ++i) {
        const Rows& a = tensors[i];
        for (size_t j = 0; j < i; ++j)
            if ((a.output || tensors[j].output) && rows_overlap(a, tensors[j], T, e)) return TF_ERR_ALIAS;
        const uintptr_t end = address(a.p) + uintptr_t(((T - 1) * a.stride + a.width) * e);
        for (const ByteRange& r : dense)
            if ((a.output || r.output) && r.lo < end && address(a.p) < r.hi) return TF_ERR_ALIAS;
    }
    return outputs_overlap_something(dense) ? TF_ERR_ALIAS : TF_OK;
}

// Calls launch(call) with the sequences of the call, longest first, as many at a time as a launch takes; the first one has the padding.
template <class F>
hipError_t attention_launches(AttentionCall& a, int32_t n_seqs, const int64_t* starts, bool narrow, F&& launch) {
    std::vector<AttentionSequence> seqs;
    for (int32_t s = 0; s < n_seqs; ++s)
        if (starts[s + 1] > starts[s]) seqs.push_back({int32_t(starts[s]), int32_t(starts[s + 1] - starts[s]), 0});
    std::stable_sort(seqs.begin(), seqs.end(), [](const AttentionSequence& x, const AttentionSequence& y) { return x.rows > y.rows; });
    for (size_t i = 0; i < seqs.size() || a.pad_blocks > 0;) {
        a.n_seqs = a.tiles = 0;
        for (; i < seqs.size() && a.n_seqs < kMaxSequences; ++i) {
            const int64_t tiles = attention_tiles(seqs[i].rows, narrow);
            if (a.n_seqs > 0 && (a.tiles + tiles) * a.hq > kMaxAttentionBlocks) break;
            a.seq[a.n_seqs] = seqs[i];
            a.seq[a.n_seqs++].tile_start = a.tiles;
            a.tiles += int32_t(tiles);
        }
        const hipError_t e = launch(a);
        if (e != hipSuccess) return e;
        a.pad_blocks = 0;
    }
    return hipSuccess;
}

void set_padding(AttentionCall& a, int64_t used) {
    constexpr int64_t kBlocks = 1024;
    a.pad_first = used;
    a.pad_blocks = int32_t(std::min(a.T - used, kBlocks));
}

// Of the workspace of a backward pass: D, then the heads' parts of dk and dv.
int64_t attention_parts_at(int64_t T, int64_t hq) { return (T * hq * 4 + 15) / 16 * 16; }

}  // namespace

extern "C" {

int tf_attention_forward(tf_ctx* ctx, void* hip_stream, int32_t n_seqs, const int64_t* seq_starts, int64_t T,
                         int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, tf_dtype io_dtype,
                         const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, float scale,
                         void* o, int64_t o_stride, float* lse) {
    const int64_t wide = int64_t(n_heads) * head_dim, narrow = int64_t(n_kv_heads) * head_dim;
    try {
        std::vector<ByteRange> dense{{address(lse), address(lse) + uintptr_t(T) * uintptr_t(n_heads) * 4, true}};
        if (const int bad = check_attention(n_seqs, seq_starts, T, n_heads, n_kv_heads, head_dim, io_dtype, scale,
                                            {{q, q_stride, wide, false}, {k, k_stride, narrow, false}, {v, v_stride, narrow, false}, {o, o_stride, wide, true}}, dense))
            return bad;
        if (!ctx) return TF_ERR_INVALID_ARG;
        if (!use_device(ctx)) return TF_ERR_HIP;
        AttentionCall a{};
        a.q = q; a.k = k; a.v = v; a.o = o; a.lse = lse;
        a.T = T; a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.o_stride = o_stride;
        a.scale = scale; a.hq = n_heads; a.group = n_heads / n_kv_heads; a.d = head_dim;
        hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        const Dtype dtype = to_dtype(io_dtype);
        ProfScope prof(ctx, stream, TF_KERNEL_ATTENTION_FORWARD);
        const bool narrow = attention_narrow(ctx, dtype, head_dim, false, n_seqs, seq_starts, n_heads);
        set_padding(a, seq_starts[n_seqs]);
        const hipError_t e = attention_launches(a, n_seqs, seq_starts, narrow, [&](const AttentionCall& c) {
            return narrow ? launch_attention_forward_narrow(stream, c, dtype) : launch_attention_forward(stream, c, dtype);
        });
        return finish(ctx, e);
    } catch (const std::bad_alloc&) {
        return TF_ERR_WORKSPACE;
    }
}

int64_t tf_attention_workspace(int64_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, tf_dtype io_dtype) {
    if (const int bad = check_attention_sizes(T, n_heads, n_kv_heads, head_dim, io_dtype)) return bad;
    return attention_parts_at(T, n_heads) + (n_heads > n_kv_heads ? 2 * T * n_heads * head_dim * 4 : 0);
}

int tf_attention_backward(tf_ctx* ctx, void* hip_stream, int32_t n_seqs, const int64_t* seq_starts, int64_t T,
                          int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, tf_dtype io_dtype,
                          const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                          const void* o, int64_t o_stride, const float* lse, const void* d_o, float scale,
                          void* dq, void* dk, void* dv, void* workspace, int64_t workspace_bytes) {
    const int64_t wide = int64_t(n_heads) * head_dim, narrow = int64_t(n_kv_heads) * head_dim;
    try {
        if (const int bad = check_attention_sizes(T, n_heads, n_kv_heads, head_dim, io_dtype)) return bad;
        const int64_t need = tf_attention_workspace(T, n_heads, n_kv_heads, head_dim, io_dtype);
        std::vector<ByteRange> dense{{address(lse), address(lse) + uintptr_t(T * n_heads * 4), false},
                                     {address(workspace), address(workspace) + uintptr_t(need), true}};
        if (const int bad = check_attention(n_seqs, seq_starts, T, n_heads, n_kv_heads, head_dim, io_dtype, scale,
                                            {{q, q_stride, wide, false}, {k, k_stride, narrow, false}, {v, v_stride, narrow, false},
                                             {o, o_stride, wide, false}, {d_o, o_stride, wide, false},
                                             {dq, q_stride, wide, true}, {dk, k_stride, narrow, true}, {dv, v_stride, narrow, true}}, dense))
            return bad;
        if (workspace_bytes < need) return TF_ERR_WORKSPACE;
        if (!ctx) return TF_ERR_INVALID_ARG;
        if (!use_device(ctx)) return TF_ERR_HIP;
        AttentionCall a{};
        a.q = q; a.k = k; a.v = v; a.o = const_cast<void*>(o); a.lse = const_cast<float*>(lse); a.go = d_o;
        a.dq = dq; a.dk = dk; a.dv = dv;
        a.minus_d = static_cast<float*>(workspace);
        a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + attention_parts_at(T, n_heads));
        a.T = T; a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.o_stride = o_stride;
        a.scale = scale; a.hq = n_heads; a.group = n_heads / n_kv_heads; a.d = head_dim;
        hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        const Dtype dtype = to_dtype(io_dtype);
        const int64_t used = seq_starts[n_seqs];
        const bool narrow = attention_narrow(ctx, dtype, a.d, true, n_seqs, seq_starts, n_heads);
        a.per = attention_heads_per_block(attention_tiles(n_seqs, seq_starts, narrow), a.hq, a.group, a.d, dtype);
        ProfScope prof(ctx, stream, TF_KERNEL_ATTENTION_BACKWARD);
        set_padding(a, used);
        hipError_t e = hipSuccess;
        if (narrow) {
            e = launch_attention_delta(stream, a, used, dtype);
            a.pad_blocks = 0;
        }
        if (e == hipSuccess)
            e = attention_launches(a, n_seqs, seq_starts, narrow, [&](const AttentionCall& c) {
                return narrow ? launch_attention_backward_narrow(stream, c, dtype) : launch_attention_backward(stream, c, dtype);
            });
        if (e == hipSuccess && a.group > a.per && used > 0) e = launch_attention_group(stream, a, used, dtype);
        return finish(ctx, e);
    } catch (const std::bad_alloc&) {
        return TF_ERR_WORKSPACE;
    }
}

int64_t tf_norm_workspace(int64_t T, int64_t d) {
    if (check_norm(T, d, 0) != TF_OK) return check_norm(T, d, 0);
    return 2 * int64_t(norm_backward_most_blocks(T, int(d))) * d * 4;
}

int tf_norm_forward(tf_ctx* ctx, void* hip_stream, int64_t T, int64_t d, tf_dtype io_dtype,
                    const void* x, const void* weight, const void* bias, float eps, int center,
                    void* y, float* mean, float* rstd) {
    if (!valid_dtype(io_dtype)) return TF_ERR_DTYPE;
    if (const int bad = check_norm(T, d, center)) return bad;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return TF_ERR_INVALID_ARG;
    const int64_t e = size_of(io_dtype);
    Tensors t;
    t.in(x, T * d * e);
    t.in(weight, d * e);
    t.in(bias, d * e, false);
    t.out(y, T * d * e);
    if (center) t.out(mean, T * 4);
    t.out(rstd, T * 4);
    if (const int bad = t.check()) return bad;
    if (!ctx) return TF_ERR_INVALID_ARG;
    if (!use_device(ctx)) return TF_ERR_HIP;
    NormRows r{};
    r.x = x; r.w = weight; r.b = bias; r.y = y;
    r.mean = center ? mean : nullptr;
    r.rstd = rstd;
    r.T = T; r.d = int32_t(d); r.center = center; r.eps = eps;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    ProfScope prof(ctx, stream, TF_KERNEL_NORM);
    return finish(ctx, launch_norm_forward(stream, r, to_dtype(io_dtype)));
}

int tf_norm_backward(tf_ctx* ctx, void* hip_stream, int64_t T, int64_t d, tf_dtype io_dtype,
                     const void* x, const void* weight, const void* dy, const float* mean, const float* rstd, int center,
                     void* dx, void* dweight, void* dbias, tf_dtype dw_dtype, int accumulate,
                     void* workspace, int64_t workspace_bytes) {
    if (const int bad = check_gradient_type(io_dtype, dw_dtype, accumulate)) return bad;
    if (const int bad = check_norm(T, d, center)) return bad;
    const int64_t e = size_of(io_dtype), w = size_of(dw_dtype);
    Tensors t;
    t.in(x, T * d * e);
    t.in(weight, d * e);
    t.in(dy, T * d * e);
    if (center) t.in(mean, T * 4);
    t.in(rstd, T * 4);
    t.out(dx, T * d * e);
    t.out(dweight, d * w, false);
    t.out(dbias, d * w, false);
    const bool sums = dweight || dbias;
    if (sums) t.out(workspace, tf_norm_workspace(T, d));
    if (const int bad = t.check()) return bad;
    if (sums && workspace_bytes < tf_norm_workspace(T, d)) return TF_ERR_WORKSPACE;
    if (!ctx) return TF_ERR_INVALID_ARG;
    if (!use_device(ctx)) return TF_ERR_HIP;
    NormRows r{};
    r.x = x; r.w = weight; r.dy = dy; r.dx = dx; r.dw = dweight; r.db = dbias;
    r.mean = const_cast<float*>(center ? mean : nullptr);
    r.rstd = const_cast<float*>(rstd);
    r.partials = static_cast<float*>(workspace);
    r.T = T; r.d = int32_t(d); r.center = center;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    ProfScope prof(ctx, stream, TF_KERNEL_NORM);
    return finish(ctx, launch_norm_backward(stream, r, to_dtype(io_dtype), to_dtype(dw_dtype), accumulate != 0));
}

int64_t tf_embedding_workspace(int64_t T, int64_t n_rows, int64_t d) {
    if (const int bad = check_embedding(T, n_rows, d, 1.f)) return bad;
    return embedding_plan(T, d).bytes;
}

int tf_embedding_forward(tf_ctx* ctx, void* hip_stream, int64_t T, int64_t n_rows, int64_t d, tf_dtype io_dtype,
                         const int32_t* ids, const void* table, float scale, void* out) {
    if (!valid_dtype(io_dtype)) return TF_ERR_DTYPE;
    if (const int bad = check_embedding(T, n_rows, d, scale)) return bad;
    const int64_t e = size_of(io_dtype);
    Tensors t;
    t.in(ids, T * 4);
    t.in(table, n_rows * d * e);
    t.out(out, T * d * e);
    if (const int bad = t.check()) return bad;
    if (!ctx) return TF_ERR_INVALID_ARG;
    if (!use_device(ctx)) return TF_ERR_HIP;
    EmbeddingCall c{};
    c.ids = ids; c.table = table; c.out = out;
    c.T = T; c.rows = int32_t(n_rows); c.d = int32_t(d); c.scale = scale;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    ProfScope prof(ctx, stream, TF_KERNEL_EMBEDDING);
    return finish(ctx, launch_embedding_forward(stream, c, to_dtype(io_dtype)));
}

int tf_embedding_backward(tf_ctx* ctx, void* hip_stream, int64_t T, int64_t n_rows, int64_t d, tf_dtype io_dtype,
                          const int32_t* ids, const void* dout, float scale, void* dtable, tf_dtype dw_dtype, int accumulate,
                          void* workspace, int64_t workspace_bytes) {
    if (const int bad = check_gradient_type(io_dtype, dw_dtype, accumulate)) return bad;
    if (const int bad = check_embedding(T, n_rows, d, scale)) return bad;
    const EmbeddingPlan plan = embedding_plan(T, d);
    Tensors t;
    t.in(ids, T * 4);
    t.in(dout, T * d * size_of(io_dtype));
    t.out(dtable, n_rows * d * size_of(dw_dtype));
    t.out(workspace, plan.bytes);
    if (const int bad = t.check()) return bad;
    if (workspace_bytes < plan.bytes) return TF_ERR_WORKSPACE;
    if (!ctx) return TF_ERR_INVALID_ARG;
    if (!use_device(ctx)) return TF_ERR_HIP;
    char* at = static_cast<char*>(workspace);
    EmbeddingCall c{};
    c.ids = ids; c.dout = dout; c.dtable = dtable;
    c.sorted_id = reinterpret_cast<int32_t*>(at);
    c.sorted_token = reinterpret_cast<int32_t*>(at + plan.tokens);
    c.merged_id = reinterpret_cast<int32_t*>(at + plan.merged);
    c.merged_token = reinterpret_cast<int32_t*>(at + plan.merged + plan.tokens);
    c.windows = reinterpret_cast<float*>(at + plan.windows);
    c.T = T;
    c.rows = int32_t(n_rows); c.d = int32_t(d); c.pitch = int32_t(plan.pitch); c.chunks = int32_t(plan.chunks); c.scale = scale;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    ProfScope prof(ctx, stream, TF_KERNEL_EMBEDDING);
    return finish(ctx, launch_embedding_backward(stream, c, to_dtype(io_dtype), to_dtype(dw_dtype), accumulate != 0));
}

int tf_distill_loss(tf_ctx* ctx, void* hip_stream, int64_t T, int64_t V, int64_t K, tf_dtype io_dtype,
                    const void* logits, const int32_t* teacher_ids, const float* teacher_logits, const float* token_weight,
                    float temperature, float grad_scale, float* loss, void* dlogits) {
    if (!valid_dtype(io_dtype)) return TF_ERR_DTYPE;
    if (T <= 0 || T > kMaxTokens || V <= 0 || V > kMaxTokens || K <= 0 || K > kDistillMaxK) return TF_ERR_SHAPE;
    if (!(temperature >= FLT_MIN) || !std::isfinite(temperature) || !std::isfinite(grad_scale)) return TF_ERR_INVALID_ARG;
    const int64_t e = size_of(io_dtype);
    Tensors t;
    t.in(logits, T * V * e);
    t.in(teacher_ids, T * K * 4);
    t.in(teacher_logits, T * K * 4);
    t.in(token_weight, T * 4, false);
    t.out(loss, T * 4);
    t.out(dlogits, T * V * e, false);
    if (const int bad = t.check()) return bad;
    if (!ctx) return TF_ERR_INVALID_ARG;
    if (!use_device(ctx)) return TF_ERR_HIP;
    DistillCall c{};
    c.logits = logits; c.ids = teacher_ids; c.teacher = teacher_logits; c.weight = token_weight;
    c.loss = loss; c.dlogits = dlogits;
    c.T = T; c.V = int32_t(V); c.K = int32_t(K);
    c.temperature = temperature; c.grad_scale = grad_scale;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    ProfScope prof(ctx, stream, TF_KERNEL_DISTILL);
    return finish(ctx, launch_distill(stream, c, to_dtype(io_dtype)));
}

}  // extern "C"

// Tests: the kernels that attention calls of this context take (0 by the rule, 1 those of 128 rows, 2 those of 32 where they exist).
extern "C" int tf_internal_attention_route(tf_ctx* ctx, int route) {
    if (!ctx || route < kAttentionByRule || route > kAttentionNarrow) return TF_ERR_INVALID_ARG;
    ctx->attention_route = route;
    return TF_OK;
}
