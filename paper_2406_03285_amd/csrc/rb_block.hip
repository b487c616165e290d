// What a block of a model computes between its matrix products, for gfx950 (MI355X): the C ABI of include/rb_block.h (host side); the kernels are
// in rb_kernels_norm.h (dropout, layer norm) and rb_kernels_attention.h (attention of packed documents).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>

#include "rb_host.h"
#include "rb_kernels_norm.h"
#include "rb_kernels_attention.h"
#include "rb_block.h"

namespace {

constexpr int64_t MAX_STRIDE = int64_t(1) << 36;       // of rows and positions, in elements: no offset passes 64 bits
inline bool known(int32_t dtype) { return dtype == RB_F32 || dtype == RB_BF16; }
inline int64_t elem_bytes(int32_t dtype) { return dtype == RB_F32 ? 4 : 2; }

bool drop_of(const rb_drop* d, Drop& to)
{
    to = Drop{};
    if (!d) return true;
    if (!(d->p >= 0.0 && d->p <= 1.0)) return false;
    to.seed_lo = (uint32_t)d->seed;
    to.seed_hi = (uint32_t)(d->seed >> 32);
    to.step_lo = (uint32_t)d->step;
    to.step_hi = (uint32_t)(d->step >> 32);
    to.least = (uint32_t)std::nearbyint(d->p * 65536.0);
    to.scale = to.least == 65536 ? 0.0f : (float)(65536.0 / (65536.0 - to.least));
    return true;
}

}  // namespace

// ---- dropout ---------------------------------------------------------------------
extern "C" int rb_dropout(const void* x, int64_t x_stride, int64_t rows, int64_t width, int32_t dtype, const rb_drop* drop, void* out, int64_t out_stride,
                          void* hip_stream)
{
    DropoutArgs a{};
    if (!x || !out || !drop || !known(dtype) || rows < 0 || rows > RB_MAX_NORM_ROWS || width < 1 || width > RB_MAX_DROP_WIDTH) return RB_EINVAL;
    if (!aligned(x, (size_t)elem_bytes(dtype)) || !aligned(out, (size_t)elem_bytes(dtype))) return RB_EINVAL;
    if (x_stride < width || out_stride < width || x_stride > MAX_STRIDE || out_stride > MAX_STRIDE || !drop_of(drop, a.drop)) return RB_EINVAL;
    if (x == out && x_stride != out_stride && rows > 1) return RB_EINVAL;
    if (rows == 0) return RB_OK;
    a.x = x;
    a.out = out;
    a.x_stride = x_stride;
    a.out_stride = out_stride;
    a.rows = (int32_t)rows;
    a.width = (int32_t)width;
    a.pieces = (int32_t)((width + NM_PIECE - 1) / NM_PIECE);
    a.at_once = std::max(1, NM_TPB / a.pieces);
    a.blocks = (a.pieces + NM_TPB - 1) / NM_TPB;
    a.items = (rows + a.at_once - 1) / a.at_once * a.blocks;
    const dim3 grid((unsigned)std::min<int64_t>(a.items, 1 << 20));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = dtype == RB_F32 ? launch(rb_dropout_kernel<float>, grid, NM_TPB, 0, st, a) : launch(rb_dropout_kernel<Bf16>, grid, NM_TPB, 0, st, a);
    return e == hipSuccess ? RB_OK : RB_EHIP;
}

// ---- layer norm ------------------------------------------------------------------
struct rb_norm {
    int32_t width, dtype, weight_dtype;
    float eps;
    float* sums;       // workspace
};

namespace {

constexpr int64_t NM_FUSED_WIDTH = 16384;      // longest rows whose sums over rows stay in registers beside them

inline bool rows_fit(const rb_norm* n, const rb_rows* r)
{
    return r && r->data && aligned(r->data, (size_t)elem_bytes(n->dtype)) && r->stride >= n->width && r->stride <= MAX_STRIDE;
}
// what is written in place has to lie as what is read
inline bool apart_or_alike(const rb_rows* a, const rb_rows* b, int64_t rows) { return !a || !b || !a->data || a->data != b->data || a->stride == b->stride || rows <= 1; }

// Workgroups of a grid that goes through `rows` rows: as many as the chip holds at once.
inline unsigned norm_groups(int64_t rows, int lanes, int waves_per_simd)
{
    const int threads = nm_threads(lanes), at_once = threads / lanes;
    return (unsigned)std::min<int64_t>((rows + at_once - 1) / at_once, 256 * std::max(1, waves_per_simd * 4 * 64 / threads));
}

template <typename T, int LANES, int PARTS>
hipError_t norm_forward(const NormArgs& a, hipStream_t st)
{
    const dim3 grid(norm_groups(a.rows, LANES, nm_waves<T>(LANES, PARTS)));
    return launch(a.total ? rb_norm_kernel<T, LANES, PARTS, true> : rb_norm_kernel<T, LANES, PARTS, false>, grid, nm_threads(LANES), 0, st, a);
}

template <int N> using Int = std::integral_constant<int, N>;

// Lanes of a row and pieces of a lane, by the row's length, which ends in the last part: `of` is called with both.  Few lanes have few exchanges to a sum (2^25
// numbers of bfloat16 with residual and dropout: rows of 256 51 us with 16 lanes and 96 with 64, of 512 50 with 32 and 54 with 64), many have few
// registers to a lane (2048: 56 with 128, 62 with 64; 8192: 54 with 512 and 66 with 256).
template <typename Of>
auto forward_by_width(int32_t width, const Of& of)
{
    if (width <= 128) return of(Int<16>(), Int<1>());
    if (width <= 256) return of(Int<16>(), Int<2>());
    if (width <= 512) return of(Int<32>(), Int<2>());
    if (width <= 1024) return of(Int<64>(), Int<2>());
    if (width <= 1536) return of(Int<64>(), Int<3>());
    if (width <= 2048) return of(Int<128>(), Int<2>());
    if (width <= 4096) return of(Int<256>(), Int<2>());
    if (width <= 6144) return of(Int<256>(), Int<3>());
    if (width <= 8192) return of(Int<512>(), Int<2>());
    if (width <= 16384) return of(Int<1024>(), Int<2>());
    if (width <= 24576) return of(Int<1024>(), Int<3>());
    return of(Int<1024>(), Int<4>());
}
// The gradients' sums and rows ahead take more registers: fewer pieces of a lane, of binary32 all the more.  (The same 2^25 numbers: rows of 384 70 us with 16
// lanes and 149 with 64; 512 72 with 32 and 121 with 64; 1536 71 with 64 and 161 with 256; 2048 76 with 128, 130 with 256 and 78 with 64; 8192 82 with 512
// and 110 with 256.)
template <typename Of>
auto grad_by_width(int32_t width, const Of& of)
{
    if (width <= 128) return of(Bf16(), Int<16>(), Int<1>());
    if (width <= 256) return of(Bf16(), Int<16>(), Int<2>());
    if (width <= 384) return of(Bf16(), Int<16>(), Int<3>());
    if (width <= 512) return of(Bf16(), Int<32>(), Int<2>());
    if (width <= 768) return of(Bf16(), Int<32>(), Int<3>());
    if (width <= 1024) return of(Bf16(), Int<64>(), Int<2>());
    if (width <= 1536) return of(Bf16(), Int<64>(), Int<3>());
    if (width <= 2048) return of(Bf16(), Int<128>(), Int<2>());
    if (width <= 4096) return of(Bf16(), Int<256>(), Int<2>());
    if (width <= 6144) return of(Bf16(), Int<256>(), Int<3>());
    if (width <= 8192) return of(Bf16(), Int<512>(), Int<2>());
    if (width <= 12288) return of(Bf16(), Int<512>(), Int<3>());
    if (width <= 16384) return of(Bf16(), Int<512>(), Int<4>());
    if (width <= 24576) return of(Bf16(), Int<1024>(), Int<3>());
    return of(Bf16(), Int<1024>(), Int<4>());
}
template <typename Of>
auto grad_by_width_wide(int32_t width, const Of& of)
{
    if (width <= 128) return of(float(), Int<16>(), Int<1>());
    if (width <= 256) return of(float(), Int<16>(), Int<2>());
    if (width <= 512) return of(float(), Int<32>(), Int<2>());
    if (width <= 1024) return of(float(), Int<64>(), Int<2>());
    if (width <= 2048) return of(float(), Int<128>(), Int<2>());
    if (width <= 4096) return of(float(), Int<256>(), Int<2>());
    if (width <= 8192) return of(float(), Int<512>(), Int<2>());
    if (width <= 12288) return of(float(), Int<512>(), Int<3>());
    if (width <= 16384) return of(float(), Int<512>(), Int<4>());
    if (width <= 24576) return of(float(), Int<1024>(), Int<3>());
    return of(float(), Int<1024>(), Int<4>());
}
template <typename Of>
auto grad_form(const rb_norm* n, const Of& of) { return n->dtype == RB_F32 ? grad_by_width_wide(n->width, of) : grad_by_width(n->width, of); }

}  // namespace

extern "C" {

int rb_norm_create(rb_norm** out, int64_t width, int32_t dtype, int32_t weight_dtype, float eps)
{
    if (!out) return RB_EINVAL;
    *out = nullptr;
    if (width < 1 || width > RB_MAX_NORM_WIDTH || !known(dtype) || !known(weight_dtype) || !std::isfinite(eps) || !(eps > 0.0f)) return RB_EINVAL;
    rb_norm* n = new (std::nothrow) rb_norm();
    if (!n) return RB_ENOMEM;
    n->width = (int32_t)width;
    n->dtype = dtype;
    n->weight_dtype = weight_dtype;
    n->eps = eps;
    *out = n;
    return RB_OK;
}

int rb_norm_query(const rb_norm* n, size_t* workspace_bytes)
{
    if (!n || !workspace_bytes) return RB_EINVAL;
    *workspace_bytes = (size_t)2 * NM_MAX_GROUPS * n->width * sizeof(float);
    return RB_OK;
}

int rb_norm_bind(rb_norm* n, void* workspace)
{
    if (!n || !workspace || !aligned(workspace, 256)) return RB_EINVAL;
    n->sums = static_cast<float*>(workspace);
    return RB_OK;
}

int rb_norm_forward(rb_norm* n, const rb_rows* x, const rb_rows* residual, const rb_drop* drop, int64_t rows, const void* weight, const void* bias,
                    const rb_rows* total, const rb_rows* y, float* mean, float* rstd, void* hip_stream)
{
    if (!n || rows < 0 || rows > RB_MAX_NORM_ROWS || !rows_fit(n, x) || !rows_fit(n, y) || (residual && !rows_fit(n, residual))) return RB_EINVAL;
    const bool sum = residual || drop;
    if (sum != (total && total->data) || (sum && !rows_fit(n, total))) return RB_EINVAL;
    const size_t size = (size_t)elem_bytes(n->weight_dtype);
    if (!weight || !aligned(weight, size) || !aligned(bias, size) || !aligned(mean, 4) || !aligned(rstd, 4)) return RB_EINVAL;
    if (!apart_or_alike(y, x, rows) || (sum && (total->data == y->data || !apart_or_alike(total, x, rows) || !apart_or_alike(total, residual, rows)))) return RB_EINVAL;
    if (residual && y->data == residual->data && rows > 0) return RB_EINVAL;
    NormArgs a{};
    if (!drop_of(drop, a.drop)) return RB_EINVAL;
    if (rows == 0) return RB_OK;
    a.x = x->data;
    a.x_stride = x->stride;
    if (residual) {
        a.residual = residual->data;
        a.residual_stride = residual->stride;
    }
    if (sum) {
        a.total = total->data;
        a.total_stride = total->stride;
    }
    a.y = y->data;
    a.y_stride = y->stride;
    a.weight = weight;
    a.bias = bias;
    a.mean = mean;
    a.rstd = rstd;
    a.rows = (int32_t)rows;
    a.width = n->width;
    a.eps = n->eps;
    a.wide_weights = n->weight_dtype == RB_F32;
    a.drops = drop != nullptr;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = forward_by_width(n->width, [&](auto lanes, auto parts) {
        return n->dtype == RB_F32 ? norm_forward<float, lanes(), parts()>(a, st) : norm_forward<Bf16, lanes(), parts()>(a, st);
    });
    return e == hipSuccess ? RB_OK : RB_EHIP;
}

int rb_norm_grad(rb_norm* n, const rb_rows* grad_y, const rb_rows* total, const rb_rows* grad_total, const float* mean, const float* rstd, const rb_drop* drop,
                 int64_t rows, const void* weight, const rb_rows* grad_sum, const rb_rows* grad_x, void* grad_weight, void* grad_bias, void* hip_stream)
{
    if (!n || rows < 0 || rows > RB_MAX_NORM_ROWS || !rows_fit(n, grad_y) || !rows_fit(n, total) || !rows_fit(n, grad_sum)) return RB_EINVAL;
    if ((grad_total && !rows_fit(n, grad_total)) || (drop != nullptr) != (grad_x && grad_x->data) || (drop && !rows_fit(n, grad_x))) return RB_EINVAL;
    const size_t size = (size_t)elem_bytes(n->weight_dtype);
    if (!mean || !rstd || !weight || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(weight, size) || !aligned(grad_weight, size) || !aligned(grad_bias, size))
        return RB_EINVAL;
    if (!apart_or_alike(grad_sum, grad_y, rows) || !apart_or_alike(grad_sum, grad_total, rows) || grad_sum->data == total->data) return RB_EINVAL;
    if (drop && (grad_x->data == grad_sum->data || grad_x->data == total->data || !apart_or_alike(grad_x, grad_y, rows) || !apart_or_alike(grad_x, grad_total, rows)))
        return RB_EINVAL;
    NormGradArgs a{};
    if (!drop_of(drop, a.drop)) return RB_EINVAL;
    const bool wanted = grad_weight || grad_bias;
    if (!n->sums) return RB_ESTATE;
    if (rows == 0 && !wanted) return RB_OK;
    a.grad_y = grad_y->data;
    a.grad_y_stride = grad_y->stride;
    a.total = total->data;
    a.total_stride = total->stride;
    if (grad_total) {
        a.grad_total = grad_total->data;
        a.grad_total_stride = grad_total->stride;
    }
    a.grad_sum = grad_sum->data;
    a.grad_sum_stride = grad_sum->stride;
    if (drop) {
        a.grad_x = grad_x->data;
        a.grad_x_stride = grad_x->stride;
    }
    a.weight = weight;
    a.mean = mean;
    a.rstd = rstd;
    a.sums = n->sums;
    a.rows = (int32_t)rows;
    a.width = n->width;
    a.wide_weights = n->weight_dtype == RB_F32;
    a.drops = drop != nullptr;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipError_t e = hipSuccess;
    const unsigned groups = grad_form(n, [&](auto, auto lanes, auto) { return norm_groups(rows, std::min(lanes(), 512), NM_SUM_WAVES); });
    const dim3 columns_grid(groups, (unsigned)(n->width + NM_TPB * NM_PIECE - 1) / (NM_TPB * NM_PIECE));
    auto columns = [&] { return n->dtype == RB_F32 ? launch(rb_norm_columns_kernel<float>, columns_grid, NM_TPB, 0, st, a) : launch(rb_norm_columns_kernel<Bf16>, columns_grid, NM_TPB, 0, st, a); };
    // long rows: their weights' gradients come from another kernel, which needs grad_y and what the rows have beside their means: behind the first kernel, that makes
    // the latter on its way, or before it where it overwrites grad_y
    const bool apart = wanted && rows > 0 && n->width > NM_FUSED_WIDTH, before = apart && (grad_sum->data == grad_y->data || (drop && grad_x->data == grad_y->data));
    if (apart) {
        constexpr int64_t GROUPS = NM_MAX_GROUPS / 2;       // (of workgroups of 512 threads; the workspace's second half is free)
        static_assert(2 * GROUPS * (NM_FUSED_WIDTH + 1) >= RB_MAX_NORM_ROWS, "a number a row");
        a.rests = n->sums + 2 * GROUPS * n->width;
    }
    if (before) {
        e = grad_form(n, [&](auto type, auto lanes, auto parts) {
            if constexpr (lanes() > 512) return launch(rb_norm_rests_kernel<decltype(type), lanes(), parts()>, dim3(norm_groups(rows, lanes(), 8)), nm_threads(lanes()), 0, st, a);
            return hipSuccess;
        });
        if (e == hipSuccess) e = columns();
    }
    if (e == hipSuccess && rows > 0)
        e = grad_form(n, [&](auto type, auto lanes, auto parts) {
            const dim3 grid(lanes() <= 512 ? groups : norm_groups(rows, lanes(), 4));
            return launch(rb_norm_grad_kernel<decltype(type), lanes(), parts()>, grid, nm_threads(lanes()), 0, st, a);
        });
    if (apart && !before && e == hipSuccess) e = columns();
    if (e == hipSuccess && wanted) {
        const dim3 grid((unsigned)(n->width + 63) / 64, 2);
        e = n->weight_dtype == RB_F32
                ? launch(rb_norm_join_kernel<float>, grid, 1024, 0, st, n->sums, (int)groups, (int)n->width, static_cast<float*>(grad_weight), static_cast<float*>(grad_bias))
                : launch(rb_norm_join_kernel<Bf16>, grid, 1024, 0, st, n->sums, (int)groups, (int)n->width, static_cast<Bf16*>(grad_weight), static_cast<Bf16*>(grad_bias));
    }
    return e == hipSuccess ? RB_OK : RB_EHIP;
}

int rb_norm_destroy(rb_norm* n)
{
    delete n;
    return RB_OK;
}

}  // extern "C"

// ---- attention of packed documents -----------------------------------------------
struct rb_attention {
    int32_t heads, kv_heads, dim, max_tokens;
    bool causal;
    float scale, cap;
    size_t off_lse2, off_delta, off_sums, bytes;
    char* ws;
};

namespace {

// Workgroups that the gradients of keys and values are cut into at least.
constexpr int64_t AT_KEY_GROUPS = 512, AT_MAX_PARTS = 16;

// Into how many parts the queries of a head of keys are cut: until all units have two workgroups, and twice as many where some have much more to do than others.
// That is so for the first keys of what is causal, and in documents of several lengths.  (Gradients of 16 heads of 128 to 8, once and twice as many: one causal
// document of 8192 1347 and 1080 us, not causal 1985 and 2027; 24 documents of any lengths in 8192 306 and 241, 8 of them 468 and 352, not causal 690 and
// 563.  The price is paid by documents of the same length, 24 of 341: 156 and 182, and by short ones, which have no such differences.)
inline int key_parts(const rb_attention* a, int64_t tokens, int64_t documents)
{
    const int64_t groups = (tokens + AT_ROWS - 1) / AT_ROWS * a->kv_heads;
    const int64_t wanted = (a->causal || documents > 1) && tokens >= documents * 160 ? 2 * AT_KEY_GROUPS : AT_KEY_GROUPS;
    // (a part of less than 4 tiles of queries would not be worth its sums)
    const int64_t most = std::min<int64_t>(AT_MAX_PARTS, std::max<int64_t>(1, tokens / std::max<int64_t>(documents, 1) * (a->heads / a->kv_heads) / (4 * AT_BLOCK)));
    return (int)std::min<int64_t>(most, (wanted + groups - 1) / groups);
}

// Heads of one die that take turns (0: dies have no heads of their own): those that read the same keys.
inline int inner_heads(int64_t heads, int64_t group)
{
    if (heads % 8 != 0) return 0;
    const int64_t of_die = heads / 8;
    return (int)(of_die % group == 0 ? group : group % of_die == 0 ? of_die : 1);
}

bool heads_fit(const rb_heads* t)
{
    if (!t || !t->data || !aligned(t->data, 16) || t->token_stride % 8 != 0 || t->head_stride % 8 != 0) return false;
    return t->token_stride >= 0 && t->head_stride >= 0 && t->token_stride <= AT_MAX_STRIDE && t->head_stride <= (int64_t(1) << 48);
}
// What is written: no two of its rows may share a number.
bool heads_apart(const rb_attention* a, const rb_heads* t, int64_t tokens, int64_t heads)
{
    if (!heads_fit(t) || t->token_stride < a->dim || t->head_stride < a->dim) return false;
    return tokens <= 1 || heads <= 1 || t->token_stride >= (heads - 1) * t->head_stride + a->dim || t->head_stride >= (tokens - 1) * t->token_stride + a->dim;
}
HeadRows rows_of(const rb_heads* t) { return HeadRows{static_cast<Bf16*>(t->data), t->token_stride, t->head_stride}; }

bool documents_fit(const rb_documents* d)
{
    if (!d || !d->offsets || d->count < 0 || d->count > RB_MAX_DOCUMENTS) return false;
    return aligned(d->offsets, 8) && aligned(d->lengths, 8) && aligned(d->prefixes, 8);
}

// Documents of less than 128 positions in the mean have the forms for short documents (FINE), and their capped scores are exact near 0, too: AT_CAPPED's are off by up
// to cap * 2^-21, which is some parts in 10^6 of lse and less where it is of 128 positions.  (64 documents of 128, 16 heads of 128: forward 35 us by
// these forms and 33 by the others, gradients 122 and 104; with a cap of 30 forward 40 and 34, gradients 135 and 110.)
inline bool is_short(int64_t tokens, int64_t documents) { return tokens < 128 * documents; }
inline int form_of(const rb_attention* a, bool fine) { return a->cap == 0.0f ? AT_PLAIN : a->cap <= AT_LOW_CAP && !fine ? AT_CAPPED : AT_HIGH_CAP; }
ScoreOf score_of(const rb_attention* a, int form)
{
    if (form == AT_PLAIN) return ScoreOf{a->scale, a->scale * AT_LOG2E, 0.0f};
    return ScoreOf{a->scale, a->cap * AT_LOG2E, a->scale / a->cap * (form == AT_CAPPED ? 2 * AT_LOG2E : 1.0f)};
}

AttentionArgs attention_args(const rb_attention* a, int form, const rb_heads* q, const rb_heads* k, const rb_heads* v, int64_t tokens, const rb_documents* d, const float* slopes)
{
    AttentionArgs g{};
    g.q = rows_of(q);
    g.k = rows_of(k);
    g.v = rows_of(v);
    g.documents = SpanArgs{d->offsets, d->lengths, d->prefixes, d->count, reinterpret_cast<Spans*>(a->ws), (int32_t)tokens, a->causal};
    g.spans = g.documents.spans;
    g.slopes = slopes;
    g.score = score_of(a, form);
    g.tokens = (int32_t)tokens;
    g.dim = a->dim;
    g.heads = a->heads;
    g.group = a->heads / a->kv_heads;
    g.tiles = (int32_t)((tokens + AT_ROWS - 1) / AT_ROWS);
    g.inner = inner_heads(a->heads, g.group);
    // (documents of any lengths in 8192 positions, 16 heads of 128: 24 of them, forward 74 -> 60 us and gradients 313 -> 241, 42 of them 49 -> 46 and 198 -> 189; 64
    // of 128 each lose by it: 33 -> 39 and 104 -> 112)
    g.ranked = d->count > 1 && tokens >= 160 * d->count && g.tiles > 1 && g.tiles <= AT_RANKED;
    return g;
}

// The kernel of a head's size, the scores' form and slopes: and whether documents are short: `of` is called with these four.
template <typename Of>
hipError_t by_form(const rb_attention* a, int form, bool slopes, bool fine, const Of& of)
{
    auto with = [&](auto dim) {
        using Plain = std::integral_constant<int, AT_PLAIN>;
        using Capped = std::integral_constant<int, AT_CAPPED>;
        using HighCap = std::integral_constant<int, AT_HIGH_CAP>;
        using Yes = std::true_type;
        using No = std::false_type;
        if (fine) return form == AT_PLAIN ? of(dim, Plain(), Yes(), Yes()) : of(dim, HighCap(), Yes(), Yes());       // (slopes of 0, and below)
        if (form == AT_PLAIN) return slopes ? of(dim, Plain(), Yes(), No()) : of(dim, Plain(), No(), No());
        if (form == AT_CAPPED) return slopes ? of(dim, Capped(), Yes(), No()) : of(dim, Capped(), No(), No());
        return of(dim, HighCap(), Yes(), No());
    };
    return a->dim <= 64 ? with(std::integral_constant<int, 64>()) : with(std::integral_constant<int, 128>());
}

}  // namespace

extern "C" {

int rb_attention_create(rb_attention** out, int64_t heads, int64_t kv_heads, int64_t head_dim, int64_t max_tokens, int32_t causal, float scale, float cap)
{
    if (!out) return RB_EINVAL;
    *out = nullptr;
    if (heads < 1 || heads > RB_MAX_HEADS || kv_heads < 1 || heads % kv_heads != 0) return RB_EINVAL;
    if (head_dim < 8 || head_dim > RB_MAX_HEAD_DIM || head_dim % 8 != 0 || max_tokens < 1 || max_tokens > RB_MAX_TOKENS || heads * max_tokens > RB_MAX_HEAD_ROWS) return RB_EINVAL;
    if (!std::isfinite(scale) || !(scale > 0.0f) || !std::isfinite(cap) || cap < 0.0f) return RB_EINVAL;
    // (what the kernels multiply by; a quotient below binary32's normal numbers would have lost bits)
    if (!std::isfinite(scale * AT_LOG2E) || !std::isfinite(cap * AT_LOG2E) || (cap > 0.0f && (!std::isfinite(2 * AT_LOG2E * (scale / cap)) || !std::isnormal(scale / cap)))) return RB_EINVAL;
    rb_attention* a = new (std::nothrow) rb_attention();
    if (!a) return RB_ENOMEM;
    a->heads = (int32_t)heads;
    a->kv_heads = (int32_t)kv_heads;
    a->dim = (int32_t)head_dim;
    a->max_tokens = (int32_t)max_tokens;
    a->causal = causal != 0;
    a->scale = scale;
    a->cap = cap;
    size_t off = round_up((size_t)max_tokens * sizeof(Spans), 256);
    a->off_lse2 = off; off += round_up((size_t)heads * (size_t)max_tokens * sizeof(float), 256);
    a->off_delta = off; off += round_up((size_t)heads * (size_t)max_tokens * sizeof(float), 256);
    a->off_sums = off;
    // (parts > 1: workgroups are less than what is wanted and one more of each)
    const size_t tiles = ((size_t)max_tokens + AT_ROWS - 1) / AT_ROWS;
    off += std::min((size_t)AT_MAX_PARTS * kv_heads * tiles, (size_t)4 * AT_KEY_GROUPS) * AT_ROWS * 2 * (head_dim <= 64 ? 64 : 128) * sizeof(float);
    a->bytes = off;
    *out = a;
    return RB_OK;
}

int rb_attention_query(const rb_attention* a, size_t* workspace_bytes)
{
    if (!a || !workspace_bytes) return RB_EINVAL;
    *workspace_bytes = a->bytes;
    return RB_OK;
}

int rb_attention_bind(rb_attention* a, void* workspace)
{
    if (!a || !workspace || !aligned(workspace, 256)) return RB_EINVAL;
    a->ws = static_cast<char*>(workspace);
    return RB_OK;
}

int rb_attention_forward(rb_attention* a, const rb_heads* q, const rb_heads* k, const rb_heads* v, int64_t tokens, const rb_documents* documents,
                         const float* slopes, const rb_heads* out, float* lse, void* hip_stream)
{
    if (!a || tokens < 0 || tokens > a->max_tokens || !documents_fit(documents) || !aligned(slopes, 4) || !aligned(lse, 4)) return RB_EINVAL;
    if (!heads_fit(q) || !heads_fit(k) || !heads_fit(v) || !heads_apart(a, out, tokens, a->heads)) return RB_EINVAL;
    if (!a->ws) return RB_ESTATE;
    if (tokens == 0) return RB_OK;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool fine = is_short(tokens, documents->count);
    const int form = form_of(a, fine);
    AttentionArgs g = attention_args(a, form, q, k, v, tokens, documents, slopes);
    g.out = rows_of(out);
    g.lse = lse;
    // one launch where a workgroup can look through the documents itself (9 documents in 160 positions: 10.2 to 12.7 us in two, 8.4 in one)
    hipError_t e = hipSuccess;
    if (documents->count < AT_NEAR_OFFSETS) g.spans = nullptr;       // (with many documents tiles take turns as they lie)
    else e = launch(rb_spans_kernel, dim3((unsigned)(tokens + AT_TPB - 1) / AT_TPB), AT_TPB, 0, st, g.documents);
    if (e == hipSuccess)
        e = by_form(a, form, slopes != nullptr, fine, [&](auto dim, auto scores, auto lowered, auto rests) {
            return launch(rb_attend_kernel<dim(), scores(), lowered(), rests()>, dim3((unsigned)(g.tiles * g.heads)), AT_TPB, 0, st, g);
        });
    return e == hipSuccess ? RB_OK : RB_EHIP;
}

int rb_attention_grad(rb_attention* a, const rb_heads* q, const rb_heads* k, const rb_heads* v, int64_t tokens, const rb_documents* documents,
                      const float* slopes, const rb_heads* out, const float* lse, const rb_heads* grad_out, const rb_heads* grad_q, const rb_heads* grad_k,
                      const rb_heads* grad_v, void* hip_stream)
{
    if (!a || tokens < 0 || tokens > a->max_tokens || !documents_fit(documents) || !aligned(slopes, 4) || !lse || !aligned(lse, 4)) return RB_EINVAL;
    if (!heads_fit(q) || !heads_fit(k) || !heads_fit(v) || !heads_fit(out) || !heads_fit(grad_out)) return RB_EINVAL;
    if (!heads_apart(a, grad_q, tokens, a->heads) || !heads_apart(a, grad_k, tokens, a->kv_heads) || !heads_apart(a, grad_v, tokens, a->kv_heads)) return RB_EINVAL;
    if (!a->ws) return RB_ESTATE;
    if (tokens == 0) return RB_OK;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool fine = is_short(tokens, documents->count);
    const int form = form_of(a, fine);
    AttentionArgs g = attention_args(a, form, q, k, v, tokens, documents, slopes);
    float *const lse2 = reinterpret_cast<float*>(a->ws + a->off_lse2), *const delta = reinterpret_cast<float*>(a->ws + a->off_delta);
    g.out = rows_of(out);
    g.lse = const_cast<float*>(lse);
    g.grad_out = rows_of(grad_out);
    g.grad_q = rows_of(grad_q);
    g.grad_k = rows_of(grad_k);
    g.grad_v = rows_of(grad_v);
    g.lse2 = lse2;
    g.delta = delta;
    g.lse_less = form == AT_CAPPED ? g.score.to_log2 : 0.0f;
    const int parts = key_parts(a, tokens, documents->count);
    AttentionArgs of_keys = g;
    of_keys.shares = a->kv_heads * parts;
    of_keys.inner = inner_heads(of_keys.shares, parts);
    of_keys.sums = parts > 1 ? reinterpret_cast<float*>(a->ws + a->off_sums) : nullptr;
    const int64_t blocks = (tokens + AT_POSITIONS - 1) / AT_POSITIONS;
    const dim3 delta_grid((unsigned)blocks, (unsigned)std::min<int64_t>((a->heads + AT_ONCE - 1) / AT_ONCE, (1024 + blocks - 1) / blocks));
    hipError_t e = launch(rb_attend_delta_kernel, delta_grid, AT_TPB, 0, st, g, lse2);
    if (e == hipSuccess)
        e = by_form(a, form, slopes != nullptr, fine, [&](auto dim, auto scores, auto lowered, auto rests) {
            // (of queries first: it makes delta exact)
            hipError_t r = launch(rb_attend_grad_q_kernel<dim(), scores(), lowered(), rests()>, dim3((unsigned)(g.tiles * g.heads)), AT_TPB, 0, st, g);
            if (r == hipSuccess)
                r = launch(rb_attend_grad_kv_kernel<dim(), scores(), lowered(), rests()>, dim3((unsigned)(g.tiles * of_keys.shares)), AT_TPB, 0, st, of_keys);
            if (r == hipSuccess && parts > 1) {
                const int64_t threads = (int64_t)a->kv_heads * tokens * (2 * dim() / 4);
                r = launch(rb_attend_join_kernel<dim()>, dim3((unsigned)std::min<int64_t>((threads + AT_TPB - 1) / AT_TPB, 1 << 16)), AT_TPB, 0, st, of_keys);
            }
            return r;
        });
    return e == hipSuccess ? RB_OK : RB_EHIP;
}

int rb_attention_destroy(rb_attention* a)
{
    delete a;
    return RB_OK;
}

}  // extern "C"
