// The training step that the rehearsal buffer feeds, for gfx950 (MI355X): the C ABI of include/rb_train.h (host side); the kernels are in
// rb_kernels_scorer.h (scores of tokens and their gradient) and rb_kernels_ortho.h (orthogonalised updates).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>

#include "rb_host.h"
#include "rb_kernels_scorer.h"
#include "rb_kernels_ortho.h"
#include "rb_train.h"

// ---- scores of tokens ----------------------------------------------------------
struct rb_scorer {
    int32_t vocab, dtype, given, top;
    uint32_t* counters;      // workspace: a counter per shared row, then the parts of the workgroups that share
    char* partials;
    bool bound;
};

namespace {

inline int64_t elem_bytes(int32_t dtype) { return dtype == RB_F32 ? 4 : 2; }
inline size_t scorer_bytes(int32_t top) { return SC_SPLIT_GROUPS * (sizeof(uint32_t) + sc_partial_bytes(top)); }

template <typename T, bool TOP>
hipError_t score(const ScoreArgs& a, bool wave_per_row, hipStream_t st)
{
    if (wave_per_row) return launch(rb_score_kernel<T, TOP, 1>, dim3((unsigned)((a.rows + SC_NWAVE - 1) / SC_NWAVE)), SC_TPB, 0, st, a);
    return launch(rb_score_kernel<T, TOP, SC_NWAVE>, dim3((unsigned)a.rows * (unsigned)a.splits), SC_TPB, 0, st, a);
}

template <typename T>
hipError_t score_grad(GradArgs& a, int64_t rows, bool vectors, hipStream_t st)
{
    const int64_t accesses = vectors ? (a.vocab + Logit<T>::N - 1) / Logit<T>::N : a.vocab;
    // a chunk: as many tiles as the bits that tell of given tokens, fewer where the rows alone are not enough workgroups
    const int64_t tiles = (accesses + SC_TPB - 1) / SC_TPB;
    const int64_t want = std::max<int64_t>(1, (2048 + rows - 1) / rows);
    const int64_t per = std::min<int64_t>(GR_MAX_TILES, std::max<int64_t>(4, (tiles + want - 1) / want));
    a.chunk = (int32_t)(per * SC_TPB);
    const dim3 grid((unsigned)rows, (unsigned)std::max<int64_t>(1, (tiles + per - 1) / per));
    if (vectors) return launch(rb_score_grad_kernel<T, Logit<T>::N>, grid, SC_TPB, 0, st, a);
    return launch(rb_score_grad_kernel<T, 1>, grid, SC_TPB, 0, st, a);
}

}  // namespace

extern "C" {

int rb_scorer_create(rb_scorer** out, int64_t vocab, int32_t dtype, int64_t given, int64_t top)
{
    if (!out) return RB_EINVAL;
    *out = nullptr;
    if (vocab < 1 || vocab > RB_MAX_VOCAB || (dtype != RB_F32 && dtype != RB_BF16)) return RB_EINVAL;
    if (given < 0 || given > RB_MAX_GIVEN || top < 0 || top > RB_MAX_TOP || top > vocab) return RB_EINVAL;
    rb_scorer* s = new (std::nothrow) rb_scorer();
    if (!s) return RB_ENOMEM;
    s->vocab = (int32_t)vocab;
    s->dtype = dtype;
    s->given = (int32_t)given;
    s->top = (int32_t)top;
    *out = s;
    return RB_OK;
}

int rb_scorer_query(const rb_scorer* s, size_t* workspace_bytes)
{
    if (!s || !workspace_bytes) return RB_EINVAL;
    *workspace_bytes = scorer_bytes(s->top);
    return RB_OK;
}

int rb_scorer_bind(rb_scorer* s, void* workspace, void* hip_stream)
{
    if (!s || !workspace || !aligned(workspace, 256)) return RB_EINVAL;
    if (launch(rb_train_clear_kernel, dim3(SC_SPLIT_GROUPS / SC_TPB), SC_TPB, 0, static_cast<hipStream_t>(hip_stream), static_cast<uint32_t*>(workspace),
               (int64_t)SC_SPLIT_GROUPS) != hipSuccess)
        return RB_EHIP;
    s->counters = static_cast<uint32_t*>(workspace);
    s->partials = static_cast<char*>(workspace) + SC_SPLIT_GROUPS * sizeof(uint32_t);
    s->bound = true;
    return RB_OK;
}

int rb_scorer_score(rb_scorer* s, const void* logits, int64_t rows, int64_t row_stride, const int64_t* tokens, float* logp, float* lse,
                    float* entropy, float* top_logp, int64_t* top_ids, void* hip_stream)
{
    if (!s || rows < 0 || rows > RB_MAX_ROWS || row_stride < s->vocab) return RB_EINVAL;
    if (!logits || !aligned(logits, (size_t)elem_bytes(s->dtype))) return RB_EINVAL;
    if (s->given > 0 && (!tokens || !logp)) return RB_EINVAL;
    if (s->top > 0 && (!top_logp || !top_ids)) return RB_EINVAL;
    if (!aligned(tokens, 8) || !aligned(logp, 4) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(top_logp, 4) || !aligned(top_ids, 8)) return RB_EINVAL;
    if (!s->bound) return RB_ESTATE;
    if (rows == 0) return RB_OK;
    const int64_t tiles = (s->vocab + SC_TILE - 1) / SC_TILE;
    ScoreArgs a{};
    a.logits = logits;
    a.stride = row_stride;
    a.tokens = tokens;
    a.logp = logp;
    a.lse = lse;
    a.entropy = entropy;
    a.top_logp = top_logp;
    a.top_ids = top_ids;
    a.counters = s->counters;
    a.partials = s->partials;
    a.rows = (int32_t)rows;
    a.vocab = s->vocab;
    a.given = s->given;
    a.top = s->top;
    a.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>({(tiles + SC_NWAVE - 1) / SC_NWAVE, (SC_SPLIT_GROUPS / 2 + rows - 1) / rows, SC_MAX_SPLITS}));
    const bool wave_per_row = tiles == 1;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipError_t e;
    if (s->dtype == RB_F32)
        e = s->top ? score<float, true>(a, wave_per_row, st) : score<float, false>(a, wave_per_row, st);
    else
        e = s->top ? score<Bf16, true>(a, wave_per_row, st) : score<Bf16, false>(a, wave_per_row, st);
    return e == hipSuccess ? RB_OK : RB_EHIP;
}

int rb_scorer_grad(rb_scorer* s, const void* logits, int64_t rows, int64_t row_stride, const int64_t* tokens, const float* lse,
                   const float* entropy, const float* grad_logp, const float* grad_entropy, void* grad_logits, int64_t grad_stride,
                   void* hip_stream)
{
    if (!s || rows < 0 || rows > RB_MAX_ROWS || row_stride < s->vocab || grad_stride < s->vocab) return RB_EINVAL;
    const int64_t size = elem_bytes(s->dtype);
    if (!logits || !grad_logits || !lse || !aligned(logits, (size_t)size) || !aligned(grad_logits, (size_t)size)) return RB_EINVAL;
    if (s->given > 0 && (!tokens || !grad_logp)) return RB_EINVAL;
    if (grad_entropy && !entropy) return RB_EINVAL;
    if (!aligned(tokens, 8) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(grad_logp, 4) || !aligned(grad_entropy, 4)) return RB_EINVAL;
    if (grad_logits == logits && grad_stride != row_stride && rows > 1) return RB_EINVAL;
    if (rows == 0) return RB_OK;
    GradArgs a{};
    a.logits = logits;
    a.grad = grad_logits;
    a.stride = row_stride;
    a.grad_stride = grad_stride;
    a.tokens = tokens;
    a.lse = lse;
    a.entropy = entropy;
    a.grad_logp = grad_logp;
    a.grad_entropy = grad_entropy;
    a.vocab = s->vocab;
    a.given = s->given;
    const uintptr_t apart = reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(grad_logits);
    const bool vectors = apart % 16 == 0 && (rows == 1 || (row_stride - grad_stride) * size % 16 == 0);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = s->dtype == RB_F32 ? score_grad<float>(a, rows, vectors, st) : score_grad<Bf16>(a, rows, vectors, st);
    return e == hipSuccess ? RB_OK : RB_EHIP;
}

int rb_scorer_destroy(rb_scorer* s)
{
    delete s;
    return RB_OK;
}

}  // extern "C"

// ---- orthogonalised updates ------------------------------------------------------
struct rb_ortho {
    int64_t matrices;
    int32_t m, n;                  // the caller's
    int32_t dtype, out_dtype;
    int32_t steps;
    float coefficients[RB_MAX_ORTHO_STEPS][3];
    float eps;
    bool tall;
    int32_t rows, cols;            // of the kept X: short and long side
    int32_t small;                 // a workgroup per matrix: its padded side (64, 128), or 0: tiled products
    int32_t prows, pcols;          // tiled: padded to whole tiles
    int32_t tile[3];               // of A, of B, of X
    size_t off_x, off_xt[2], off_a, off_b, bytes;
    char* ws;
};

namespace {

// Tiles of a product: 64 x 64 by 4 wavefronts, 128 x 128 by 8, 256 x 256 by 8.
template <int KIND, typename OUT, int BM, int WM, int WN, int STAGES, int WAVES_PER_SIMD>
hipError_t product_of(const ProductArgs& a, unsigned tiles, unsigned matrices, hipStream_t st)
{
    return launch(rb_ortho_product_kernel<KIND, OUT, BM, BM, WM, WN, STAGES, WAVES_PER_SIMD>, dim3(tiles, matrices), BM / WM * (BM / WN) * 64,
                  (size_t)STAGES * 2 * BM * 128, st, a);
}

template <int KIND, typename OUT>
hipError_t product(const rb_ortho* o, ProductArgs a, int tile, bool symmetric, hipStream_t st)
{
    a.tiles_i = o->prows / tile;
    a.tiles_j = (symmetric ? o->prows : o->pcols) / tile;
    const unsigned tiles = symmetric ? (unsigned)a.tiles_i * (a.tiles_i + 1) / 2 : (unsigned)a.tiles_i * a.tiles_j, n = (unsigned)o->matrices;
    switch (tile) {
    case 256: return product_of<KIND, OUT, 256, 128, 64, 2, 2>(a, tiles, n, st);
    case 128: return product_of<KIND, OUT, 128, 64, 32, 2, 4>(a, tiles, n, st);
    default: return product_of<KIND, OUT, 64, 32, 32, 3, 3>(a, tiles, n, st);
    }
}

// What a product takes, in us, by its tile, measured on 256 compute units: a launch with its epilogue, and a tile's block of 32 of the summed
// index on a compute unit that has one workgroup (64: 0.25, 128: 0.51, 256: 2.1) or is full (two of 128 together 1.58, 256: 2.65).
double product_us(int tile, double tiles, int kblocks)
{
    const double per = tiles / 256;
    if (tile == 64) return 5 + kblocks * 0.25 * std::max(1.0, per);
    if (tile == 128) {
        const double pairs = std::floor(per / 2), rest = per - 2 * pairs;
        return 8 + kblocks * (1.58 * pairs + (rest == 0 ? 0 : rest <= 1 ? 0.51 : 1.58));
    }
    return 15 + kblocks * (per <= 0.75 ? 2.1 : 2.65 * std::ceil(per));
}

// The padding and the three products' tiles that take least.
void choose_tiles(rb_ortho* o)
{
    double best = 1e300;
    for (int pad = 64; pad <= 256; pad *= 2) {
        const int64_t R = (int64_t)round_up((size_t)o->rows, (size_t)pad), C = (int64_t)round_up((size_t)o->cols, (size_t)pad);
        double total = 0;
        int chosen[3] = {};
        for (int kind = 0; kind < 3; ++kind) {
            double least = 1e300;
            for (int tile = 64; tile <= pad; tile *= 2) {
                const double n = (double)(R / tile), tiles = (double)o->matrices * (kind < 2 ? n * (n + 1) / 2 : n * (double)(C / tile));
                const double us = product_us(tile, tiles, (int)((kind == 0 ? C : R) / NS_KBLOCK));
                if (us < least) {
                    least = us;
                    chosen[kind] = tile;
                }
            }
            total += least;
        }
        if (total < best) {
            best = total;
            o->prows = (int32_t)R;
            o->pcols = (int32_t)C;
            for (int kind = 0; kind < 3; ++kind) o->tile[kind] = chosen[kind];
        }
    }
}

template <typename T>
hipError_t first_pass(const rb_ortho* o, const UpdateArgs& u, const KeptArgs& q, hipStream_t st)
{
    double* parts = reinterpret_cast<double*>(o->ws);
    const int64_t items = (int64_t)((o->m + 7) / 8) * ((o->n + NS_TPB - 1) / NS_TPB);
    const int nparts = (int)std::min<int64_t>(items, NS_PARTS);
    hipError_t e = launch(rb_ortho_norm_kernel<T>, dim3((unsigned)nparts, (unsigned)o->matrices), NS_TPB, 0, st, u, parts);
    if (e != hipSuccess) return e;
    return launch(rb_ortho_split_kernel<T>, dim3((unsigned)(o->pcols / 64), (unsigned)(o->prows / 64), (unsigned)o->matrices), NS_TPB, 0, st, u, q,
                  static_cast<const double*>(parts), nparts);
}

template <typename T, typename OUT>
hipError_t whole(const rb_ortho* o, const UpdateArgs& u, const ResultArgs& result, hipStream_t st)
{
    SmallArgs a{};
    a.update = u;
    a.result = result;
    a.steps = o->steps;
    for (int s = 0; s < o->steps; ++s)
        for (int i = 0; i < 3; ++i) a.coefficients[s][i] = o->coefficients[s][i];
    const size_t lds = (size_t)2 * o->small * o->small * 4;
    if (o->small == 64) return launch(rb_ortho_small_kernel<T, OUT, 64, 32>, dim3((unsigned)o->matrices), 256, lds, st, a);
    return launch(rb_ortho_small_kernel<T, OUT, 128, 64>, dim3((unsigned)o->matrices), 512, lds, st, a);
}

hipError_t orthogonalize(const rb_ortho* o, const UpdateArgs& u, const ResultArgs& result, hipStream_t st)
{
    if (o->small) {
        if (o->dtype == RB_F32) return o->out_dtype == RB_F32 ? whole<float, float>(o, u, result, st) : whole<float, Bf16>(o, u, result, st);
        return o->out_dtype == RB_F32 ? whole<Bf16, float>(o, u, result, st) : whole<Bf16, Bf16>(o, u, result, st);
    }
    const int64_t R = o->prows, C = o->pcols;
    _Float16* x = reinterpret_cast<_Float16*>(o->ws + o->off_x);
    _Float16* xt[2] = {reinterpret_cast<_Float16*>(o->ws + o->off_xt[0]), reinterpret_cast<_Float16*>(o->ws + o->off_xt[1])};
    _Float16* ma = reinterpret_cast<_Float16*>(o->ws + o->off_a);
    _Float16* mb = reinterpret_cast<_Float16*>(o->ws + o->off_b);
    const KeptArgs kept{x, xt[0], 2 * R * C, 2 * R * C, (int32_t)R, (int32_t)C};
    hipError_t e = o->dtype == RB_F32 ? first_pass<float>(o, u, kept, st) : first_pass<Bf16>(o, u, kept, st);
    for (int s = 0; s < o->steps && e == hipSuccess; ++s) {
        const float* c = o->coefficients[s];
        ProductArgs g{};                                   // A = X X^T
        g.p = x; g.q = x; g.p_matrix = g.q_matrix = 2 * R * C;
        g.kblocks = (int32_t)(C / NS_KBLOCK);
        g.out = ma; g.out_t = ma;
        g.out_matrix = g.out_t_matrix = 2 * R * R;
        g.out_pitch = g.out_t_pitch = 2 * R;
        g.beta = NS_SCALE_A / (NS_SCALE_X * NS_SCALE_X);
        if ((e = product<NS_GRAM, float>(o, g, o->tile[0], true, st)) != hipSuccess) break;
        ProductArgs p = g;                                 // B = b A + c A A
        p.p = ma; p.q = ma; p.p_matrix = p.q_matrix = 2 * R * R;
        p.kblocks = (int32_t)(R / NS_KBLOCK);
        p.old = ma; p.old_matrix = 2 * R * R; p.old_pitch = 2 * R;
        p.out = mb; p.out_t = mb;
        p.alpha = c[1] * (NS_SCALE_B / NS_SCALE_A);
        p.beta = c[2] * (NS_SCALE_B / (NS_SCALE_A * NS_SCALE_A));
        if ((e = product<NS_POLY, float>(o, p, o->tile[1], true, st)) != hipSuccess) break;
        ProductArgs q{};                                   // X <- a X + B X
        q.p = mb; q.p_matrix = 2 * R * R;
        q.q = xt[s & 1]; q.q_matrix = 2 * R * C;
        q.kblocks = (int32_t)(R / NS_KBLOCK);
        q.old = xt[s & 1]; q.old_matrix = 2 * R * C; q.old_pitch = 2 * R;
        q.out = x; q.out_matrix = 2 * R * C; q.out_pitch = 2 * C;
        q.out_t = xt[(s + 1) & 1]; q.out_t_matrix = 2 * R * C; q.out_t_pitch = 2 * R;
        q.alpha = c[0];
        q.beta = 1.0f / NS_SCALE_B;
        if (s + 1 < o->steps) {
            e = product<NS_APPLY, float>(o, q, o->tile[2], false, st);
            continue;
        }
        q.alpha = c[0] / NS_SCALE_X;
        q.beta = 1.0f / (NS_SCALE_B * NS_SCALE_X);
        q.result = result;
        e = o->out_dtype == RB_F32 ? product<NS_LAST, float>(o, q, o->tile[2], false, st) : product<NS_LAST, Bf16>(o, q, o->tile[2], false, st);
    }
    return e;
}

inline bool strides_fit(const rb_ortho* o, int64_t matrix_stride, int64_t row_stride, bool written)
{
    if (row_stride < o->n || matrix_stride < 0 || row_stride > INT64_MAX / RB_MAX_DIM / 8 || matrix_stride > INT64_MAX / RB_MAX_MATRICES / 8) return false;
    return !written || o->matrices == 1 || matrix_stride >= o->n;
}

}  // namespace

extern "C" {

int rb_ortho_create(rb_ortho** out, int64_t matrices, int64_t m, int64_t n, int32_t dtype, int32_t out_dtype, const float* coefficients,
                    int64_t steps, float eps)
{
    if (!out) return RB_EINVAL;
    *out = nullptr;
    if (!coefficients || matrices < 1 || matrices > RB_MAX_MATRICES || m < 1 || n < 1 || m > RB_MAX_DIM || n > RB_MAX_DIM) return RB_EINVAL;
    if ((dtype != RB_F32 && dtype != RB_BF16) || (out_dtype != RB_F32 && out_dtype != RB_BF16)) return RB_EINVAL;
    if (steps < 1 || steps > RB_MAX_ORTHO_STEPS || !std::isfinite(eps) || eps < 0.0f) return RB_EINVAL;
    for (int64_t i = 0; i < 3 * steps; ++i)
        if (!std::isfinite(coefficients[i])) return RB_EINVAL;
    for (int i = 0; i <= 1024; ++i) {                      // where the steps lead the singular values (at most 1 at first)
        double v = i / 1024.0;
        for (int64_t s = 0; s < steps; ++s) {
            const double l = v * v, q = coefficients[3 * s + 1] * l + coefficients[3 * s + 2] * l * l;
            v *= coefficients[3 * s] + q;
            if (!(std::fabs(v) <= 4.0) || !(std::fabs(q) <= 60.0)) return RB_EINVAL;
        }
    }
    rb_ortho* o = new (std::nothrow) rb_ortho();
    if (!o) return RB_ENOMEM;
    o->matrices = matrices;
    o->m = (int32_t)m;
    o->n = (int32_t)n;
    o->dtype = dtype;
    o->out_dtype = out_dtype;
    o->steps = (int32_t)steps;
    for (int64_t i = 0; i < 3 * steps; ++i) o->coefficients[i / 3][i % 3] = coefficients[i];
    o->eps = eps;
    o->tall = m > n;
    o->rows = (int32_t)std::min(m, n);
    o->cols = (int32_t)std::max(m, n);
    o->small = o->cols <= 64 ? 64 : o->cols <= 128 ? 128 : 0;
    o->bytes = 256;
    if (!o->small) {
        choose_tiles(o);
        const size_t kept = (size_t)matrices * o->prows * o->pcols * 4, square = (size_t)matrices * o->prows * o->prows * 4;
        size_t off = round_up((size_t)matrices * NS_PARTS * sizeof(double), 256);
        o->off_x = off; off += kept;
        o->off_xt[0] = off; off += kept;
        o->off_xt[1] = off; off += kept;
        o->off_a = off; off += square;
        o->off_b = off; off += square;
        o->bytes = off;
    }
    *out = o;
    return RB_OK;
}

int rb_ortho_query(const rb_ortho* o, size_t* workspace_bytes)
{
    if (!o || !workspace_bytes) return RB_EINVAL;
    *workspace_bytes = o->bytes;
    return RB_OK;
}

int rb_ortho_bind(rb_ortho* o, void* workspace)
{
    if (!o || !workspace || !aligned(workspace, 256)) return RB_EINVAL;
    o->ws = static_cast<char*>(workspace);
    return RB_OK;
}

int rb_ortho_apply(rb_ortho* o, const void* update, int64_t update_matrix_stride, int64_t update_row_stride, void* out,
                   int64_t out_matrix_stride, int64_t out_row_stride, void* hip_stream)
{
    if (!o || !update || !out) return RB_EINVAL;
    if (!aligned(update, (size_t)elem_bytes(o->dtype)) || !aligned(out, (size_t)elem_bytes(o->out_dtype))) return RB_EINVAL;
    if (!strides_fit(o, update_matrix_stride, update_row_stride, false) || !strides_fit(o, out_matrix_stride, out_row_stride, true)) return RB_EINVAL;
    if (!o->ws) return RB_ESTATE;
    UpdateArgs u{update, update_matrix_stride, update_row_stride, nullptr, 0.0f, 0, o->m, o->n, o->tall, o->eps};
    const ResultArgs w{out, out_matrix_stride, out_row_stride, o->rows, o->cols, o->tall, 0, 0.0f, 0.0f};
    return orthogonalize(o, u, w, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? RB_OK : RB_EHIP;
}

int rb_ortho_step(rb_ortho* o, void* weight, int64_t weight_matrix_stride, int64_t weight_row_stride, const void* grad,
                  int64_t grad_matrix_stride, int64_t grad_row_stride, float* momentum, float lr, float beta, int32_t nesterov,
                  float weight_decay, float scale, void* hip_stream)
{
    if (!o || !weight || !grad || !momentum) return RB_EINVAL;
    if (!aligned(grad, (size_t)elem_bytes(o->dtype)) || !aligned(weight, (size_t)elem_bytes(o->out_dtype)) || !aligned(momentum, 4)) return RB_EINVAL;
    if (!strides_fit(o, grad_matrix_stride, grad_row_stride, false) || !strides_fit(o, weight_matrix_stride, weight_row_stride, true)) return RB_EINVAL;
    if (!std::isfinite(lr) || !std::isfinite(beta) || !std::isfinite(weight_decay) || !std::isfinite(scale)) return RB_EINVAL;
    if (!o->ws) return RB_ESTATE;
    UpdateArgs u{grad, grad_matrix_stride, grad_row_stride, momentum, beta, nesterov != 0, o->m, o->n, o->tall, o->eps};
    const ResultArgs w{weight, weight_matrix_stride, weight_row_stride, o->rows, o->cols, o->tall, 1, (float)(1.0 - (double)lr * weight_decay),
                       (float)((double)lr * scale)};
    return orthogonalize(o, u, w, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? RB_OK : RB_EHIP;
}

int rb_ortho_destroy(rb_ortho* o)
{
    delete o;
    return RB_OK;
}

}  // extern "C"
