// The training step that the rehearsal buffer feeds, for gfx950 (MI355X): the C ABI of include/rb_train.h (host side); the kernels are in
// rb_kernels_scorer.h (scores of tokens and their gradient) and rb_kernels_ortho.h (orthogonalised updates).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
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

constexpr int64_t MAX_STRIDE = INT64_MAX / RB_MAX_ROWS / 8;      // of rows of logits: no offset passes 64 bits
inline int64_t elem_bytes(int32_t dtype) { return dtype == RB_F32 ? 4 : 2; }
inline size_t scorer_bytes(int32_t top) { return SC_SPLIT_GROUPS * (sizeof(uint32_t) + sc_partial_bytes(top)); }

template <typename T, bool TOP>
hipError_t score(const ScoreArgs& a, int waves, hipStream_t st)
{
    if (waves == 1) return launch(rb_score_kernel<T, TOP, 1>, dim3((unsigned)((a.rows + SC_NWAVE - 1) / SC_NWAVE)), SC_TPB, 0, st, a);
    const dim3 grid((unsigned)a.rows * (unsigned)a.splits);
    if (waves == 2) return launch(rb_score_kernel<T, TOP, 2>, grid, 2 * SC_WAVE, 0, st, a);
    if (waves == SC_NWAVE) return launch(rb_score_kernel<T, TOP, SC_NWAVE>, grid, SC_TPB, 0, st, a);
    return launch(rb_score_kernel<T, TOP, SC_MANY_WAVES>, grid, SC_MANY_WAVES * SC_WAVE, 0, st, a);
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
    if (vectors) return launch(a.grad_entropy ? rb_score_grad_kernel<T, Logit<T>::N, true> : rb_score_grad_kernel<T, Logit<T>::N, false>, grid, SC_TPB, 0, st, a);
    return launch(a.grad_entropy ? rb_score_grad_kernel<T, 1, true> : rb_score_grad_kernel<T, 1, false>, grid, SC_TPB, 0, st, a);
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
    if (!s || rows < 0 || rows > RB_MAX_ROWS || row_stride < s->vocab || row_stride > MAX_STRIDE) return RB_EINVAL;
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
    // Wavefronts per row: one tile is a wavefront's.  Rows that fill the chip get few, since each has a list of its own to sort and join, and four when
    // they are long.  Two where there are more rows than 7 workgroups of four on each of 256 compute units (bfloat16, 50001 with 16 alternatives, two
    // and four: 1700 rows 48.6 and 47.8 us, 1750 48.3 and 48.2, 1800 48.1 and 50.2, 2500 57.5 and 62.4; of 10000 1800 rows 18.8 and 22.4; without
    // alternatives 50001 1750 33.4 and 31.9, 1900 34.8 and 34.9).  Binary32 rows are twice the bytes, which long ones wait for rather than for lists (1800
    // rows of 10000 with 16 21.0 and 23.6, of 20000 32.1 and 33.3, of 30001 43.3 and 41.5; 3000 of 65000 152 and 144).  Fewer rows get 16.
    const bool two = rows > 7 * 256 && tiles <= (s->dtype == RB_BF16 ? 32 : 12);
    const int waves = tiles == 1 || (tiles <= 8 && rows >= 4096) ? 1 : two ? 2 : rows >= 512 || tiles <= SC_NWAVE ? SC_NWAVE : SC_MANY_WAVES;
    // Rows shared by workgroups: what the last one waits for (the others' parts have to reach memory) costs more with every workgroup, so the
    // more rows, the more tiles for each wavefront: one, two, and four from 33 rows (bfloat16, 20 alternatives, unshared and shared: one row
    // of 131072 20.0 and 13.2 us, 16 rows of 131072 20.7 and 18.0, 64 rows of 262144 34.5 and 26.3; at two tiles each 64 rows of 131072
    // without alternatives would take 15.3 us, not 11.4).
    const int64_t each = rows > 32 ? 4 : rows > 8 ? 2 : 1, splits = waves == SC_MANY_WAVES ? tiles / (each * SC_MANY_WAVES) : 1;
    a.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>({splits, SC_SPLIT_GROUPS / rows, SC_MAX_SPLITS}));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipError_t e;
    if (s->dtype == RB_F32)
        e = s->top ? score<float, true>(a, waves, st) : score<float, false>(a, waves, st);
    else
        e = s->top ? score<Bf16, true>(a, waves, st) : score<Bf16, false>(a, waves, st);
    return e == hipSuccess ? RB_OK : RB_EHIP;
}

int rb_scorer_grad(rb_scorer* s, const void* logits, int64_t rows, int64_t row_stride, const int64_t* tokens, const float* lse,
                   const float* entropy, const float* grad_logp, const float* grad_entropy, void* grad_logits, int64_t grad_stride,
                   void* hip_stream)
{
    if (!s || rows < 0 || rows > RB_MAX_ROWS || row_stride < s->vocab || grad_stride < s->vocab || row_stride > MAX_STRIDE || grad_stride > MAX_STRIDE)
        return RB_EINVAL;
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
    int32_t kept_rows, kept_cols;  // tiled: with room for whole tiles of every product
    int32_t tile[3], slices[3];    // of A, of B, of X
    bool pairs;                    // two steps are made on A before X is multiplied
    size_t off_x, off_xt[2], off_square[4], off_sums, bytes;
    char* ws;
};

namespace {

// A kernel that asks for more dynamic LDS than it gets by default: allowed once per kernel and device.
template <auto kernel>
hipError_t allow_lds(size_t bytes)
{
    static std::atomic<bool> allowed[64] = {};      // (handles of several host threads)
    int dev = 0;
    if (bytes <= 65536) return hipSuccess;
    if (hipGetDevice(&dev) != hipSuccess) return hipErrorInvalidDevice;
    if (dev >= 0 && dev < 64 && allowed[dev]) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess && dev >= 0 && dev < 64) allowed[dev] = true;
    return e;
}

enum { OF_A = 0, OF_B = 1, OF_X = 2 };

template <int KIND, typename OUT, int BM, int WM, int WN, int WAVES_PER_SIMD>
hipError_t product_of(const Operands& o, const ProductArgs& a, unsigned tiles, hipStream_t st)
{
    constexpr int STAGES = BM == 64 ? 3 : 2;
    constexpr size_t LDS = (size_t)STAGES * 2 * BM * 128;
    constexpr auto kernel = rb_ortho_product_kernel<KIND, OUT, BM, WM, WN, STAGES, WAVES_PER_SIMD>;
    hipError_t e = allow_lds<kernel>(LDS);
    if (e != hipSuccess) return e;
    e = launch(kernel, dim3(tiles * (unsigned)a.slices), BM / WM * (BM / WN) * 64, LDS, st, o.p, o.q, o.p_lines, o.q_lines, o.p_matrix, o.q_matrix,
               o.kblocks, a.tiles_i, a.tiles_j, a.tiles, a.slices, a);
    if (e != hipSuccess || a.slices == 1) return e;
    return launch(rb_ortho_join_kernel<KIND, OUT, BM>, dim3(tiles * (BM / 32) * (BM / 32) / (NS_TPB / 64)), NS_TPB, 0, st, a);
}

template <int KIND, typename OUT>
hipError_t product(const rb_ortho* o, const Operands& of, ProductArgs a, int which, hipStream_t st)
{
    const int tile = o->tile[which];
    a.tiles_i = (o->rows + tile - 1) / tile;
    a.tiles_j = which == OF_X ? (o->cols + tile - 1) / tile : a.tiles_i;
    a.tiles = which == OF_X ? a.tiles_i * a.tiles_j : a.tiles_i * (a.tiles_i + 1) / 2;
    a.slices = o->slices[which];
    a.sums = reinterpret_cast<float*>(o->ws + o->off_sums);
    const unsigned tiles = (unsigned)(a.tiles * o->matrices);
    switch (tile) {
    case 256: return product_of<KIND, OUT, 256, 128, 64, 2>(of, a, tiles, st);
    case 192: return product_of<KIND, OUT, 192, 96, 96, 1>(of, a, tiles, st);
    case 128: return product_of<KIND, OUT, 128, 64, 32, 4>(of, a, tiles, st);
    default: return product_of<KIND, OUT, 64, 32, 32, 3>(of, a, tiles, st);
    }
}

// What a product takes, in us, by its tile and slices: a launch with its ends, and per block of 32 of the summed index what 256 compute units were
// measured to take, by how many tiles there are per unit (64: 0.23 for one, 0.25 each for more; 128: 0.57 for one while others idle,
// 0.74, 0.8; 192: 1.2, 1.55 and 256: 1.85, 2.0, 2.5, one at a time).  Slices add a launch that reads what they have written.
double product_us(int tile, double tiles, int kblocks, int slices)
{
    const double per = tiles * slices / 256, whole = std::floor(per), part = per - whole;
    const double shared = whole + (part > 0 ? 0.35 + 0.65 * part : 0);       // several at a time: the last of them have the unit to themselves
    double us = 0;
    if (tile == 64) us = 5 + kblocks / (double)slices * (per <= 1 ? 0.23 : 0.25 * shared);
    if (tile == 128) us = 8 + kblocks / (double)slices * (per <= 0.5 ? 0.57 : per <= 1 ? 0.57 + 0.34 * (per - 0.5) : 0.8 * shared);
    if (tile == 192) us = 12 + kblocks / (double)slices * (per <= 0.5 ? 1.2 : 1.55) * std::ceil(per);
    if (tile == 256) us = 16 + kblocks / (double)slices * (per <= 0.5 ? 1.85 : per <= 0.75 ? 2.0 : 2.5) * std::ceil(per);
    return slices == 1 ? us : us + 6 + tiles * slices * tile * tile * 8 / 1e7;
}

// Whether P of every step, and of every pair the product of both, stay within what is kept (60 in NS_SCALE_B).
bool pairs_fit(const rb_ortho* o)
{
    for (int i = 0; i <= 1024; ++i) {
        double v = i / 1024.0, first = 1.0;
        for (int s = 0; s < o->steps; ++s) {
            const float* c = o->coefficients[s];
            const double l = v * v, p = c[0] + c[1] * l + c[2] * l * l;
            v *= p;
            if (!(std::fabs(p) <= 60.0) || (s % 2 != 0 && !(std::fabs(first * p) <= 60.0))) return false;
            first = p;
        }
    }
    return true;
}

// The tiles and slices that take least, whether pairs of steps are made on A, and the room that all products need.
void choose_tiles(rb_ortho* o)
{
    int64_t rows = round_up((size_t)o->rows, 64), cols = round_up((size_t)o->cols, 64);
    size_t sums = 0;
    double us[3];
    for (int which = 0; which < 3; ++which) {
        us[which] = 1e300;
        for (int tile = 64; tile <= 256; tile += 64) {
            const int64_t n = (o->rows + tile - 1) / tile, m = (o->cols + tile - 1) / tile, tiles = o->matrices * (which == OF_X ? n * m : n * (n + 1) / 2);
            const int kblocks = ((which == OF_A ? o->cols : o->rows) + NS_KBLOCK - 1) / NS_KBLOCK;
            for (int slices = 1; slices <= 16 && (slices == 1 || (kblocks / slices >= 8 && tiles * slices <= 512)); ++slices) {
                const double t = product_us(tile, (double)tiles, kblocks, slices);
                if (t >= us[which]) continue;
                us[which] = t;
                o->tile[which] = tile;
                o->slices[which] = slices;
            }
        }
        const size_t tile = (size_t)o->tile[which], n = (o->rows + tile - 1) / tile, m = (o->cols + tile - 1) / tile;
        rows = std::max(rows, (int64_t)(n * tile));
        cols = std::max(cols, (int64_t)((which == OF_X ? m : n) * tile));
        if (o->slices[which] > 1) sums = std::max(sums, (size_t)o->matrices * (which == OF_X ? n * m : n * (n + 1) / 2) * o->slices[which] * tile * tile * sizeof(float));
    }
    // two steps: A, five squares (in LDS: 0.9 or 2.3 us each, and 5 for the launch) and R X instead of twice A, B and B X
    const double five = o->rows > 128 ? 5 * us[OF_B] : 5 + 5 * (o->rows <= 64 ? 0.9 : 2.3) * (double)((o->matrices + 255) / 256);
    o->pairs = o->steps > 1 && five < us[OF_A] + 2 * us[OF_B] + us[OF_X] && pairs_fit(o);
    o->kept_rows = (int32_t)rows;
    o->kept_cols = (int32_t)cols;
    const size_t n = (size_t)o->matrices * sizeof(_Float16), xp = (size_t)ns_pitch(cols), tp = (size_t)ns_pitch(rows);
    size_t off = round_up((size_t)o->matrices * NS_PARTS * sizeof(double), 256);
    o->off_x = off; off += n * (size_t)rows * xp;
    o->off_xt[0] = off; off += n * (size_t)cols * tp;
    o->off_xt[1] = off; off += n * (size_t)cols * tp;
    for (int i = 0; i < 4; ++i) {                          // A, B (P); of pairs also the first P and what P A and R share
        o->off_square[i] = off;
        if (i < 2 || (o->pairs && o->rows > 128)) off += n * (size_t)rows * tp;
    }
    o->off_sums = off; off += sums;
    o->bytes = off;
}

template <typename T, int V>
hipError_t first_passes(const rb_ortho* o, const UpdateArgs& u, const KeptArgs& q, hipStream_t st)
{
    double* parts = reinterpret_cast<double*>(o->ws);
    const int64_t items = (int64_t)((o->m + NS_ROWS_AT_ONCE - 1) / NS_ROWS_AT_ONCE) * ((o->n + V * NS_TPB - 1) / (V * NS_TPB));
    const int nparts = (int)std::min<int64_t>(items, NS_PARTS);
    hipError_t e = launch(rb_ortho_norm_kernel<T, V>, dim3((unsigned)nparts, (unsigned)o->matrices), NS_TPB, 0, st, u, parts);
    if (e != hipSuccess) return e;
    return launch(rb_ortho_split_kernel<T, V>, dim3((unsigned)(o->cols + 63) / 64, (unsigned)(o->rows + 63) / 64, (unsigned)o->matrices), NS_TPB, 0, st, u, q,
                  static_cast<const double*>(parts), nparts);
}

template <typename T>
hipError_t first_pass(const rb_ortho* o, const UpdateArgs& u, const KeptArgs& q, hipStream_t st)
{
    const bool vectors = o->n % 4 == 0 && u.row_stride % 4 == 0 && u.matrix_stride % 4 == 0 && aligned(u.grad, 4 * sizeof(T)) &&
                         aligned(u.momentum, 16);
    return vectors ? first_passes<T, 4>(o, u, q, st) : first_passes<T, 1>(o, u, q, st);
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
    if (o->small == 64) return launch(rb_ortho_small_kernel<T, OUT, 64>, dim3((unsigned)o->matrices), 256, lds, st, a);
    constexpr auto kernel = rb_ortho_small_kernel<T, OUT, 128>;
    const hipError_t e = allow_lds<kernel>(lds);
    return e != hipSuccess ? e : launch(kernel, dim3((unsigned)o->matrices), 1024, lds, st, a);
}

// R of steps s and s + 1, from A, of short sides that fit one workgroup.
hipError_t pair_in_lds(const rb_ortho* o, const _Float16* a, _Float16* r, int64_t pitch, int s, hipStream_t st)
{
    PairArgs g{};
    g.a = a;
    g.r = r;
    g.matrix = o->kept_rows * pitch;
    g.pitch = pitch;
    g.rows = o->rows;
    for (int i = 0; i < 2; ++i)
        for (int k = 0; k < 3; ++k) g.coefficients[i][k] = o->coefficients[s + i][k];
    if (o->rows <= 64) return launch(rb_ortho_pair_kernel<64>, dim3((unsigned)o->matrices), 256, 2 * LdsMatrices<64>::BYTES, st, g);
    const hipError_t e = allow_lds<rb_ortho_pair_kernel<128>>(2 * LdsMatrices<128>::BYTES);
    return e != hipSuccess ? e : launch(rb_ortho_pair_kernel<128>, dim3((unsigned)o->matrices), 1024, 2 * LdsMatrices<128>::BYTES, st, g);
}

hipError_t orthogonalize(const rb_ortho* o, const UpdateArgs& u, const ResultArgs& result, hipStream_t st)
{
    if (o->small) {
        if (o->dtype == RB_F32) return o->out_dtype == RB_F32 ? whole<float, float>(o, u, result, st) : whole<float, Bf16>(o, u, result, st);
        return o->out_dtype == RB_F32 ? whole<Bf16, float>(o, u, result, st) : whole<Bf16, Bf16>(o, u, result, st);
    }
    const int64_t R = o->kept_rows, C = o->kept_cols;
    const int64_t xp = ns_pitch(C), tp = ns_pitch(R);     // halves between rows of X; of X^T and the squares
    auto place = [&](size_t off) { return reinterpret_cast<_Float16*>(o->ws + off); };
    _Float16 *const x = place(o->off_x), *const xt[2] = {place(o->off_xt[0]), place(o->off_xt[1])};
    const KeptArgs kept{x, xt[0], R * xp, C * tp, xp, tp, (int32_t)R, (int32_t)C};
    hipError_t e = o->dtype == RB_F32 ? first_pass<float>(o, u, kept, st) : first_pass<Bf16>(o, u, kept, st);
    const int by_rows = (o->rows + NS_KBLOCK - 1) / NS_KBLOCK, by_cols = (o->cols + NS_KBLOCK - 1) / NS_KBLOCK;
    const int32_t xl = (int32_t)(xp / NS_KHALVES), tl = (int32_t)(tp / NS_KHALVES);
    const uint32_t x_matrix = (uint32_t)(R * xl), t_matrix = (uint32_t)(C * tl), square_matrix = (uint32_t)(R * tl);
    // to <- beta * p q^T of two squares that commute: symmetric
    auto squares = [&](const _Float16* p, const _Float16* q) { return Operands{p, q, tl, tl, square_matrix, square_matrix, by_rows}; };
    auto to_square = [&](_Float16* to, float beta) {
        ProductArgs a{};
        a.out = to; a.out_t = to; a.out_matrix = a.out_t_matrix = R * tp; a.out_pitch = a.out_t_pitch = tp;
        a.beta = beta;
        return a;
    };
    _Float16 *const ma = place(o->off_square[0]), *const mb = place(o->off_square[1]);
    // to <- b A + c A A of step s, and P of a pair's: a I too
    auto polynomial = [&](int s, bool whole, _Float16* to) {
        const float* c = o->coefficients[s];
        ProductArgs p = to_square(to, c[2] * (NS_SCALE_B / (NS_SCALE_A * NS_SCALE_A)));
        p.old = ma; p.old_matrix = R * tp; p.old_pitch = tp;
        p.alpha = c[1] * (NS_SCALE_B / NS_SCALE_A);
        p.diagonal = whole ? c[0] * NS_SCALE_B : 0.0f;
        return product<NS_POLY, float>(o, squares(ma, ma), p, OF_B, st);
    };
    for (int s = 0, n = 0, now = 0; s < o->steps && e == hipSuccess; s += n, now ^= 1) {
        n = o->pairs && s + 1 < o->steps ? 2 : 1;
        // A = X X^T
        e = product<NS_GRAM, float>(o, Operands{x, x, xl, xl, x_matrix, x_matrix, by_cols}, to_square(ma, NS_SCALE_A / (NS_SCALE_X * NS_SCALE_X)), OF_A, st);
        // B and then a X + B X; or, of a pair, R and R X
        const _Float16* left_of_x = mb;
        if (n == 1 && e == hipSuccess) e = polynomial(s, false, mb);
        if (n == 2 && o->rows <= 128 && e == hipSuccess) e = pair_in_lds(o, ma, mb, tp, s, st);
        if (n == 2 && o->rows > 128) {
            _Float16 *const first = place(o->off_square[2]), *const t = place(o->off_square[3]);
            if (e == hipSuccess) e = polynomial(s, true, first);
            if (e == hipSuccess) e = product<NS_GRAM, float>(o, squares(first, ma), to_square(t, 1.0f / NS_SCALE_B), OF_B, st);       // A <- P (P A)
            if (e == hipSuccess) e = product<NS_GRAM, float>(o, squares(first, t), to_square(ma, 1.0f / NS_SCALE_B), OF_B, st);
            if (e == hipSuccess) e = polynomial(s + 1, true, mb);
            if (e == hipSuccess) e = product<NS_GRAM, float>(o, squares(mb, first), to_square(t, 1.0f / NS_SCALE_B), OF_B, st);      // R
            left_of_x = t;
        }
        if (e != hipSuccess) break;
        const Operands of{left_of_x, xt[now], tl, tl, square_matrix, t_matrix, by_rows};
        ProductArgs q{};
        if (n == 1) {
            q.old = xt[now]; q.old_matrix = C * tp; q.old_pitch = tp;
            q.alpha = o->coefficients[s][0];
        }
        q.out = x; q.out_matrix = R * xp; q.out_pitch = xp;
        q.out_t = xt[now ^ 1]; q.out_t_matrix = C * tp; q.out_t_pitch = tp;
        q.beta = 1.0f / NS_SCALE_B;
        if (s + n < o->steps) {
            e = product<NS_APPLY, float>(o, of, q, OF_X, st);
            continue;
        }
        q.alpha /= NS_SCALE_X;
        q.beta /= NS_SCALE_X;
        q.result = result;
        e = o->out_dtype == RB_F32 ? product<NS_LAST, float>(o, of, q, OF_X, st) : product<NS_LAST, Bf16>(o, of, q, OF_X, st);
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
    if (!o->small) choose_tiles(o);
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
