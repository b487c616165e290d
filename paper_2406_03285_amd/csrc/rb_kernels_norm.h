// Dropout (rb_dropout), layer norm of a residual sum (rb_norm_forward) and its gradients (rb_norm_grad).  Included by rb_block.hip only.
//
// All are bound by HBM: what they read and write once is all they move.  A row stays in registers between its sums and its results: LANES lanes hold
// PARTS pieces of 8 numbers each, and the sums go over them twice, for the mean and then for the squares of what is left without it (one pass over both
// would lose the variance of rows that lie far from 0).  The mean is made exact to its last bit by a second sum, over the differences.
// The weights' gradients are sums over rows: a workgroup goes through rows that are the grid's width apart and keeps its columns' sums in registers; what
// the workgroups have is added up by a second launch, in the same order every time.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>
#include <type_traits>

#include "rb_lanes.h"

namespace {

constexpr int NM_TPB = 256;
constexpr int NM_PIECE = 8;                        // numbers of a lane's piece: 16 bytes of bfloat16, 32 of binary32; one draw of dropout
constexpr int NM_MAX_GROUPS = 512;                 // most workgroups whose sums of the weights' gradients are kept: two for each compute unit

// ---- numbers -------------------------------------------------------------------

// Eight numbers of a row as they lie in memory, at any alignment (the hardware's accesses of 16 bytes take any address).
template <typename T> struct Piece;
template <> struct Piece<float> {
    float v[8];
    __device__ __forceinline__ float get(int i) const { return v[i]; }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = x[i];
    }
    __device__ __forceinline__ void load(const float* p) { memcpy(v, p, 32); }
    __device__ __forceinline__ void store(float* p) const { memcpy(p, v, 32); }
    __device__ __forceinline__ void put(float* p, float x) const { *p = x; }
    __device__ __forceinline__ void keep()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(v[i]));
    }
};
template <> struct Piece<Bf16> {
    sc_vec w;
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = sc_bf16_pair(x[2 * i], x[2 * i + 1]);
    }
    __device__ __forceinline__ void load(const Bf16* p) { memcpy(&w, p, 16); }
    __device__ __forceinline__ void store(Bf16* p) const { memcpy(p, &w, 16); }
    __device__ __forceinline__ void put(Bf16* p, float x) const { p->bits = (uint16_t)sc_bf16_bits(x); }
    // From here on the numbers are taken apart anew (otherwise the compiler keeps all of them as binary32 beside the row).
    __device__ __forceinline__ void keep() { asm volatile("" : "+v"(w)); }
};

__device__ __forceinline__ float nm_number(float x) { return x; }
__device__ __forceinline__ float nm_number(Bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }

// A row's pieces: lane `lane` of LANES has the pieces p * LANES + lane, p < PARTS, and the row ends among those of the last part.  Where it does not end with
// a piece, the last one is the row's last eight numbers: the first `skip` of them are another lane's too, which makes the same of them; sums leave them out
// here.  (Lanes behind the row's end have its last eight numbers as well, and skip all.)  Rows of less than eight numbers come one by one.
template <int LANES, int PARTS>
struct Row {
    int width, lane, skip, last;       // of the last part: where it is
    __device__ __forceinline__ Row(int width_, int lane_) : width(width_), lane(lane_)
    {
        const int column = ((PARTS - 1) * LANES + lane) * NM_PIECE;
        last = max(min(column, width - NM_PIECE), 0);
        skip = column < width ? column - last : NM_PIECE;
    }
    __device__ __forceinline__ bool tiny() const { return LANES == 16 && PARTS == 1 && width < NM_PIECE; }
    __device__ __forceinline__ int column(int p) const { return p < PARTS - 1 ? (p * LANES + lane) * NM_PIECE : last; }
    __device__ __forceinline__ bool counts(int p, int i) const { return p < PARTS - 1 || (i >= skip && (LANES != 16 || PARTS != 1 || i < width)); }
    template <typename T>
    __device__ __forceinline__ void load(const T* row, int p, Piece<T>& x) const
    {
        if (tiny()) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < width ? nm_number(row[i]) : 0.0f;
            x.set(v);
        } else {
            x.load(row + column(p));
        }
    }
    template <typename T>
    __device__ __forceinline__ void store(T* row, int p, const Piece<T>& x) const
    {
        if (p == PARTS - 1 && skip == NM_PIECE) return;
        if (tiny()) {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < width) x.put(row + i, x.get(i));
        } else {
            x.store(row + column(p));
        }
    }
    // Weights are binary32 or bfloat16, as the handle says (the same for all lanes).
    __device__ __forceinline__ void weights(const void* w, bool wide, int p, float (&v)[8]) const
    {
        if (wide) {
            Piece<float> x;
            load(static_cast<const float*>(w), p, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = x.get(i);
        } else {
            Piece<Bf16> x;
            load(static_cast<const Bf16*>(w), p, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = x.get(i);
        }
    }
};

// ---- dropout -------------------------------------------------------------------

struct Drop {
    uint32_t seed_lo, seed_hi, step_lo, step_hi;
    uint32_t least;            // what 16 bits have to be to stay: 0 (all stay) .. 65536 (none does)
    float scale;
};

// Philox4x32-10 (Salmon et al., SC'11) of a row and a piece of it, 16 bits an element.
__device__ __forceinline__ void nm_draw(const Drop& d, uint32_t row, uint32_t piece, uint32_t (&x)[4])
{
    uint32_t x0 = row, x1 = 0x80000000u | piece, x2 = d.step_lo, x3 = d.step_hi, ka = d.seed_lo, kb = d.seed_hi;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t pa = (uint64_t)0xD2511F53u * x0, pb = (uint64_t)0xCD9E8D57u * x2;
        x0 = (uint32_t)(pb >> 32) ^ x1 ^ ka;
        x2 = (uint32_t)(pa >> 32) ^ x3 ^ kb;
        x1 = (uint32_t)pb;
        x3 = (uint32_t)pa;
        ka += 0x9E3779B9u;
        kb += 0xBB67AE85u;
    }
    x[0] = x0; x[1] = x1; x[2] = x2; x[3] = x3;
}

// What stays of the eight numbers from `column` on.  Those of a row's end may be parts of two pieces (ENDS: it may be the end).
template <bool ENDS>
__device__ __forceinline__ void nm_drop(const Drop& d, uint32_t row, int column, float (&v)[8])
{
    if (d.least == 0) return;
    uint32_t x[4];
    nm_draw(d, row, (uint32_t)column / NM_PIECE, x);
    const int by = column % NM_PIECE;
    if (ENDS && __any(by != 0)) {
        uint32_t more[4];
        nm_draw(d, row, (uint32_t)column / NM_PIECE + 1, more);
        // the sixteen halves move down by as many as the first number is behind its piece's begin
        const bool one = by & 1, two = by & 2, four = by & 4;
        const uint32_t a0 = one ? x[0] >> 16 | x[1] << 16 : x[0], a1 = one ? x[1] >> 16 | x[2] << 16 : x[1], a2 = one ? x[2] >> 16 | x[3] << 16 : x[2];
        const uint32_t a3 = one ? x[3] >> 16 | more[0] << 16 : x[3], a4 = one ? more[0] >> 16 | more[1] << 16 : more[0];
        const uint32_t a5 = one ? more[1] >> 16 | more[2] << 16 : more[1], a6 = one ? more[2] >> 16 | more[3] << 16 : more[2];
        const uint32_t b0 = two ? a1 : a0, b1 = two ? a2 : a1, b2 = two ? a3 : a2, b3 = two ? a4 : a3, b4 = two ? a5 : a4, b5 = two ? a6 : a5;
        x[0] = four ? b2 : b0;
        x[1] = four ? b3 : b1;
        x[2] = four ? b4 : b2;
        x[3] = four ? b5 : b3;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = (x[i] & 0xffffu) >= d.least ? v[2 * i] * d.scale : 0.0f;
        v[2 * i + 1] = (x[i] >> 16) >= d.least ? v[2 * i + 1] * d.scale : 0.0f;
    }
}

struct DropoutArgs {
    const void* x;
    void* out;
    int64_t x_stride, out_stride;
    int64_t items;                     // of a workgroup's work
    int32_t rows, width, pieces;       // pieces of a row
    int32_t at_once, blocks;           // an item: this many short rows, or this part of a row
    Drop drop;
};

// A thread has eight numbers, that is one draw: ten rounds of two multiplications hide behind the reading.  Short rows share a workgroup; long grids go round.
// Bound by HBM: 8191 x 10007 bfloat16 63.3 us, 5.2 TB/s, what a copy reaches.  Of 128 x 192 binary32 the launch (3.0 us of a call's 5.7).
template <typename T>
__global__ void __launch_bounds__(NM_TPB) rb_dropout_kernel(DropoutArgs a)
{
    int r = 0, p = threadIdx.x;
    if (a.at_once > 1) {
        r = (int)((uint32_t)threadIdx.x / (uint32_t)a.pieces);
        p = threadIdx.x - r * a.pieces;
        if (r >= a.at_once) return;
    }
    for (int64_t item = blockIdx.x; item < a.items; item += gridDim.x) {
        const int64_t line = item / a.blocks;
        const int64_t row = line * a.at_once + r;
        const int piece = (int)(item - line * a.blocks) * NM_TPB + p, column = piece * NM_PIECE;
        if (row >= a.rows || piece >= a.pieces) continue;
        const T* const from = static_cast<const T*>(a.x) + row * a.x_stride + column;
        T* const to = static_cast<T*>(a.out) + row * a.out_stride + column;
        const int there = a.width - column;
        Piece<T> x;
        float v[8];
        if (there >= NM_PIECE) {
            x.load(from);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < there ? nm_number(from[i]) : 0.0f;
            x.set(v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = x.get(i);
        nm_drop<false>(a.drop, (uint32_t)row, column, v);
        x.set(v);
        if (there >= NM_PIECE) {
            x.store(to);
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < there) x.put(to + i, x.get(i));
        }
    }
}

// ---- sums over a row ------------------------------------------------------------

// Sums over the LANES lanes of a row, the same in all of them.  `places`: 2 sums of each wavefront, for this call alone.
template <int LANES, int N>
__device__ __forceinline__ void nm_sum(float (&v)[N], float* places)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] += sc_xor<1>(v[i]);
        v[i] += sc_xor<2>(v[i]);
        v[i] += sc_xor<4>(v[i]);
        v[i] += sc_xor<8>(v[i]);
        if (LANES >= 32) v[i] += sc_xor<16>(v[i]);
        if (LANES >= 64) v[i] += sc_xor<32>(v[i]);
    }
    if (LANES > 64) {
        constexpr int WAVES = LANES / 64;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) places[threadIdx.x / 64 * N + i] = v[i];
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // (not for what is on its way from memory)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v[i] += places[(threadIdx.x / LANES * WAVES + w) * N + i];
        }
    }
}

// ---- forward -------------------------------------------------------------------

struct NormArgs {
    const void *x, *residual, *weight, *bias;
    void *total, *y;
    float *mean, *rstd;
    int64_t x_stride, residual_stride, total_stride, y_stride;
    int32_t rows, width;
    float eps;
    bool wide_weights, drops;
    Drop drop;
};

// Wavefronts that share a SIMD, so how many workgroups of how many threads a grid that fills the chip once has.  More hide more of memory's latency until a row and the
// next one no longer fit their registers (forward, one less each: 8192 x 8192 bfloat16 118 -> 129 us, 13000 x 5003 153 -> 171; one more: 118 -> 158, 153 -> 169).
constexpr int nm_threads(int lanes) { return lanes > NM_TPB ? lanes : NM_TPB; }
template <typename T>
constexpr int nm_waves(int lanes, int parts)
{
    const int registers = parts * (int)sizeof(T) / 2;      // of a row, by fours
    return lanes > 512 || registers <= 2 ? 4 : registers <= 4 ? 3 : 2;
}

// A workgroup goes through rows that are the grid's width apart; the next row is on its way while one is worked on.  What is kept of a row is as it lies in
// memory (the sum is rounded to that type anyway).  SUMMED: there is a residual or dropout.  The sum is stored when all of the row has been read (a lane that
// has numbers of another one reads them in its own time).
// Bound by HBM: 8192 x 8192 bfloat16 with residual and dropout 110 us (4.9 TB/s), or 118 where one call follows another at once and the clock falls;
// 5120 x 2048 binary32 alone 17.3 us (4.85 TB/s).  One row: the launch and one chain of reading, sums and writing, 3.0 us of a call's 6.1.
template <typename T, int LANES, int PARTS, bool SUMMED>
__global__ void __launch_bounds__(nm_threads(LANES), nm_waves<T>(LANES, PARTS)) rb_norm_kernel(NormArgs a)
{
    constexpr int ROWS = nm_threads(LANES) / LANES;
    constexpr bool KEPT = PARTS * sizeof(T) <= 4;              // weights stay in registers between rows
    __shared__ float places[2][2][32];
    const Row<LANES, PARTS> of(a.width, threadIdx.x % LANES);
    const int line = threadIdx.x / LANES;
    Piece<T> x[PARTS], next[PARTS], next_r[SUMMED ? PARTS : 1];
    auto row_of = [&](int64_t first) { return min(first + line, (int64_t)a.rows - 1); };       // (of the last rows some are made twice, alike)
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) of.load(static_cast<const T*>(a.x) + row * a.x_stride, p, next[p]);
        if (SUMMED && a.residual) {
#pragma unroll
            for (int p = 0; p < PARTS; ++p) of.load(static_cast<const T*>(a.residual) + row * a.residual_stride, p, next_r[p]);
        }
    };
    int64_t first = (int64_t)blockIdx.x * ROWS;
    fetch(row_of(first));
    float w[KEPT ? PARTS : 1][8], b[KEPT ? PARTS : 1][8];
    auto fetch_weights = [&](int p, float (&ww)[8], float (&bb)[8]) {
        of.weights(a.weight, a.wide_weights, p, ww);
        if (a.bias) of.weights(a.bias, a.wide_weights, p, bb);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) bb[i] = 0.0f;
        }
    };
    if constexpr (KEPT) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) fetch_weights(p, w[p], b[p]);
    }
    const float width = (float)a.width;
    for (int turn = 0; first < a.rows; first += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const int64_t row = row_of(first);
        const bool mine = first + line < a.rows;
        float sum[1] = {0.0f};
        // part by part: all parts' draws side by side would not fit
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            x[p] = next[p];
            if constexpr (SUMMED) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = x[p].get(i);
                if (a.drops) {
                    if (p == PARTS - 1) nm_drop<true>(a.drop, (uint32_t)row, of.column(p), v);
                    else nm_drop<false>(a.drop, (uint32_t)row, of.column(p), v);
                }
                if (a.residual) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] += next_r[p].get(i);
                }
                x[p].set(v);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += of.counts(p, i) ? x[p].get(i) : 0.0f;
            x[p].keep();
            __builtin_amdgcn_sched_barrier(0);
        }
        if (first + (int64_t)gridDim.x * ROWS < a.rows) fetch(row_of(first + (int64_t)gridDim.x * ROWS));
        nm_sum<LANES>(sum, places[turn][0]);
        if constexpr (SUMMED) {
            if (mine) {
#pragma unroll
                for (int p = 0; p < PARTS; ++p) of.store(static_cast<T*>(a.total) + row * a.total_stride, p, x[p]);
            }
        }
        const float mean = sum[0] / width;
        float off[2] = {0.0f, 0.0f};               // sums of the differences and of their squares
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = of.counts(p, i) ? x[p].get(i) - mean : 0.0f;
                off[0] += d;
                off[1] = fmaf(d, d, off[1]);
            }
            x[p].keep();
        }
        nm_sum<LANES>(off, places[turn][1]);
        const float more = off[0] / width;
        float rstd = 1.0f / sqrtf(fmaxf(fmaf(-more, more, off[1] / width), 0.0f) + a.eps);
        if (off[1] != off[1]) rstd = off[1];       // (a NaN is none of fmaxf's)
        if (mine && of.lane == 0) {
            if (a.mean) a.mean[row] = mean + more;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            float out[8], ww[8], bb[8];
            if constexpr (!KEPT) fetch_weights(p, ww, bb);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float h = (x[p].get(i) - mean - more) * rstd;        // (the mean as two numbers: rows far from 0)
                if constexpr (KEPT) out[i] = fmaf(h, w[p][i], b[p][i]);
                else out[i] = fmaf(h, ww[i], bb[i]);
            }
            Piece<T> y;
            y.set(out);
            if (mine) of.store(static_cast<T*>(a.y) + row * a.y_stride, p, y);
        }
    }
}

// ---- gradients -----------------------------------------------------------------

constexpr int NM_SUM_WAVES = 2;

// What a row has beside its mean, from the sum of the differences: half a step of the mean at most.  (More would be what that sum's own roundings leave, which
// rows near 0 are better without.)
__device__ __forceinline__ float nm_rest(float sum, int width, float mean)
{
    const float most = fabsf(mean) * 0x1p-24f;
    return fminf(fmaxf(sum / (float)width, -most), most);
}

struct NormGradArgs {
    const void *grad_y, *total, *grad_total, *weight;
    const float *mean, *rstd;
    void *grad_sum, *grad_x;
    float* sums;                       // [2][groups][width]: of the weight's and of the bias's gradient
    float* rests;                      // [rows]: what the rows have beside `mean`, for rb_norm_columns_kernel; null: not wanted
    int64_t grad_y_stride, total_stride, grad_total_stride, grad_sum_stride, grad_x_stride;
    int32_t rows, width;
    bool wide_weights, drops;
    Drop drop;
};

// As forward; the gradients of the next row's y and that row are on their way while one is worked on.  SUMS: the weights' gradients are summed on the way (of rows
// that leave room for the sums).
// Bound by HBM where rows are of 1024 to 8192: 16384 x 4096 bfloat16 with residual and dropout 140 us of the call's 145 (4.8 TB/s).  Where there are few or
// short rows, by the sums between lanes (65536 x 512 73 us, 4.6 TB/s; 65536 x 100 30 us, 2.1 TB/s); of more than 8192, by the registers (4096 x 16384 196 us, 3.4 TB/s), of more
// than 16384 by reading grad_y and total twice, too (4096 x 32768 634 us, 2.1 TB/s).
//
// `mean` is one number, so of rows far from 0 half a step of it may be as large as what the rows differ by (a mean of 10^4 with a deviation of 10^-3: h off by 0.15).
// The forward pass normalises with the mean as two numbers; the second one, `rest`, is made again here, as a third sum over the row, and h is that of the forward
// pass.  The sums of g h are made without it and put right: sum of g (h - rest rstd).
template <typename T, int LANES, int PARTS>
__global__ void __launch_bounds__(nm_threads(LANES), LANES > 512 ? 4 : NM_SUM_WAVES) rb_norm_grad_kernel(NormGradArgs a)
{
    constexpr bool SUMS = LANES <= 512;
    constexpr int TPB = nm_threads(LANES), ROWS = TPB / LANES;
    constexpr bool KEPT = SUMS && PARTS * sizeof(T) <= (sizeof(T) == 2 ? 6 : 8);       // weights stay in registers between rows
    __shared__ float places[2][48];
    const Row<LANES, PARTS> of(a.width, threadIdx.x % LANES);
    const int line = threadIdx.x / LANES;
    Piece<T> next_y[PARTS], next_t[PARTS];
    auto row_of = [&](int64_t first) { return min(first + line, (int64_t)a.rows - 1); };
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            of.load(static_cast<const T*>(a.grad_y) + row * a.grad_y_stride, p, next_y[p]);
            of.load(static_cast<const T*>(a.total) + row * a.total_stride, p, next_t[p]);
        }
    };
    int64_t first = (int64_t)blockIdx.x * ROWS;
    fetch(row_of(first));
    float w[KEPT ? PARTS : 1][8];
    float gw[SUMS ? PARTS : 1][8], gb[SUMS ? PARTS : 1][8];
    if constexpr (KEPT) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) of.weights(a.weight, a.wide_weights, p, w[p]);
    }
    if constexpr (SUMS) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) gw[p][i] = gb[p][i] = 0.0f;
    }
    for (int turn = 0; first < a.rows; first += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const int64_t row = row_of(first);
        const bool mine = first + line < a.rows;
        const float mean = a.mean[row], rstd = a.rstd[row];
        Piece<T> y[PARTS], t[PARTS], more[PARTS];
        if (a.grad_total) {
#pragma unroll
            for (int p = 0; p < PARTS; ++p) of.load(static_cast<const T*>(a.grad_total) + row * a.grad_total_stride, p, more[p]);
        }
        float sum[3] = {0.0f, 0.0f, 0.0f};
        auto part = [&](int p, float rest, float (&g)[8], float (&h)[8]) {       // grad_y * weight and the normalised row
            float ww[8];
            if constexpr (!KEPT) of.weights(a.weight, a.wide_weights, p, ww);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[i] = (t[p].get(i) - mean - rest) * rstd;
                if constexpr (KEPT) g[i] = y[p].get(i) * w[p][i];
                else g[i] = y[p].get(i) * ww[i];
            }
        };
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            float g[8], h[8];
            y[p] = next_y[p];
            t[p] = next_t[p];
            part(p, 0.0f, g, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool counts = of.counts(p, i);
                sum[0] += counts ? g[i] : 0.0f;
                sum[1] += counts ? g[i] * h[i] : 0.0f;
                sum[2] += counts ? t[p].get(i) - mean : 0.0f;
            }
            y[p].keep();
            t[p].keep();
            __builtin_amdgcn_sched_barrier(0);
        }
        if (first + (int64_t)gridDim.x * ROWS < a.rows) fetch(row_of(first + (int64_t)gridDim.x * ROWS));
        if (a.grad_total) more[PARTS - 1].keep();          // (has been read before any lane may write there)
        nm_sum<LANES>(sum, places[turn]);
        const float rest = nm_rest(sum[2], a.width, mean);
        const float c0 = sum[0] / (float)a.width, c1 = fmaf(-rest * rstd, sum[0], sum[1]) / (float)a.width;
        if (!SUMS && a.rests && threadIdx.x == 0) a.rests[row] = rest;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            float g[8], h[8], d[8];
            part(p, rest, g, h);
            if constexpr (SUMS) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool adds = of.counts(p, i) && (ROWS == 1 || mine);
                    gw[p][i] += adds ? y[p].get(i) * h[i] : 0.0f;
                    gb[p][i] += adds ? y[p].get(i) : 0.0f;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = rstd * (g[i] - c0 - h[i] * c1);
            if (a.grad_total) {
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] += more[p].get(i);
            }
            Piece<T> out;
            out.set(d);
            if (mine) of.store(static_cast<T*>(a.grad_sum) + row * a.grad_sum_stride, p, out);
            if (a.drops) {
                if (p == PARTS - 1) nm_drop<true>(a.drop, (uint32_t)row, of.column(p), d);
                else nm_drop<false>(a.drop, (uint32_t)row, of.column(p), d);
                out.set(d);
                if (mine) of.store(static_cast<T*>(a.grad_x) + row * a.grad_x_stride, p, out);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if constexpr (SUMS) {
        // the workgroup's rows together, and its sums to memory
        float* const to_w = a.sums + (int64_t)blockIdx.x * a.width;
        float* const to_b = a.sums + ((int64_t)gridDim.x + blockIdx.x) * a.width;
        if constexpr (ROWS > 1) {
            __shared__ float join[ROWS][LANES * PARTS * 8];
            for (int which = 0; which < 2; ++which) {
                __syncthreads();
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (of.counts(p, i)) join[line][of.column(p) + i] = which ? gb[p][i] : gw[p][i];
                __syncthreads();
                for (int c = threadIdx.x; c < a.width; c += TPB) {
                    float s = 0.0f;
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) s += join[r][c];
                    (which ? to_b : to_w)[c] = s;
                }
            }
        } else {
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (of.counts(p, i)) {
                        to_w[of.column(p) + i] = gw[p][i];
                        to_b[of.column(p) + i] = gb[p][i];
                    }
        }
    }
}

// What rows have beside their means, as rb_norm_grad_kernel makes it (the same sums in the same order), where the next kernel has to come before that one.
template <typename T, int LANES, int PARTS>
__global__ void __launch_bounds__(nm_threads(LANES), 4) rb_norm_rests_kernel(NormGradArgs a)
{
    static_assert(LANES == nm_threads(LANES), "a row a workgroup");
    __shared__ float places[2][48];
    const Row<LANES, PARTS> of(a.width, threadIdx.x);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const float mean = a.mean[row];
        Piece<T> t[PARTS];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) of.load(static_cast<const T*>(a.total) + row * a.total_stride, p, t[p]);
        float sum[1] = {0.0f};
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += of.counts(p, i) ? t[p].get(i) - mean : 0.0f;
        nm_sum<LANES>(sum, places[turn]);
        if (threadIdx.x == 0) a.rests[row] = nm_rest(sum[0], a.width, mean);
    }
}

// The weights' gradients of rows too long for the sums to stay in registers beside them: a workgroup has 2048 columns of some rows.
template <typename T>
__global__ void __launch_bounds__(NM_TPB) rb_norm_columns_kernel(NormGradArgs a)
{
    const int column = (blockIdx.y * NM_TPB + threadIdx.x) * NM_PIECE;
    if (column >= a.width) return;
    const int last = min(column, a.width - NM_PIECE);          // (the row's last piece as Row says)
    float gw[8] = {}, gb[8] = {};
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float mean = a.mean[row], rest = a.rests[row], rstd = a.rstd[row];
        Piece<T> y, t;
        y.load(static_cast<const T*>(a.grad_y) + row * a.grad_y_stride + last);
        t.load(static_cast<const T*>(a.total) + row * a.total_stride + last);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            gw[i] = fmaf(y.get(i), (t.get(i) - mean - rest) * rstd, gw[i]);
            gb[i] += y.get(i);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (last + i >= column) {
            a.sums[(int64_t)blockIdx.x * a.width + last + i] = gw[i];
            a.sums[((int64_t)gridDim.x + blockIdx.x) * a.width + last + i] = gb[i];
        }
}

// The workgroups' sums together: 64 columns of a workgroup, 16 parts of the groups for each, 16 groups on their way at a time (4096 columns of 512 groups 9.5 us
// one by one, 4.5 so: 3.7 TB/s, mostly from the last cache).  Kept with the first kernel's atomics instead, results would depend on the order.
template <typename W>
__global__ void __launch_bounds__(1024) rb_norm_join_kernel(const float* sums, int groups, int width, W* grad_weight, W* grad_bias)
{
    __shared__ float parts[16][64];
    W* const to = blockIdx.y ? grad_bias : grad_weight;
    if (!to) return;
    const int column = blockIdx.x * 64 + (threadIdx.x & 63), part = threadIdx.x / 64;
    float s = 0.0f;
    if (column < width) {
        const float* const from = sums + (int64_t)blockIdx.y * groups * width + column;
        for (int first = part; first < groups; first += 16 * 16) {
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = from[(int64_t)min(first + 16 * i, groups - 1) * width];
#pragma unroll
            for (int i = 0; i < 16; ++i) s += first + 16 * i < groups ? v[i] : 0.0f;
        }
    }
    parts[part][threadIdx.x & 63] = s;
    __syncthreads();
    if (part != 0 || column >= width) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += parts[i][threadIdx.x];
    if constexpr (std::is_same_v<W, float>) to[column] = s;
    else to[column].bits = (uint16_t)sc_bf16_bits(s);
}

}  // namespace
