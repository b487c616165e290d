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

// Pieces of a row at any alignment (the hardware's 16-byte accesses take any address); the last one of a row may be shorter.
template <typename T> __device__ __forceinline__ void nm_load(const T* p, int there, float (&v)[8]);
template <> __device__ __forceinline__ void nm_load<float>(const float* p, int there, float (&v)[8])
{
    if (there >= 8) {
        memcpy(v, p, 32);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < there ? p[i] : 0.0f;
}
template <> __device__ __forceinline__ void nm_load<Bf16>(const Bf16* p, int there, float (&v)[8])
{
    if (there >= 8) {
        sc_vec w;
        memcpy(&w, p, 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < there ? __uint_as_float((uint32_t)p[i].bits << 16) : 0.0f;
}

__device__ __forceinline__ void nm_store(float* p, int there, const float (&v)[8])
{
    if (there >= 8) {
        memcpy(p, v, 32);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < there) p[i] = v[i];
}
__device__ __forceinline__ void nm_store(Bf16* p, int there, const float (&v)[8])
{
    if (there >= 8) {
        sc_vec w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = sc_bf16_pair(v[2 * i], v[2 * i + 1]);
        memcpy(p, &w, 16);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < there) p[i].bits = (uint16_t)sc_bf16_bits(v[i]);
}

template <typename T> __device__ __forceinline__ float nm_round(float x)
{
    if constexpr (std::is_same_v<T, float>) return x;
    else return __uint_as_float(sc_bf16_bits(x) << 16);
}

// Weights are binary32 or bfloat16, as the handle says (the same for all lanes).
__device__ __forceinline__ void nm_weights(const void* w, bool wide, int column, int there, float (&v)[8])
{
    if (wide) nm_load(static_cast<const float*>(w) + column, there, v);
    else nm_load(static_cast<const Bf16*>(w) + column, there, v);
}

// ---- dropout -------------------------------------------------------------------

struct Drop {
    uint32_t seed_lo, seed_hi, step_lo, step_hi;
    uint32_t least;            // what 16 bits have to be to stay: 0 (all stay) .. 65536 (none does)
    float scale;
};

// Which of the eight elements of a piece stay: Philox4x32-10 (Salmon et al., SC'11) of the row and the piece, 16 bits an element.
__device__ __forceinline__ void nm_drop(const Drop& d, uint32_t row, uint32_t piece, float (&v)[8])
{
    if (d.least == 0) return;
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
    const uint32_t x[4] = {x0, x1, x2, x3};
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
        const int piece = (int)(item - line * a.blocks) * NM_TPB + p;
        if (row >= a.rows || piece >= a.pieces) continue;
        const int there = a.width - piece * NM_PIECE;
        float v[8];
        nm_load(static_cast<const T*>(a.x) + row * a.x_stride + piece * NM_PIECE, there, v);
        nm_drop(a.drop, (uint32_t)row, (uint32_t)piece, v);
        nm_store(static_cast<T*>(a.out) + row * a.out_stride + piece * NM_PIECE, there, v);
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
        if (LANES >= 64) {
            v[i] += sc_xor<16>(v[i]);
            v[i] += sc_xor<32>(v[i]);
        }
    }
    if (LANES > 64) {
        constexpr int WAVES = LANES / 64;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) places[threadIdx.x / 64 * N + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v[i] += places[w * N + i];
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

template <typename T, int LANES, int PARTS>
__global__ void __launch_bounds__(LANES > NM_TPB ? LANES : NM_TPB) rb_norm_kernel(NormArgs a)
{
    constexpr int TPB = LANES > NM_TPB ? LANES : NM_TPB, ROWS = TPB / LANES;
    constexpr bool KEPT = PARTS <= 4 && LANES <= NM_TPB;       // weights stay in registers between rows
    __shared__ float places[2][2][32];
    const int lane = threadIdx.x % LANES;
    float w[KEPT ? PARTS : 1][8], b[KEPT ? PARTS : 1][8];
    if constexpr (KEPT) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const int piece = p * LANES + lane, there = a.width - piece * NM_PIECE;
            nm_weights(a.weight, a.wide_weights, piece * NM_PIECE, there, w[p]);
            if (a.bias) nm_weights(a.bias, a.wide_weights, piece * NM_PIECE, there, b[p]);
            else
                for (int i = 0; i < 8; ++i) b[p][i] = 0.0f;
        }
    }
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const int64_t row = min(first + threadIdx.x / LANES, (int64_t)a.rows - 1);       // (of the last rows some are made twice, alike)
        const bool mine = first + threadIdx.x / LANES < a.rows;
        float v[PARTS][8];
        float sum[1] = {0.0f};
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const int piece = p * LANES + lane, there = a.width - piece * NM_PIECE;
            nm_load(static_cast<const T*>(a.x) + row * a.x_stride + piece * NM_PIECE, there, v[p]);
        }
        if (a.total) {
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                const int piece = p * LANES + lane, there = a.width - piece * NM_PIECE;
                if (a.drops) nm_drop(a.drop, (uint32_t)row, (uint32_t)piece, v[p]);
                if (a.residual) {
                    float r[8];
                    nm_load(static_cast<const T*>(a.residual) + row * a.residual_stride + piece * NM_PIECE, there, r);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[p][i] += r[i];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) v[p][i] = nm_round<T>(v[p][i]);
                if (mine) nm_store(static_cast<T*>(a.total) + row * a.total_stride + piece * NM_PIECE, there, v[p]);
            }
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += v[p][i];
        nm_sum<LANES>(sum, places[turn][0]);
        const float width = (float)a.width;
        float mean = sum[0] / width;
        float off[2] = {0.0f, 0.0f};               // sums of the differences and of their squares
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const int there = a.width - (p * LANES + lane) * NM_PIECE;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = i < there ? v[p][i] - mean : 0.0f;
                v[p][i] = d;
                off[0] += d;
                off[1] = fmaf(d, d, off[1]);
            }
        }
        nm_sum<LANES>(off, places[turn][1]);
        const float more = off[0] / width;
        const float rstd = 1.0f / sqrtf(fmaxf(fmaf(-more, more, off[1] / width), 0.0f) + a.eps);
        mean += more;
        if (mine && lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = off[1] != off[1] ? off[1] : rstd;
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const int piece = p * LANES + lane, there = a.width - piece * NM_PIECE;
            float out[8], ww[8], bb[8];
            if constexpr (!KEPT) {
                nm_weights(a.weight, a.wide_weights, piece * NM_PIECE, there, ww);
                if (a.bias) nm_weights(a.bias, a.wide_weights, piece * NM_PIECE, there, bb);
                else
                    for (int i = 0; i < 8; ++i) bb[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float h = (v[p][i] - more) * rstd;
                if constexpr (KEPT) out[i] = fmaf(h, w[p][i], b[p][i]);
                else out[i] = fmaf(h, ww[i], bb[i]);
            }
            if (mine) nm_store(static_cast<T*>(a.y) + row * a.y_stride + piece * NM_PIECE, there, out);
        }
    }
}

// ---- gradients -----------------------------------------------------------------

struct NormGradArgs {
    const void *grad_y, *total, *grad_total, *weight;
    const float *mean, *rstd;
    void *grad_sum, *grad_x;
    float* sums;                       // [2][groups][width]: of the weight's and of the bias's gradient; null: none is wanted
    int64_t grad_y_stride, total_stride, grad_total_stride, grad_sum_stride, grad_x_stride;
    int32_t rows, width;
    bool wide_weights, drops;
    Drop drop;
};

// SUMS: the weights' gradients are summed on the way.
template <typename T, int LANES, int PARTS, bool SUMS>
__global__ void __launch_bounds__(LANES > NM_TPB ? LANES : NM_TPB) rb_norm_grad_kernel(NormGradArgs a)
{
    constexpr int TPB = LANES > NM_TPB ? LANES : NM_TPB, ROWS = TPB / LANES;
    constexpr bool KEPT = PARTS <= 4 && LANES <= NM_TPB;
    __shared__ float places[2][32];
    const int lane = threadIdx.x % LANES;
    float w[KEPT ? PARTS : 1][8];
    float gw[SUMS ? PARTS : 1][8], gb[SUMS ? PARTS : 1][8];
    if constexpr (KEPT) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) nm_weights(a.weight, a.wide_weights, (p * LANES + lane) * NM_PIECE, a.width - (p * LANES + lane) * NM_PIECE, w[p]);
    }
    if constexpr (SUMS) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) gw[p][i] = gb[p][i] = 0.0f;
    }
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const int64_t row = min(first + threadIdx.x / LANES, (int64_t)a.rows - 1);
        const bool mine = first + threadIdx.x / LANES < a.rows;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float g[PARTS][8], h[PARTS][8];
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const int piece = p * LANES + lane, there = a.width - piece * NM_PIECE;
            nm_load(static_cast<const T*>(a.grad_y) + row * a.grad_y_stride + piece * NM_PIECE, there, g[p]);
            nm_load(static_cast<const T*>(a.total) + row * a.total_stride + piece * NM_PIECE, there, h[p]);
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const int piece = p * LANES + lane, there = a.width - piece * NM_PIECE;
            float ww[8];
            if constexpr (!KEPT) nm_weights(a.weight, a.wide_weights, piece * NM_PIECE, there, ww);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[p][i] = i < there ? (h[p][i] - mean) * rstd : 0.0f;
                if constexpr (SUMS) {
                    if (mine) {
                        gw[p][i] = fmaf(g[p][i], h[p][i], gw[p][i]);
                        gb[p][i] += g[p][i];
                    }
                }
                if constexpr (KEPT) g[p][i] *= w[p][i];
                else g[p][i] *= ww[i];
                sum[0] += g[p][i];
                sum[1] = fmaf(g[p][i], h[p][i], sum[1]);
            }
        }
        nm_sum<LANES>(sum, places[turn]);
        const float c0 = sum[0] / (float)a.width, c1 = sum[1] / (float)a.width;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const int piece = p * LANES + lane, there = a.width - piece * NM_PIECE;
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = rstd * (g[p][i] - c0 - h[p][i] * c1);
            if (a.grad_total) {
                float r[8];
                nm_load(static_cast<const T*>(a.grad_total) + row * a.grad_total_stride + piece * NM_PIECE, there, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] += r[i];
            }
            if (mine) nm_store(static_cast<T*>(a.grad_sum) + row * a.grad_sum_stride + piece * NM_PIECE, there, d);
            if (a.drops) {
                nm_drop(a.drop, (uint32_t)row, (uint32_t)piece, d);
                if (mine) nm_store(static_cast<T*>(a.grad_x) + row * a.grad_x_stride + piece * NM_PIECE, there, d);
            }
        }
    }
    if constexpr (SUMS) {
        // the workgroup's rows together, and its sums to memory
        if constexpr (ROWS > 1) {
            __shared__ float join[ROWS][LANES * PARTS * 8];
            for (int which = 0; which < 2; ++which) {
                __syncthreads();
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int i = 0; i < 8; ++i) join[threadIdx.x / LANES][(p * LANES + lane) * 8 + i] = which ? gb[p][i] : gw[p][i];
                __syncthreads();
                for (int c = threadIdx.x; c < a.width; c += TPB) {
                    float s = 0.0f;
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) s += join[r][c];
                    a.sums[((int64_t)which * gridDim.x + blockIdx.x) * a.width + c] = s;
                }
            }
        } else {
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                const int column = (p * LANES + lane) * NM_PIECE, there = a.width - column;
                nm_store(a.sums + (int64_t)blockIdx.x * a.width + column, there, gw[p]);
                nm_store(a.sums + ((int64_t)gridDim.x + blockIdx.x) * a.width + column, there, gb[p]);
            }
        }
    }
}

// The weights' gradients of rows too long for the sums to stay in registers beside them: a workgroup has 2048 columns of some rows.
template <typename T>
__global__ void __launch_bounds__(NM_TPB) rb_norm_columns_kernel(NormGradArgs a)
{
    const int column = (blockIdx.y * NM_TPB + threadIdx.x) * NM_PIECE, there = a.width - column;
    if (there <= 0) return;
    float gw[8] = {}, gb[8] = {};
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float g[8], h[8];
        nm_load(static_cast<const T*>(a.grad_y) + row * a.grad_y_stride + column, there, g);
        nm_load(static_cast<const T*>(a.total) + row * a.total_stride + column, there, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            gw[i] = fmaf(g[i], (h[i] - mean) * rstd, gw[i]);
            gb[i] += g[i];
        }
    }
    nm_store(a.sums + (int64_t)blockIdx.x * a.width + column, there, gw);
    nm_store(a.sums + ((int64_t)gridDim.x + blockIdx.x) * a.width + column, there, gb);
}

// The workgroups' sums together: 64 columns of a workgroup, 16 parts of the groups for each.
template <typename W>
__global__ void __launch_bounds__(1024) rb_norm_join_kernel(const float* sums, int groups, int width, W* grad_weight, W* grad_bias)
{
    __shared__ float parts[16][64];
    W* const to = blockIdx.y ? grad_bias : grad_weight;
    if (!to) return;
    const int column = blockIdx.x * 64 + (threadIdx.x & 63), part = threadIdx.x / 64;
    float s = 0.0f;
    if (column < width)
        for (int g = part; g < groups; g += 16) s += sums[((int64_t)blockIdx.y * groups + g) * width + column];
    parts[part][threadIdx.x & 63] = s;
    __syncthreads();
    if (part != 0 || column >= width) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += parts[i][threadIdx.x];
    if constexpr (std::is_same_v<W, float>) to[column] = s;
    else to[column].bits = (uint16_t)sc_bf16_bits(s);
}

}  // namespace
