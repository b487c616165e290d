// Updates orthogonalised by Newton-Schulz products (rb_ortho_apply, rb_ortho_step).  Included by rb_train.hip only.
//
// X = G / (|G| + eps), short side first; per step A = X X^T, B = b A + c A A, X <- a X + B X.  The iteration multiplies a small singular
// value by a (3.4 in the usual coefficients) in every step, and a rounding error in its direction as well: by 140 in four steps.  Operands
// rounded to one 16-bit number would leave errors of per cents; so an operand is kept as the sum of two binary16 numbers (hi + lo, 22
// bits), a product is three matrix instructions (hi hi + hi lo + lo hi; lo lo is below the last bit), and sums are binary32.
//
// Every product is P Q^T of two row-major matrices with the summed index contiguous: X and X^T are both kept, A and B are symmetric, and of
// the symmetric results only the tiles on and above the diagonal are computed, each written to its place and mirrored.
//
// A row of a kept matrix is cut into blocks of 32 elements, hi before lo: 128 bytes, one line of memory.  Matrices are padded with zeros
// to whole tiles, so that products need no bounds.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint32_t ns_vec __attribute__((ext_vector_type(4)));

constexpr int NS_TPB = 256;
constexpr int NS_KBLOCK = 32;                  // elements of a block: hi, then lo
constexpr int NS_KHALVES = 2 * NS_KBLOCK;
constexpr int NS_TILE = 128;                   // rows and columns of a product's tile
constexpr int NS_PARTS = 256;                  // partial sums of a norm per matrix
// What is kept is scaled by powers of two, so that lo is a normal binary16 number for elements of the size that occurs, and a singular
// value of 4 (A: 16, B: 60) is still below 65504.
constexpr float NS_SCALE_X = 4096.0f, NS_SCALE_A = 2048.0f, NS_SCALE_B = 1024.0f;

__device__ __forceinline__ void ns_split(float x, _Float16& hi, _Float16& lo)
{
    hi = (_Float16)x;
    lo = (_Float16)(x - (float)hi);
}
__device__ __forceinline__ int64_t ns_at(int64_t row, int col, int64_t pitch) { return row * pitch + (col >> 5) * NS_KHALVES + (col & 31); }

template <typename T> __device__ __forceinline__ float ns_load(const T* p);
template <> __device__ __forceinline__ float ns_load<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float ns_load<Bf16>(const Bf16* p) { return __uint_as_float((uint32_t)p->bits << 16); }
__device__ __forceinline__ void ns_store(float* p, float x) { *p = x; }
__device__ __forceinline__ void ns_store(Bf16* p, float x) { p->bits = (uint16_t)sc_bf16_bits(x); }

// The update that is orthogonalised: a tensor as it is, or a gradient with its momentum.
struct UpdateArgs {
    const void* grad;
    int64_t matrix_stride, row_stride;      // elements
    float* momentum;                        // null: the gradient itself is the update
    float beta;
    int32_t nesterov;
    int32_t m, n;                           // as the caller has them
    int32_t tall;                           // m > n: the kept matrices are of the transpose
    float eps;
};

// First pass over the update: the squares' partial sums (binary64: no square of a binary32 number overflows or vanishes), and the momentum.
template <typename T>
__global__ __launch_bounds__(NS_TPB) void rb_ortho_norm_kernel(const UpdateArgs a, double* parts)
{
    __shared__ double sums[NS_TPB / 64];
    const int64_t k = blockIdx.y;
    const T* g = static_cast<const T*>(a.grad) + k * a.matrix_stride;
    float* mom = a.momentum != nullptr ? a.momentum + k * a.m * (int64_t)a.n : nullptr;
    double sum = 0.0;
    for (int i = blockIdx.x; i < a.m; i += gridDim.x) {
        for (int j = threadIdx.x; j < a.n; j += NS_TPB) {
            float u = ns_load(g + i * a.row_stride + j);
            if (mom != nullptr) {
                const float v = fmaf(a.beta, mom[(int64_t)i * a.n + j], u);
                mom[(int64_t)i * a.n + j] = v;
                u = a.nesterov ? fmaf(a.beta, v, u) : v;
            }
            sum = fma((double)u, (double)u, sum);
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0) parts[k * NS_PARTS + blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

struct KeptArgs {
    _Float16 *x, *xt;                       // X: rows x 2 cols halves, X^T: cols x 2 rows
    int64_t x_matrix, xt_matrix;            // halves between matrices
    int32_t rows, cols;                     // padded
};

// Second pass: X and X^T, 64 x 64 elements per workgroup.
template <typename T>
__global__ __launch_bounds__(NS_TPB) void rb_ortho_split_kernel(const UpdateArgs a, const KeptArgs q, const double* parts, int32_t nparts)
{
    __shared__ float tile[64][65];
    __shared__ double sums[NS_TPB / 64];
    const int64_t k = blockIdx.z;
    double sum = (int)threadIdx.x < nparts ? parts[k * NS_PARTS + threadIdx.x] : 0.0;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = sum;
    __syncthreads();
    const double norm = sqrt((sums[0] + sums[1]) + (sums[2] + sums[3])) + (double)a.eps;
    const double inverse = norm > 0.0 || norm != norm ? (double)NS_SCALE_X / norm : 0.0;      // a zero update stays zero
    // the tile in the caller's orientation: rows i0.., columns j0..
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, i0 = a.tall ? c0 : r0, j0 = a.tall ? r0 : c0;
    const T* g = static_cast<const T*>(a.grad) + k * a.matrix_stride;
    const float* mom = a.momentum != nullptr ? a.momentum + k * a.m * (int64_t)a.n : nullptr;
    const int tx = threadIdx.x & 63, ty = threadIdx.x / 64;
    for (int y = ty; y < 64; y += NS_TPB / 64) {
        const int i = i0 + y, j = j0 + tx;
        float u = 0.0f;
        if (i < a.m && j < a.n) {
            u = ns_load(g + i * a.row_stride + j);
            if (mom != nullptr) {
                const float v = mom[(int64_t)i * a.n + j];
                u = a.nesterov ? fmaf(a.beta, v, u) : v;
            }
        }
        tile[y][tx] = (float)((double)u * inverse);
    }
    __syncthreads();
    // which of the two kept matrices has its rows along the caller's rows
    _Float16* along = a.tall ? q.xt + k * q.xt_matrix : q.x + k * q.x_matrix;
    _Float16* across = a.tall ? q.x + k * q.x_matrix : q.xt + k * q.xt_matrix;
    const int64_t along_pitch = 2 * (int64_t)(a.tall ? q.rows : q.cols), across_pitch = 2 * (int64_t)(a.tall ? q.cols : q.rows);
    for (int y = ty; y < 64; y += NS_TPB / 64) {
        _Float16 hi, lo;
        ns_split(tile[y][tx], hi, lo);
        int64_t at = ns_at(i0 + y, j0 + tx, along_pitch);
        along[at] = hi;
        along[at + NS_KBLOCK] = lo;
        ns_split(tile[tx][y], hi, lo);
        at = ns_at(j0 + y, i0 + tx, across_pitch);
        across[at] = hi;
        across[at + NS_KBLOCK] = lo;
    }
}

enum { NS_GRAM = 0, NS_POLY = 1, NS_APPLY = 2, NS_LAST = 3 };

struct ProductArgs {
    const _Float16 *p, *q;                  // P: tiles_i * NS_TILE rows, Q: tiles_j * NS_TILE rows, kblocks blocks each
    int64_t p_matrix, q_matrix;             // halves between matrices
    int32_t kblocks, tiles_i, tiles_j;
    const _Float16* old;                    // POLY: A; APPLY, LAST: X^T, of which a * X is added
    int64_t old_matrix, old_pitch;
    _Float16 *out, *out_t;                  // the result and its transpose, as hi and lo
    int64_t out_matrix, out_t_matrix, out_pitch, out_t_pitch;
    float alpha, beta;                      // result = alpha * old + beta * product, in the scales of what is kept
    // LAST: the caller's result
    void* dst;
    int64_t dst_matrix, dst_row;
    int32_t m, n, tall;                     // of the kept X, and whether the caller has its transpose
    int32_t update;                         // dst <- keep * dst - gain * result
    float keep, gain;
};

// C = P Q^T of one tile of 128 x 128; a wavefront has 64 x 64 of it as 2 x 2 blocks of 32 x 32.
template <int KIND, typename OUT>
__global__ __launch_bounds__(NS_TPB, 2) void rb_ortho_product_kernel(const ProductArgs a)
{
    __shared__ __align__(16) char lds[2][2 * NS_TILE * 128];
    const int64_t k = blockIdx.y;
    int ti, tj;
    if (KIND == NS_GRAM || KIND == NS_POLY) {
        // tiles on and above the diagonal, row by row
        int t = blockIdx.x;
        ti = 0;
        while (t >= a.tiles_j - ti) {
            t -= a.tiles_j - ti;
            ++ti;
        }
        tj = ti + t;
    } else {
        ti = blockIdx.x / a.tiles_j;
        tj = blockIdx.x % a.tiles_j;
    }
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const int wi = (wave >> 1) * 64, wj = (wave & 1) * 64;
    const int64_t pitch = (int64_t)a.kblocks * NS_KHALVES;
    const _Float16* p = a.p + k * a.p_matrix + (int64_t)ti * NS_TILE * pitch;
    const _Float16* q = a.q + k * a.q_matrix + (int64_t)tj * NS_TILE * pitch;

    // 2048 pieces of 16 bytes per block of both operands, eight per thread
    const int piece_row = threadIdx.x / 8, piece = threadIdx.x % 8;
    const _Float16* src_p = p + piece_row * pitch + piece * 8;
    const _Float16* src_q = q + piece_row * pitch + piece * 8;
    const int dst = piece_row * 128 + ((piece ^ (piece_row & 7)) * 16);
    ns_vec stage_p[4], stage_q[4];
    auto fetch = [&](int block) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            stage_p[s] = *reinterpret_cast<const ns_vec*>(src_p + block * NS_KHALVES + s * 32 * pitch);
            stage_q[s] = *reinterpret_cast<const ns_vec*>(src_q + block * NS_KHALVES + s * 32 * pitch);
        }
    };
    auto put = [&](int to) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            *reinterpret_cast<ns_vec*>(lds[to] + dst + s * 32 * 128) = stage_p[s];
            *reinterpret_cast<ns_vec*>(lds[to] + NS_TILE * 128 + dst + s * 32 * 128) = stage_q[s];
        }
    };

    float16v acc[2][2] = {};
    fetch(0);
    put(0);
    __syncthreads();
    for (int block = 0; block < a.kblocks; ++block) {
        const bool more = block + 1 < a.kblocks;
        if (more) fetch(block + 1);
        const char* at = lds[block & 1];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            half8 ph[2], pl[2], qh[2], ql[2];
            const int row = lane & 31, c = ks * 2 + lane / 32;
            const int hi = ((c ^ (row & 7)) * 16), lo = (((c + 4) ^ (row & 7)) * 16);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const char* pr = at + (wi + b * 32 + row) * 128;
                const char* qr = at + NS_TILE * 128 + (wj + b * 32 + row) * 128;
                ph[b] = *reinterpret_cast<const half8*>(pr + hi);
                pl[b] = *reinterpret_cast<const half8*>(pr + lo);
                qh[b] = *reinterpret_cast<const half8*>(qr + hi);
                ql[b] = *reinterpret_cast<const half8*>(qr + lo);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl[i], qh[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[i], ql[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[i], qh[j], acc[i][j], 0, 0, 0);
                }
        }
        if (more) put((block + 1) & 1);
        __syncthreads();
    }

    // Block element i of a lane: row 8 (i / 4) + 4 (lane / 32) + i % 4, column lane % 32.
    const bool mirror = (KIND == NS_GRAM || KIND == NS_POLY) ? ti != tj : true;
    const _Float16* old = a.old + k * a.old_matrix;
    _Float16* out = a.out + k * a.out_matrix;
    _Float16* out_t = a.out_t + k * a.out_t_matrix;
#pragma unroll
    for (int bi = 0; bi < 2; ++bi)
#pragma unroll
        for (int bj = 0; bj < 2; ++bj)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int r = ti * NS_TILE + wi + bi * 32 + g * 8 + (lane / 32) * 4, c = tj * NS_TILE + wj + bj * 32 + (lane & 31);
                float v[4];
                half4 hi, lo;
                if (KIND != NS_GRAM) {
                    // what is added lies transposed (A is symmetric): four rows of this column are neighbours there
                    const int64_t o = ns_at(c, r, a.old_pitch);
                    hi = *reinterpret_cast<const half4*>(old + o);
                    lo = *reinterpret_cast<const half4*>(old + o + NS_KBLOCK);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = a.beta * acc[bi][bj][g * 4 + e];
                    if (KIND != NS_GRAM) v[e] = fmaf(a.alpha, (float)hi[e] + (float)lo[e], v[e]);
                }
                if (KIND == NS_LAST) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (r + e >= a.m || c >= a.n) continue;
                        OUT* d = static_cast<OUT*>(a.dst) + k * a.dst_matrix + (a.tall ? c * a.dst_row + r + e : (r + e) * a.dst_row + c);
                        ns_store(d, a.update ? a.keep * ns_load(d) - a.gain * v[e] : v[e]);
                    }
                    continue;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    _Float16 h, l;
                    ns_split(v[e], h, l);
                    hi[e] = h;
                    lo[e] = l;
                    const int64_t o = ns_at(r + e, c, a.out_pitch);
                    out[o] = h;
                    out[o + NS_KBLOCK] = l;
                }
                if (mirror) {
                    const int64_t o = ns_at(c, r, a.out_t_pitch);
                    *reinterpret_cast<half4*>(out_t + o) = hi;
                    *reinterpret_cast<half4*>(out_t + o + NS_KBLOCK) = lo;
                }
            }
}

}  // namespace
