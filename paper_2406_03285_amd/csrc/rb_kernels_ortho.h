// Updates orthogonalised by Newton-Schulz products (rb_ortho_apply, rb_ortho_step).  Included by rb_train.hip only.
//
// X = G / (|G| + eps), short side first; per step A = X X^T, B = b A + c A A, X <- a X + B X.  The iteration multiplies a small singular
// value by a (3.4 in the usual coefficients) in every step, and a rounding error in its direction as well: by 140 in four steps.  Operands
// rounded to one 16-bit number would leave errors of per cents; so an operand is kept as the sum of two binary16 numbers (hi + lo: 22
// bits, as far as binary16's range goes), a product is three matrix instructions (hi hi + hi lo + lo hi; lo lo is below the last bit), and sums are binary32.
//
// Where one side is much the longer one, most of the work is in the two products with X.  Then steps are made in pairs on A alone: a step
// multiplies X from the left by P = a I + b A + c A A, and A, a polynomial of the same symmetric matrix, by P twice; R, the product of the
// pair's P, is applied to X at its end.  That is 5 symmetric products of the short side for two steps instead of 2, one more A and one more B X.
// Three steps at a time would let A's rounding errors grow once more by a^2, which they do where a few directions are much stronger than the
// rest (errors of 3 to 20 times those of the plain form in binary32 were measured); in pairs they stay within 1.7 times, and from 200 rows on at or
// below the plain form's.
//
// Every product is P Q^T of two row-major matrices with the summed index contiguous: X and X^T are both kept, A and B are symmetric, and of
// the symmetric results only the tiles on and above the diagonal are computed, each written to its place and mirrored.
//
// A row of a kept matrix is cut into blocks of 32 elements, hi before lo: 128 bytes, one line of memory.  The matrices have room for whole
// tiles, so that products need no bounds: what lies beyond the last row and column up to a multiple of 32 is zero (it starts so, and the
// products keep it so); what lies beyond that is whatever it is, enters no sum and is in no result.
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
constexpr int NS_ROWS_AT_ONCE = 4;             // rows a thread of the first pass has on their way
constexpr int NS_PARTS = 1024;                 // most partial sums of a norm per matrix
// What is kept is scaled by powers of two so that a singular value of 4 (A: 16, B: 60) is still below 65504.  lo is a normal binary16 number, and the sum
// has its 22 bits, for elements of X from 2^-14 on (of 4096 x 4096 a typical one is 2^-12); below, it goes in steps of 2^-24 over the scale.
constexpr float NS_SCALE_X = 4096.0f, NS_SCALE_A = 2048.0f, NS_SCALE_B = 1024.0f;

template <typename H, int N>      // of N neighbours, a vector of N binary16 numbers each (conversions go in pairs)
__device__ __forceinline__ void ns_split(const float* x, H& hi, H& lo)
{
    typedef float floats __attribute__((ext_vector_type(N)));
    floats v, rest;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = x[i];
    hi = __builtin_convertvector(v, H);
#pragma unroll
    for (int i = 0; i < N; ++i) rest[i] = v[i] - (float)hi[i];
    lo = __builtin_convertvector(rest, H);
}
__device__ __forceinline__ int64_t ns_at(int64_t row, int col, int64_t pitch) { return row * pitch + (col >> 5) * NS_KHALVES + (col & 31); }

// What an update is multiplied by; a zero update stays zero.
__device__ __forceinline__ double ns_inverse(double norm) { return norm == 0.0 ? 0.0 : (double)NS_SCALE_X / norm; }

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

// V neighbours of a row, V = 4 where all rows of all tensors are whole and aligned vectors, else 1.
template <typename T, int V> struct Run;
template <typename T> struct Run<T, 1> {
    static __device__ __forceinline__ void load(const T* p, float* x) { x[0] = ns_load(p); }
    static __device__ __forceinline__ void store(T* p, const float* x) { ns_store(p, x[0]); }
};
template <> struct Run<float, 4> {
    static __device__ __forceinline__ void load(const float* p, float* x)
    {
        const float4 v = *reinterpret_cast<const float4*>(p);
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    }
    static __device__ __forceinline__ void store(float* p, const float* x) { *reinterpret_cast<float4*>(p) = float4{x[0], x[1], x[2], x[3]}; }
};
template <> struct Run<Bf16, 4> {
    static __device__ __forceinline__ void load(const Bf16* p, float* x)
    {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
    }
};

// First pass over the update: the squares' partial sums (binary64: no square of a binary32 number overflows or vanishes), and the momentum.
// A thread has V neighbours of a row; some rows are on their way at once.
template <typename T, int V>
__global__ __launch_bounds__(NS_TPB) void rb_ortho_norm_kernel(const UpdateArgs a, double* parts)
{
    constexpr int AT_ONCE = NS_ROWS_AT_ONCE;
    __shared__ double sums[NS_TPB / 64];
    const int64_t k = blockIdx.y;
    const T* g = static_cast<const T*>(a.grad) + k * a.matrix_stride;
    float* mom = a.momentum != nullptr ? a.momentum + k * a.m * (int64_t)a.n : nullptr;
    double sum = 0.0;
    // the matrix in pieces of AT_ONCE rows by V NS_TPB columns
    const int spans = (a.n + V * NS_TPB - 1) / (V * NS_TPB);
    const int items = (a.m + AT_ONCE - 1) / AT_ONCE * spans;             // (at most 2^14 * 2^8)
    for (int it = blockIdx.x; it < items; it += gridDim.x) {
        const int i0 = (int)((uint32_t)it / (uint32_t)spans) * AT_ONCE, j = ((int)((uint32_t)it % (uint32_t)spans) * NS_TPB + threadIdx.x) * V;
        if (j >= a.n) continue;
        float u[AT_ONCE][V] = {};
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e)
            if (i0 + e < a.m) Run<T, V>::load(g + (i0 + e) * a.row_stride + j, u[e]);
        if (mom != nullptr) {
            float v[AT_ONCE][V] = {};
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e)
                if (i0 + e < a.m) Run<float, V>::load(mom + (int64_t)(i0 + e) * a.n + j, v[e]);
#pragma unroll
            for (int e = 0; e < AT_ONCE; ++e) {
#pragma unroll
                for (int x = 0; x < V; ++x) v[e][x] = fmaf(a.beta, v[e][x], u[e][x]);
                if (i0 + e < a.m) Run<float, V>::store(mom + (int64_t)(i0 + e) * a.n + j, v[e]);
#pragma unroll
                for (int x = 0; x < V; ++x) u[e][x] = a.nesterov ? fmaf(a.beta, v[e][x], u[e][x]) : v[e][x];
            }
        }
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e)
#pragma unroll
            for (int x = 0; x < V; ++x) sum = fma((double)u[e][x], (double)u[e][x], sum);
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
    int64_t x_pitch, xt_pitch;              // halves between rows
    int32_t rows, cols;                     // padded
};

// Halves between the rows of a kept matrix of so many columns: an odd number of lines, so that a tile's lines of one block do not all
// begin at multiples of one power of two.
__host__ __device__ inline int64_t ns_pitch(int64_t cols) { return (cols / NS_KBLOCK | 1) * NS_KHALVES; }

// Second pass: X and X^T, 64 x 64 elements per workgroup, 8 neighbours of a row per thread and store.
template <typename T, int V>
__global__ __launch_bounds__(NS_TPB) void rb_ortho_split_kernel(const UpdateArgs a, const KeptArgs q, const double* parts, int32_t nparts)
{
    constexpr int ACROSS = 64 / V, ROWS = NS_TPB / ACROSS, ITEMS = 64 / ROWS;      // threads of a row, rows at a time, how often
    __shared__ float tile[64][65];
    __shared__ double sums[NS_TPB / 64];
    const int64_t k = blockIdx.z;
    // the tile in the caller's orientation: rows i0.., columns j0..
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, i0 = a.tall ? c0 : r0, j0 = a.tall ? r0 : c0;
    const T* g = static_cast<const T*>(a.grad) + k * a.matrix_stride;
    const float* mom = a.momentum != nullptr ? a.momentum + k * a.m * (int64_t)a.n : nullptr;
    const int tx = threadIdx.x % ACROSS * V, ty = threadIdx.x / ACROSS;
    float u[ITEMS][V] = {};
#pragma unroll
    for (int e = 0; e < ITEMS; ++e)
        if (i0 + ty + e * ROWS < a.m && j0 + tx < a.n) Run<T, V>::load(g + (i0 + ty + e * ROWS) * a.row_stride + j0 + tx, u[e]);
    if (mom != nullptr) {
        float v[ITEMS][V] = {};
#pragma unroll
        for (int e = 0; e < ITEMS; ++e)
            if (i0 + ty + e * ROWS < a.m && j0 + tx < a.n) Run<float, V>::load(mom + (int64_t)(i0 + ty + e * ROWS) * a.n + j0 + tx, v[e]);
#pragma unroll
        for (int e = 0; e < ITEMS; ++e)
#pragma unroll
            for (int x = 0; x < V; ++x) u[e][x] = a.nesterov ? fmaf(a.beta, v[e][x], u[e][x]) : v[e][x];
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < NS_PARTS / NS_TPB; ++i)
        if ((int)threadIdx.x + i * NS_TPB < nparts) sum += parts[k * NS_PARTS + threadIdx.x + i * NS_TPB];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = sum;
    __syncthreads();
    const double inverse = ns_inverse(sqrt((sums[0] + sums[1]) + (sums[2] + sums[3])) + (double)a.eps);
#pragma unroll
    for (int e = 0; e < ITEMS; ++e)
#pragma unroll
        for (int x = 0; x < V; ++x) tile[ty + e * ROWS][tx + x] = (float)((double)u[e][x] * inverse);
    __syncthreads();
    // which of the two kept matrices has its rows along the caller's rows
    _Float16* along = a.tall ? q.xt + k * q.xt_matrix : q.x + k * q.x_matrix;
    _Float16* across = a.tall ? q.x + k * q.x_matrix : q.xt + k * q.xt_matrix;
    const int64_t along_pitch = a.tall ? q.xt_pitch : q.x_pitch, across_pitch = a.tall ? q.x_pitch : q.xt_pitch;
    const int row = threadIdx.x / 4, first = threadIdx.x % 4 * 8;
#pragma unroll
    for (int b = 0; b < 64; b += NS_KBLOCK) {
        half8 hi, lo;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[row][b + first + e];
        ns_split<half8, 8>(v, hi, lo);
        _Float16* to = along + ns_at(i0 + row, j0 + b + first, along_pitch);
        *reinterpret_cast<half8*>(to) = hi;
        *reinterpret_cast<half8*>(to + NS_KBLOCK) = lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[b + first + e][row];
        ns_split<half8, 8>(v, hi, lo);
        to = across + ns_at(j0 + row, i0 + b + first, across_pitch);
        *reinterpret_cast<half8*>(to) = hi;
        *reinterpret_cast<half8*>(to + NS_KBLOCK) = lo;
    }
}

// Where the result goes.
struct ResultArgs {
    void* dst;
    int64_t matrix_stride, row_stride;      // elements
    int32_t rows, cols, tall;               // of the kept X, and whether the caller has its transpose
    int32_t update;                         // dst <- keep * dst - gain * result
    float keep, gain;
};

// 16 numbers of a lane to their places: all that is read of them first (an update), then all that is written.  They are `stride` apart, number i
// step(i) of these from `at`, where there are `count`.
struct StepRows { static constexpr int of(int i) { return (i / 4) * 8 + i % 4; } };      // the rows of a lane's elements
struct StepPairs { static constexpr int of(int i) { return 2 * i; } };
template <typename STEP, typename OUT>
__device__ __forceinline__ void ns_result(const ResultArgs& a, OUT* at, int64_t stride, int count, float* v)
{
    if (a.update) {
        float w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = STEP::of(i) < count ? ns_load(at + STEP::of(i) * stride) : 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = a.keep * w[i] - a.gain * v[i];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (STEP::of(i) < count) ns_store(at + STEP::of(i) * stride, v[i]);
}

enum { NS_GRAM = 0, NS_POLY = 1, NS_APPLY = 2, NS_LAST = 3 };

// What the first instructions of a product need: as arguments in front of the structure it is in registers when a wavefront starts.
struct Operands {
    const _Float16 *p, *q;                  // P: tiles_i tiles of rows, Q: tiles_j
    int32_t p_lines, q_lines;               // lines of 128 bytes between rows
    uint32_t p_matrix, q_matrix;            // lines between matrices
    int32_t kblocks;                        // of the summed index
};

struct ProductArgs {
    int32_t tiles_i, tiles_j;
    int32_t tiles, slices;                  // of one matrix; of the summed index
    float* sums;                            // of the slices, if there are several
    const _Float16* old;                    // POLY: A; APPLY, LAST: X^T, of which a * X is added (null: nothing is)
    int64_t old_matrix, old_pitch;
    _Float16 *out, *out_t;                  // the result and its transpose, as hi and lo
    int64_t out_matrix, out_t_matrix, out_pitch, out_t_pitch;
    float alpha, beta;                      // result = alpha * old + beta * product, in the scales of what is kept,
    float diagonal;                         // and, POLY, this much on the diagonal
    ResultArgs result;                      // LAST
};

// Asynchronous loads into LDS.  The wavefront's 64 lanes bring 16 bytes each, which land behind each other from `to` on.
__device__ __forceinline__ void ns_load_to_lds(const char* from, char* to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
// Waits until at most COUNT of them are on their way and everything read from LDS is there, then for the workgroup's other wavefronts.
template <int COUNT>
__device__ __forceinline__ void ns_arrived()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(COUNT) : "memory");
}

// Which tile a workgroup has.  Workgroups go to the 8 dies in turn, and each die has its own L2: a die gets tiles that are neighbours, in groups
// of 8 tile rows walked column by column, so that the panels it reads at a time are few.
__device__ __forceinline__ int ns_rank(int id, int count)
{
    const int die = id & 7, whole = count >> 3, more = count & 7;
    return die * whole + min(die, more) + (id >> 3);
}
constexpr int NS_GROUP = 8;
__device__ __forceinline__ void ns_in_group(int t, int height, int& row, int& col)          // (divisions take long where little else is to be done)
{
    if (height == NS_GROUP) {
        row = t % NS_GROUP;
        col = t / NS_GROUP;
    } else {
        col = (int)((uint32_t)t / (uint32_t)height);
        row = t - col * height;
    }
}
__device__ __forceinline__ void ns_tile_of(int t, int rows, int cols, int& ti, int& tj)
{
    const int g = rows <= NS_GROUP ? 0 : (int)((uint32_t)t / (uint32_t)(NS_GROUP * cols)), first = g * NS_GROUP;
    ns_in_group(t - first * cols, min(NS_GROUP, rows - first), ti, tj);
    ti += first;
}
__device__ __forceinline__ void ns_tile_above(int t, int rows, int& ti, int& tj)          // on and above the diagonal only
{
    for (int first = 0;; first += NS_GROUP) {
        const int height = min(NS_GROUP, rows - first), corner = height * (height + 1) / 2, count = corner + (rows - first - height) * height;
        if (t < count) {
            int col = 0;
            if (t < corner) {
                while (t > col) t -= ++col;
                ti = first + t;
            } else {
                ns_in_group(t - corner, height, ti, col);
                ti += first;
                col += height;
            }
            tj = first + col;
            return;
        }
        t -= count;
    }
}
// Matrix, tile and slice of the `rank`-th workgroup.
__device__ __forceinline__ void ns_share(int rank, int tiles, int slices, int& tile, int& slice, int& k)
{
    tile = rank;
    slice = k = 0;
    if (slices > 1) {
        tile = (int)((uint32_t)rank / (uint32_t)slices);
        slice = rank - tile * slices;
    }
    if (tile >= tiles) k = (int)((uint32_t)tile / (uint32_t)tiles);
}

// ---- a block of 32 x 32 of a result -------------------------------------------
//
// Element i of a lane: row 8 (i / 4) + 4 (lane / 32) + i % 4, column lane % 32.  The block is 32 lines of 128 bytes of the kept matrix, and 32 of its
// transpose: they are put together in LDS (each wavefront has a place of its own, lines 144 bytes apart) and moved 16 bytes a lane.
constexpr int NS_PLACE_PITCH = 144, NS_PLACE = 32 * NS_PLACE_PITCH;

// What is added to the product lies transposed (A is symmetric): the four rows of a lane's column are neighbours there.
__device__ __forceinline__ void ns_fetch_old(const ProductArgs& a, int64_t k, int r0, int c0, ns_vec* old)
{
    const int lane = threadIdx.x & 63, line = lane >> 3, part = (lane & 7) * 16;
    const _Float16* from = a.old + k * a.old_matrix;
    if (a.old == nullptr) {
#pragma unroll
        for (int l = 0; l < 4; ++l) old[l] = ns_vec{0, 0, 0, 0};
        return;
    }
#pragma unroll
    for (int l = 0; l < 4; ++l)
        old[l] = *reinterpret_cast<const ns_vec*>(reinterpret_cast<const char*>(from + ns_at(c0 + l * 8 + line, r0, a.old_pitch)) + part);
}

template <int KIND, typename OUT>
__device__ __forceinline__ void ns_finish(const ProductArgs& a, int64_t k, int r0, int c0, const float16v& acc, const ns_vec* old, bool mirror, char* mine)
{
    const int lane = threadIdx.x & 63, half = lane / 32, col = lane & 31, line = lane >> 3, part = (lane & 7) * 16;
    float v[16];
    if (KIND != NS_GRAM) {
#pragma unroll
        for (int l = 0; l < 4; ++l) *reinterpret_cast<ns_vec*>(mine + (l * 8 + line) * NS_PLACE_PITCH + part) = old[l];
        sc_lds_wait();
    }
    half4 hi[4], lo[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        char* const at = mine + col * NS_PLACE_PITCH + (g * 8 + half * 4) * 2;
        if (KIND != NS_GRAM) {
            hi[g] = *reinterpret_cast<const half4*>(at);
            lo[g] = *reinterpret_cast<const half4*>(at + 64);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[g * 4 + e] = a.beta * acc[g * 4 + e];
            if (KIND != NS_GRAM) v[g * 4 + e] = fmaf(a.alpha, (float)hi[g][e] + (float)lo[g][e], v[g * 4 + e]);
        }
    }
    if (KIND == NS_POLY && r0 == c0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] += (i / 4) * 8 + half * 4 + i % 4 == col ? a.diagonal : 0.0f;
    }
    if (KIND == NS_LAST) {
        // 32 numbers of a row of what the caller has, by half a wavefront
        OUT* const dst = static_cast<OUT*>(a.result.dst) + k * a.result.matrix_stride;
        if (!a.result.tall) {
            const int r = r0 + half * 4, c = c0 + col;
            ns_result<StepRows>(a.result, dst + r * a.result.row_stride + c, a.result.row_stride, c < a.result.cols ? a.result.rows - r : 0, v);
        } else {
            sc_lds_wait();
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4*>(mine + col * NS_PLACE_PITCH + (g * 8 + half * 4) * 4) = float4{v[g * 4], v[g * 4 + 1], v[g * 4 + 2], v[g * 4 + 3]};
            sc_lds_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = *reinterpret_cast<const float*>(mine + (2 * i + half) * NS_PLACE_PITCH + col * 4);
            const int r = r0 + col, c = c0 + half;
            ns_result<StepPairs>(a.result, dst + c * a.result.row_stride + r, a.result.row_stride, r < a.result.rows ? a.result.cols - c : 0, v);
        }
        sc_lds_wait();
        return;
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) ns_split<half4, 4>(v + g * 4, hi[g], lo[g]);
    if (mirror) {
        char* to = reinterpret_cast<char*>(a.out_t + k * a.out_t_matrix + ns_at(c0 + line, r0, a.out_t_pitch)) + part;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            *reinterpret_cast<half4*>(mine + col * NS_PLACE_PITCH + (g * 8 + half * 4) * 2) = hi[g];
            *reinterpret_cast<half4*>(mine + col * NS_PLACE_PITCH + (g * 8 + half * 4) * 2 + 64) = lo[g];
        }
        sc_lds_wait();
#pragma unroll
        for (int l = 0; l < 4; ++l) *reinterpret_cast<ns_vec*>(to + l * 8 * a.out_t_pitch * 2) = *reinterpret_cast<const ns_vec*>(mine + (l * 8 + line) * NS_PLACE_PITCH + part);
        sc_lds_wait();
    }
    char* to = reinterpret_cast<char*>(a.out + k * a.out_matrix + ns_at(r0 + line, c0, a.out_pitch)) + part;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        _Float16* at = reinterpret_cast<_Float16*>(mine + ((i / 4) * 8 + half * 4 + i % 4) * NS_PLACE_PITCH) + col;
        at[0] = hi[i / 4][i % 4];
        at[NS_KBLOCK] = lo[i / 4][i % 4];
    }
    sc_lds_wait();
#pragma unroll
    for (int l = 0; l < 4; ++l) *reinterpret_cast<ns_vec*>(to + l * 8 * a.out_pitch * 2) = *reinterpret_cast<const ns_vec*>(mine + (l * 8 + line) * NS_PLACE_PITCH + part);
    sc_lds_wait();
}

// Block b of 32 x 32 of a tile, tile t of slice s: 1024 sums, 16 of a lane as 4 times 4.
__device__ __forceinline__ float4* ns_sums(const ProductArgs& a, int64_t tile, int slice, int blocks, int b)
{
    return reinterpret_cast<float4*>(a.sums) + ((tile * a.slices + slice) * blocks + b) * 256 + (threadIdx.x & 63);
}

// C = P Q^T of one tile of BM x BM; a wavefront has WM x WN of it in blocks of 32 x 32.  A block of 32 of the summed index is 2 BM lines of 128
// bytes; STAGES of them are in LDS or on their way there.  Where the tiles are few the summed index is cut into slices, a workgroup each.
// Large products run the matrix instructions at what power leaves of the clock: 4096 x 4096 348 us (1.19 PFLOP/s of binary16) by tiles of 256, which
// need the least of L2 and LDS; A of it 215 us by 253 tiles of 192, one per compute unit.  Small ones (1024 x 1024: 11 to 14 us by tiles of 64) are
// bound by a launch's start and end (5 us) and by loads and matrix instructions that one wavefront per SIMD hardly overlaps.
template <int KIND, typename OUT, int BM, int WM, int WN, int STAGES, int WAVES_PER_SIMD>
__global__ __launch_bounds__((BM / WM) * (BM / WN) * 64, WAVES_PER_SIMD) void rb_ortho_product_kernel(
    const _Float16* of_p, const _Float16* of_q, int32_t p_lines, int32_t q_lines, uint32_t p_matrix, uint32_t q_matrix, int32_t all_blocks,
    int32_t tiles_i, int32_t tiles_j, int32_t tiles, int32_t slices, const ProductArgs a)
{
    constexpr int BN = BM, WAVES = (BM / WM) * (BN / WN), MI = WM / 32, MJ = WN / 32;
    constexpr int STAGE = (BM + BN) * 128, PIECES = (BM + BN) / 8, PER_WAVE = PIECES / WAVES;
    static_assert(PIECES % (4 * WAVES) == 0, "pairs of pieces of 8 lines of either operand per wavefront");
    extern __shared__ __align__(16) char lds[];
    int tile, slice, k, ti, tj;                                    // tile: counted over all matrices
    ns_share(ns_rank(blockIdx.x, gridDim.x), tiles, slices, tile, slice, k);
    if (KIND == NS_GRAM || KIND == NS_POLY)
        ns_tile_above(tile - k * tiles, tiles_i, ti, tj);
    else
        ns_tile_of(tile - k * tiles, tiles_i, tiles_j, ti, tj);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
    int kbegin = 0, kblocks = all_blocks;
    if (slices > 1) {
        kbegin = (int)((uint32_t)(all_blocks * slice) / (uint32_t)slices);
        kblocks = (int)((uint32_t)(all_blocks * (slice + 1)) / (uint32_t)slices) - kbegin;
    }
    const int wi = (wave / (BN / WN)) * WM, wj = (wave % (BN / WN)) * WN;

    // A piece is 8 lines; the 16-byte part c of line r stands at place c ^ (r / 2 % 8) of its line in LDS, so that 16 lanes that read one part of
    // 16 lines read all 64 banks once.  (Of an odd piece r / 2 is 4 more.)  A wavefront fetches neighbouring pieces of both operands.
    constexpr int HALF = PER_WAVE / 2;
    const char* p = reinterpret_cast<const char*>(of_p) + ((int64_t)p_matrix * k + (int64_t)(ti * BM + wave * HALF * 8) * p_lines + kbegin) * 128;
    const char* q = reinterpret_cast<const char*>(of_q) + ((int64_t)q_matrix * k + (int64_t)(tj * BN + wave * HALF * 8) * q_lines + kbegin) * 128;
    const uint32_t place = ((lane & 7) ^ (lane >> 4)) * 16, p_lane = (lane >> 3) * p_lines * 128, q_lane = (lane >> 3) * q_lines * 128;
    auto fetch = [&](int block, int stage) {
        char* to = lds + stage * STAGE + wave * (HALF * 1024);
#pragma unroll
        for (int i = 0; i < HALF; ++i) {
            ns_load_to_lds(p + (int64_t)(i * 8 * p_lines + block) * 128 + (p_lane + (place ^ (i & 1) * 64)), to + i * 1024);
            ns_load_to_lds(q + (int64_t)(i * 8 * q_lines + block) * 128 + (q_lane + (place ^ (i & 1) * 64)), to + BM * 128 + i * 1024);
        }
    };
    // what is added to a single block is on its way before anything else (the wait for the first stage is one for it too)
    constexpr bool EARLY = KIND != NS_GRAM && MI * MJ == 1;
    ns_vec early[4];
    if (EARLY) ns_fetch_old(a, k, ti * BM + wi, tj * BN + wj, early);

    // The fragments of 16 of the summed index: a lane has 8 of them of row lane % 32 of every block, hi and lo.
    struct Fragments { half8 ph[MI], pl[MI], qh[MJ], ql[MJ]; };
    const int row = lane & 31;
    auto read = [&](Fragments& f, int stage, int ks) {
        const int c = ks * 2 + lane / 32, hi = (c ^ (row / 2 & 7)) * 16, lo = ((c + 4) ^ (row / 2 & 7)) * 16;
        const char* at = lds + stage * STAGE;
#pragma unroll
        for (int b = 0; b < MI; ++b) {
            f.ph[b] = *reinterpret_cast<const half8*>(at + (wi + b * 32 + row) * 128 + hi);
            f.pl[b] = *reinterpret_cast<const half8*>(at + (wi + b * 32 + row) * 128 + lo);
        }
#pragma unroll
        for (int b = 0; b < MJ; ++b) {
            f.qh[b] = *reinterpret_cast<const half8*>(at + (BM + wj + b * 32 + row) * 128 + hi);
            f.ql[b] = *reinterpret_cast<const half8*>(at + (BM + wj + b * 32 + row) * 128 + lo);
        }
    };
    float16v acc[MI][MJ] = {};
    auto multiply = [&](const Fragments& f) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < MJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.pl[i], f.qh[j], acc[i][j], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < MJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.ph[i], f.ql[j], acc[i][j], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < MJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.ph[i], f.qh[j], acc[i][j], 0, 0, 0);
    };

    // While the second half of a block is multiplied the next block's first half is read, and its second half while that is multiplied; a block's
    // place is free for the block STAGES further on as soon as all wavefronts have read its second half.
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
        if (s < kblocks) fetch(s, s);
    if (kblocks >= STAGES)
        ns_arrived<PER_WAVE * (STAGES - 1)>();
    else
        ns_arrived<0>();
    Fragments first, second;
    read(first, 0, 0);
    int stage = 0;
    for (int block = 0; block < kblocks; ++block) {
        read(second, stage, 1);
        multiply(first);
        const int next = stage + 1 == STAGES ? 0 : stage + 1;
        if (block + STAGES < kblocks) {
            ns_arrived<PER_WAVE * (STAGES - 2)>();
            fetch(block + STAGES, stage);
        } else {
            ns_arrived<0>();
        }
        if (block + 1 < kblocks) read(first, next, 0);
        multiply(second);
        stage = next;
    }

    if (slices > 1) {                          // a slice's sums: rb_ortho_join_kernel adds them up
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < MJ; ++j) {
                float4* to = ns_sums(a, tile, slice, (BM / 32) * (BM / 32), ((wi / 32) + i) * (BM / 32) + wj / 32 + j);
#pragma unroll
                for (int g = 0; g < 4; ++g) to[g * 64] = float4{acc[i][j][g * 4], acc[i][j][g * 4 + 1], acc[i][j][g * 4 + 2], acc[i][j][g * 4 + 3]};
            }
        return;
    }
    static_assert(WAVES * NS_PLACE <= STAGES * STAGE, "the wavefronts' places fit what the stages leave");
    char* mine = lds + wave * NS_PLACE;
    const bool mirror = (KIND == NS_GRAM || KIND == NS_POLY) ? tj > ti : true;
    // (what is added: all of it at once while that is four blocks, a row of blocks at a time of a larger tile, which would not fit the registers)
    constexpr int AHEAD = MI * MJ <= 4 ? MI : 1;
    ns_vec old[AHEAD][MJ][4];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        if (KIND != NS_GRAM && !EARLY && (i == 0 || AHEAD == 1)) {
#pragma unroll
            for (int b = 0; b < AHEAD; ++b)
#pragma unroll
                for (int j = 0; j < MJ; ++j) ns_fetch_old(a, k, ti * BM + wi + (i + b) * 32, tj * BN + wj + j * 32, old[b][j]);
        }
#pragma unroll
        for (int j = 0; j < MJ; ++j)
            ns_finish<KIND, OUT>(a, k, ti * BM + wi + i * 32, tj * BN + wj + j * 32, acc[i][j], EARLY ? early : old[AHEAD == 1 ? 0 : i][j], mirror, mine);
    }
}

// The sums of the slices, in their order, and what is left of the product: a wavefront per block of 32 x 32.
template <int KIND, typename OUT, int BM>
__global__ __launch_bounds__(NS_TPB) void rb_ortho_join_kernel(const ProductArgs a)
{
    __shared__ __align__(16) char places[NS_TPB / 64][NS_PLACE];
    constexpr int SIDE = BM / 32;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t item = (int64_t)blockIdx.x * (NS_TPB / 64) + wave, tile = item / (SIDE * SIDE);
    const int b = (int)(item % (SIDE * SIDE));
    const int64_t k = tile / a.tiles;
    int ti, tj;
    if (KIND == NS_GRAM || KIND == NS_POLY)
        ns_tile_above((int)(tile - k * a.tiles), a.tiles_i, ti, tj);
    else
        ns_tile_of((int)(tile - k * a.tiles), a.tiles_i, a.tiles_j, ti, tj);
    const int r0 = ti * BM + b / SIDE * 32, c0 = tj * BM + b % SIDE * 32;
    ns_vec old[4];
    if (KIND != NS_GRAM) ns_fetch_old(a, k, r0, c0, old);
    float16v acc = {};
    for (int s = 0; s < a.slices; ++s) {
        const float4* from = ns_sums(a, tile, s, SIDE * SIDE, b);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 v = from[g * 64];
            acc[g * 4] += v.x;
            acc[g * 4 + 1] += v.y;
            acc[g * 4 + 2] += v.z;
            acc[g * 4 + 3] += v.w;
        }
    }
    ns_finish<KIND, OUT>(a, k, r0, c0, acc, old, (KIND == NS_GRAM || KIND == NS_POLY) ? tj > ti : true, places[wave]);
}

// ---- matrices of up to P x P in the LDS of one workgroup ------------------------
//
// A wavefront per block of 32 x 32 of the result, whose element i of a lane is as above.  A matrix is P * P / 32 lines of 128 bytes, line (block of
// 32 columns, row), its 16-byte parts at c ^ (row / 2 % 8).
template <int P>
struct LdsMatrices {
    static constexpr int WAVES = (P / 32) * (P / 32), BYTES = P * P * 4;
    int lane, half, col, wi, wj;
    uint32_t across_at, along_at;

    __device__ __forceinline__ LdsMatrices()
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        lane = threadIdx.x & 63;
        half = lane / 32;
        col = lane & 31;
        wi = wave / (P / 32) * 32;
        wj = wave % (P / 32) * 32;
        // The part of a line is the only thing in bits 4 to 6 of an address, so that its turn by the row is one exclusive or, and what is left of
        // an address a constant.
        across_at = (uint32_t)((wi / 32 * P + wj + col) * 128 + (col / 2 & 7) * 16 + half * 8);
        along_at = (uint32_t)((wj / 32 * P + wi + half * 4) * 128 + ((col / 8) ^ (half * 2)) * 16 + col % 8 * 2);
    }
    __device__ __forceinline__ int row(int i) const { return wi + (i / 4) * 8 + half * 4 + i % 4; }
    __device__ __forceinline__ int column() const { return wj + col; }

    // v, scaled already, to the transposed place (4 rows of a column are neighbours there) and, unless null, to its own.
    __device__ __forceinline__ void put(char* across, char* along, const float* v) const
    {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            half4 hi, lo;
            ns_split<half4, 4>(v + g * 4, hi, lo);
            if (along != nullptr) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int turn = (g & 1) * 4 + e / 2, off = (g * 8 + e) * 128;
                    *reinterpret_cast<_Float16*>(along + (along_at ^ (turn * 16)) + off) = hi[e];
                    *reinterpret_cast<_Float16*>(along + (along_at ^ ((turn ^ 4) * 16)) + off) = lo[e];
                }
            }
            *reinterpret_cast<half4*>(across + (across_at ^ (g * 16))) = hi;
            *reinterpret_cast<half4*>(across + (across_at ^ ((g ^ 4) * 16))) = lo;
        }
    }
    // The same where another wavefront may still be reading, for all to read.
    __device__ __forceinline__ void replace(char* across, char* along, const float* v) const
    {
        __syncthreads();
        put(across, along, v);
        __syncthreads();
    }

    struct Fragments { half8 ph, pl, qh, ql; };
    __device__ __forceinline__ void read(Fragments& f, const char* p, const char* q, int block, int ks) const
    {
        const int at = ks * 2 + half, hi = (at ^ (col / 2 & 7)) * 16, lo = ((at + 4) ^ (col / 2 & 7)) * 16;
        const char* pr = p + (block * P + wi + col) * 128;
        const char* qr = q + (block * P + wj + col) * 128;
        f.ph = *reinterpret_cast<const half8*>(pr + hi);
        f.pl = *reinterpret_cast<const half8*>(pr + lo);
        f.qh = *reinterpret_cast<const half8*>(qr + hi);
        f.ql = *reinterpret_cast<const half8*>(qr + lo);
    }
    static __device__ __forceinline__ void multiply(const Fragments& f, float16v& acc)
    {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.pl, f.qh, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.ph, f.ql, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.ph, f.qh, acc, 0, 0, 0);
    }
    // The wavefront's block of P Q^T over so many blocks of 32 of the summed index.
    __device__ __forceinline__ float16v product(const char* p, const char* q, int blocks) const
    {
        float16v acc = {};
        if (WAVES > 4) {                                        // four wavefronts a SIMD: one multiplies while another reads
            for (int block = 0; block < blocks; ++block) {
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    Fragments f;
                    read(f, p, q, block, ks);
                    multiply(f, acc);
                }
            }
        } else {                                                // one: half of a block is read while the other half is multiplied
            Fragments first, second;
            read(first, p, q, 0, 0);
            for (int block = 0; block < blocks; ++block) {
                read(second, p, q, block, 1);
                multiply(first, acc);
                if (block + 1 < blocks) read(first, p, q, block + 1, 0);
                multiply(second, acc);
            }
        }
        return acc;
    }
};

// A whole matrix of up to P x P: X, or A, or B in one half of the LDS, X^T in the other; X itself in registers.  One launch from the update to the
// result.  The products need 19 us at 128 x 128 and five steps, the rest is the conversions and barriers between them (43 us in all).
struct SmallArgs {
    UpdateArgs update;
    ResultArgs result;
    int32_t steps;
    float coefficients[16][3];
};

template <typename T, typename OUT, int P>
__global__ __launch_bounds__(LdsMatrices<P>::WAVES * 64) void rb_ortho_small_kernel(const SmallArgs a)
{
    extern __shared__ __align__(16) char lds[];
    __shared__ double sums[LdsMatrices<P>::WAVES];
    const LdsMatrices<P> mat;
    char* const one = lds;                                      // X, A, B
    char* const two = lds + LdsMatrices<P>::BYTES;              // X^T
    const int64_t k = blockIdx.x;
    const UpdateArgs& u = a.update;
    const int rows = a.result.rows, cols = a.result.cols, c = mat.column();

    float x[16];
    const T* grad = static_cast<const T*>(u.grad) + k * u.matrix_stride;
    float* mom = u.momentum != nullptr ? u.momentum + k * u.m * (int64_t)u.n : nullptr;
    // the place of the lane's element i in the caller's tensors
    auto at = [&](int i, int64_t stride) { return u.tall ? c * stride + mat.row(i) : mat.row(i) * stride + c; };
    auto there = [&](int i) { return mat.row(i) < rows && c < cols; };
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = there(i) ? ns_load(grad + at(i, u.row_stride)) : 0.0f;
    if (mom != nullptr) {
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = there(i) ? mom[at(i, u.n)] : 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            v[i] = fmaf(u.beta, v[i], x[i]);
            if (there(i)) mom[at(i, u.n)] = v[i];
            x[i] = u.nesterov ? fmaf(u.beta, v[i], x[i]) : v[i];
        }
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum = fma((double)x[i], (double)x[i], sum);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if (mat.lane == 0) sums[threadIdx.x / 64] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < LdsMatrices<P>::WAVES; ++w) sum += sums[w];
    const double inverse = ns_inverse(sqrt(sum) + (double)u.eps);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = (float)((double)x[i] * inverse);

    const int row_blocks = (rows + 31) / 32, col_blocks = (cols + 31) / 32;
    mat.put(two, one, x);
    __syncthreads();
    for (int s = 0; s < a.steps; ++s) {
        const float ca = a.coefficients[s][0], cb = a.coefficients[s][1], cc = a.coefficients[s][2];
        float v[16];
        float16v acc = mat.product(one, one, col_blocks);       // A
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = acc[i] * (NS_SCALE_A / (NS_SCALE_X * NS_SCALE_X));
        mat.replace(one, nullptr, v);
        acc = mat.product(one, one, row_blocks);                // B = b A + c A A
#pragma unroll
        for (int i = 0; i < 16; ++i)
            v[i] = fmaf(cb * (NS_SCALE_B / NS_SCALE_A), v[i], cc * (NS_SCALE_B / (NS_SCALE_A * NS_SCALE_A)) * acc[i]);
        mat.replace(one, nullptr, v);
        acc = mat.product(one, two, row_blocks);                // X <- a X + B X
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = fmaf(ca, x[i], acc[i] * (1.0f / NS_SCALE_B));
        if (s + 1 < a.steps) mat.replace(two, one, x);
    }
    OUT* dst = static_cast<OUT*>(a.result.dst) + k * a.result.matrix_stride;
    const int r = mat.row(0);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] *= 1.0f / NS_SCALE_X;
    if (!a.result.tall)
        ns_result<StepRows>(a.result, dst + r * a.result.row_stride + c, a.result.row_stride, c < cols ? rows - r : 0, x);
    else
        ns_result<StepRows>(a.result, dst + c * a.result.row_stride + r, 1, c < cols ? rows - r : 0, x);
}

// Two steps on A alone, of a short side of up to P: R = P2 P1 with P = a I + b A + c A A, the second of P1 A P1.  A launch instead of five of a few
// microseconds each.  What is put is there transposed, so a product's operands are the other way round: P1 A P1 and P2 P1 as they are
// written.  P1 P1 A and P1 P2 would be the same but for their rounding errors, which P1 multiplies by up to a a and by a in the weak singular
// directions (results of up to twice the error).
struct PairArgs {
    const _Float16* a;
    _Float16* r;
    int64_t matrix, pitch;      // halves between matrices, and between rows, of both
    int32_t rows;
    float coefficients[2][3];
};

template <int P>
__global__ __launch_bounds__(LdsMatrices<P>::WAVES * 64) void rb_ortho_pair_kernel(const PairArgs a)
{
    extern __shared__ __align__(16) char lds[];
    const LdsMatrices<P> mat;
    char* const one = lds;                                      // A, P1 A, P1 A P1, P1
    char* const two = lds + LdsMatrices<P>::BYTES;              // P1, P2
    const int c = mat.column(), blocks = (a.rows + 31) / 32;
    const _Float16* from = a.a + blockIdx.x * a.matrix + ns_at(c, mat.row(0), a.pitch);          // (A is symmetric)
    float m[16], p[16], r[16];                                  // A, the step's P, the first P and R
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const half4 hi = *reinterpret_cast<const half4*>(from + g * 8), lo = *reinterpret_cast<const half4*>(from + g * 8 + NS_KBLOCK);
#pragma unroll
        for (int e = 0; e < 4; ++e) m[g * 4 + e] = mat.row(g * 4 + e) < a.rows && c < a.rows ? (float)hi[e] + (float)lo[e] : 0.0f;
    }
    auto polynomial = [&](const float* k, const float16v& acc) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[i] = fmaf(k[1] * (NS_SCALE_B / NS_SCALE_A), m[i], k[2] * (NS_SCALE_B / (NS_SCALE_A * NS_SCALE_A)) * acc[i]);
            if (mat.row(i) == c) p[i] += k[0] * NS_SCALE_B;
        }
    };
    auto of_p = [&](float* to, const float16v& acc) {
#pragma unroll
        for (int i = 0; i < 16; ++i) to[i] = acc[i] * (1.0f / NS_SCALE_B);
    };
    mat.put(one, nullptr, m);
    __syncthreads();
    polynomial(a.coefficients[0], mat.product(one, one, blocks));
    mat.replace(two, nullptr, p);
    of_p(m, mat.product(one, two, blocks));
    mat.replace(one, nullptr, m);
    of_p(m, mat.product(two, one, blocks));
    mat.replace(one, nullptr, m);
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = p[i];
    polynomial(a.coefficients[1], mat.product(one, one, blocks));
    __syncthreads();
    mat.put(two, nullptr, p);
    mat.put(one, nullptr, r);
    __syncthreads();
    of_p(r, mat.product(one, two, blocks));
    _Float16* to = a.r + blockIdx.x * a.matrix + ns_at(c, mat.row(0), a.pitch);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        half4 hi, lo;
        ns_split<half4, 4>(r + g * 4, hi, lo);
        *reinterpret_cast<half4*>(to + g * 8) = hi;
        *reinterpret_cast<half4*>(to + g * 8 + NS_KBLOCK) = lo;
    }
}

}  // namespace
