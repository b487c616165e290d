// Attention of packed documents (rb_attention_forward) and its gradients (rb_attention_grad).  Included by rb_block.hip only.
//
// Masks.  What a position sees - its document up to itself, or the prefix, or all of the document - is one interval of positions, and so is what sees
// it.  A workgroup of the forward pass finds those of its rows in LDS (of many documents a small kernel finds them first), the first kernel of the gradients
// those of all positions; what follows compares with them and knows no documents.  Tiles that every row of a wavefront sees whole
// are not compared at all, tiles that none sees are passed over.
//
// Products.  Matrix instructions of 32 x 32 x 16 give a lane 16 elements of one column, in rows 8 (i / 4) + 4 (lane / 32) + i % 4.  The scores are made
// transposed (keys x queries), so that a lane has one query: maximum and sum of the softmax are its own but for one exchange with lane ^ 32.  The next
// product sums over the keys, and may take them in any order as long as both operands do: the lane's elements, rounded to bfloat16, are that
// operand as they are, and the other one (values, transposed) is read from LDS in the same order by transposing reads.  The gradients of keys
// and values have keys for columns (a lane has one key) and sum over queries in the same way.
//
// LDS.  Tiles are 64 rows of 128 or 256 bytes, loaded straight into LDS, 16 bytes a lane; the 16-byte pieces of a row are permuted by the row's number so
// that both the reads of rows (one piece each of 32 rows) and the transposing reads (four neighbouring pieces of eight rows) meet all banks.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "rb_lanes.h"

namespace {

constexpr int AT_TPB = 256;
constexpr int AT_WAVES = AT_TPB / 64;
constexpr int AT_BLOCK = 32;                       // rows of a wavefront
constexpr int AT_ROWS = AT_WAVES * AT_BLOCK;       // rows of a workgroup
constexpr int AT_TILE = 64;                        // rows that are in LDS at a time
constexpr float AT_LOG2E = 1.44269504088896340736f;
constexpr int64_t AT_MAX_STRIDE = 1 << 26;         // of positions, in numbers: 31 strides are less than 2^32 bytes
constexpr int AT_NEAR_OFFSETS = 2048;              // offsets of documents that a workgroup looks through in LDS
constexpr float AT_LN2 = 0.69314718055994530942f;

typedef __bf16 at_bf8 __attribute__((ext_vector_type(8)));
typedef float at_acc __attribute__((ext_vector_type(16)));
typedef short at_s4 __attribute__((ext_vector_type(4)));
typedef short at_s8 __attribute__((ext_vector_type(8)));

struct HeadRows {
    Bf16* data;
    int64_t token, head;       // strides in elements
    __device__ __forceinline__ Bf16* at(int64_t t, int64_t h) const { return data + t * token + h * head; }
};

struct Span { int32_t lo, hi; };
struct Spans { Span sees, seen; };      // of a position: what it sees, and what sees it

struct SpanArgs {
    const int64_t *offsets, *lengths, *prefixes;
    int64_t count;
    Spans* spans;
    int32_t tokens, causal;
};

// How many documents begin at or before position t.
template <typename Offsets>
__host__ __device__ inline int64_t at_begun(Offsets offsets, int64_t count, int32_t t)
{
    int64_t low = 0, high = count;
    while (low < high) {
        const int64_t mid = (low + high) / 2;
        if (offsets[mid] <= t) low = mid + 1;
        else high = mid;
    }
    return low;
}

// Of position t.  Its document is the last one that begins at or before it (those behind that one with the same begin are empty).  Positions
// in no document get empty intervals at themselves, so that neighbouring positions' intervals still rise.  Whatever the numbers are, intervals
// lie within the positions there are, and one that is not empty holds t.
template <typename Offsets>
__host__ __device__ inline Spans at_spans_of(const SpanArgs& a, Offsets offsets, int32_t t)
{
    auto lower = [](int64_t x, int64_t y) { return x < y ? x : y; };
    auto higher = [](int64_t x, int64_t y) { return x < y ? y : x; };
    Spans s{{t, t}, {t, t}};
    const int64_t d = at_begun(offsets, a.count, t) - 1;
    if (d < 0) return s;
    const int64_t begin = higher(offsets[d], 0);
    int64_t end = lower(offsets[d + 1], a.tokens);
    if (a.lengths) end = lower(end, begin + lower(higher(a.lengths[d], 0), a.tokens));
    if (t >= end) return s;
    const int64_t prefix = a.prefixes ? begin + lower(higher(a.prefixes[d], 0), end - begin) : begin;
    s.sees.lo = (int32_t)begin;
    s.sees.hi = (int32_t)(a.causal ? higher((int64_t)t + 1, prefix) : end);
    s.seen.lo = (int32_t)(a.causal && t >= prefix ? t : begin);
    s.seen.hi = (int32_t)end;
    return s;
}

// A thread per position.
__global__ void __launch_bounds__(AT_TPB) rb_spans_kernel(SpanArgs a)
{
    const int t = blockIdx.x * AT_TPB + threadIdx.x;
    if (t < a.tokens) a.spans[t] = at_spans_of(a, a.offsets, t);
}

// ---- tiles in LDS --------------------------------------------------------------

// Where piece c (16 bytes) of row r of a tile lies: in place c ^ at_turn(r) of the row.
template <int D>
__device__ __forceinline__ int at_turn(int r)
{
    return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

// Asynchronous loads into LDS: the wavefront's lanes bring BYTES each, which land behind each other from `to` on (the same for all of them).  Written
// out, since for the builtin the compiler has every later read from LDS wait for all of them, also of the tile that is complete; at_arrived waits.
// (There are no registers that such a load writes.)  Two forms: an address a lane, and one for all with an offset in bytes a lane, which takes a third of
// the registers.
__device__ __forceinline__ uint32_t at_place_of(const void* to)       // as LDS counts, the same for all lanes
{
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)to);
}
__device__ __forceinline__ uint64_t at_scalar(uint64_t v)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
}
template <int BYTES>
__device__ __forceinline__ void at_load_to_lds(const void* from, uint32_t to)
{
    to = (uint32_t)__builtin_amdgcn_readfirstlane((int)to);
    if constexpr (BYTES == 16) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory", "m0");
    else asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(to) : "memory", "m0");
}
__device__ __forceinline__ void at_load_to_lds(uint64_t base, uint32_t offset, uint32_t to)
{
    to = (uint32_t)__builtin_amdgcn_readfirstlane((int)to);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(to) : "memory", "m0");
}

// A lane's part in bringing tiles of ROWS rows of a tensor: the same pieces of every tile.
template <int D, int ROWS = AT_TILE>
struct Bring {
    static constexpr int PIECES = D / 8, LOADS = ROWS * PIECES / AT_TPB, STEP = ROWS / LOADS;
    int row, piece, wave;
    bool there;                // (pieces behind the head's last number are left as they are: 0)
    __device__ __forceinline__ Bring(int wave_, int dim) : wave(wave_)
    {
        const int lane = threadIdx.x & 63;
        row = (wave * 64 + lane) / PIECES;
        piece = (lane % PIECES) ^ at_turn<D>(row);
        there = piece * 8 < dim;
    }
    // Where the lane's piece of a tile's first rows is, in bytes behind the tile's first row (a lane's row is one of 32: strides are at most AT_MAX_STRIDE).
    __device__ __forceinline__ uint32_t offset(int64_t stride) const
    {
        uint32_t bytes = 2 * ((uint32_t)row * (uint32_t)stride + (uint32_t)piece * 8);
        asm volatile("" : "+v"(bytes));                 // (one register, and not half of a product's two)
        return bytes;
    }
    // Rows first .. first + ROWS - 1 of the tensor that begins at `from`, no further than row `last`.
    __device__ __forceinline__ void operator()(const Bf16* from, int64_t stride, uint32_t offset, int first, int last, uint32_t tile) const
    {
        if (!there) return;
        if (first + ROWS <= last + 1) {
            const uint64_t base = at_scalar(reinterpret_cast<uint64_t>(from + first * stride)), step = at_scalar(2 * STEP * (uint64_t)stride);
#pragma unroll
            for (int j = 0; j < LOADS; ++j) at_load_to_lds(base + j * step, offset, tile + (j * AT_WAVES + wave) * 1024);
        } else {
            int r = first + row, p = piece * 8;
            asm volatile("" : "+v"(r), "+v"(p));        // (nothing of this is kept for the next tile)
#pragma unroll
            for (int j = 0; j < LOADS; ++j)
                at_load_to_lds<16>(from + (int64_t)min(r + j * STEP, last) * stride + p, tile + (j * AT_WAVES + wave) * 1024);
        }
    }
};

// 32 binary32 numbers of a lane half each, to places behind one another.
__device__ __forceinline__ void at_bring_numbers(const float* from, int first, int last, uint32_t to)
{
    at_load_to_lds<4>(from + min(first + (int)(threadIdx.x & 31), last), to);
}

// Waits until a wavefront's loads into LDS and its reads from there are done, then for the workgroup's other wavefronts.
__device__ __forceinline__ void at_arrived() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// What a lane reads of tiles: rows (an operand whose rows are the tile's, summed over the head's numbers) and columns (one whose rows are the head's
// numbers, summed over the tile's rows in the order of a result's elements).
template <int D>
struct Reads {
    int row_at, row_turn, col_at, col_turn;
    __device__ __forceinline__ Reads()
    {
        const int lane = threadIdx.x & 63, half = lane / 32, r = lane & 31;
        row_at = r * D * 2;
        row_turn = half ^ at_turn<D>(r);
        // 16 lanes read four rows of 16 numbers; lane i gets column i of them
        const int i = lane & 15, c = (lane >> 4) & 1, rr = 4 * half + i / 4;
        col_at = rr * D * 2 + (i & 1) * 8;
        col_turn = (2 * c + (i & 3) / 2) ^ at_turn<D>(rr);
    }
    // numbers 16 s + 8 (lane / 32) .. of row 32 b + lane % 32
    __device__ __forceinline__ at_bf8 rows(const char* tile, int b, int s) const
    {
        return *reinterpret_cast<const at_bf8*>(tile + b * 32 * D * 2 + row_at + ((row_turn ^ (2 * s)) << 4));
    }
    // number 32 n + lane % 32 of the rows 16 c + 4 (lane / 32) .. + 3 and 8 behind these
    __device__ __forceinline__ at_bf8 columns(const char* tile, int n, int c) const
    {
        typedef __attribute__((address_space(3))) at_s4* place;
        const char* const first = tile + c * 16 * D * 2 + col_at;
        const int turn = col_turn ^ (4 * n);
        const at_s4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((place)(first + (turn << 4)));
        const at_s4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((place)(first + 8 * D * 2 + ((turn ^ 2) << 4)));
        return __builtin_bit_cast(at_bf8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

__device__ __forceinline__ at_acc at_mma(at_bf8 a, at_bf8 b, at_acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// Elements 8 c .. 8 c + 7 of a lane as an operand.
__device__ __forceinline__ at_bf8 at_pack(const at_acc& v, int c)
{
    sc_vec w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = sc_bf16_pair(v[8 * c + 2 * i], v[8 * c + 2 * i + 1]);
    return __builtin_bit_cast(at_bf8, w);
}

// What that rounding left, rounded: both together are the elements to within 2^-17 of each.
__device__ __forceinline__ at_bf8 at_pack_rest(const at_acc& v, const at_bf8& rounded, int c)
{
    const sc_vec r = __builtin_bit_cast(sc_vec, rounded);
    sc_vec w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = sc_bf16_pair(v[8 * c + 2 * i] - __uint_as_float(r[i] << 16), v[8 * c + 2 * i + 1] - __uint_as_float(r[i] & 0xffff0000u));
    return __builtin_bit_cast(at_bf8, w);
}
// sum + the eight numbers of an operand, two at a time.  (Each pair through a register of its own: from within the operand's the compiler takes the first pair
// four times.)
__device__ __forceinline__ float at_sum(const at_bf8& v, float sum)
{
    typedef __bf16 at_bf2 __attribute__((ext_vector_type(2)));
    const sc_vec w = __builtin_bit_cast(sc_vec, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t pair = w[i];
        asm volatile("" : "+v"(pair));
        sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(at_bf2, pair), __builtin_bit_cast(at_bf2, 0x3f803f80u), sum, false);
    }
    return sum;
}

// The wavefront's 32 of the workgroup's 128 rows in two tiles, as operands.
template <int D>
__device__ __forceinline__ void at_own(const Reads<D>& reads, const char (&tiles)[2][AT_TILE * D * 2], int wave, at_bf8 (&f)[D / 16])
{
#pragma unroll
    for (int n = 0; n < D / 16; ++n) f[n] = reads.rows(tiles[wave / 2], wave % 2, n);
}
// The workgroup's 128 rows into two tiles.
template <int D>
__device__ __forceinline__ void at_bring_own(const Bring<D>& bring, const Bf16* from, int64_t stride, int tile, int last, uint32_t tiles)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) bring(from, stride, bring.offset(stride), min(tile * AT_ROWS + i * AT_TILE, last), last, tiles + i * AT_TILE * D * 2);
}

// sum[n] += columns of the tile's rows 16 (c0 + c) .. times factors[c], for the head's numbers 32 n ..  AHEAD: the next columns are on their way while the last
// ones are multiplied (left to itself the compiler waits for each; where it has no registers left that is better, the other wavefront fills in).
template <int D, int C, bool AHEAD>
__device__ __forceinline__ void at_add(at_acc (&sum)[D / 32], const at_bf8 (&factors)[C], const Reads<D>& reads, const char* tile, int c0)
{
    if constexpr (!AHEAD) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int n = 0; n < D / 32; ++n) sum[n] = at_mma(reads.columns(tile, n, c0 + c), factors[c], sum[n]);
        return;
    }
    at_bf8 v[2][D / 32];
#pragma unroll
    for (int n = 0; n < D / 32; ++n) v[0][n] = reads.columns(tile, n, c0);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (c + 1 < C) {
#pragma unroll
            for (int n = 0; n < D / 32; ++n) v[(c + 1) & 1][n] = reads.columns(tile, n, c0 + c + 1);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < D / 32; ++n) sum[n] = at_mma(v[c & 1][n], factors[c], sum[n]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// ---- what is not finite where something is masked --------------------------------
//
// A masked factor is 0, and 0 times an infinity or a NaN is no 0.  So in tiles of which a row of the workgroup does not see all, the workgroup
// makes what is not finite 0 before it is multiplied by factors, and notes the rows it was in: who sees one of them makes up for it.

struct Noted {
    uint32_t rows[2][2];       // of this tile and the next, 64 bits each
};

// The pieces of a tile that the thread has brought.  (Between two waits for the workgroup.)
template <int D, int ROWS = AT_TILE>
__device__ __forceinline__ void at_make_finite(char* tile, int wave, uint32_t (&noted)[2])
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                      // (as above)
#pragma unroll
    for (int j = 0; j < Bring<D, ROWS>::LOADS; ++j) {
        const int at = (j * AT_WAVES + wave) * 64 + lane;
        sc_vec w = *reinterpret_cast<const sc_vec*>(tile + at * 16);
        uint32_t found = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) found |= (w[i] & 0x7f807f80u) + 0x00800080u;       // (an exponent of ones carries into the sign's place)
        if (found & 0x80008000u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t m = (((w[i] & 0x7f807f80u) + 0x00800080u) >> 15) & 0x00010001u;
                w[i] &= ~((m << 16) - m);
            }
            *reinterpret_cast<sc_vec*>(tile + at * 16) = w;
            const int row = at / Bring<D, ROWS>::PIECES;
            atomicOr(&noted[row / 32], 1u << (row % 32));
        }
    }
}
__device__ __forceinline__ void at_wait_for_all() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The noted rows among from .. to - 1.
__device__ __forceinline__ uint64_t at_noted(const uint32_t (&noted)[2], int from, int to)
{
    const uint64_t rows = (uint64_t)noted[1] << 32 | noted[0];
    const int f = min(max(from, 0), 64), t = min(max(to, 0), 64);
    const uint64_t below_to = t == 64 ? ~0ull : (1ull << t) - 1, below_from = f == 64 ? ~0ull : (1ull << f) - 1;
    return rows & below_to & ~below_from;
}

// ---- scores ------------------------------------------------------------------
//
// All in base 2.  With r = 1 / (1 + e^2x), tanh x = 1 - 2 r to within 2^-21 (and its slope 4 r (1 - r)), so that a capped score is off by cap * 2^-21 at
// most: less than what rounding e^score to bfloat16 puts in for caps of up to 32, where more is not worth it.  There the cap is also the maximum
// that the softmax needs: e^(score - cap) is at least e^-64 for what lies next to a position, and its sums are normal numbers.  Larger caps have
// scores that are exact near 0, too, and a running maximum; a slope below 0 raises scores beyond any cap and has one as well.  (16384 positions, 8 heads of 128: a
// cap of 30 613 us and gradients 2424, one of 33 926 and 2905.)
//
// Short documents.  p and ds are rounded to bfloat16 for the products over positions.  The errors of many positions are as independent as those of the results'
// own rounding, and as large.  Of a handful of positions they may be twice as large, so there (FINE) what the rounding left is multiplied too: an error
// of 2^-17, for products that cost nothing where a launch has a few tiles of positions.
enum { AT_PLAIN = 0, AT_CAPPED = 1, AT_HIGH_CAP = 2 };
constexpr float AT_LOW_CAP = 32.0f;

struct ScoreOf {
    float scale;               // of a product
    float to_log2;             // plain: scale * log2 e; else cap * log2 e
    float to_tanh;             // 2 log2 e scale / cap: 2^(to_tanh * product) = e^2x; of a high cap: scale / cap
};

// tanh within 2^-21 of itself (eight half steps): below 0.4 by a polynomial, x + x^3 times one of three terms in x^2 that is nearest to tanh there (2^-23, and 2^-22.2 with
// its roundings); from there on 1 - 2 r, where an exponential and a reciprocal that are off by their last bits put 2^-21 into 0.38.  (The polynomial with one
// term more, up to 0.5, would be within 2^-21.4, and costs 2.5 % of 16384 positions with a cap of 33.)
__device__ __forceinline__ float at_tanh(float x)
{
    const float x2 = x * x;
    const float near = x * fmaf(x2, fmaf(x2, fmaf(x2, -0.0478118619f, 0.1327802241f), -0.3333190084f), 1.0f);
    const float e = __builtin_amdgcn_exp2f(x * (2 * AT_LOG2E));
    const float far = 1.0f - 2.0f * __builtin_amdgcn_rcpf(e + 1.0f);
    return fabsf(x) < 0.4f ? near : far;
}

// A score (of AT_CAPPED: less the cap) in base 2, and the cap's slope.
template <int FORM>
__device__ __forceinline__ float at_score(const ScoreOf& of, float product, float& slope)
{
    if (FORM == AT_PLAIN) return product * of.to_log2;
    if (FORM == AT_CAPPED) {
        const float r = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(product * of.to_tanh));
        const float four = 4.0f * r;
        slope = fmaf(-four, r, four);
        return r * (-2.0f * of.to_log2);
    }
    const float t = at_tanh(product * of.to_tanh);
    slope = 1.0f - t * t;
    return t * of.to_log2;
}

struct AttentionArgs {
    HeadRows q, k, v;
    const Spans* spans;                    // null: from the documents
    SpanArgs documents;
    const float* slopes;
    ScoreOf score;
    int32_t tokens, dim, heads, group;     // group: heads of queries to one of keys
    int32_t tiles, inner;
    bool ranked;                           // tiles take turns by what they see, not by where they are
    int32_t shares;                        // gradients of keys: heads of keys, times the parts that their queries are cut into
    float* sums;                           // of the parts: [shares][tokens][2][D]; null: there is one
    // forward: written; gradients: read
    HeadRows out;
    float* lse;
    // gradients
    HeadRows grad_out, grad_q, grad_k, grad_v;
    const float* lse2;                     // [heads][tokens]: lse in base 2, less lse_less (+inf where nothing is seen)
    float* delta;                          // [heads][tokens]: the sum of grad_out * out; then of p dp
    float lse_less;                        // what scores are less by: of AT_CAPPED the cap
};

// Which tile and head the workgroup has.  Workgroups go to the 8 dies in turn, and each die has its own L2: a die gets heads of its own (where their number
// allows it), those that read the same keys at a time.  `inner` of them take turns; their longest tiles come first: the last of a causal document for
// queries, the first for keys (UP).
template <bool UP>
__device__ __forceinline__ void at_place(int id, int tiles, int heads, int inner, int& tile, int& head)
{
    const int i = id >> 3;
    int t;
    if (inner > 0) {
        const int outer = i / inner;
        const int round = outer / tiles;
        t = outer - round * tiles;
        head = (id & 7) * (heads >> 3) + round * inner + (i - outer * inner);
    } else {
        t = id / heads;
        head = id - t * heads;
    }
    tile = __builtin_amdgcn_readfirstlane(UP ? t : tiles - 1 - t);             // (the turn's, where tiles are ranked)
    head = __builtin_amdgcn_readfirstlane(head);
}

// What rows see: all of it lies in [lo, hi), and [all_lo, all_hi) is seen by every row that sees anything.  Intervals of rows behind one another rise, so the
// first and the last row that see anything tell.  (Where documents cannot be, what comes of it is unspecified, and within the positions like every interval.)
struct Reach {
    int lo, hi, all_lo, all_hi;
    __device__ __forceinline__ Reach(Span first, Span last, bool any) : lo(any ? first.lo : 0), hi(any ? last.hi : 0), all_lo(any ? last.lo : 0), all_hi(any ? first.hi : 0) {}
    __device__ __forceinline__ bool meets(int first, int rows = AT_TILE) const { return first < hi && first + rows > lo; }
    __device__ __forceinline__ bool whole(int first, int rows = AT_TILE) const { return first >= all_lo && first + rows <= all_hi; }
    __device__ __forceinline__ int tiles(int rows) const { return lo < hi ? (hi - lo + rows - 1) / rows : 0; }
};
__device__ __forceinline__ Span at_lane(Span s, int lane) { return Span{__builtin_amdgcn_readlane(s.lo, lane), __builtin_amdgcn_readlane(s.hi, lane)}; }
// Of the wavefront's rows, one a lane and the same 32 in both halves.
__device__ __forceinline__ Reach at_reach(Span s)
{
    const uint64_t some = __ballot(s.lo < s.hi);
    const int first = some ? __builtin_ctzll(some) : 0, last = some ? 63 - __builtin_clzll(some) : 0;
    return Reach(at_lane(s, first), at_lane(s, last), some != 0);
}
// Of the workgroup's rows: those of its lanes, `low`, and the 64 behind them, `high`.
static_assert(AT_ROWS == 128, "two a lane");
__device__ __forceinline__ Reach at_reach(Span low, Span high)
{
    const uint64_t in_low = __ballot(low.lo < low.hi), in_high = __ballot(high.lo < high.hi);
    const Span first = in_low ? at_lane(low, __builtin_ctzll(in_low)) : at_lane(high, in_high ? __builtin_ctzll(in_high) : 0);
    const Span last = in_high ? at_lane(high, 63 - __builtin_clzll(in_high)) : at_lane(low, in_low ? 63 - __builtin_clzll(in_low) : 0);
    return Reach(first, last, (in_low | in_high) != 0);
}
// The same from all positions' intervals (SEEN: of what sees the rows).
template <bool SEEN>
__device__ __forceinline__ Reach at_reach(const Spans* spans, int first, int tokens)
{
    const int t = first + (threadIdx.x & 63), u = t + 64;
    const Span none{0, 0};
    const Span low = t < tokens ? SEEN ? spans[t].seen : spans[t].sees : none, high = u < tokens ? SEEN ? spans[u].seen : spans[u].sees : none;
    return at_reach(low, high);
}

// The tile whose turn it is where there are several documents: the one with the turn's place among all, by what its rows see (or are seen by), the longest first.
// `lengths`: of all tiles, one a thread (at most AT_RANKED; 24 documents in 8192 positions, 16 heads of 128: 74 -> 60 us).
constexpr int AT_RANKED = AT_TPB;
__device__ __forceinline__ int at_ranked(int turn, int tiles, int length, char* lds)
{
    int* const lengths = reinterpret_cast<int*>(lds);
    int* const found = lengths + AT_RANKED;
    lengths[threadIdx.x] = (int)threadIdx.x < tiles ? length : -1;
    __syncthreads();
    int before = 0;
    for (int i = 0; i < tiles; i += 4) {
        const int4 l = *reinterpret_cast<const int4*>(lengths + i);
        before += l.x > length || (l.x == length && i < (int)threadIdx.x);
        before += l.y > length || (l.y == length && i + 1 < (int)threadIdx.x);
        before += l.z > length || (l.z == length && i + 2 < (int)threadIdx.x);
        before += l.w > length || (l.w == length && i + 3 < (int)threadIdx.x);
    }
    if ((int)threadIdx.x < tiles && before == turn) *found = threadIdx.x;
    __syncthreads();
    const int tile = __builtin_amdgcn_readfirstlane(*found);
    __syncthreads();
    return tile;
}
// How far the first and the last of a tile's rows reach.
__device__ __forceinline__ int at_length(Span first, Span last) { return max(last.hi - first.lo, 0); }
template <bool SEEN>
__device__ __forceinline__ int at_ranked_by_spans(const Spans* spans, int turn, int tiles, int tokens, char* lds)
{
    const int first = min((int)threadIdx.x, tiles - 1) * AT_ROWS, last = min(first + AT_ROWS, tokens) - 1;
    const int length = SEEN ? at_length(spans[first].seen, spans[last].seen) : at_length(spans[first].sees, spans[last].sees);
    return at_ranked(turn, tiles, length, lds);
}

template <int D>
__device__ __forceinline__ void at_clear(char* lds, int bytes, int dim)
{
    if (dim == D) return;
    for (int i = threadIdx.x * 16; i < bytes; i += AT_TPB * 16) *reinterpret_cast<sc_vec*>(lds + i) = sc_vec{0, 0, 0, 0};
    __syncthreads();
}

// 32 rows of a result, of which a lane has one (lane % 32) with its numbers 32 n + 8 (i / 4) + 4 (lane / 32) + i % 4: through LDS (`place`, the wavefront's own),
// so that whole rows go to memory (eight bytes a lane at a time cost a quarter of the time of short documents).
template <int D>
__device__ __forceinline__ void at_store(char* place, Bf16* first, int64_t stride, int rows, int dim, const at_acc (&v)[D / 32], float factor, bool zero)
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                      // (nothing is kept for this over the tiles)
    const int half = lane / 32, r = lane & 31;
    char* const mine = place + r * D * 2 + half * 8;
    const int turn = at_turn<D>(r);
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            uint2 w{0, 0};
            if (!zero) w = uint2{sc_bf16_pair(v[n][4 * g] * factor, v[n][4 * g + 1] * factor), sc_bf16_pair(v[n][4 * g + 2] * factor, v[n][4 * g + 3] * factor)};
            *reinterpret_cast<uint2*>(mine + (((4 * n + g) ^ turn) << 4)) = w;
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
        const int at = j * 64 + lane, row = at / (D / 8), piece = at % (D / 8);
        const sc_vec w = *reinterpret_cast<const sc_vec*>(place + row * D * 2 + ((piece ^ at_turn<D>(row)) << 4));
        if (row < rows && piece * 8 < dim) *reinterpret_cast<sc_vec*>(first + row * stride + piece * 8) = w;
    }
}

// The same unrounded.
template <int D>
__device__ __forceinline__ void at_store_sum(float* row, const at_acc (&v)[D / 32], float factor, bool zero)
{
    const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float4 w{0.0f, 0.0f, 0.0f, 0.0f};
            if (!zero) w = float4{v[n][4 * g] * factor, v[n][4 * g + 1] * factor, v[n][4 * g + 2] * factor, v[n][4 * g + 3] * factor};
            *reinterpret_cast<float4*>(row + 32 * n + 8 * g + 4 * half) = w;
        }
}

// ---- forward -------------------------------------------------------------------

// A workgroup has 128 queries of one head, 32 a wavefront, and goes through the keys that they see, 64 at a time, with the next 64 keys and values on their
// way into the other half of LDS.  One pass: p = e^(s - m) with the running maximum m, l the sum of p, o the sum of p v; o and l are scaled where m
// has grown by more than 2^8.  Two workgroups a unit (256 registers a lane, 64 KB of LDS): while a wavefront makes its softmax, another one multiplies.  That
// they do not do both at the same time is what the wavefronts' priorities are for: scores and softmax go before the second product (16 heads of 128 that see all of 8192 positions
// 526 us without, 503 with both products before the softmax, 497 so; 16384 positions, 8 heads, a cap of 30: 662, 661 and 602).
// Bound by the matrix instructions and the softmax's vector instructions beside them: the 497 us are 1.11 PFLOP/s (a large product of the library runs at 1.3); one
// document of 16384 with 8 heads 510 us causal, 602 with capped scores; 24 documents of any lengths in 8192 positions 60 us, half of it starts, ends and
// tiles that are masked in part.  64 documents of 128 33 us.
template <int D, int FORM, bool SLOPES, bool FINE>
__global__ void __launch_bounds__(AT_TPB, 2) rb_attend_kernel(AttentionArgs a)
{
    __shared__ __align__(1024) char lds[2][2][AT_TILE * D * 2];
    __shared__ Noted noted;
    constexpr uint32_t BYTES = AT_TILE * D * 2;
    const uint32_t place = at_place_of(&lds[0][0][0]);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, half = lane / 32;
    int tile, head;
    at_place<false>(blockIdx.x, a.tiles, a.heads, a.inner, tile, head);
    const int kv = __builtin_amdgcn_readfirstlane(head / a.group);
    // what the workgroup's rows see, in LDS before the tiles come
    Span* const spans = reinterpret_cast<Span*>(&lds[0][0][0]);
    if (a.spans == nullptr) {
        static_assert(AT_ROWS * sizeof(Span) + AT_NEAR_OFFSETS * 8 + (AT_RANKED + 1) * 4 <= sizeof(lds), "intervals, offsets, ranks");
        int64_t* const near = reinterpret_cast<int64_t*>(&lds[0][0][0] + AT_ROWS * sizeof(Span));
        for (int i = threadIdx.x; i <= a.documents.count; i += AT_TPB) near[i] = a.documents.offsets[i];
        __syncthreads();
        if (a.ranked) {
            const int first = min((int)threadIdx.x, a.tiles - 1) * AT_ROWS, end = min(first + AT_ROWS, a.tokens);
            const int64_t d = at_begun(near, a.documents.count, first);
            const int length = end - (d > 0 ? (int)min(max(near[d - 1], (int64_t)0), (int64_t)a.tokens) : first);
            tile = at_ranked(a.tiles - 1 - tile, a.tiles, length, reinterpret_cast<char*>(near + AT_NEAR_OFFSETS));
        }
        if (threadIdx.x < AT_ROWS) {
            const int t = tile * AT_ROWS + threadIdx.x;
            spans[threadIdx.x] = t < a.tokens ? at_spans_of(a.documents, near, t).sees : Span{0, 0};
        }
    } else if (threadIdx.x < AT_ROWS) {
        const int t = tile * AT_ROWS + threadIdx.x;
        spans[threadIdx.x] = t < a.tokens ? a.spans[t].sees : Span{0, 0};
    }
    __syncthreads();
    const int row = tile * AT_ROWS + wave * AT_BLOCK + (lane & 31);
    const Span mine = spans[wave * AT_BLOCK + (lane & 31)];
    const Reach all = at_reach(spans[lane], spans[64 + lane]), reach = at_reach(mine);
    __syncthreads();
    const int last = a.tokens - 1;
    const Bf16 *const keys = a.k.at(0, kv), *const values = a.v.at(0, kv);
    const float slope2 = SLOPES && a.slopes ? a.slopes[head] * AT_LOG2E : 0.0f;
    at_bf8 q[D / 16];
    if (threadIdx.x < 4) noted.rows[threadIdx.x / 2][threadIdx.x % 2] = 0;
    at_clear<D>(&lds[0][0][0], sizeof(lds), a.dim);
    const Bring<D> bring(wave, a.dim);
    const Reads<D> reads;
    const uint32_t k_offset = bring.offset(a.k.token), v_offset = bring.offset(a.v.token);
    at_acc o[D / 32]{};
    // capped scores need no maximum, but where a slope below 0 raises what is far away (16384 positions, 8 heads of 128, a cap of 30, slopes above 0: 584 us, with a
    // maximum 736)
    constexpr bool MAY_RISE = FORM == AT_CAPPED && SLOPES;
    const bool moves = FORM != AT_CAPPED || (MAY_RISE && __builtin_amdgcn_readfirstlane(slope2 < 0.0f));
    float m = moves ? sc_neg_inf() : 0.0f, l = 0.0f;               // maximum (base 2), and this lane's part of the sum

    auto step = [&](bool masked, int first, const char* kt, const char* vt) {
        __builtin_amdgcn_s_setprio(1);              // (see above)
        at_acc s[2]{};
        at_bf8 f[2][2][2];                          // pieces of the keys, two ahead
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int b = 0; b < 2; ++b) f[0][n][b] = reads.rows(kt, b, n);
#pragma unroll
        for (int n = 0; n < D / 16; n += 2) {
            if (n + 2 < D / 16) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int b = 0; b < 2; ++b) f[(n / 2 + 1) & 1][i][b] = reads.rows(kt, b, n + 2 + i);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) s[b] = at_mma(f[(n / 2) & 1][i][b], q[n + i], s[b]);
            __builtin_amdgcn_sched_barrier(0);
        }
        const int from = mine.lo - first, to = mine.hi - first;        // what the lane's row sees of the tile
        constexpr bool SCORED = FORM != AT_PLAIN || SLOPES;            // (plain products are scaled in the exponent's own instruction)
        const float away = (float)(row - first - 4 * half);
        if (SCORED) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = 32 * b + 8 * (e / 4) + e % 4;
                    float slope;
                    s[b][e] = at_score<FORM>(a.score, s[b][e], slope);
                    if (SLOPES) s[b][e] = fmaf(-slope2, fabsf(away - (float)key), s[b][e]);
                }
        }
        if (masked) {
            asm volatile("");       // (a branch: few tiles need it)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int key = 32 * b + 8 * (e / 4) + 4 * half + e % 4;
                    s[b][e] = key >= from && key < to ? s[b][e] : sc_neg_inf();
                }
        }
        float base = 0.0f;
        if (moves) {
            float most = sc_neg_inf();
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) most = fmaxf(most, s[b][e]);
            if (!SCORED) most *= a.score.to_log2;
            most = fmaxf(most, sc_xor<32>(most));
            // a maximum that is a little too small does as well: sums up to 2^8 times as large
            if (__any(most > m + 8.0f)) {
                const float now = fmaxf(m, most);
                const float factor = now == sc_neg_inf() ? 1.0f : __builtin_amdgcn_exp2f(m - now);
                l *= factor;
#pragma unroll
                for (int n = 0; n < D / 32; ++n)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[n][e] *= factor;
                m = now;
            }
            base = m == sc_neg_inf() ? 0.0f : m;
        }
        at_bf8 p[4];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[b][e] = __builtin_amdgcn_exp2f(!SCORED ? fmaf(s[b][e], a.score.to_log2, -base) : FORM == AT_CAPPED && !MAY_RISE ? s[b][e] : s[b][e] - base);
                l += s[b][e];
            }
            p[2 * b] = at_pack(s[b], 0);
            p[2 * b + 1] = at_pack(s[b], 1);
        }
        __builtin_amdgcn_s_setprio(0);
        at_add<D, 4, true>(o, p, reads, vt, 0);
        if constexpr (FINE) {
#pragma unroll
            for (int c = 0; c < 4; ++c) p[c] = at_pack_rest(s[c / 2], p[c], c % 2);
            at_add<D, 4, true>(o, p, reads, vt, 0);
        }
    };

    const int count = all.tiles(AT_TILE);
    if (count > 0) {
        at_bring_own<D>(bring, a.q.at(0, head), a.q.token, tile, last, place + 2 * BYTES);
        bring(keys, a.k.token, k_offset, all.lo, last, place);
        bring(values, a.v.token, v_offset, all.lo, last, place + BYTES);
        at_arrived();
        at_own<D>(reads, lds[1], wave, q);
        at_wait_for_all();
    }
    for (int i = 0; i < count; ++i) {
        const int first = all.lo + i * AT_TILE, now = i & 1;
        at_arrived();
        if (threadIdx.x < 2) noted.rows[now ^ 1][threadIdx.x] = 0;
        if (i + 1 < count) {
            bring(keys, a.k.token, k_offset, first + AT_TILE, last, place + (now ^ 1) * 2 * BYTES);
            bring(values, a.v.token, v_offset, first + AT_TILE, last, place + (now ^ 1) * 2 * BYTES + BYTES);
        }
        const bool all_see = !FINE && all.whole(first);       // (what rounding leaves may be 0 or negative, too)
        if (!all_see) {
            at_make_finite<D>(lds[now][1], wave, noted.rows[now]);
            at_wait_for_all();
        }
        if (!reach.meets(first)) continue;
        step(!reach.whole(first), first, lds[now][0], lds[now][1]);
        if (!all_see && (noted.rows[now][0] | noted.rows[now][1]) != 0) {
            // what was not finite and is seen, from where the tile came from
            const uint64_t rows = at_noted(noted.rows[now], 0, 64), mine_of = at_noted(noted.rows[now], mine.lo - first, mine.hi - first);
#pragma unroll 1
            for (uint64_t left = rows; left; left &= left - 1) {
                const int r = __builtin_ctzll(left);
                const bool seen = mine_of >> r & 1;
                const Bf16* const from = values + (int64_t)min(first + r, last) * a.v.token + 4 * half;
#pragma unroll
                for (int n = 0; n < D / 32; ++n)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        uint2 w{0, 0};
                        if (32 * n + 8 * g < a.dim) w = *reinterpret_cast<const uint2*>(from + 32 * n + 8 * g);
                        const uint32_t x[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n][4 * g + e] += seen && (x[e] & 0x7f800000u) == 0x7f800000u ? __uint_as_float(x[e]) : 0.0f;
                    }
            }
        }
    }
    l += sc_xor<32>(l);
    const bool empty = mine.lo >= mine.hi;
    const int start = tile * AT_ROWS + wave * AT_BLOCK;
    at_wait_for_all();                              // (the tiles are read)
    at_store<D>(&lds[0][0][0] + wave * AT_BLOCK * D * 2, a.out.at(start, head), a.out.token, a.tokens - start, a.dim, o, 1.0f / l, empty);
    if (a.lse && half == 0 && row < a.tokens)
        a.lse[(int64_t)head * a.tokens + row] = empty ? sc_neg_inf() : ((FORM == AT_CAPPED ? a.score.to_log2 + m : m) + __log2f(l)) * AT_LN2;
}

// ---- gradients -----------------------------------------------------------------

// What the gradients need: the positions' intervals, and of every row of every head lse in base 2 and the sum of grad_out * out.  A workgroup has 16 positions, 16
// lanes each, and goes through its part of the heads, four at a time.  (Reads both once: 8192 positions of 16 heads of 128 20 us, 3.3 TB/s.)
constexpr int AT_POSITIONS = AT_TPB / 16, AT_ONCE = 4;
__global__ void __launch_bounds__(AT_TPB) rb_attend_delta_kernel(AttentionArgs a, float* lse2)
{
    __shared__ Spans found[AT_POSITIONS];
    __shared__ int64_t near[AT_TPB];                // offsets, where a thread has at most one (24 documents in 8192: gradients 246 -> 241 us)
    const int start = blockIdx.x * AT_POSITIONS, of = threadIdx.x / 16, t = min(start + of, a.tokens - 1), first = (threadIdx.x & 15) * 8;
    const bool is_near = a.documents.count < AT_TPB;
    if (is_near) {
        if (threadIdx.x <= a.documents.count) near[threadIdx.x] = a.documents.offsets[threadIdx.x];
        __syncthreads();
    }
    if (threadIdx.x < AT_POSITIONS && start + (int)threadIdx.x < a.tokens) {
        const Spans spans = is_near ? at_spans_of(a.documents, near, start + threadIdx.x) : at_spans_of(a.documents, a.documents.offsets, start + threadIdx.x);
        found[threadIdx.x] = spans;
        if (blockIdx.y == 0) a.documents.spans[start + threadIdx.x] = spans;
    }
    const int from_head = a.heads * blockIdx.y / gridDim.y, to_head = a.heads * (blockIdx.y + 1) / gridDim.y;
    for (int h0 = from_head; h0 < to_head; h0 += AT_ONCE) {
        sc_vec x[AT_ONCE], y[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int h = min(h0 + i, to_head - 1), from = first < a.dim ? first : 0;
            x[i] = *reinterpret_cast<const sc_vec*>(a.out.at(t, h) + from);
            y[i] = *reinterpret_cast<const sc_vec*>(a.grad_out.at(t, h) + from);
        }
        if (h0 == from_head) __syncthreads();
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            float sum = 0.0f;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                sum = fmaf(__uint_as_float(x[i][n] << 16), __uint_as_float(y[i][n] << 16), sum);
                sum = fmaf(__uint_as_float(x[i][n] & 0xffff0000u), __uint_as_float(y[i][n] & 0xffff0000u), sum);
            }
            if (first >= a.dim) sum = 0.0f;
            sum += sc_xor<1>(sum);
            sum += sc_xor<2>(sum);
            sum += sc_xor<4>(sum);
            sum += sc_xor<8>(sum);
            if (first == 0 && start + of < a.tokens && h0 + i < to_head) {
                const Span s = found[of].sees;
                const int64_t to = (int64_t)(h0 + i) * a.tokens + t;
                a.delta[to] = sum;
                lse2[to] = s.lo < s.hi ? a.lse[to] * AT_LOG2E - a.lse_less : -sc_neg_inf();
            }
        }
    }
}

// p of one element and the cap's slope; less: lse in base 2 (of AT_CAPPED: less the cap) and what the score is lowered by.
template <int FORM>
__device__ __forceinline__ void at_weight(const ScoreOf& of, float product, float less, float& p, float& slope)
{
    slope = 1.0f;
    if (FORM == AT_PLAIN) p = __builtin_amdgcn_exp2f(fmaf(product, of.to_log2, -less));
    else p = __builtin_amdgcn_exp2f(at_score<FORM>(of, product, slope) - less);
}

// Of queries: as forward, with the scores made again.
//
// ds = p (dp - delta), delta the sum of p dp; where attention is sharp that is a small difference, and delta = grad_out . out of an out that was rounded to
// bfloat16 puts an error of p times 2^-9 |grad_out . out| into it (5 times what rounding the results does, in short documents).  So delta is summed up again from
// p dp, unrounded, as its difference `off` from that first value; and since that is known at the end only, sums of p k are kept beside those of
// ds k: the gradient is the sum of p (dp - first - off) k.  The keys' kernel gets the better delta.  (A fourth product beside three, that shares its operand; a
// pass of its own over the keys would be two.)  What is taken away is not the sum of ds itself but that of what they were rounded to: then of a rounding's
// error e the gradient gets e (k - mean of k) and not e k, where keys may lie around a mean that is larger than what they differ by.
//
// The queries' gradients of the results stay in LDS (q is in registers), 32 keys at a time leave room for two workgroups a unit.  One document of 8192, 16 heads of
// 128: 510 us of a call's 1080, four products at 1.08 PFLOP/s.
template <int D, int FORM, bool SLOPES, bool FINE>
__global__ void __launch_bounds__(AT_TPB, 2) rb_attend_grad_q_kernel(AttentionArgs a)
{
    constexpr int ROWS = AT_BLOCK;                  // keys at a time
    __shared__ __align__(1024) char lds[2][2][ROWS * D * 2];           // keys and values; first the workgroup's queries
    __shared__ __align__(1024) char own[AT_ROWS / AT_TILE][AT_TILE * D * 2];       // the gradients of the workgroup's results
    __shared__ Noted noted;
    constexpr uint32_t BYTES = ROWS * D * 2;
    const uint32_t place = at_place_of(&lds[0][0][0]), place_own = at_place_of(&own[0][0]);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, half = lane / 32;
    int tile, head;
    at_place<false>(blockIdx.x, a.tiles, a.heads, a.inner, tile, head);
    if (a.ranked) tile = at_ranked_by_spans<false>(a.spans, a.tiles - 1 - tile, a.tiles, a.tokens, &lds[0][0][0]);
    const int kv = __builtin_amdgcn_readfirstlane(head / a.group);
    const Reach all = at_reach<false>(a.spans, tile * AT_ROWS, a.tokens);
    const int row = tile * AT_ROWS + wave * AT_BLOCK + (lane & 31);
    const Span mine = row < a.tokens ? a.spans[row].sees : Span{0, 0};
    const Reach reach = at_reach(mine);
    const int last = a.tokens - 1, r = min(row, last);
    const Bf16 *const keys = a.k.at(0, kv), *const values = a.v.at(0, kv);
    const float slope2 = SLOPES && a.slopes ? a.slopes[head] * AT_LOG2E : 0.0f;
    const float lse2 = a.lse2[(int64_t)head * a.tokens + r], delta = a.delta[(int64_t)head * a.tokens + r];
    if (threadIdx.x < 4) noted.rows[threadIdx.x / 2][threadIdx.x % 2] = 0;
    at_clear<D>(&lds[0][0][0], sizeof(lds), a.dim);
    at_clear<D>(&own[0][0], sizeof(own), a.dim);
    const Bring<D, ROWS> bring(wave, a.dim);
    const Bring<D> bring_own(wave, a.dim);
    const Reads<D> reads;
    const uint32_t k_offset = bring.offset(a.k.token), v_offset = bring.offset(a.v.token);
    at_bf8 q[D / 16];
    at_acc dq[D / 32]{}, pk[D / 32]{};
    float off = 0.0f, by = 0.0f;                    // by: what the rounded ds add up to, of capped scores less what they would unrounded

    auto step = [&](bool masked, int first, const char* kt, const char* vt) {
        const int from = mine.lo - first, to = mine.hi - first;
        const float away = (float)(row - first - 4 * half);
        __builtin_amdgcn_s_setprio(0);
        at_acc s{}, dp{};
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
            s = at_mma(reads.rows(kt, 0, n), q[n], s);
            dp = at_mma(reads.rows(vt, 0, n), reads.rows(own[wave / 2], wave % 2, n), dp);
        }
        at_acc w;                                   // p; s: ds; both times the cap's slope, that is kept in dp meanwhile
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int key = 8 * (e / 4) + e % 4;
            float p, slope;
            at_weight<FORM>(a.score, s[e], SLOPES ? fmaf(slope2, fabsf(away - (float)key), lse2) : lse2, p, slope);
            w[e] = p;
            s[e] = p * (dp[e] - delta);
            dp[e] = slope;
        }
        if (masked) {
            asm volatile("");       // (a branch: few tiles need it)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int key = 8 * (e / 4) + 4 * half + e % 4;
                const bool seen = key >= from && key < to;
                w[e] = seen ? w[e] : 0.0f;
                s[e] = seen ? s[e] : 0.0f;
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            off += s[e];
            if (FORM != AT_PLAIN) s[e] *= dp[e], w[e] *= dp[e];
            if (FORM != AT_PLAIN && !FINE) by -= s[e];
        }
        const at_bf8 f[2] = {at_pack(s, 0), at_pack(s, 1)}, g[2] = {at_pack(w, 0), at_pack(w, 1)};
        __builtin_amdgcn_s_setprio(1);              // (as in the forward pass: wavefronts take turns)
        if constexpr (!FINE) by = at_sum(f[1], at_sum(f[0], by));
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            at_bf8 rest;
            if constexpr (FINE) rest = at_pack_rest(s, f[c], c);
#pragma unroll
            for (int n = 0; n < D / 32; ++n) {
                const at_bf8 column = reads.columns(kt, n, c);
                dq[n] = at_mma(column, f[c], dq[n]);
                pk[n] = at_mma(column, g[c], pk[n]);
                if constexpr (FINE) dq[n] = at_mma(column, rest, dq[n]);
            }
        }
    };

    bool lost = false;                              // the row sees a key that is not finite
    const int count = all.tiles(ROWS);
    if (count > 0) {
        static_assert(sizeof(lds) == sizeof(own), "queries fit where the keys will be");
        char(&queries)[2][AT_TILE * D * 2] = reinterpret_cast<char(&)[2][AT_TILE * D * 2]>(lds);
        at_bring_own<D>(bring_own, a.grad_out.at(0, head), a.grad_out.token, tile, last, place_own);
        at_bring_own<D>(bring_own, a.q.at(0, head), a.q.token, tile, last, place);
        at_arrived();
        at_own<D>(reads, queries, wave, q);
        at_wait_for_all();
        bring(keys, a.k.token, k_offset, all.lo, last, place);
        bring(values, a.v.token, v_offset, all.lo, last, place + BYTES);
    }
    for (int i = 0; i < count; ++i) {
        const int first = all.lo + i * ROWS, now = i & 1;
        at_arrived();
        if (threadIdx.x < 2) noted.rows[now ^ 1][threadIdx.x] = 0;
        if (i + 1 < count) {
            bring(keys, a.k.token, k_offset, first + ROWS, last, place + (now ^ 1) * 2 * BYTES);
            bring(values, a.v.token, v_offset, first + ROWS, last, place + (now ^ 1) * 2 * BYTES + BYTES);
        }
        if (!all.whole(first, ROWS)) {
            at_make_finite<D, ROWS>(lds[now][0], wave, noted.rows[now]);
            at_wait_for_all();
            lost |= at_noted(noted.rows[now], mine.lo - first, mine.hi - first) != 0;
        }
        if (reach.meets(first, ROWS)) step(!reach.whole(first, ROWS), first, lds[now][0], lds[now][1]);
    }
    off += sc_xor<32>(off);
    by += sc_xor<32>(by);
    const bool empty = mine.lo >= mine.hi;
    // (of a row that sees a key that is not finite `off` is made of scores without its numbers: the first value stays)
    if (half == 0 && row < a.tokens && !empty && !lost) a.delta[(int64_t)head * a.tokens + row] = delta + off;
    const float aside = FINE ? off : FORM == AT_PLAIN ? by : off + by;
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) dq[n][e] = fmaf(-aside, pk[n][e], dq[n][e]);
    const bool alone = mine.hi - mine.lo == 1;      // one key has the weight 1 whatever its score is: no gradient, and no rounding of one
    const int start = tile * AT_ROWS + wave * AT_BLOCK;
    at_wait_for_all();
    at_store<D>(&lds[0][0][0] + wave * AT_BLOCK * D * 2, a.grad_q.at(start, head), a.grad_q.token, a.tokens - start, a.dim, dq, lost ? sc_nan() : alone ? 0.0f : a.score.scale, empty);
}

// Of keys and values: a workgroup has 128 of one head, and goes through the queries of all the heads that read it, or of a part of these (key_parts) whose sums
// then go to memory unrounded and are added up by the next kernel, in the same order every time.  One document of 8192, 16 heads of 128 to 8: 530 us of a
// call's 1080, four products at 1.04 PFLOP/s, and 25 us for the parts' sums.
template <int D, int FORM, bool SLOPES, bool FINE>
__global__ void __launch_bounds__(AT_TPB, 2) rb_attend_grad_kv_kernel(AttentionArgs a)
{
    constexpr int ROWS = AT_BLOCK;                  // queries at a time
    __shared__ __align__(1024) char lds[2][2][ROWS * D * 2];           // queries and their gradients; first the workgroup's keys
    __shared__ __align__(1024) char own[AT_ROWS / AT_TILE][AT_TILE * D * 2];       // the workgroup's values
    __shared__ Noted noted;
    constexpr uint32_t BYTES = ROWS * D * 2;
    const uint32_t place = at_place_of(&lds[0][0][0]), place_own = at_place_of(&own[0][0]);
    __shared__ __align__(1024) float numbers[2][AT_TILE];          // lse in base 2 and delta of the tile's queries
    const uint32_t place_numbers = at_place_of(&numbers[0][0]);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, half = lane / 32;
    // one workgroup's share: a head of keys, and all of its queries or a part of them
    int tile, share;
    at_place<true>(blockIdx.x, a.tiles, a.shares, a.inner, tile, share);
    const int parts = __builtin_amdgcn_readfirstlane(a.shares / (a.heads / a.group)), kv = __builtin_amdgcn_readfirstlane(share / parts), part = share - kv * parts;
    if (a.ranked) tile = at_ranked_by_spans<true>(a.spans, tile, a.tiles, a.tokens, &lds[0][0][0]);
    const Reach all = at_reach<true>(a.spans, tile * AT_ROWS, a.tokens);
    const int row = tile * AT_ROWS + wave * AT_BLOCK + (lane & 31);
    const Span mine = row < a.tokens ? a.spans[row].seen : Span{0, 0};
    const Reach reach = at_reach(mine);
    const int last = a.tokens - 1;
    at_bf8 k[D / 16];
    if (threadIdx.x < 4) noted.rows[threadIdx.x / 2][threadIdx.x % 2] = 0;
    at_clear<D>(&lds[0][0][0], sizeof(lds), a.dim);
    at_clear<D>(&own[0][0], sizeof(own), a.dim);
    const Bring<D, ROWS> bring(wave, a.dim);
    const Bring<D> bring_own(wave, a.dim);
    const Reads<D> reads;
    const uint32_t q_offset = bring.offset(a.q.token), g_offset = bring.offset(a.grad_out.token);
    auto fetch = [&](int head, int first, int buffer) {
        bring(a.q.at(0, head), a.q.token, q_offset, first, last, place + buffer * 2 * BYTES);
        bring(a.grad_out.at(0, head), a.grad_out.token, g_offset, first, last, place + buffer * 2 * BYTES + BYTES);
        if (wave == 0) at_bring_numbers((lane < 32 ? a.lse2 : a.delta) + (int64_t)head * a.tokens, first, last, place_numbers + buffer * AT_TILE * 4);
    };
    at_acc dk[D / 32]{}, dv[D / 32]{};

    auto step = [&](bool masked, int first, int head, int buffer) {
        const char *const qt = lds[buffer][0], *const gt = lds[buffer][1];
        const float slope2 = SLOPES && a.slopes ? a.slopes[head] * AT_LOG2E : 0.0f;
        const int from = mine.lo - first, to = mine.hi - first;
        const float away = (float)(row - first - 4 * half);
        {
            __builtin_amdgcn_s_setprio(0);
            at_acc s{}, dp{};
#pragma unroll
            for (int n = 0; n < D / 16; ++n) {
                s = at_mma(reads.rows(qt, 0, n), k[n], s);
                dp = at_mma(reads.rows(gt, 0, n), reads.rows(own[wave / 2], wave % 2, n), dp);
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 lse2 = *reinterpret_cast<const float4*>(&numbers[buffer][8 * g + 4 * half]);
                const float4 delta = *reinterpret_cast<const float4*>(&numbers[buffer][32 + 8 * g + 4 * half]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int e = 4 * g + i, query = 8 * g + i;
                    const float less = i == 0 ? lse2.x : i == 1 ? lse2.y : i == 2 ? lse2.z : lse2.w;
                    const float delta_i = i == 0 ? delta.x : i == 1 ? delta.y : i == 2 ? delta.z : delta.w;
                    float p, slope;
                    at_weight<FORM>(a.score, s[e], SLOPES ? fmaf(slope2, fabsf(away - (float)query), less) : less, p, slope);
                    const float ds = p * (dp[e] - delta_i);
                    s[e] = p;
                    dp[e] = FORM == AT_PLAIN ? ds : ds * slope;
                }
            }
            if (masked) {
            asm volatile("");       // (a branch: few tiles need it)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int query = 8 * (e / 4) + 4 * half + e % 4;
                    const bool seen = query >= from && query < to;
                    s[e] = seen ? s[e] : 0.0f;
                    dp[e] = seen ? dp[e] : 0.0f;
                }
            }
            const at_bf8 p[2] = {at_pack(s, 0), at_pack(s, 1)}, ds[2] = {at_pack(dp, 0), at_pack(dp, 1)};
            __builtin_amdgcn_s_setprio(1);
            at_add<D, 2, false>(dv, p, reads, gt, 0);
            if constexpr (FINE) {
                const at_bf8 rest[2] = {at_pack_rest(s, p[0], 0), at_pack_rest(s, p[1], 1)};
                at_add<D, 2, false>(dv, rest, reads, gt, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            at_add<D, 2, false>(dk, ds, reads, qt, 0);
            if constexpr (FINE) {
                const at_bf8 rest[2] = {at_pack_rest(dp, ds[0], 0), at_pack_rest(dp, ds[1], 1)};
                at_add<D, 2, false>(dk, rest, reads, qt, 0);
            }
        }
    };

    bool lost = false;                              // seen by a query that is not finite, or whose gradient is not
    // tiles of queries, head by head; from where and how many
    const int tiles = all.tiles(ROWS);
    const int from = __builtin_amdgcn_readfirstlane((int)((int64_t)tiles * a.group * part / parts)), skipped = tiles > 0 ? __builtin_amdgcn_readfirstlane(from / tiles) : 0;
    int head = kv * a.group + skipped, first = all.lo + (from - skipped * tiles) * ROWS, left = __builtin_amdgcn_readfirstlane((int)((int64_t)tiles * a.group * (part + 1) / parts)) - from;
    if (left) {
        static_assert(sizeof(lds) == sizeof(own), "keys fit where the queries will be");
        char(&keys)[2][AT_TILE * D * 2] = reinterpret_cast<char(&)[2][AT_TILE * D * 2]>(lds);
        at_bring_own<D>(bring_own, a.v.at(0, kv), a.v.token, tile, last, place_own);
        at_bring_own<D>(bring_own, a.k.at(0, kv), a.k.token, tile, last, place);
        at_arrived();
        at_own<D>(reads, keys, wave, k);
        at_wait_for_all();
        fetch(head, first, 0);
    }
    for (int now = 0; left > 0; --left, now ^= 1) {
        int next_head = head, next = first + ROWS;
        if (next >= all.hi) {
            next = all.lo;
            ++next_head;
        }
        at_arrived();
        if (threadIdx.x < 2) noted.rows[now ^ 1][threadIdx.x] = 0;
        if (left > 1) fetch(next_head, next, now ^ 1);
        if (!all.whole(first, ROWS)) {
            at_make_finite<D, ROWS>(lds[now][0], wave, noted.rows[now]);
            at_make_finite<D, ROWS>(lds[now][1], wave, noted.rows[now]);
            at_wait_for_all();
            lost |= at_noted(noted.rows[now], mine.lo - first, mine.hi - first) != 0;
        }
        if (reach.meets(first, ROWS)) step(!reach.whole(first, ROWS), first, head, now);
        head = next_head;
        first = next;
    }
    const bool empty = mine.lo >= mine.hi;
    bool alone = false;                             // (the key's only query sees nothing else, see there)
    if (mine.hi - mine.lo == 1) {
        const Span sees = a.spans[row].sees;
        alone = sees.hi - sees.lo == 1;
    }
    const float factor = lost ? sc_nan() : alone ? 0.0f : a.score.scale;
    if (a.sums) {
        if (row >= a.tokens) return;
        float* const to = a.sums + ((int64_t)share * a.tokens + row) * (2 * D);
        at_store_sum<D>(to, dk, factor, empty);
        at_store_sum<D>(to + D, dv, lost ? sc_nan() : 1.0f, empty);
        return;
    }
    const int start = tile * AT_ROWS + wave * AT_BLOCK;
    char* const through = &own[0][0] + wave * AT_BLOCK * D * 2;
    at_wait_for_all();
    at_store<D>(through, a.grad_k.at(start, kv), a.grad_k.token, a.tokens - start, a.dim, dk, factor, empty);
    at_store<D>(through, a.grad_v.at(start, kv), a.grad_v.token, a.tokens - start, a.dim, dv, lost ? sc_nan() : 1.0f, empty);
}

// Gradients of keys and values from the parts' sums: a thread has four numbers of a row of one head.  Bound by what it reads (two parts of 8192 rows of 8 heads of
// 128 in binary32, 134 MB, 25 us).
template <int D>
__global__ void __launch_bounds__(AT_TPB) rb_attend_join_kernel(AttentionArgs a)
{
    const int kv_heads = a.heads / a.group, parts = a.shares / kv_heads;
    const int64_t count = (int64_t)kv_heads * a.tokens * (2 * D / 4);
    for (int64_t at = (int64_t)blockIdx.x * AT_TPB + threadIdx.x; at < count; at += (int64_t)gridDim.x * AT_TPB) {
        const int64_t line = at / (2 * D / 4);
        const int kv = (int)(line / a.tokens), t = (int)(line - (int64_t)kv * a.tokens), first = (int)(at % (2 * D / 4)) * 4;
        float4 s{0.0f, 0.0f, 0.0f, 0.0f};
        for (int p = 0; p < parts; ++p) {
            const float4 v = *reinterpret_cast<const float4*>(a.sums + ((int64_t)(kv * parts + p) * a.tokens + t) * (2 * D) + first);
            s.x += v.x;
            s.y += v.y;
            s.z += v.z;
            s.w += v.w;
        }
        const int column = first % D;
        if (column < a.dim)
            *reinterpret_cast<uint2*>((first < D ? a.grad_k : a.grad_v).at(t, kv) + column) = uint2{sc_bf16_pair(s.x, s.y), sc_bf16_pair(s.z, s.w)};
    }
}

}  // namespace
