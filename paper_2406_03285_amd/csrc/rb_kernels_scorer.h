// Scores of tokens under rows of logits (rb_scorer_score) and their gradient (rb_scorer_grad).  Included by rb_train.hip only.
//
// Score.  A row of logits is read once, 16 bytes per lane and load.  Every lane keeps the running maximum m of what it has seen, s = sum
// of e^(z - m) and t = sum of e^(z - m) (z - m), rescaled when a tile of 32 elements brings a larger maximum; lanes, wavefronts and
// workgroups are joined by the same rule, and lse = m + log s, entropy = log s - t / s.
// Bound by HBM without alternatives (8192 x 131072 bfloat16: 368 us, 5.8 TB/s; 8.7 vector instructions per logit), by vector instructions with them
// (2048 x 50001 with 16: 51 us, 4.0 TB/s, 14.4 per logit; 5120 x 10000 binary32 with 5: 40 us, 5.2 TB/s).
// Alternatives.  A wavefront keeps its best 64 elements so far as one 64-bit key per lane, sorted: the logit in an order-preserving 32-bit
// form above the inverted index, so that equal logits order by index and no two keys are equal.  A lane whose tile holds nothing above the
// smallest key that still counts (which the running maximum tells at no cost) goes on; the others put their tile into LDS, half a wavefront
// looks at one of them at a time, what passes is queued, and a full queue is sorted and merged into the list.  So the time depends on the order of
// the logits: of rows that rise along their indices all pass (20 from end to end; 2048 x 50001 bfloat16 with 16: 114 us; one row of 32000 with 20: 15.8
// for 10.1; 5120 x 10000 binary32 with 5: 43); falling or equal ones take less than random ones (40 and 43 for 2048 x 50001).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace {

constexpr int SC_WAVE = 64;
constexpr int SC_TPB = 256;
constexpr int SC_NWAVE = SC_TPB / SC_WAVE;
constexpr int SC_MANY_WAVES = 16;                  // of a workgroup that has a row to itself while most of the chip is idle
constexpr int SC_LANE_ELEMS = 32;                  // elements of a tile per lane: 4 loads of 8 bfloat16, 8 of 4 binary32
constexpr int SC_TILE = SC_WAVE * SC_LANE_ELEMS;   // elements of a wavefront's tile
constexpr int SC_MAX_SPLITS = 64;                  // most workgroups that share a row (the last one's lanes join them)
constexpr int SC_SPLIT_GROUPS = 256;               // most workgroups of a launch whose rows are shared
constexpr float SC_LOG2E = 1.44269504088896340736f;
constexpr float SC_FLOOR = -200.0f;                // e^-200 is 0 in binary32: what is further below the maximum adds nothing, and 0 * floor is 0

typedef uint32_t sc_vec __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float sc_neg_inf() { return -__builtin_huge_valf(); }
__device__ __forceinline__ float sc_nan() { return __builtin_nanf(""); }

template <typename T> struct Logit;
template <> struct Logit<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    static __device__ __forceinline__ void unpack(const sc_vec v, float* z)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = __uint_as_float(v[i]);
    }
    static __device__ __forceinline__ float round(float x) { return x; }
    static __device__ __forceinline__ sc_vec pack(const float* z)
    {
        return sc_vec{__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3])};
    }
};
struct Bf16 { uint16_t bits; };
typedef __bf16 sc_bf16x2 __attribute__((ext_vector_type(2)));
typedef float sc_floatx2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t sc_bf16_pair(float a, float b)      // to nearest, ties to even; NaN stays NaN (one instruction)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((sc_floatx2{a, b}), sc_bf16x2));
}
__device__ __forceinline__ uint32_t sc_bf16_bits(float x) { return sc_bf16_pair(x, x) & 0xffffu; }
template <> struct Logit<Bf16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float one(const Bf16* p) { return __uint_as_float((uint32_t)p->bits << 16); }
    static __device__ __forceinline__ void unpack(const sc_vec v, float* z)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            z[2 * i] = __uint_as_float(v[i] << 16);
            z[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ Bf16 round(float x) { return Bf16{(uint16_t)sc_bf16_bits(x)}; }
    static __device__ __forceinline__ sc_vec pack(const float* z)
    {
        sc_vec v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = sc_bf16_pair(z[2 * i], z[2 * i + 1]);
        return v;
    }
};

// A row cut into what lies before the first 16-byte boundary, whole 16-byte vectors, and the rest.
template <typename T>
struct RowSpan {
    int head, vectors, tail;
    const sc_vec* body;
    __device__ __forceinline__ RowSpan(const T* row, int vocab)
    {
        const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        head = off ? min(Logit<T>::N - off, vocab) : 0;
        vectors = (vocab - head) / Logit<T>::N;
        tail = vocab - head - vectors * Logit<T>::N;
        body = reinterpret_cast<const sc_vec*>(row + head);
    }
};

// ---- between lanes -----------------------------------------------------------

// The value of lane ^ D, without a trip through LDS.
template <int D>
__device__ __forceinline__ uint32_t sc_xor(uint32_t v)
{
    static_assert(D == 1 || D == 2 || D == 4 || D == 8 || D == 16 || D == 32, "a power of two within a wavefront");
    const int x = (int)v;
    if constexpr (D == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, false);             // quad_perm 1 0 3 2
    if constexpr (D == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, false);             // quad_perm 2 3 0 1
    if constexpr (D == 4) return (uint32_t)__builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, false), 0x1B, 0xf, 0xf, false);   // halves of a row mirrored, quads mirrored
    if constexpr (D == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false);            // rows of 16 turned by 8
    if constexpr (D == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);      // [0]: odd rows hold the even ones, [1]: even rows the odd ones
        return threadIdx.x & 16 ? r[0] : r[1];
    }
    if constexpr (D == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
}
template <int D> __device__ __forceinline__ float sc_xor(float v) { return __uint_as_float(sc_xor<D>(__float_as_uint(v))); }
template <int D> __device__ __forceinline__ uint64_t sc_xor(uint64_t v)
{
    return ((uint64_t)sc_xor<D>((uint32_t)(v >> 32)) << 32) | sc_xor<D>((uint32_t)v);
}
// Lane i's value in lane 63 - i.
__device__ __forceinline__ uint64_t sc_reverse(uint64_t v)
{
    auto mirror = [](uint32_t x) { return sc_xor<32>(sc_xor<16>((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, false))); };   // row_mirror
    return ((uint64_t)mirror((uint32_t)(v >> 32)) << 32) | mirror((uint32_t)v);
}
__device__ __forceinline__ uint64_t sc_lane(uint64_t v, int lane)          // the same lane for all
{
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// ---- running maximum and sums ------------------------------------------------

struct Stats {
    float m, s, t;      // maximum (NaN left out), sum of e^(z - m), sum of e^(z - m) (z - m)
};

// m as something to subtract: 0 where there is nothing but -inf (every e^(-inf - 0) is 0)
__device__ __forceinline__ float sc_base(float m) { return m == sc_neg_inf() ? 0.0f : m; }

__device__ __forceinline__ Stats sc_rebase(const Stats a, float m)
{
    const float d = fmaxf(a.m - sc_base(m), SC_FLOOR);             // a.m <= m; -inf and NaN (inf - inf) go to the floor
    const float f = a.m == m ? 1.0f : __builtin_amdgcn_exp2f(d * SC_LOG2E);
    return Stats{m, a.s * f, f * fmaf(a.s, a.m == m ? 0.0f : d, a.t)};
}

__device__ __forceinline__ Stats sc_join(const Stats a, const Stats b)
{
    const float m = fmaxf(a.m, b.m);
    const Stats x = sc_rebase(a, m), y = sc_rebase(b, m);
    return Stats{m, x.s + y.s, x.t + y.t};
}

template <int D>
__device__ __forceinline__ Stats sc_join_xor(const Stats a) { return sc_join(a, Stats{sc_xor<D>(a.m), sc_xor<D>(a.s), sc_xor<D>(a.t)}); }
__device__ __forceinline__ Stats sc_join_wave(const Stats a)
{
    return sc_join_xor<1>(sc_join_xor<2>(sc_join_xor<4>(sc_join_xor<8>(sc_join_xor<16>(sc_join_xor<32>(a))))));
}

template <int COUNT>
__device__ __forceinline__ float sc_max(const float* z)
{
    float m = z[0];
#pragma unroll
    for (int i = 1; i < COUNT; ++i) m = fmaxf(m, z[i]);
    return m;
}

template <int COUNT>
__device__ __forceinline__ void sc_absorb(Stats& a, const float* z, float tile_max)
{
    a = sc_rebase(a, fmaxf(a.m, tile_max));
    const float base = sc_base(a.m);
    float s0 = 0.0f, s1 = 0.0f, t0 = 0.0f, t1 = 0.0f;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const float d = z[i] - base, e = __builtin_amdgcn_exp2f(d * SC_LOG2E), c = fmaxf(d, SC_FLOOR);
        if (i & 1) {
            s1 += e;
            t1 = fmaf(e, c, t1);
        } else {
            s0 += e;
            t0 = fmaf(e, c, t0);
        }
    }
    a.s += s0 + s1;
    a.t += t0 + t1;
}

// ---- the best elements -------------------------------------------------------

__device__ __forceinline__ uint32_t sc_order(float z)              // orders as the numbers do, -0 as +0
{
    const uint32_t u = __float_as_uint(z + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float sc_unorder(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ uint64_t sc_key(float z, uint32_t index) { return ((uint64_t)sc_order(z) << 32) | (uint32_t)~index; }

template <int D, typename K>
__device__ __forceinline__ K sc_exchange(K key, bool keep_larger)
{
    const K other = sc_xor<D>(key);
    return (key > other) == keep_larger ? key : other;             // (equal keys: either)
}

// Runs of SIZE lanes whose keys rise and then fall (or the other way round), put in order: downwards where `down`.
template <int SIZE, typename K>
__device__ __forceinline__ K sc_bitonic(K key, bool down)
{
    if constexpr (SIZE > 1) {
        constexpr int D = SIZE / 2;
        key = sc_exchange<D>(key, ((threadIdx.x & D) == 0) == down);
        return sc_bitonic<D>(key, down);
    }
    return key;
}

// The keys of the wavefront's first `count` lanes, largest in lane 0; the others' are 0.
template <typename K>
__device__ __forceinline__ K sc_sort(K key, int count)
{
    key = sc_bitonic<2>(key, (threadIdx.x & 2) == 0);
    key = sc_bitonic<4>(key, (threadIdx.x & 4) == 0);
    key = sc_bitonic<8>(key, (threadIdx.x & 8) == 0);
    key = sc_bitonic<16>(key, (threadIdx.x & 16) == 0);
    if (count > 16) key = sc_bitonic<32>(key, (threadIdx.x & 32) == 0);
    if (count > 32) key = sc_bitonic<64>(key, true);
    return key;
}

// The 64 largest of two sorted lists, sorted.
__device__ __forceinline__ uint64_t sc_merge(uint64_t a, uint64_t b)
{
    b = sc_reverse(b);
    return sc_bitonic<64>(a > b ? a : b, true);
}

__device__ __forceinline__ void sc_lds_wait() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// A wavefront's list and the queue in LDS before it.  WAVES that share a row tell each other what they hold: the value that `share` of a
// wavefront's elements reach.  WAVES * share >= top elements reach the least of these, and what is below that is wanted by none.
template <int WAVES>
struct Best {
    uint64_t list;        // lane i: the (i + 1)-th largest key so far, 0: none
    uint64_t least;       // the key of the last place that counts: what is not above it is not wanted
    uint64_t* queue;      // 2 * SC_WAVE keys
    uint32_t* told;       // sc_order of the values, one per wavefront, 0: nothing told yet
    int queued, top, share;

    __device__ __forceinline__ Best(uint64_t* q, uint32_t* told_, int top_)
        : list(0), least(0), queue(q), told(told_), queued(0), top(top_), share((top_ + WAVES - 1) / WAVES) {}

    __device__ __forceinline__ void tell(uint32_t order)
    {
        if (WAVES > 1 && (threadIdx.x & (SC_WAVE - 1)) == 0) __hip_atomic_store(told + threadIdx.x / SC_WAVE, order, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    // sc_order of the least value that is still wanted: above the list's last (an element that equals it comes with a higher index), and what all reach
    __device__ __forceinline__ uint32_t wanted() const
    {
        const uint32_t own = least == 0 ? 0 : (uint32_t)(least >> 32) + 1;
        if (WAVES == 1) return own;
        uint32_t all = __hip_atomic_load(told + threadIdx.x % WAVES, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        if (WAVES > 1) all = min(all, sc_xor<1>(all));
        if (WAVES > 2) all = min(all, sc_xor<2>(all));
        if (WAVES > 4) all = min(all, sc_xor<4>(all));
        if (WAVES > 8) all = min(all, sc_xor<8>(all));
        return max(own, (uint32_t)__builtin_amdgcn_readfirstlane((int)all));
    }
    __device__ __forceinline__ void merge_first()
    {
        const int lane = threadIdx.x & (SC_WAVE - 1), now = min(queued, SC_WAVE);
        sc_lds_wait();
        uint64_t key = lane < queued ? queue[lane] : 0;
        const uint64_t rest = SC_WAVE + lane < queued ? queue[SC_WAVE + lane] : 0;
        sc_lds_wait();
        queue[lane] = rest;
        queued = max(queued - SC_WAVE, 0);
        key = sc_sort(key, now);
        list = sc_lane(list, 0) == 0 ? key : sc_merge(list, key);
        least = sc_lane(list, top - 1);
        if (WAVES > 1) tell((uint32_t)(sc_lane(list, share - 1) >> 32));
    }
    __device__ __forceinline__ void push(uint64_t key, bool wanted)
    {
        const uint64_t who = __ballot(wanted && key > least);
        if (who == 0) return;
        if (wanted && key > least) queue[queued + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = key;
        queued += __popcll(who);
        if (queued >= SC_WAVE) merge_first();
    }
    __device__ __forceinline__ void flush()
    {
        while (queued > 0) merge_first();
    }
};

// ---- one row's share of a wavefront ------------------------------------------

constexpr int SC_STAGED = 16;        // lanes whose elements are in LDS at a time

template <typename T>
struct Staged {
    T elements[SC_STAGED][SC_LANE_ELEMS];
    int32_t lanes[SC_STAGED];
};

// Tiles part, part + parts, ... of the row; the elements at its unaligned ends fall to part 0.
template <typename T, bool TOP, int WAVES>
__device__ __forceinline__ void sc_scan(const T* row, int vocab, int part, int parts, Stats& stats, Best<WAVES>& best, Staged<T>* staged)
{
    constexpr int N = Logit<T>::N, U = SC_LANE_ELEMS / N;
    const int lane = threadIdx.x & (SC_WAVE - 1);
    const RowSpan<T> span(row, vocab);
    const int tiles = (span.vectors + SC_WAVE * U - 1) / (SC_WAVE * U);
    bool first = true;
    if (TOP && WAVES > 1 && part >= tiles) __syncthreads();        // a wavefront without a tile tells nothing, and is met all the same
    for (int tile = part; tile < tiles; tile += parts) {
        const int v0 = tile * (SC_WAVE * U) + lane;
        sc_vec v[U];
        if (v0 - lane + SC_WAVE * U <= span.vectors) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = span.body[v0 + u * SC_WAVE];
        } else {
            const uint32_t none = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;      // -inf: two bfloat16 or one binary32
#pragma unroll
            for (int u = 0; u < U; ++u) {
                v[u] = sc_vec{none, none, none, none};
                if (v0 + u * SC_WAVE < span.vectors) v[u] = span.body[v0 + u * SC_WAVE];
            }
        }
        float z[SC_LANE_ELEMS];
#pragma unroll
        for (int u = 0; u < U; ++u) Logit<T>::unpack(v[u], z + u * N);
        const float tile_max = sc_max<SC_LANE_ELEMS>(z);
        sc_absorb<SC_LANE_ELEMS>(stats, z, tile_max);
        if (TOP) {
            const bool any = v0 < span.vectors;
            const bool meet = WAVES > 1 && first;                  // (all wavefronts meet once, behind their first tile)
            uint32_t least = meet ? 0 : best.wanted();
            const uint32_t highest = any ? sc_order(tile_max) : 0;
            uint64_t who = __ballot(any && highest >= least);
            if (who != 0) {
                if (first || __popcll(who) > 16) {
                    // At least `top` elements reach the top-th largest of the lanes' maxima (fewer lanes than that: all are looked at).
                    const uint32_t sorted = sc_sort(highest, SC_WAVE);
                    least = max(least, (uint32_t)__builtin_amdgcn_readlane((int)sorted, best.top - 1));
                    if (meet) {
                        best.tell((uint32_t)__builtin_amdgcn_readlane((int)sorted, best.share - 1));
                        __syncthreads();
                        least = max(least, best.wanted());
                    }
                    who = __ballot(any && highest >= least);
                }
                while (who != 0) {
                    // the first lanes of them put their elements into LDS; then half a wavefront looks at one lane's
                    const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
                    const bool mine = ((who >> lane) & 1) != 0 && rank < SC_STAGED;
                    if (mine) {
#pragma unroll
                        for (int u = 0; u < U; ++u) *reinterpret_cast<sc_vec*>(&staged->elements[rank][u * N]) = v[u];
                        staged->lanes[rank] = lane;
                    }
                    const int count = min(__popcll(who), SC_STAGED);
                    who &= ~__ballot(mine);
                    sc_lds_wait();
                    for (int at = lane / SC_LANE_ELEMS; at - lane / SC_LANE_ELEMS < count; at += 2) {
                        const int from = min(at, count - 1), e = lane & (SC_LANE_ELEMS - 1);
                        const int vector = tile * (SC_WAVE * U) + e / N * SC_WAVE + staged->lanes[from];
                        const float x = Logit<T>::one(&staged->elements[from][e]);
                        best.push(sc_key(x, (uint32_t)(span.head + vector * N + e % N)), at < count && vector < span.vectors && sc_order(x) >= least);
                    }
                }
                if (first) best.flush();
                first = false;
            }
        }
    }
    if (part == 0 && span.head + span.tail > 0) {
        const int j = lane < span.head ? lane : lane >= SC_WAVE / 2 && lane - SC_WAVE / 2 < span.tail ? vocab - span.tail + lane - SC_WAVE / 2 : -1;
        const float x = j >= 0 ? Logit<T>::one(row + j) : sc_neg_inf();
        sc_absorb<1>(stats, &x, fmaxf(x, sc_neg_inf()));
        if (TOP) best.push(sc_key(x, (uint32_t)j), j >= 0);
    }
    if (TOP) best.flush();
}

struct ScoreArgs {
    const void* logits;
    int64_t stride;                 // elements between rows
    const int64_t* tokens;
    float *logp, *lse, *entropy, *top_logp;
    int64_t* top_ids;
    uint32_t* counters;             // per row that is shared: workgroups that have left their part (0 between launches)
    char* partials;                 // per workgroup of a shared row: Stats, then `top` keys
    int32_t rows, vocab, given, top, splits;
};

__host__ __device__ inline size_t sc_partial_bytes(int top) { return 16 + 8 * (size_t)top; }

// The logit of the lane's given token, fetched before the row is gone through.
struct Given {
    float logit;
    bool there;
};
template <typename T>
__device__ __forceinline__ Given sc_given(const ScoreArgs& a, const T* z, int64_t row)
{
    Given g{0.0f, false};
    const int lane = threadIdx.x & (SC_WAVE - 1);
    if (lane < a.given) {
        const int64_t t = a.tokens[row * a.given + lane];
        g.there = t >= 0 && t < a.vocab;
        if (g.there) g.logit = Logit<T>::one(z + t);
    }
    return g;
}

// What a wavefront that knows a whole row writes.
__device__ __forceinline__ void sc_finish(const ScoreArgs& a, int64_t row, const Stats st, uint64_t list, const Given& given)
{
    const int lane = threadIdx.x & (SC_WAVE - 1);
    const bool empty = st.m == sc_neg_inf() && st.s == 0.0f;
    const float log_s = logf(st.s);
    const float lse = empty ? sc_neg_inf() : st.m + log_s;
    const bool broken = lse != lse;
    if (lane == 0) {
        if (a.lse != nullptr) a.lse[row] = lse;
        if (a.entropy != nullptr) a.entropy[row] = empty ? 0.0f : broken ? lse : log_s - st.t / st.s;
    }
    if (lane < a.given) {
        const float x = given.logit;
        a.logp[row * a.given + lane] = !given.there ? 0.0f : broken ? lse : x == sc_neg_inf() ? x : (x - st.m) - log_s;      // (x - lse would be off by lse's last bit)
    }
    if (lane < a.top) {
        const float x = sc_unorder((uint32_t)(list >> 32));
        a.top_logp[row * a.top + lane] = broken ? lse : x == sc_neg_inf() ? x : (x - st.m) - log_s;
        a.top_ids[row * a.top + lane] = broken ? -1 : (int64_t)(uint32_t)~(uint32_t)list;
    }
}

// A wavefront per row (WAVES 1, in workgroups of four: short rows), or a workgroup of WAVES per row or per 1 / splits of one.
template <typename T, bool TOP, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? SC_TPB : WAVES * SC_WAVE) void rb_score_kernel(const ScoreArgs a)
{
    constexpr int LISTS = WAVES == 1 ? SC_NWAVE : WAVES;
    __shared__ uint64_t queues[LISTS][TOP ? 2 * SC_WAVE : 1];
    __shared__ __align__(16) Staged<T> staged[TOP ? LISTS : 1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / SC_WAVE), lane = threadIdx.x & (SC_WAVE - 1);
    Stats st{sc_neg_inf(), 0.0f, 0.0f};
    if (WAVES == 1) {
        const int64_t row = (int64_t)blockIdx.x * SC_NWAVE + wave;
        if (row >= a.rows) return;
        const T* z = static_cast<const T*>(a.logits) + row * a.stride;
        Best<1> best(queues[wave], nullptr, a.top);
        const Given given = sc_given(a, z, row);
        sc_scan<T, TOP, 1>(z, a.vocab, 0, 1, st, best, &staged[TOP ? wave : 0]);
        sc_finish(a, row, sc_join_wave(st), best.list, given);
        return;
    }
    __shared__ Stats stats[LISTS];
    __shared__ uint32_t told[WAVES];
    const int64_t row = blockIdx.x / (uint32_t)a.splits;
    const int split = blockIdx.x % (uint32_t)a.splits;
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    if (TOP) {
        if (threadIdx.x < WAVES) told[threadIdx.x] = 0;
        __syncthreads();
    }
    Best<WAVES> best(queues[wave], told, a.top);
    Given given{};
    if (wave == 0) given = sc_given(a, z, row);
    sc_scan<T, TOP, WAVES>(z, a.vocab, split * WAVES + wave, a.splits * WAVES, st, best, &staged[TOP ? wave : 0]);
    st = sc_join_wave(st);
    if (lane == 0) stats[wave] = st;
    uint64_t list = best.list;
    if (TOP) {
        // half of the lists into the other half, and so on
        queues[wave][lane] = list;
#pragma unroll
        for (int d = WAVES / 2; d > 0; d >>= 1) {
            __syncthreads();
            if (wave < d) {
                list = sc_merge(list, queues[wave + d][lane]);
                queues[wave][lane] = list;
            }
        }
    } else {
        __syncthreads();
    }
    if (wave != 0) return;
    st = sc_join_wave(lane < WAVES ? stats[lane] : Stats{sc_neg_inf(), 0.0f, 0.0f});
    if (a.splits > 1) {
        // Every workgroup leaves its part; the one that is last to do so joins them, in the order of the parts whoever it is.
        const size_t bytes = sc_partial_bytes(a.top);
        char* mine = a.partials + (size_t)blockIdx.x * bytes;
        if (lane == 0) *reinterpret_cast<Stats*>(mine) = st;
        if (TOP && lane < a.top) reinterpret_cast<uint64_t*>(mine + 16)[lane] = list;
        __threadfence();
        uint32_t before = 0;
        if (lane == 0) before = __hip_atomic_fetch_add(a.counters + row, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        before = __builtin_amdgcn_readfirstlane(before);
        if (before != (uint32_t)a.splits - 1) return;
        __threadfence();
        if (lane == 0) __hip_atomic_store(a.counters + row, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const char* parts = a.partials + (size_t)row * a.splits * bytes;
        st = Stats{sc_neg_inf(), 0.0f, 0.0f};
        if (lane < a.splits) st = *reinterpret_cast<const Stats*>(parts + lane * bytes);
        st = sc_join_wave(st);
        if (TOP) {
            list = 0;
            for (int p = 0; p < a.splits; ++p) list = sc_merge(list, lane < a.top ? reinterpret_cast<const uint64_t*>(parts + p * bytes + 16)[lane] : 0);
        }
    }
    sc_finish(a, row, st, list, given);
}

// ---- gradient ----------------------------------------------------------------

struct GradArgs {
    const void* logits;
    void* grad;
    int64_t stride, grad_stride;
    const int64_t* tokens;
    const float *lse, *entropy, *grad_logp, *grad_entropy;
    int32_t vocab, given, chunk;    // chunk: accesses (vectors, or elements) of a row per workgroup
};

constexpr int GR_MAX_TILES = 32;    // tiles of SC_TPB accesses in a chunk: one bit each says whether a given token is in it

// Bound by HBM: each logit read once, each gradient written once (8192 x 131072 bfloat16: 814 us, 5.3 TB/s; 1024 x 50001 with 17 given tokens: 38 us).
// A workgroup per row (blockIdx.x) and chunk of the row (blockIdx.y).  N elements per access: 16 bytes, or one element where logits and
// gradient lie differently relative to 16 bytes.  Which of a thread's accesses hold a given token is one word of bits, so that the rest
// costs one test; the tokens' sums are made in the order in which they were given.
template <typename T, int N, bool ENTROPY>
__global__ __launch_bounds__(SC_TPB) void rb_score_grad_kernel(const GradArgs a)
{
    __shared__ uint32_t hit[SC_TPB];
    __shared__ int32_t ids[64];
    __shared__ float weights[64];
    const int64_t row = blockIdx.x;
    const T* z = static_cast<const T*>(a.logits) + row * a.stride;
    T* dz = static_cast<T*>(a.grad) + row * a.grad_stride;
    const float lse = a.lse[row];
    const float h = ENTROPY ? a.grad_entropy[row] : 0.0f, entropy = ENTROPY ? a.entropy[row] : 0.0f;
    int head = 0, count = a.vocab, tail = 0;
    if (N > 1) {
        const RowSpan<T> span(z, a.vocab);
        head = span.head;
        count = span.vectors;
        tail = span.tail;
    }
    const int begin = blockIdx.y * a.chunk, end = min(begin + a.chunk, count);
    const int lane = threadIdx.x & (SC_WAVE - 1);
    int id = -1;
    float w = 0.0f;
    if (lane < a.given) {
        const int64_t t = a.tokens[row * a.given + lane];
        if (t >= 0 && t < a.vocab) {
            id = (int)t;
            w = a.grad_logp[row * a.given + lane];
        }
    }
    float sum = w;
    sum += sc_xor<32>(sum);
    sum += sc_xor<16>(sum);
    sum += sc_xor<8>(sum);
    sum += sc_xor<4>(sum);
    sum += sc_xor<2>(sum);
    sum += sc_xor<1>(sum);
    hit[threadIdx.x] = 0;
    __syncthreads();
    if (threadIdx.x < 64) {
        ids[lane] = id;
        weights[lane] = w;
        const int at = id < head ? -1 : (id - head) / N;
        if (id >= 0 && at >= begin && at < end) atomicOr(&hit[(at - begin) % SC_TPB], 1u << ((at - begin) / SC_TPB));
    }
    __syncthreads();
    const uint32_t mine = hit[threadIdx.x];
    const bool dead = lse == sc_neg_inf();
    const float rest = fmaf(h, entropy, sum);
    auto value = [&](float x) {
        const float d = x - lse, p = __builtin_amdgcn_exp2f(d * SC_LOG2E);
        return -p * (ENTROPY ? fmaf(h, fmaxf(d, SC_FLOOR), rest) : sum);
    };
    // what is given for COUNT elements from `first` on
    auto given = [&](float* x, int first, auto count) {
        for (int g = 0; g < a.given; ++g) {
            const int at = ids[g] - first;
            const float v = weights[g];
#pragma unroll
            for (int i = 0; i < decltype(count)::value; ++i) x[i] += at == i ? v : 0.0f;
        }
    };
    using One = std::integral_constant<int, 1>;
    if (N > 1) {
        constexpr int U = 4;
        const sc_vec* src = reinterpret_cast<const sc_vec*>(z + head);
        sc_vec* dst = reinterpret_cast<sc_vec*>(dz + head);
        int tile = 0;
        for (int i0 = begin + threadIdx.x; i0 < end; i0 += U * SC_TPB, tile += U) {
            sc_vec v[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u * SC_TPB < end) v[u] = src[i0 + u * SC_TPB];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i0 + u * SC_TPB >= end) continue;
                float x[Logit<T>::N];
                Logit<T>::unpack(v[u], x);
#pragma unroll
                for (int i = 0; i < Logit<T>::N; ++i) x[i] = value(x[i]);
                if ((mine >> (tile + u)) & 1u) given(x, head + (i0 + u * SC_TPB) * N, std::integral_constant<int, Logit<T>::N>());
                if (dead) {
#pragma unroll
                    for (int i = 0; i < Logit<T>::N; ++i) x[i] = 0.0f;
                }
                dst[i0 + u * SC_TPB] = Logit<T>::pack(x);
            }
        }
        if (blockIdx.y == 0 && threadIdx.x < head + tail) {
            const int j = threadIdx.x < head ? threadIdx.x : a.vocab - tail + (int)threadIdx.x - head;
            float x = value(Logit<T>::one(z + j));
            given(&x, j, One());
            dz[j] = Logit<T>::round(dead ? 0.0f : x);
        }
    } else {
        int tile = 0;
        for (int i = begin + threadIdx.x; i < end; i += SC_TPB, ++tile) {
            float x = value(Logit<T>::one(z + i));
            if ((mine >> tile) & 1u) given(&x, i, One());
            dz[i] = Logit<T>::round(dead ? 0.0f : x);
        }
    }
}

__global__ __launch_bounds__(SC_TPB) void rb_train_clear_kernel(uint32_t* p, int64_t words)
{
    for (int64_t i = (int64_t)blockIdx.x * SC_TPB + threadIdx.x; i < words; i += (int64_t)gridDim.x * SC_TPB) p[i] = 0;
}

}  // namespace
