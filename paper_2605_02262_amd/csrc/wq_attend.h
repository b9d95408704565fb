// What the attention kernels of many query rows over plain rows and over packed caches are made of (wq_attend.hip, wq_tree.hip; what it
// computes and what bounds it stand there): a wavefront's products and weights, tiles on their way into LDS, a packed cache's walk, the parts' merge.
#pragma once
#include <float.h>
#include <math.h>
#include <type_traits>

#include "wq_internal.h"

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

struct Bf16 {};
struct F16 {};
struct F32 {};

constexpr int COLS = 2;                            // 16-row columns of a wavefront
// fp32: four wavefronts of 32 rows, 32 keys at a time.  16-bit types: two groups of four wavefronts, 64 keys at a time.
template <typename CT> constexpr int WAVES = std::is_same_v<CT, F32> ? 4 : 8;
template <typename CT> constexpr int KEYS = std::is_same_v<CT, F32> ? 32 : 64;
// The reference of a row's exponents moves only when a logit exceeds it by SLACK (weights of up to 2^SLACK); fp16 weights are kept 2^SHIFT too
// large, so that one is lost only below 2^-34 of the largest (SHIFT + SLACK < 16).  Other types have the range of fp32, which their
// values use too: their numerators are kept as small as can be.
constexpr float SLACK = 5.f;
template <typename CT> constexpr float SHIFT = std::is_same_v<CT, F16> ? 10.f : 0.f;

template <typename CT> constexpr int ESIZE = std::is_same_v<CT, F32> ? 4 : 2;
template <typename CT, int HD> constexpr int STEPS = HD * ESIZE<CT> / 64;          // products of a key tile: 32 (16) channels each
template <typename CT> constexpr int VSTEPS = KEYS<CT> * ESIZE<CT> / 64;           // products over a tile's keys: 32 (16) keys each
template <typename CT, int HD> constexpr int TILE_BYTES = KEYS<CT> * HD * ESIZE<CT>;   // a staged tile of keys, or of values
template <typename CT, int HD, int N> using QueryRows = u4[N][STEPS<CT, HD>];      // B operands of N columns of rows
template <typename CT, int HD> using Query = QueryRows<CT, HD, COLS>;              // ... of a wavefront's
typedef __attribute__((address_space(3))) char* Lds;
typedef __attribute__((address_space(3))) u4* Lds4;
typedef __attribute__((address_space(3))) uint32_t* Lds1;

template <typename CT>
__device__ __forceinline__ f4 product(u4 a, u4 b, f4 c)
{
    if constexpr (std::is_same_v<CT, Bf16>) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
    } else if constexpr (std::is_same_v<CT, F16>) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
        return c;
    }
}

// (one conversion instruction per pair, to nearest even)
__device__ __forceinline__ uint32_t pack2(float x, float y, Bf16)
{
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, b2{(__bf16)x, (__bf16)y});
}
__device__ __forceinline__ uint32_t pack2(float x, float y, F16)
{
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, h2{(_Float16)x, (_Float16)y});
}

// ---- a wavefront's part of the arithmetic ------------------------------------------------------------------------------
template <int HD>
struct Rows {
    f4 o[HD / 16][COLS];       // numerators: channel 16 ct + 4 (lane / 16) + i of row lane % 16
    float ref[COLS];           // reference of the exponents (log2), -inf before the first visible key
    float sum[COLS];           // this lane's part of the sum of weights
    float scale[COLS];         // log2(e) * sm_scale, times the power of two that the query was divided by
    int limit[COLS];           // the row sees the keys below it
};

template <int HD>
__device__ __forceinline__ void clear(Rows<HD>& r)
{
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        r.ref[n] = -INFINITY;
        r.sum[n] = 0.f;
#pragma unroll
        for (int ct = 0; ct < HD / 16; ct++) r.o[ct][n] = f4{0.f, 0.f, 0.f, 0.f};
    }
}

// (a scalar: what follows from it is one branch for the wavefront, not a mask)
__device__ __forceinline__ int this_wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

__device__ __forceinline__ float max_of_column(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16, 64));
    return fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float sum_of_column(float x)
{
    x += __shfl_xor(x, 16, 64);
    return x + __shfl_xor(x, 32, 64);
}

// The order in which a tile's weights go into the value product's operand: register e holds the weights of the keys first(e) and
// second(e) of the lane's eight (its four of the first 16 keys, then of the second).  Free, as long as the values' operand has the
// same: a packed class is expanded fastest with the pairs that its masks leave in the two halves of a register.
struct Natural {
    static constexpr int first(int e) { return 2 * e; }
    static constexpr int second(int e) { return 2 * e + 1; }
};
struct Far {                   // 2- and 4-bit codes
    static constexpr int first(int e) { return e; }
    static constexpr int second(int e) { return e + 4; }
};
struct Near {                  // 8-bit codes
    static constexpr int first(int e) { return 4 * (e >> 1) + (e & 1); }
    static constexpr int second(int e) { return first(e) + 2; }
};

template <typename CT> using Products = f4[KEYS<CT> / 16][COLS];          // of a tile's keys and a wavefront's rows
template <typename CT> using Weights = u4[VSTEPS<CT>][COLS];              // B operands of the value products

// keys(t, st): this lane's part of the A operand.  Operands are read from LDS one 16-key tile ahead (and no more: left to itself the compiler
// reads all of them first, and spills).
template <typename CT, int HD, typename Keys>
__device__ __forceinline__ void multiply_keys(Products<CT>& s, const Query<CT, HD>& q, const Keys& keys)
{
    constexpr int T = KEYS<CT> / 16, ST = STEPS<CT, HD>;
    u4 a[2][ST];
#pragma unroll
    for (int st = 0; st < ST; st++) a[0][st] = keys(0, st);
#pragma unroll
    for (int t = 0; t < T; t++) {
        if (t + 1 < T) {
#pragma unroll
            for (int st = 0; st < ST; st++) a[(t + 1) & 1][st] = keys(t + 1, st);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < COLS; n++) s[t][n] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < ST; st++)
#pragma unroll
            for (int n = 0; n < COLS; n++) s[t][n] = product<CT>(a[t & 1][st], q[n][st], s[t][n]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// A packed class's codes as they are, for fp16 queries: the group's scale and minimum are applied to the sums in fp32,
//     q.k^ = sum over the head's groups g of  s_g (q.code)_g + m_g (sum of q)_g
// A key rounded to fp16 would be off by 3.0e-4 of a result whose own rounding is 2.1e-4, for two vector operations less per logit and group: us per call of
// 64 requests over 51200 tokens, rounded -> as codes: heads of 128 in one, two and four groups 92 -> 97, 103, 119, heads of 64 in one and two 44 -> 48, 52.
// metas(t, g): the scales and minima of this lane's four keys, read one group ahead.  A group's sums are finished behind the products of the next (all groups
// of 16 keys at once, or the minima as one more matrix product, took more registers than there are: 107, 106 for two groups).
template <int HD, int G, typename Keys, typename Metas>
__device__ __forceinline__ void multiply_codes(Products<F16>& s, const Query<F16, HD>& q, const float (&q_sum)[COLS][G], const Keys& keys, const Metas& metas)
{
    constexpr int T = KEYS<F16> / 16, ST = STEPS<F16, HD>, PER = ST / G;
    u4 a[2][ST];
    u4 sm[2];
    f4 x[2][COLS];
    sm[0] = metas(0, 0);
#pragma unroll
    for (int st = 0; st < ST; st++) a[0][st] = keys(0, st);
#pragma unroll
    for (int j = 0; j <= T * G; j++) {
        const int t = j / G, g = j % G;
        if (g == 0 && t + 1 < T) {
#pragma unroll
            for (int st = 0; st < ST; st++) a[(t + 1) & 1][st] = keys(t + 1, st);
        }
        if (j > 0 && j < T * G) sm[j & 1] = metas(t, g);
        __builtin_amdgcn_sched_barrier(0);
        if (t < T) {
#pragma unroll
            for (int n = 0; n < COLS; n++) x[j & 1][n] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = g * PER; st < (g + 1) * PER; st++)
#pragma unroll
                for (int n = 0; n < COLS; n++) x[j & 1][n] = product<F16>(a[t & 1][st], q[n][st], x[j & 1][n]);
        }
        if (j > 0) {
            const int bt = (j - 1) / G, bg = (j - 1) % G;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t word = sm[(j - 1) & 1][i];      // (the cast of a vector's element would read its first)
                const h2 f = __builtin_bit_cast(h2, word);
#pragma unroll
                for (int n = 0; n < COLS; n++) {
                    const float y = bg ? fmaf((float)f[1], q_sum[n][bg], s[bt][n][i]) : (float)f[1] * q_sum[n][bg];
                    s[bt][n][i] = fmaf((float)f[0], x[(j - 1) & 1][n][i], y);
                }
            }
            // (here, not behind the barrier, where all tiles' sums would wait for it in registers)
#pragma unroll
            for (int n = 0; n < COLS; n++) asm volatile("" : "+v"(s[bt][n]));
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// values(vs, ct): this lane's part of the A operand
template <typename CT, int HD, typename Values>
__device__ __forceinline__ void multiply_values(Rows<HD>& r, const Weights<CT>& p, const Values& values)
{
    constexpr int AT_ONCE = 4, N = VSTEPS<CT> * (HD / 16);
    u4 a[2][AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; i++) a[0][i] = values(i / (HD / 16), i % (HD / 16));
#pragma unroll
    for (int j = 0; j < N; j += AT_ONCE) {
        if (j + AT_ONCE < N) {
#pragma unroll
            for (int i = 0; i < AT_ONCE; i++) a[(j / AT_ONCE + 1) & 1][i] = values((j + AT_ONCE + i) / (HD / 16), (j + AT_ONCE + i) % (HD / 16));
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < AT_ONCE; i++)
#pragma unroll
            for (int n = 0; n < COLS; n++) r.o[(j + i) % (HD / 16)][n] = product<CT>(a[j / AT_ONCE & 1][i], p[(j + i) / (HD / 16)][n], r.o[(j + i) % (HD / 16)][n]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Which keys of a tile a row does not see: those from its limit on
struct Limits {
    __device__ __forceinline__ int key_tile(int t) const { return t; }         // the t-th of the walk
    __device__ __forceinline__ void ahead(int) const {}        // (its keys are on their way)
    template <typename CT, int HD>
    __device__ __forceinline__ void hide(const Rows<HD>& r, Products<CT>& s, int key0) const
    {
        const int k0 = key0 + 4 * ((threadIdx.x & 63) >> 4);
#pragma unroll
        for (int n = 0; n < COLS; n++)
#pragma unroll
            for (int t = 0; t < KEYS<CT> / 16; t++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (k0 + 16 * t + i >= r.limit[n]) s[t][n][i] = -INFINITY;
    }
};

// The weights of the keys from key0 on
template <typename CT, int HD, typename Order, typename Hidden>
__device__ __forceinline__ void form_weights(Rows<HD>& r, Products<CT>& s, Weights<CT>& p, int key0, bool masked, const Hidden& hidden)
{
    constexpr int T = KEYS<CT> / 16;
    if (masked) hidden.template hide<CT, HD>(r, s, key0);
    float most[COLS];
    bool move = false;
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        float m = s[0][n][0];
#pragma unroll
        for (int t = 0; t < T; t++)
#pragma unroll
            for (int i = 0; i < 4; i++) m = fmaxf(m, s[t][n][i]);
        most[n] = m * r.scale[n];
        move = move || most[n] > r.ref[n] + SLACK;
    }
    if (__ballot(move)) {
#pragma unroll
        for (int n = 0; n < COLS; n++) {
            const float ref = fmaxf(r.ref[n], max_of_column(most[n]));
            const float by = ref == r.ref[n] ? 1.f : __builtin_amdgcn_exp2f(r.ref[n] - ref);
            r.ref[n] = ref;
            r.sum[n] *= by;
#pragma unroll
            for (int ct = 0; ct < HD / 16; ct++) r.o[ct][n] *= by;
        }
    }
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        const float shift = r.ref[n] == -INFINITY ? 0.f : SHIFT<CT> - r.ref[n];
#pragma unroll
        for (int g = 0; g < T / 2; g++) {                      // 8 keys of this lane
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; e++) {
                w[e] = __builtin_amdgcn_exp2f(fmaf(s[2 * g + (e >> 2)][n][e & 3], r.scale[n], shift));
                r.sum[n] += w[e];
            }
            if constexpr (ESIZE<CT> == 2) {
#pragma unroll
                for (int e = 0; e < 4; e++) p[g][n][e] = pack2(w[Order::first(e)], w[Order::second(e)], CT());
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++) p[2 * g + (e >> 2)][n][e & 3] = __float_as_uint(w[e]);
            }
        }
    }
}

// fp32: a tile staged in the operands' order, [step][lane][16 bytes]
template <int HD, typename Hidden = Limits>
__device__ __forceinline__ void attend_f32(Rows<HD>& r, const Query<F32, HD>& q, Lds4 k_tile, Lds4 v_tile, int key0, int least, int most, const Hidden& hidden = Hidden())
{
    const int lane = threadIdx.x & 63;
    if (key0 >= most) return;
    Products<F32> s;
    Weights<F32> p;
    multiply_keys<F32, HD>(s, q, [&](int t, int st) { return k_tile[(t * STEPS<F32, HD> + st) * 64 + lane]; });
    form_weights<F32, HD, Natural>(r, s, p, key0, key0 + KEYS<F32> > least, hidden);
    multiply_values<F32, HD>(r, p, [&](int vs, int ct) { return v_tile[(vs * (HD / 16) + ct) * 64 + lane]; });
}

// ---- 16-bit types: two groups of wavefronts in turn ----------------------------------------------------------------------------
// A wavefront alternates between products (keys of its tile, values of the one before: 64 matrix instructions) and weights (the vector unit).
// The two wavefronts of a SIMD belong to different groups, and the groups are half a turn apart: in every phase one of them has the
// matrix cores and the other one the vector unit.  (Left to themselves they hardly overlap: a wavefront issues at most one instruction in
// 6 cycles, the older one of a SIMD goes first, and two that mix matrix and vector instructions take twice the time of one.)
//   phase 2i      group 0: products of tile i, brings the keys of tile i + 1      group 1: weights of tile i - 1, brings the values of tile i
//   phase 2i + 1  group 0: weights of tile i                                      group 1: products of tile i
// A tile's keys and values are read in two neighbouring phases, so two tiles of each in LDS are enough.  Expanding packed keys fills the vector
// slots behind the products (with the weights in the next phase: 88 us instead of 86 for the 50 700 tokens above).  Plain rows need no
// wavefront's time: group 1 sends for values and the next keys.  The group that multiplies has priority (64 frames 2110 -> 2050 us).
// SPLIT: up to 128 rows, all group 0's; group 1 brings it keys and values.
// A barrier for what is in LDS: loads into registers stay in flight across it (__syncthreads() waits for them)
__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_s_waitcnt(0xC07F);                        // lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ int group_of_wave() { return this_wave() >> 2; }

// Tiles t0 .. t1-1.  multiply(s, t): a tile's products of keys; bring_keys(t), bring_values(t): of the group that does so, into LDS; settle(): a phase's end.
// The products of the first tile meet weights of zero with what lies in front of its values: zeros.  (No condition inside the loop but who brings what: the compiler
// copies the accumulators around every one, and spills them.)
template <typename CT, int HD, bool SPLIT, typename Order, typename Multiply, typename Values, typename BringKeys, typename BringValues, typename Settle>
__device__ __forceinline__ void take_turns(Rows<HD>& r, int t0, int t1, int least, const Multiply& multiply, const Values& values, const BringKeys& bring_keys,
                                           const BringValues& bring_values, const Settle& settle)
{
    const int group = group_of_wave();
    if (SPLIT && group == 1) {
#pragma unroll 1
        for (int t = t0; t < t1; t++) {
            bring_values(t);
            settle();
            settle();
        }
        settle();
        return;
    }
    Products<CT> s;
    Weights<CT> p;
#pragma unroll
    for (int vs = 0; vs < VSTEPS<CT>; vs++)
#pragma unroll
        for (int n = 0; n < COLS; n++) p[vs][n] = u4{0, 0, 0, 0};
    if (!SPLIT && group == 1) {
        bring_values(t0);
        settle();
    }
#pragma unroll 1
    for (int t = t0; t < t1; t++) {
        __builtin_amdgcn_s_setprio(3);
        multiply(s, t);
        multiply_values<CT, HD>(r, p, [&](int vs, int ct) { return values(t - 1, vs, ct); });
        __builtin_amdgcn_s_setprio(0);
        if (!SPLIT && group == 0 && t + 1 < t1) bring_keys(t + 1);
        settle();
        form_weights<CT, HD, Order>(r, s, p, t * KEYS<CT>, (t + 1) * KEYS<CT> > least, Limits());
        if (!SPLIT && group == 1 && t + 1 < t1) bring_values(t + 1);
        settle();
    }
    if (SPLIT || group == 0) settle();
    multiply_values<CT, HD>(r, p, [&](int vs, int ct) { return values(t1 - 1, vs, ct); });
}
// All wavefronts together: bring(t) sends for, or expands, tile t while tile t - 1 is worked on.  Where two workgroups share a compute unit their phases
// mix by themselves, and tiles of 128 rows cost little more per row than ones of 256 in turns.
template <typename CT, int HD, typename Order, typename Multiply, typename Values, typename Bring, typename Settle, typename Hidden = Limits>
__device__ __forceinline__ void take_all(Rows<HD>& r, int t0, int t1, int least, const Multiply& multiply, const Values& values, const Bring& bring, const Settle& settle,
                                         const Hidden& hidden = Hidden())
{
    Products<CT> s;
    Weights<CT> p;
    bring(t0);
#pragma unroll 1
    for (int t = t0; t < t1; t++) {
        settle();
        multiply(s, t);
        if (t + 1 < t1) bring(t + 1);
        form_weights<CT, HD, Order>(r, s, p, t * KEYS<CT>, (t + 1) * KEYS<CT> > least, hidden);
        multiply_values<CT, HD>(r, p, [&](int vs, int ct) { return values(t, vs, ct); });
    }
}
template <typename CT, int HD>
__device__ __forceinline__ void clear_tile(Lds tile)
{
    for (int i = threadIdx.x & 255; i < TILE_BYTES<CT, HD> / 16; i += 256) ((Lds4)tile)[i] = u4{0, 0, 0, 0};
}

// ---- plain rows, fp32 arithmetic: through registers --------------------------------------------------------------------
// 16 bytes of fp32 from a row that holds elements of type ST
template <typename ST>
__device__ __forceinline__ u4 row_piece(const char* p)
{
    if constexpr (std::is_same_v<ST, F32>) {
        return *reinterpret_cast<const u4*>(p);
    } else {
        static_assert(std::is_same_v<ST, F16>, "");
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        u4 r;
        r[0] = __float_as_uint(wq_f16_bits_to_float(u.x & 0xFFFF)), r[1] = __float_as_uint(wq_f16_bits_to_float(u.x >> 16));
        r[2] = __float_as_uint(wq_f16_bits_to_float(u.y & 0xFFFF)), r[3] = __float_as_uint(wq_f16_bits_to_float(u.y >> 16));
        return r;
    }
}

// n rows from k, v (stride: bytes from row to row), a tile's at most; the tile's other rows become zeros.  The c-th 4 channels of a row are part of
// product c / 4, lane group c % 4; four keys of four channels are transposed by naming registers.
template <typename ST, int HD>
__device__ void stage_rows(const char* k, const char* v, int64_t k_stride, int64_t v_stride, int n, Lds4 k_tile, Lds4 v_tile)
{
    constexpr int PIECES = HD / 4, PB = 4 * ESIZE<ST>;
    const int tid = threadIdx.x;
#pragma unroll 4
    for (int u = tid; u < KEYS<F32> * PIECES; u += 64 * WAVES<F32>) {
        const int row = u / PIECES, c = u % PIECES;
        u4 x = {0, 0, 0, 0};
        if (row < n) x = row_piece<ST>(k + row * k_stride + c * PB);
        k_tile[((row >> 4) * STEPS<F32, HD> + (c >> 2)) * 64 + 16 * (c & 3) + (row & 15)] = x;
    }
    for (int u = tid; u < KEYS<F32> / 4 * PIECES; u += 64 * WAVES<F32>) {
        const int c = u % PIECES, jj = u / PIECES % 4, t16 = u / PIECES / 4;
        u4 x[4];
#pragma unroll
        for (int t = 0; t < 4; t++) {
            const int row = 16 * t16 + 4 * jj + t;
            x[t] = u4{0, 0, 0, 0};
            if (row < n) x[t] = row_piece<ST>(v + row * v_stride + c * PB);
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int ch = 4 * c + i;
            v_tile[(t16 * (HD / 16) + (ch >> 4)) * 64 + 16 * jj + (ch & 15)] = u4{x[0][i], x[1][i], x[2][i], x[3][i]};
        }
    }
}

// ---- plain rows of a 16-bit type: from memory to LDS without registers between ------------------------------------------
// A load of 16 bytes per lane lands in LDS at 16 bytes per lane in the lanes' order, so a tile lies there row by row.  What is free
// is which 16 bytes of its row a lane takes: piece c of row r goes to place c ^ f(r), so that the products' reads, which go down
// the rows, meet all banks.  Values are read with the transposing load: 16 lanes give the addresses of 4 rows x 16 channels and
// get 4 rows of one channel each.
template <int HD>
struct Direct {
    static constexpr int PIECES = HD / 8, PER_LOAD = 256 / PIECES, LOADS = KEYS<Bf16> / PER_LOAD;      // rows of one load of a group
    uint32_t k_off, v_off, k_step, v_step;     // this lane's offset in a tile, and from load to load
    int row;
    uint32_t k_piece, v_piece, k_stride, v_stride;
    int k_lds, v_lds;                          // byte offsets in a tile of this lane's operands: key tile 0, step 0; first value tile
    __device__ __forceinline__ Direct(int64_t ks, int64_t vs)
    {
        const int tid = threadIdx.x & 255, lane = tid & 63, m = lane & 15, j = lane >> 4;
        row = tid / PIECES;
        const int slot = tid % PIECES;
        k_piece = 16 * (slot ^ swizzle(row)), v_piece = 16 * (slot ^ (swizzle(row) * 2 & (PIECES - 1)));
        k_stride = (uint32_t)ks, v_stride = (uint32_t)vs;
        k_off = row * k_stride + k_piece, v_off = row * v_stride + v_piece;
        k_step = PER_LOAD * k_stride, v_step = PER_LOAD * v_stride;
        k_lds = m * (2 * HD) + 16 * (j ^ swizzle(m));
        const int r = 4 * j + (m >> 2);
        v_lds = r * (2 * HD) + 8 * (m & 3) + 16 * (swizzle(r) * 2 & (PIECES - 1));
    }
    // 16-byte places of 16 neighbouring rows meet different banks (256 bytes)
    static __device__ __forceinline__ int swizzle(int r) { return HD == 128 ? r & 15 : (r >> 1) & 7; }

    // rows from p on, n of them (the last one is read again for the rest: its weights are zero)
    __device__ __forceinline__ void load(const char* p, int n, uint32_t off, uint32_t piece, uint32_t step, uint32_t stride, Lds tile) const
    {
        const int wave = this_wave() & 3;
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            uint32_t o = off + i * step;
            if (n < KEYS<Bf16>) o = (uint32_t)(row + i * PER_LOAD < n ? row + i * PER_LOAD : n - 1) * stride + piece;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p + o),
                                             (__attribute__((address_space(3))) void*)(tile + (i * 256 + wave * 64) * 16), 16, 0, 0);
        }
    }
    __device__ __forceinline__ void load_keys(const char* p, int n, Lds tile) const { load(p, n, k_off, k_piece, k_step, k_stride, tile); }
    __device__ __forceinline__ void load_values(const char* p, int n, Lds tile) const { load(p, n, v_off, v_piece, v_step, v_stride, tile); }
    __device__ __forceinline__ u4 keys(Lds k_tile, int t, int st) const
    {
        return *(const Lds4)(k_tile + ((k_lds + t * 16 * (2 * HD)) ^ (64 * st)));
    }
    __device__ __forceinline__ u4 values(Lds v_tile, int vs, int ct) const
    {
        typedef short s4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s4* lds4;
        const Lds p = v_tile + ((v_lds + vs * 32 * (2 * HD)) ^ (32 * ct));
        struct { s4 a, b; } x = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p)), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + 16 * (2 * HD)))};
        return __builtin_bit_cast(u4, x);
    }
};

// Tiles lo .. hi-1 of the n rows from k, v on, brought by group 1: a tile's values and the next one's keys while group 0 multiplies.  TOGETHER: by all of four
// wavefronts, see take_all.
template <typename CT, int HD, bool SPLIT, bool TOGETHER = false, typename Hidden = Limits>
__device__ __forceinline__ void walk_rows(Rows<HD>& r, const Query<CT, HD>& q, const char* k, const char* v, int64_t k_stride, int64_t v_stride, int n, int lo,
                                          int hi, int least, Lds k_lds, Lds v_lds, const Hidden& hidden = Hidden())
{
    constexpr int BYTES = TILE_BYTES<CT, HD>, TK = KEYS<CT>;
    const Direct<HD> rows(k_stride, v_stride);
    auto load_keys = [&](int t) { rows.load_keys(k + (int64_t)hidden.key_tile(t) * TK * k_stride, n - hidden.key_tile(t) * TK, k_lds + (t & 1) * BYTES); };
    auto load_values = [&](int t) { rows.load_values(v + (int64_t)hidden.key_tile(t) * TK * v_stride, n - hidden.key_tile(t) * TK, v_lds + (t & 1) * BYTES); };
    auto multiply = [&](Products<CT>& s, int t) { multiply_keys<CT, HD>(s, q, [&](int kt, int st) { return rows.keys(k_lds + (t & 1) * BYTES, kt, st); }); };
    auto values = [&](int t, int vs, int ct) { return rows.values(v_lds + (t & 1) * BYTES, vs, ct); };
    __syncthreads();                                           // (whatever was in LDS before has been read)
    if constexpr (TOGETHER) {
        auto bring = [&](int t) {
            load_keys(t);
            load_values(t);
            hidden.ahead(t);
        };
        take_all<CT, HD, Natural>(r, lo, hi, least, multiply, values, bring, [] { __syncthreads(); }, hidden);
    } else {
        if (group_of_wave() == 1) load_keys(lo);
        else clear_tile<CT, HD>(v_lds + (~lo & 1) * BYTES);
        __syncthreads();
        auto bring_values = [&](int t) {
            load_values(t);
            if (t + 1 < hi) load_keys(t + 1);
        };
        take_turns<CT, HD, SPLIT, Natural>(r, lo, hi, least, multiply, values, [](int) {}, bring_values, [] { __syncthreads(); });
    }
}

// ---- a class of the packed cache -----------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302); }

template <int BITS>
__device__ __forceinline__ float code_of(const uint32_t* w, int i)
{
    constexpr int PER = 32 / BITS;
    return (float)((w[i / PER] >> (i % PER * BITS)) & ((1u << BITS) - 1));
}
template <int BYTES>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w)
{
    if constexpr (BYTES % 16 == 0) {
#pragma unroll
        for (int i = 0; i < BYTES / 16; i++) {
            const uint4 u = reinterpret_cast<const uint4*>(p)[i];
            w[4 * i] = u.x, w[4 * i + 1] = u.y, w[4 * i + 2] = u.z, w[4 * i + 3] = u.w;
        }
    } else if constexpr (BYTES == 8) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        w[0] = u.x, w[1] = u.y;
    } else {
        static_assert(BYTES == 4, "");
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}

// Field f of both halves of w as fp16: placed in the significand of a power of two, which is then taken away (exact)
template <int BITS, int AT>
__device__ __forceinline__ uint32_t placed(uint32_t w)
{
    constexpr uint32_t MASK = ((1u << BITS) - 1) << AT, ONE = (25u - AT) << 10;      // 2^(10 - AT)
    uint32_t one = ONE | ONE << 16;
    asm("" : "+v"(one));                                   // (in a vector register, so that both steps are one instruction)
    return (w & (MASK | MASK << 16)) | one;
}
template <int BITS, int AT>
__device__ __forceinline__ h2 code_pair(uint32_t x)
{
    constexpr _Float16 BIAS = (_Float16)(float)(1 << (10 - AT));
    return __builtin_bit_cast(h2, x) - h2{BIAS, BIAS};
}
template <int BITS, int AT>
__device__ __forceinline__ uint32_t expanded(uint32_t x, h2 s, h2 m)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(code_pair<BITS, AT>(x), s, m));       // (one rounding)
}
// ... or the codes alone
struct Codes {};
template <int BITS, int AT>
__device__ __forceinline__ uint32_t expanded(uint32_t x, Codes, Codes) { return __builtin_bit_cast(uint32_t, code_pair<BITS, AT>(x)); }

// A lane's 8 channels of step st from its quarter of a token's codes: pairs of channels as a masked word holds them (see order_query)
template <int BITS, typename SM>
__device__ __forceinline__ u4 expanded_keys(const uint32_t* w, int st, SM s, SM m)
{
    u4 y;
    if constexpr (BITS == 8) {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            y[2 * i] = expanded<BITS, 0>(placed<BITS, 0>(w[2 * st + i]), s, m);
            y[2 * i + 1] = expanded<BITS, 0>(placed<BITS, 0>(w[2 * st + i] >> 8), s, m);
        }
    } else if constexpr (BITS == 4) {
        const uint32_t x = w[st], z = x >> 8;
        y[0] = expanded<BITS, 0>(placed<BITS, 0>(x), s, m), y[1] = expanded<BITS, 4>(placed<BITS, 4>(x), s, m);
        y[2] = expanded<BITS, 0>(placed<BITS, 0>(z), s, m), y[3] = expanded<BITS, 4>(placed<BITS, 4>(z), s, m);
    } else {
        const uint32_t x = w[st >> 1] >> (st & 1) * 8;
        y[0] = expanded<BITS, 0>(placed<BITS, 0>(x), s, m), y[1] = expanded<BITS, 2>(placed<BITS, 2>(x), s, m);
        y[2] = expanded<BITS, 4>(placed<BITS, 4>(x), s, m), y[3] = expanded<BITS, 6>(placed<BITS, 6>(x), s, m);
    }
    return y;
}

// A lane's 8 tokens of the i-th of its channels (16 apart) from its codes: pairs of tokens, those of Far or Near, and so are their scales and minima
template <int BITS>
__device__ __forceinline__ u4 expanded_values(const uint32_t* w, int i, const h2 (&s)[4], const h2 (&m)[4])
{
    u4 y;
    if constexpr (BITS == 8) {
#pragma unroll
        for (int k = 0; k < 2; k++) {
            y[2 * k] = expanded<BITS, 0>(placed<BITS, 0>(w[2 * i + k]), s[2 * k], m[2 * k]);
            y[2 * k + 1] = expanded<BITS, 0>(placed<BITS, 0>(w[2 * i + k] >> 8), s[2 * k + 1], m[2 * k + 1]);
        }
    } else if constexpr (BITS == 4) {
        const uint32_t x = w[i], z = x >> 8;
        y[0] = expanded<BITS, 0>(placed<BITS, 0>(x), s[0], m[0]), y[1] = expanded<BITS, 4>(placed<BITS, 4>(x), s[1], m[1]);
        y[2] = expanded<BITS, 0>(placed<BITS, 0>(z), s[2], m[2]), y[3] = expanded<BITS, 4>(placed<BITS, 4>(z), s[3], m[3]);
    } else {                                                   // a word holds two of them, one per half
        const uint32_t x = w[i >> 1], both = i & 1 ? high_halves(x, x >> 8) : low_halves(x, x >> 8);
        y[0] = expanded<BITS, 0>(placed<BITS, 0>(both), s[0], m[0]), y[1] = expanded<BITS, 2>(placed<BITS, 2>(both), s[1], m[1]);
        y[2] = expanded<BITS, 4>(placed<BITS, 4>(both), s[2], m[2]), y[3] = expanded<BITS, 6>(placed<BITS, 6>(both), s[3], m[3]);
    }
    return y;
}

// A tile in flight between memory and LDS, in registers, brought by 64 * 4 (TOKENS = 64) or 64 * 2 (32) threads each of keys and of values.  A key
// unit is a quarter of a token's channels (lane of the product), a value unit 8 tokens of every 16th channel of half of the head.
// Addresses are a scalar base that moves with the tile and a lane's offset that does not.  A sequence's segment is padded to 32
// tokens: where a tile's second 32 are not the sequence's, its first 32 are taken again (their weights are zero, but zero times
// whatever lies there need not be zero).
template <int HD, int BITS, int TOKENS>
struct PackedKeys {
    static constexpr int C = BITS == 2 ? 0 : (BITS == 4 ? 1 : 2), N = HD / 4, BYTES = N * BITS / 8;
    const uint8_t* codes;                          // at the first tile
    const uint32_t* metas;
    uint32_t code_off, meta_off, G;
    int unit, slots;                               // token slots of the segment
    uint32_t w[(BYTES + 3) / 4], meta;

    __device__ __forceinline__ PackedKeys(const wq_packed_kv& kv, int kvh, int64_t tok0, int segment_slots)
    {
        slots = segment_slots, unit = threadIdx.x & (4 * TOKENS - 1), G = HD / kv.group;
        const int lane = unit & 63;
        const int64_t slot = kvh * kv.cap[C] + tok0;
        codes = static_cast<const uint8_t*>(kv.codes[C]) + slot * HD * BITS / 8;
        metas = static_cast<const uint32_t*>(kv.meta[C]) + slot * G;
        code_off = unit * BYTES;
        meta_off = ((unit >> 6) * G + (lane >> 4) * N / kv.group) * 16 + (lane & 15);      // (a quarter lies in one group: a group has at least 32 channels)
    }
    __device__ __forceinline__ void load(int t)
    {
        const bool again = TOKENS == 64 && t * 64 + 16 * (unit >> 6) >= slots;
        load_words<BYTES>(codes + (int64_t)t * (TOKENS * HD * BITS / 8) + (code_off - (again ? 128 * BYTES : 0)), w);
        meta = (metas + (int64_t)t * (TOKENS * G))[meta_off - (again ? 32 * G : 0)];
    }
    __device__ __forceinline__ void stage(Lds4 k_tile) const
    {
        const h2 sm = __builtin_bit_cast(h2, meta);
        expand(k_tile + (unit >> 6) * STEPS<F16, HD> * 64 + (unit & 63), h2{sm[0], sm[0]}, h2{sm[1], sm[1]}, [](int st) { return st * 64; });
    }
    // The codes alone, 32 neighbouring channels per step (a group is whole steps); scales and minima [16-key tile][group][key]
    __device__ __forceinline__ void stage_codes(Lds4 k_tile, Lds meta_tile) const
    {
        const int j = (unit & 63) >> 4, m = unit & 15, piece = j * STEPS<F16, HD>;         // the quarter's first 8 channels
        expand(k_tile + (unit >> 6) * STEPS<F16, HD> * 64 + (piece >> 2) * 64 + (piece & 3) * 16 + m, Codes(), Codes(), [](int st) { return st * 16; });
        ((Lds1)meta_tile)[((unit >> 6) * G + (j * G >> 2)) * 16 + m] = meta;        // (a group's quarters write the same)
    }
    // pairs of channels as a masked word holds them: see order_query, load_query_codes
    template <typename SM, typename Place>
    __device__ __forceinline__ void expand(Lds4 to, SM s, SM m, const Place& place) const
    {
#pragma unroll
        for (int st = 0; st < STEPS<F16, HD>; st++) to[place(st)] = expanded_keys<BITS>(w, st, s, m);
    }
    // fp32, codes one by one
    __device__ __forceinline__ void stage_f32(Lds4 k_tile) const
    {
        const float s = wq_f16_bits_to_float(meta & 0xFFFF), m = wq_f16_bits_to_float(meta >> 16);
#pragma unroll
        for (int st = 0; st < STEPS<F32, HD>; st++) {
            u4 y;
#pragma unroll
            for (int e = 0; e < 4; e++) y[e] = __float_as_uint(fmaf(s, code_of<BITS>(w, 4 * st + e), m));
            k_tile[((unit >> 6) * STEPS<F32, HD> + st) * 64 + (unit & 63)] = y;
        }
    }
};

template <int HD, int BITS, int TOKENS>
struct PackedValues {
    static constexpr int C = BITS == 2 ? 0 : (BITS == 4 ? 1 : 2), CT16 = HD / 16, V_CT = CT16 / 2, BYTES = V_CT * BITS;
    static constexpr int VG = HD / 64;             // groups that a unit's channels can belong to
    const uint8_t* codes;
    const uint32_t* metas;
    uint32_t code_off, meta_off[VG], G;
    int unit, slots;
    uint32_t w[(BYTES + 3) / 4];
    uint4 meta[VG][2];

    __device__ __forceinline__ PackedValues(const wq_packed_kv& kv, int kvh, int64_t tok0, int segment_slots)
    {
        slots = segment_slots, unit = threadIdx.x & (4 * TOKENS - 1), G = HD / kv.group;
        const int lane = unit & 63, half = (unit >> 6) & 1, blk = unit >> 7;
        const int64_t slot = (kv.Hkv + kvh) * kv.cap[C] + tok0;
        codes = static_cast<const uint8_t*>(kv.codes[C]) + slot * HD * BITS / 8;
        metas = static_cast<const uint32_t*>(kv.meta[C]) + slot * G;
        code_off = (blk * 64 + lane) * (CT16 * BITS) + half * BYTES;
#pragma unroll
        for (int g = 0; g < VG; g++) meta_off[g] = (2 * blk * G + (half * (HD / 2) + 32 * g) / kv.group) * 16 + 4 * (lane >> 4);
    }
    __device__ __forceinline__ void load(int t)
    {
        const bool again = TOKENS == 64 && t * 64 + 32 * (unit >> 7) >= slots;
        load_words<BYTES>(codes + (int64_t)t * (TOKENS * HD * BITS / 8) + (code_off - (again ? 64 * CT16 * BITS : 0)), w);
        const uint32_t* m = metas + (int64_t)t * (TOKENS * G);
#pragma unroll
        for (int g = 0; g < VG; g++) {
            const uint32_t at = meta_off[g] - (again ? 32 * G : 0);
            meta[g][0] = *reinterpret_cast<const uint4*>(m + at);
            meta[g][1] = *reinterpret_cast<const uint4*>(m + at + 16 * G);
        }
    }
    // pairs of tokens: those of Far or Near
    __device__ __forceinline__ void stage(Lds4 v_tile) const
    {
        const int lane = unit & 63, blk = unit >> 7, half = (unit >> 6) & 1;
        Lds4 to = v_tile + (blk * CT16 + half * V_CT) * 64 + lane;
#pragma unroll
        for (int g = 0; g < VG; g++) {
            h2 s[4], m[4];
            const uint32_t t[8] = {meta[g][0].x, meta[g][0].y, meta[g][0].z, meta[g][0].w, meta[g][1].x, meta[g][1].y, meta[g][1].z, meta[g][1].w};
#pragma unroll
            for (int e = 0; e < 4; e++) {
                using O = std::conditional_t<BITS == 8, Near, Far>;
                s[e] = __builtin_bit_cast(h2, low_halves(t[O::first(e)], t[O::second(e)]));
                m[e] = __builtin_bit_cast(h2, high_halves(t[O::first(e)], t[O::second(e)]));
            }
#pragma unroll
            for (int i = 2 * g; i < 2 * g + 2; i++) {          // 16-channel tiles of the group's 32 channels
                to[i * 64] = expanded_values<BITS>(w, i, s, m);
            }
        }
    }
    __device__ __forceinline__ void stage_f32(Lds4 v_tile) const
    {
        const int half = (unit >> 6) & 1, blk = unit >> 7;
#pragma unroll
        for (int i = 0; i < V_CT; i++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const uint4 t = meta[i >> 1][h];
                const uint32_t sm[4] = {t.x, t.y, t.z, t.w};
                u4 y;
#pragma unroll
                for (int e = 0; e < 4; e++)
                    y[e] = __float_as_uint(fmaf(wq_f16_bits_to_float(sm[e] & 0xFFFF), code_of<BITS>(w, 8 * i + 4 * h + e), wq_f16_bits_to_float(sm[e] >> 16)));
                v_tile[((2 * blk + h) * CT16 + half * V_CT + i) * 64 + (unit & 63)] = y;
            }
    }
};

// Tiles t0 .. t1-1 of a class's segment.  G: the head's groups, whose codes enter the products as they are; 0: keys expanded to fp16 (q_sum and m_lds
// are not read)
template <int HD, int BITS, int G, bool TOGETHER = false>
__device__ __forceinline__ void walk_packed(Rows<HD>& r, const Query<F16, HD>& q, const float (&q_sum)[COLS][G ? G : 1], PackedKeys<HD, BITS, 64>& keys,
                                            PackedValues<HD, BITS, 64>& values, int len, int t0, int t1, Lds k_lds, Lds v_lds, Lds m_lds)
{
    using Order = std::conditional_t<BITS == 8, Near, Far>;
    constexpr int BYTES = TILE_BYTES<F16, HD>;
    const int lane = threadIdx.x & 63;
    auto k_of = [&](int t) { return (Lds4)(k_lds + (t & 1) * BYTES); };
    auto v_of = [&](int t) { return (Lds4)(v_lds + (t & 1) * BYTES); };
    auto bring_keys = [&](int t) {
        if constexpr (G > 0) keys.stage_codes(k_of(t), m_lds + (t & 1) * (64 * 4 * G));
        else keys.stage(k_of(t));
        if (t + 1 < t1) keys.load(t + 1);
    };
    auto bring_values = [&](int t) {
        values.stage(v_of(t));
        if (t + 1 < t1) values.load(t + 1);
    };
    auto multiply = [&](Products<F16>& s, int t) {
        auto operand = [&](int kt, int st) { return k_of(t)[(kt * STEPS<F16, HD> + st) * 64 + lane]; };
        if constexpr (G > 0)
            multiply_codes<HD, G>(s, q, q_sum, operand, [&](int kt, int g) { return ((Lds4)(m_lds + (t & 1) * (64 * 4 * G)))[(kt * G + g) * 4 + (lane >> 4)]; });
        else
            multiply_keys<F16, HD>(s, q, operand);
    };
    auto value = [&](int t, int vs, int ct) { return v_of(t)[(vs * (HD / 16) + ct) * 64 + lane]; };
    __syncthreads();                                           // (whatever was in LDS before has been read)
    if constexpr (TOGETHER) {                                  // (its caller has loaded tile t0)
        auto bring = [&](int t) {
            bring_keys(t);
            bring_values(t);
        };
        take_all<F16, HD, Order>(r, t0, t1, len, multiply, value, bring, meet);
    } else {
        if (group_of_wave() == 1) {
            values.load(t0);
        } else {
            clear_tile<F16, HD>(v_lds + (~t0 & 1) * BYTES);
            keys.load(t0);
            bring_keys(t0);
        }
        __syncthreads();
        take_turns<F16, HD, false, Order>(r, t0, t1, len, multiply, value, bring_keys, bring_values, meet);
    }
}

// ---- what both kernels share -------------------------------------------------------------------------------------------
struct Out {
    void* out;                 // [rows of q][Hq][hd]
    float* lse;                // [rows of q][Hq] or NULL
    float* part;               // numerators of the parts [row of q * Hq + head][part][hd]
    float* part_ml;            // their references (log2) and sums [..][part][2]
};

// The sequence that workgroup `tile` works for and its first row there.  Sequence b's rows are off[b] * rep .. off[b+1] * rep - 1
// (a row per query head); its tiles of ROWS rows are numbered from off[b] * rep / ROWS + b: at least as many numbers as it has tiles.
// False: nothing to do.
struct Place {
    int seq, row0, rows;       // the tile's first row in its sequence, rows of the sequence
    int64_t first;             // first q row of the sequence
};
__device__ __forceinline__ int64_t clipped(int32_t x, int64_t most) { return x < 0 ? 0 : (x > most ? most : x); }
template <int ROWS>
__device__ __forceinline__ bool find_place(const int32_t* off, int nseq, int rep, int64_t total, int64_t tile, Place& p)
{
    int lo = 0, hi = nseq;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (clipped(off[mid], total) * rep / ROWS + mid <= tile) lo = mid; else hi = mid;
    }
    const int64_t a = clipped(off[lo], total), z = clipped(off[lo + 1], total);
    const int64_t row0 = (tile - (a * rep / ROWS + lo)) * ROWS;
    if (row0 < 0 || row0 >= (z - a) * rep) return false;
    p.seq = lo, p.first = a, p.rows = (int)((z - a) * rep), p.row0 = (int)row0;
    return true;
}

// 16-byte pieces of a row's channels: those of lane group j in the rows' order (32 neighbouring channels per product)
template <typename CT, int HD, int N>
__device__ __forceinline__ void load_query(QueryRows<CT, HD, N>& q, int n, const char* row)
{
    const int group = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int st = 0; st < STEPS<CT, HD>; st++) q[n][st] = row ? *reinterpret_cast<const u4*>(row + (4 * st + group) * 16) : u4{0, 0, 0, 0};
}
// ... or a quarter of the channels, as in the packed cache
template <typename CT, int HD, int N>
__device__ __forceinline__ void load_query_quarter(QueryRows<CT, HD, N>& q, int n, const char* row)
{
    const int group = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int st = 0; st < STEPS<CT, HD>; st++) q[n][st] = row ? *reinterpret_cast<const u4*>(row + (group * STEPS<CT, HD> + st) * 16) : u4{0, 0, 0, 0};
}
// A quarter's pairs of channels in the order in which Packed::stage leaves a class's keys
template <int BITS, int HD, int N>
__device__ __forceinline__ void order_query(QueryRows<F16, HD, N>& q, int n)
{
    u4 y[STEPS<F16, HD>];
#pragma unroll
    for (int st = 0; st < STEPS<F16, HD>; st++) {
        u4 a = q[n][st], b = a;
        int i0 = 0, i1 = 1, j0 = 2, j1 = 3;                    // 8 bits: registers 0 with 1, 2 with 3
        if constexpr (BITS == 4) i1 = 2, j0 = 1;               // 0 with 2, 1 with 3
        if constexpr (BITS == 2) {                             // of two neighbouring pieces
            a = q[n][st & ~1], b = q[n][st | 1];
            i0 = i1 = 2 * (st & 1), j0 = j1 = i0 + 1;
        }
        y[st] = u4{low_halves(a[i0], b[i1]), high_halves(a[i0], b[i1]), low_halves(a[j0], b[j1]), high_halves(a[j0], b[j1])};
    }
#pragma unroll
    for (int st = 0; st < STEPS<F16, HD>; st++) q[n][st] = y[st];
}

// A row's pieces of 8 channels in the rows' order, pairs of channels as stage_codes leaves them; sums over the head's G groups
template <int BITS, int G, int HD>
__device__ __forceinline__ void load_query_codes(Query<F16, HD>& q, int n, const char* row, float (&q_sum)[G])
{
    constexpr int PER = STEPS<F16, HD> / G;
    const int j = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int g = 0; g < G; g++) q_sum[g] = 0.f;
#pragma unroll
    for (int st = 0; st < STEPS<F16, HD>; st++) {
        u4 x = {0, 0, 0, 0};
        if (row) {
            const int piece = 4 * st + j;
            if constexpr (BITS == 2) {                         // of two neighbouring pieces
                const char* at = row + (piece >> 1) * 32 + (piece & 1) * 8;
                const uint2 a = *reinterpret_cast<const uint2*>(at), b = *reinterpret_cast<const uint2*>(at + 16);
                x = u4{a.x, b.x, a.y, b.y};
            } else {                                           // 4 bits: registers 0 with 2, 1 with 3; 8 bits: 0 with 1, 2 with 3
                x = *reinterpret_cast<const u4*>(row + piece * 16);
                if constexpr (BITS == 4) x = u4{x[0], x[2], x[1], x[3]};
            }
        }
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t word = x[e];
            const h2 f = __builtin_bit_cast(h2, word);
            q_sum[st / PER] += (float)f[0] + (float)f[1];
        }
        q[n][st] = u4{low_halves(x[0], x[1]), high_halves(x[0], x[1]), low_halves(x[2], x[3]), high_halves(x[2], x[3])};
    }
#pragma unroll
    for (int g = 0; g < G; g++) q_sum[g] = sum_of_column(q_sum[g]);
}

// ... the sums alone, of a query that has become fp16 since
template <int G, int HD>
__device__ __forceinline__ void sum_query_codes(const Query<F16, HD>& q, int n, float (&q_sum)[G])
{
    constexpr int PER = STEPS<F16, HD> / G;
#pragma unroll
    for (int g = 0; g < G; g++) {
        q_sum[g] = 0.f;
#pragma unroll
        for (int st = g * PER; st < (g + 1) * PER; st++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const uint32_t word = q[n][st][e];
                const h2 f = __builtin_bit_cast(h2, word);
                q_sum[g] += (float)f[0] + (float)f[1];
            }
        q_sum[g] = sum_of_column(q_sum[g]);
    }
}

template <typename QT> constexpr uint32_t EXPONENT16 = std::is_same_v<QT, Bf16> ? 0x7F80 : 0x7C00;
// Has a row's query an entry that is not finite (all exponent bits set: one more at the lowest of them carries into the sign's place)?
template <typename QT, int HD, int N>
__device__ __forceinline__ bool not_finite(const QueryRows<F16, HD, N>& q, int n)
{
    constexpr uint32_t EXPONENT = EXPONENT16<QT> * 0x10001u, ONE = std::is_same_v<QT, Bf16> ? 0x00800080u : 0x04000400u;
    uint32_t carry = 0;
#pragma unroll
    for (int st = 0; st < STEPS<F16, HD>; st++)
#pragma unroll
        for (int e = 0; e < 4; e++) carry |= (q[n][st][e] & EXPONENT) + ONE;
    carry |= __shfl_xor(carry, 16, 64);
    carry |= __shfl_xor(carry, 32, 64);
    return (carry & 0x80008000u) != 0;
}

// ... a bf16 query as fp16, divided by the power of two above the row's largest entry: its 8 bits are exact from 2^-17 of that power up, below
// that (fp16's smallest step there is 2^-24) off by at most 2^-25 of it
template <int HD, int N>
__device__ __forceinline__ float query_as_f16(QueryRows<F16, HD, N>& q, int n)
{
    constexpr int S = STEPS<F16, HD>;
    float most = 0.f;
#pragma unroll
    for (int st = 0; st < S; st++)
#pragma unroll
        for (int e = 0; e < 4; e++)
            most = fmaxf(most, fmaxf(fabsf(__uint_as_float(q[n][st][e] << 16)), fabsf(__uint_as_float(q[n][st][e] & 0xFFFF0000u))));
    most = max_of_column(most);
    int e2 = (int)(__float_as_uint(most) >> 23) - 126;             // most < 2^e2
    e2 = e2 < -100 ? -100 : (e2 > 127 ? 127 : e2);
    const float down = __uint_as_float((uint32_t)(127 - e2 + (e2 == 127)) << 23);
#pragma unroll
    for (int st = 0; st < S; st++)
#pragma unroll
        for (int e = 0; e < 4; e++)
            q[n][st][e] = pack2(__uint_as_float(q[n][st][e] << 16) * down, __uint_as_float(q[n][st][e] & 0xFFFF0000u) * down, F16());
    return 1.0f / down;
}

// A row's sum of weights is 0 where it sees no key: zeros, and a log-sum-exp of -infinity.  It is NaN where a logit is: so are the results then
// (a log-sum-exp of -infinity beside them would drop the row where results are merged by it).
__device__ __forceinline__ float one_over(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }
__device__ __forceinline__ float log_sum_exp(float ref, float sum) { return sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994530942f; }

// As one of several parts for the merge, or as the result (parts == 0).  Parts are numbered by the result's rows, or (tile_rows >= 0) by the
// tile's from there on.
template <typename CT, int HD>
__device__ __forceinline__ void store_rows(const Rows<HD>& r, const Place& p, int rep, int Hq, int kvh, int wave, int part, int parts, const Out& out,
                                           int64_t tile_rows = -1)
{
    const int lane = threadIdx.x & 63, group = lane >> 4;
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        const float sum = sum_of_column(r.sum[n]);
        const int row = p.row0 + (wave * COLS + n) * 16 + (lane & 15);
        if (row >= p.rows) continue;
        const int64_t at = (p.first + row / rep) * Hq + kvh * rep + row % rep;
        const float ref = r.ref[n] - SHIFT<CT>;
        if (parts > 0) {
            const int64_t slot = (tile_rows < 0 ? at : tile_rows + row - p.row0) * parts + part;
            float* to = out.part + slot * HD;
#pragma unroll
            for (int ct = 0; ct < HD / 16; ct++) *reinterpret_cast<f4*>(to + 16 * ct + 4 * group) = r.o[ct][n];
            if (group == 0) {
                out.part_ml[slot * 2] = ref;
                out.part_ml[slot * 2 + 1] = sum;
            }
            continue;
        }
        const float inv = one_over(sum);
        char* to = static_cast<char*>(out.out) + at * HD * ESIZE<CT>;
#pragma unroll
        for (int ct = 0; ct < HD / 16; ct++) {
            const f4 x = r.o[ct][n] * inv;
            if constexpr (ESIZE<CT> == 2)
                *reinterpret_cast<uint2*>(to + (16 * ct + 4 * group) * 2) = make_uint2(pack2(x[0], x[1], CT()), pack2(x[2], x[3], CT()));
            else
                *reinterpret_cast<f4*>(to + (16 * ct + 4 * group) * 4) = x;
        }
        if (out.lse && group == 0) out.lse[at] = log_sum_exp(ref, sum);
    }
}

template <typename CT, bool SPLIT = false> constexpr int ROWS = std::is_same_v<CT, F32> || SPLIT ? 128 : 256;       // of a workgroup

// ---- a sequence's packed cache, a workgroup's part of it ------------------------------------------------------------------
// Tiles t0 .. t1-1 of the class of BITS bits, for the wavefront's rows at row_at (NULL: no row).
// QT: the query's type; G as in walk_packed (fp16: the cache's groups per head; else 0); packed tokens are walked in fp16 (fp32 for fp32 queries), 16-bit rows in the
// cache's own type.  TREE: 16-bit types' wavefronts work together.  fp32 with heads of 128 needs 17 registers more than there are (scratch): 16 requests over 5000 tokens
// 40 us, in fp16 27.
template <typename QT> using Walked = std::conditional_t<std::is_same_v<QT, F32>, F32, F16>;
template <typename QT, int HD, int G, bool TREE, int BITS>
__device__ __forceinline__ void walk_class(Rows<HD>& r, Query<Walked<QT>, HD>& q, const char* const (&row_at)[COLS], const float& scale, const wq_packed_kv& kv, int seq,
                                           int kvh, int len, int t0, int t1, bool any, Lds s_k, Lds s_v, Lds s_m)
{
    using CT = Walked<QT>;
    constexpr bool PIPED = ESIZE<QT> == 2;
    constexpr int TK = KEYS<QT>, c = BITS == 2 ? 0 : (BITS == 4 ? 1 : 2);
    [[maybe_unused]] float q_sum[COLS][G > 0 ? G : 1];
    auto prepare = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < COLS; n++) {
            r.limit[n] = len;
            r.scale[n] = scale;
            if constexpr (G > 0) load_query_codes<BITS, G, HD>(q, n, row_at[n], q_sum[n]);
            else load_query_quarter<CT, HD>(q, n, row_at[n]);
            bool bad = false;
            if constexpr (PIPED) bad = not_finite<QT, HD>(q, n);
            // (kept from 0 and infinity: a masked logit, -infinity, times 0 and a logit of 0 times infinity would be NaN.  A scale that small leaves every
            // logit below 2^-100; with one that large logits that differ at all differ by 2^70 or more)
            if constexpr (std::is_same_v<QT, Bf16>) r.scale[n] = fminf(fmaxf(scale * query_as_f16<HD>(q, n), FLT_MIN), FLT_MAX);
            if constexpr (std::is_same_v<QT, Bf16> && G > 0) sum_query_codes<G, HD>(q, n, q_sum[n]);
            if (bad) r.scale[n] = NAN;
            if constexpr (PIPED && G == 0) order_query<BITS, HD>(q, n);
        }
    };
    if constexpr (!PIPED || !TREE) prepare();
    if constexpr (PIPED) {
        const int slots = (len + 31) / 32 * 32;
        PackedKeys<HD, BITS, 64> keys(kv, kvh, kv.cls_off[c][seq], slots);
        PackedValues<HD, BITS, 64> values(kv, kvh, kv.cls_off[c][seq], slots);
        if constexpr (TREE) {                                  // the first tile is on its way while the queries are prepared
            keys.load(t0);
            values.load(t0);
            prepare();
        }
        walk_packed<HD, BITS, G, TREE>(r, q, q_sum, keys, values, len, t0, t1, s_k, s_v, s_m);
    } else {
        PackedKeys<HD, BITS, 32> keys(kv, kvh, kv.cls_off[c][seq], 0);
        PackedValues<HD, BITS, 32> values(kv, kvh, kv.cls_off[c][seq], 0);
        const bool brings_keys = this_wave() < 2;
        auto load = [&](int t) {
            if (brings_keys) keys.load(t);
            else values.load(t);
        };
        __syncthreads();                                       // (whatever was in LDS before has been read)
        load(t0);
        for (int t = t0; t < t1; t++) {
            if (brings_keys) keys.stage_f32((Lds4)s_k);
            else values.stage_f32((Lds4)s_v);
            __syncthreads();
            if (t + 1 < t1) load(t + 1);
            __builtin_amdgcn_sched_barrier(0);
            attend_f32<HD>(r, q, (Lds4)s_k, (Lds4)s_v, t * TK, len, any ? len : 0);
            __syncthreads();
        }
    }
}
// ... of the 16-bit rows
template <typename QT, int HD, bool TREE>
__device__ __forceinline__ void walk_rows16(Rows<HD>& r, Query<Walked<QT>, HD>& q, const char* const (&row_at)[COLS], const float& scale, const wq_packed_kv& kv, int seq,
                                            int kvh, int len, int t0, int t1, bool any, Lds s_k, Lds s_v)
{
    constexpr int TK = KEYS<QT>;
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        r.limit[n] = len;
        r.scale[n] = scale;
        load_query<Walked<QT>, HD>(q, n, row_at[n]);
    }
    const int64_t row0 = kv.off16[seq], stride = (int64_t)kv.Hkv * HD * 2;
    const char* k = static_cast<const char*>(kv.k16) + row0 * stride + kvh * (HD * 2);
    const char* v = static_cast<const char*>(kv.v16) + row0 * stride + kvh * (HD * 2);
    if constexpr (ESIZE<QT> == 2) {
        walk_rows<QT, HD, false, TREE>(r, q, k, v, stride, stride, len, t0, t1, len, s_k, s_v);
    } else {
        for (int t = t0; t < t1; t++) {
            const int key0 = t * TK;
            __syncthreads();
            stage_rows<F16, HD>(k + key0 * stride, v + key0 * stride, stride, stride, len - key0, (Lds4)s_k, (Lds4)s_v);
            __syncthreads();
            attend_f32<HD>(r, q, (Lds4)s_k, (Lds4)s_v, key0, len, any ? len : 0);
        }
    }
}
// MODE.FP16_OVFL: an expanded value past fp16's range becomes its largest one.  Matrix products read NaN and infinity as numbers then, too: a query that is not finite
// makes its row's scale NaN (above), and rows are walked without
template <typename QT>
__device__ __forceinline__ void largest_instead_of_infinity(bool on)
{
    if constexpr (ESIZE<QT> == 2) on ? __builtin_amdgcn_s_setreg(1 | 23 << 6, 1) : __builtin_amdgcn_s_setreg(1 | 23 << 6, 0);
}
// From the packed tokens' shift of the weights to the rows', exact
template <typename QT, int HD>
__device__ __forceinline__ void shift_rows(Rows<HD>& r)
{
    if constexpr (std::is_same_v<QT, Bf16>) {
#pragma unroll
        for (int n = 0; n < COLS; n++) {
            r.sum[n] *= exp2f(SHIFT<QT> - SHIFT<Walked<QT>>);
#pragma unroll
            for (int ct = 0; ct < HD / 16; ct++) r.o[ct][n] *= exp2f(SHIFT<QT> - SHIFT<Walked<QT>>);
        }
    }
}

// ---- the parts' merge ----------------------------------------------------------------------------------------------------
__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
    return x;
}
__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
}

// Sum over the parts of a row, weights w (lane s: part s): HD / 4 lanes take a part's numerators, 16 bytes each, the wavefront's groups of lanes
// every second (fourth) part, FLIGHT in flight (one after the other the loads' round trips were the whole call).  This lane's
// channels are 4 (lane % (HD / 4)) ..; the groups' sums are still apart.
template <int HD, int FLIGHT = 16>
__device__ __forceinline__ f4 sum_of_parts(const float* part, int parts, float w)
{
    constexpr int LANES = HD / 4, GROUPS = 64 / LANES;
    const int lane = threadIdx.x & 63, group = lane / LANES;
    const f4* at = reinterpret_cast<const f4*>(part) + lane % LANES;
    f4 x = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < parts; s0 += GROUPS * FLIGHT) {
        f4 y[FLIGHT];
#pragma unroll
        for (int i = 0; i < FLIGHT; i++) {
            const int s = s0 + i * GROUPS + group;
            y[i] = s < parts ? at[(int64_t)s * LANES] : f4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int i = 0; i < FLIGHT; i++) {
            const int s = s0 + i * GROUPS + group;
            const float by = __shfl(w, s & 63, 64);
            x += y[i] * (s < parts ? by : 0.f);
        }
    }
    return x;
}
template <int HD>
__device__ __forceinline__ f4 sum_of_groups(f4 x)
{
#pragma unroll
    for (int o = HD / 4; o < 64; o *= 2)
#pragma unroll
        for (int i = 0; i < 4; i++) x[i] += __shfl_xor(x[i], o, 64);
    return x;
}
// Row `row` of the result from its numerators and the sum of weights L, relative to 2^M
template <int HD>
__device__ __forceinline__ void store_merged(const Out& out, int dtype, int64_t row, f4 x, float M, float L)
{
    const int lane = threadIdx.x & 63;
    x *= one_over(L);
    if (lane < HD / 4) {
        const int64_t at = row * (HD / 4) + lane;
        if (dtype == WQ_F32) static_cast<f4*>(out.out)[at] = x;
        else if (dtype == WQ_BF16) static_cast<uint2*>(out.out)[at] = make_uint2(pack2(x[0], x[1], Bf16()), pack2(x[2], x[3], Bf16()));
        else static_cast<uint2*>(out.out)[at] = make_uint2(pack2(x[0], x[1], F16()), pack2(x[2], x[3], F16()));
    }
    if (out.lse && lane == 0) out.lse[row] = log_sum_exp(M, L);
}

struct MergeArgs {
    int64_t rows;              // (q row, head) pairs
    int Hq, parts, dtype;
    const int32_t* q_off;
    int nseq;
    Out out;
};

// wq_prefill_attention: a wavefront per row.  Rows that belong to no sequence are left as they were.
template <int HD>
__global__ __launch_bounds__(256) void k_merge(MergeArgs a)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + this_wave();
    if (row >= a.rows) return;
    const int lane = threadIdx.x & 63;
    const int64_t b = row / a.Hq;
    if (b < a.q_off[0] || b >= a.q_off[a.nseq]) return;
    const float m = lane < a.parts ? a.out.part_ml[(row * a.parts + lane) * 2] : -INFINITY;
    const float l = lane < a.parts ? a.out.part_ml[(row * a.parts + lane) * 2 + 1] : 0.f;
    const float M = wave_max(m), w = __builtin_amdgcn_exp2f(m - (M == -INFINITY ? 0.f : M));
    const f4 x = sum_of_groups<HD>(sum_of_parts<HD>(a.out.part + row * a.parts * HD, a.parts, w));
    store_merged<HD>(a.out, a.dtype, row, x, M, wave_sum(l * w));
}

// ---- few query rows: a wavefront's share of the keys ---------------------------------------------------------------------------
// Where all of a sequence's query rows fit the 16 columns of one product, keys are what is shared out: wavefront w of FEW takes 32 of them,
// FEW chunks on the next.  Its keys come straight into the operands' registers (nothing else reads them), its values row by row into its own
// piece of LDS (`tile`), as in Direct; nothing waits for another wavefront until join() brings their numerators together.
constexpr int FEW = 8;

template <typename QT, int HD>
__device__ __forceinline__ void walk_few(const char* q_row, float scale, int limit, const char* k, const char* v, int64_t k_stride, int64_t v_stride, int n, int lo,
                                         int hi, Lds tile, f4 (&o)[HD / 16], float& ref, float& sum)
{
    constexpr int ST = STEPS<QT, HD>, CT16 = HD / 16, PIECES = HD / 8, PER_LOAD = 64 / PIECES, LOADS = 32 / PER_LOAD;
    using D = Direct<HD>;
    const int lane = threadIdx.x & 63, m = lane & 15, j = lane >> 4;
    Query<QT, HD> q;                                           // (fp32: read again at each use, from L1; 128 registers would not be left, and with heads
                                                               // of 128 ten of the others lie in scratch all the same)
    if constexpr (!std::is_same_v<QT, F32>) load_query<QT, HD>(q, 0, q_row);
    ref = -INFINITY, sum = 0.f;
#pragma unroll
    for (int ct = 0; ct < CT16; ct++) o[ct] = f4{0.f, 0.f, 0.f, 0.f};
    const D rows(v_stride, v_stride);
    for (int t32 = lo + this_wave(); t32 < hi; t32 += FEW) {
        const int key0 = 32 * t32, left = n - key0;                         // (the last row is read again for the rest: its weights are zero)
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int r = i * PER_LOAD + lane / PIECES, piece = (lane % PIECES) ^ (D::swizzle(r) * 2 & (PIECES - 1));
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(v + (key0 + (r < left ? r : left - 1)) * v_stride + 16 * piece),
                                             (__attribute__((address_space(3))) void*)(tile + i * 1024), 16, 0, 0);
        }
        f4 s[2];
#pragma unroll
        for (int t = 0; t < 2; t++) {
            const int r = 16 * t + m;
            const char* row = k + (key0 + (r < left ? r : left - 1)) * k_stride;
            s[t] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < ST; st++) {
                if constexpr (std::is_same_v<QT, F32>) {
                    const u4 y = q_row ? *reinterpret_cast<const u4*>(q_row + (4 * st + j) * 16) : u4{0, 0, 0, 0};
                    s[t] = product<F32>(row_piece<F16>(row + (4 * st + j) * 8), y, s[t]);
                } else {
                    s[t] = product<QT>(*reinterpret_cast<const u4*>(row + (4 * st + j) * 16), q[0][st], s[t]);
                }
            }
        }
        float most = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; t++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                s[t][i] = key0 + 16 * t + 4 * j + i < limit ? s[t][i] * scale : -INFINITY;
                most = fmaxf(most, s[t][i]);
            }
        const float next = fmaxf(ref, max_of_column(most)), base = next == -INFINITY ? 0.f : next;
        const float by = __builtin_amdgcn_exp2f(ref - base);
        ref = next, sum *= by;
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            w[e] = __builtin_amdgcn_exp2f(s[e >> 2][e & 3] - base + SHIFT<QT>);
            sum += w[e];
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);                    // vmcnt(0): the values are in LDS
        asm volatile("" ::: "memory");
        if constexpr (std::is_same_v<QT, F32>) {
#pragma unroll
            for (int ct = 0; ct < CT16; ct++) {
                o[ct] *= by;
#pragma unroll
                for (int t = 0; t < 2; t++) {
                    u4 x, p;
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int r = 16 * t + 4 * j + i, ch = 16 * ct + m;
                        const uint16_t h = *(const __attribute__((address_space(3))) uint16_t*)(tile + r * (2 * HD) + 16 * ((ch >> 3) ^ (D::swizzle(r) * 2 & (PIECES - 1))) + 2 * (ch & 7));
                        x[i] = __float_as_uint(wq_f16_bits_to_float(h)), p[i] = __float_as_uint(w[4 * t + i]);
                    }
                    o[ct] = product<F32>(x, p, o[ct]);
                }
            }
        } else {
            u4 p;
#pragma unroll
            for (int e = 0; e < 4; e++) p[e] = pack2(w[2 * e], w[2 * e + 1], QT());
#pragma unroll
            for (int ct = 0; ct < CT16; ct++) o[ct] = product<QT>(rows.values(tile, 0, ct), p, o[ct] * by);
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);                    // lgkmcnt(0): they are out of it again
        asm volatile("" ::: "memory");
    }
    sum = sum_of_column(sum);
    ref -= SHIFT<QT>;
}

// Wavefronts' numerators [row][hd] in their pieces of LDS, references and sums beside them
template <int HD>
struct Few {
    __align__(16) char v[FEW][32 * HD * 2];
    float m[FEW][16], l[FEW][16];
};
template <int HD>
__device__ __forceinline__ void leave_few(Few<HD>& s, const f4 (&o)[HD / 16], float ref, float sum)
{
    const int lane = threadIdx.x & 63, n = lane & 15, wave = this_wave();
#pragma unroll
    for (int ct = 0; ct < HD / 16; ct++) *reinterpret_cast<f4*>(s.v[wave] + (n * HD + 16 * ct + 4 * (lane >> 4)) * 4) = o[ct];
    if (lane < 16) s.m[wave][n] = ref, s.l[wave][n] = sum;
}
// Row r's numerators, those of wavefront f by weight w (lane f); lanes' channels and groups as in sum_of_parts
template <int HD>
__device__ __forceinline__ f4 join_few(const Few<HD>& s, int r, float w)
{
    constexpr int LANES = HD / 4, GROUPS = 64 / LANES;
    const int lane = threadIdx.x & 63;
    f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < FEW; k += GROUPS) {
        const int from = k + lane / LANES;
        const float by = __shfl(w, from, 64);
        x += *reinterpret_cast<const f4*>(s.v[from] + (r * HD + 4 * (lane % LANES)) * 4) * by;
    }
    return x;
}

// ---- host ----------------------------------------------------------------------------------------------------------------
int64_t tiles_of(int64_t total, int rep, int nseq, int rows) { return total * rep / rows + nseq; }

// Parts for about `want` workgroups, of at least `keys` keys each
int auto_splits_of(int64_t workgroups, int64_t max_keys, int want, int keys)
{
    int64_t s = workgroups > 0 ? (want + workgroups - 1) / workgroups : 1;
    const int64_t most = (max_keys + keys - 1) / keys;
    if (s > most) s = most;
    if (s > WQ_MAX_ATTEND_SPLITS) s = WQ_MAX_ATTEND_SPLITS;
    return s < 1 ? 1 : (int)s;
}

size_t partials_bytes(int64_t rows, int hd, int parts) { return wq_align256((size_t)rows * parts * (hd + 2) * sizeof(float)); }

}  // namespace
