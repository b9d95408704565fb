// Attention of many query rows of one KV head over one sequence: wq_prefill_attention (keys and values are plain rows, a
// row sees the keys up to its own position and the sequence's prefix) and the shared part of wq_decode_attention_shared
// (keys and values are a packed cache that the requests of a group all attend to).
//
// A row is a (token, query head) pair or a (request, query head) pair: the rep query heads of a KV head are neighbouring
// rows of one product, so a tile of keys and values is staged once for all of them.  A workgroup of four wavefronts owns
// 128 rows (32 per wavefront) and walks the keys 64 at a time:
//   S^T = K Q^T    A operand: 16 keys, B operand: 16 rows   -> a lane holds 4 x 4 keys of one row
//   online softmax in the lane's own registers (running reference and sum, fp32)
//   O^T += V^T P^T A operand: 16 channels, B operand: 16 rows: P^T needs no exchange between lanes, because the keys'
//                  order inside a product is free: V's operand takes them in the order in which S^T left them
// Tiles are staged in LDS in the operands' own order, [step][lane][16 bytes], so that every LDS read of the products is one
// conflict-free 16-byte load per lane.
//
// fp32 queries take the fp32 matrix instruction throughout.  16-bit queries take the 16-bit ones: the weights are rounded to
// the value's type (the sum of weights is not), packed keys and values to fp16 (2^-11 of a value whose own step is its
// scale; below the output's own rounding).
#include <math.h>
#include <type_traits>

#include "wq_internal.h"

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

struct Bf16 {};
struct F16 {};
struct F32 {};

constexpr int WAVES = 4, COLS = 2;                 // wavefronts per workgroup, 16-row columns per wavefront
constexpr int ROWS = WAVES * COLS * 16;            // query rows of a workgroup
constexpr int KEYS = 64;                           // keys of a tile
constexpr float LOG2E = 1.44269504088896340736f;
// The reference of a row's exponents moves only when a logit exceeds it by 2^SLACK; weights are kept 2^SHIFT too large, so that
// in fp16 one is lost only below 2^-34 of the largest (SHIFT + SLACK < 16).
constexpr float SLACK = 5.f, SHIFT = 10.f;

template <typename CT> constexpr int ESIZE = std::is_same_v<CT, F32> ? 4 : 2;
template <typename CT, int HD> constexpr int STEPS = HD * ESIZE<CT> / 64;          // products of a key tile: 32 (16) channels each
template <typename CT> constexpr int VSTEPS = KEYS * ESIZE<CT> / 64;               // products over a tile's keys: 32 (16) keys each
template <typename CT, int HD> constexpr int K_PIECES = KEYS / 16 * STEPS<CT, HD> * 64;     // 16-byte pieces of a staged key tile
template <typename CT, int HD> constexpr int V_PIECES = VSTEPS<CT> * (HD / 16) * 64;

template <typename CT, int HD> using Query = u4[COLS][STEPS<CT, HD>];             // B operands of a wavefront's rows

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
// a value of a packed group: rounding of the group's scale can carry its largest value past fp16's range
__device__ __forceinline__ float in_range(float x) { return fminf(fmaxf(x, -65504.f), 65504.f); }

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

// keys(t, st), values(vs, ct): this lane's part of the A operands
template <typename CT, int HD, typename Keys, typename Values>
__device__ __forceinline__ void attend_tile(Rows<HD>& r, const Query<CT, HD>& q, const Keys& keys, const Values& values, int key0, bool masked)
{
    const int lane = threadIdx.x & 63;
    f4 s[KEYS / 16][COLS];
#pragma unroll
    for (int t = 0; t < KEYS / 16; t++) {
#pragma unroll
        for (int n = 0; n < COLS; n++) s[t][n] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < STEPS<CT, HD>; st++) {
            const u4 a = keys(t, st);
#pragma unroll
            for (int n = 0; n < COLS; n++) s[t][n] = product<CT>(a, q[n][st], s[t][n]);
        }
    }
    if (masked) {
        const int k0 = key0 + 4 * (lane >> 4);
#pragma unroll
        for (int n = 0; n < COLS; n++)
#pragma unroll
            for (int t = 0; t < KEYS / 16; t++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (k0 + 16 * t + i >= r.limit[n]) s[t][n][i] = -INFINITY;
    }
    float most[COLS];
    bool move = false;
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        float m = s[0][n][0];
#pragma unroll
        for (int t = 0; t < KEYS / 16; t++)
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
    constexpr int PER = ESIZE<CT> == 2 ? 8 : 4;       // keys of a lane per product
    u4 p[VSTEPS<CT>][COLS];
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        const float shift = r.ref[n] == -INFINITY ? 0.f : SHIFT - r.ref[n];
#pragma unroll
        for (int vs = 0; vs < VSTEPS<CT>; vs++) {
            float w[PER];
#pragma unroll
            for (int e = 0; e < PER; e++) {
                const int t = vs * PER / 4 + e / 4;
                w[e] = __builtin_amdgcn_exp2f(fmaf(s[t][n][e & 3], r.scale[n], shift));
                r.sum[n] += w[e];
            }
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if constexpr (ESIZE<CT> == 2) p[vs][n][e] = pack2(w[2 * e], w[2 * e + 1], CT());
                else p[vs][n][e] = __float_as_uint(w[e]);
            }
        }
    }
#pragma unroll
    for (int vs = 0; vs < VSTEPS<CT>; vs++)
#pragma unroll
        for (int ct = 0; ct < HD / 16; ct++) {
            const u4 a = values(vs, ct);
#pragma unroll
            for (int n = 0; n < COLS; n++) r.o[ct][n] = product<CT>(a, p[vs][n], r.o[ct][n]);
        }
}

// ... from a tile staged in the operands' order
template <typename CT, int HD>
__device__ __forceinline__ void attend_staged(Rows<HD>& r, const Query<CT, HD>& q, const u4* __restrict__ k_tile, const u4* __restrict__ v_tile, int key0,
                                              bool masked)
{
    const int lane = threadIdx.x & 63;
    attend_tile<CT, HD>(r, q, [&](int t, int st) { return k_tile[(t * STEPS<CT, HD> + st) * 64 + lane]; },
                        [&](int vs, int ct) { return v_tile[(vs * (HD / 16) + ct) * 64 + lane]; }, key0, masked);
}

// ---- staging: plain rows -----------------------------------------------------------------------------------------------
// 16 bytes of elements of type CT from a row that holds elements of type ST
template <typename CT, typename ST>
__device__ __forceinline__ u4 row_piece(const char* p)
{
    if constexpr (std::is_same_v<CT, ST>) {
        return *reinterpret_cast<const u4*>(p);
    } else {                                           // fp16 rows, fp32 arithmetic
        static_assert(std::is_same_v<CT, F32> && std::is_same_v<ST, F16>, "");
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        u4 r;
        r[0] = __float_as_uint(wq_f16_bits_to_float(u.x & 0xFFFF)), r[1] = __float_as_uint(wq_f16_bits_to_float(u.x >> 16));
        r[2] = __float_as_uint(wq_f16_bits_to_float(u.y & 0xFFFF)), r[3] = __float_as_uint(wq_f16_bits_to_float(u.y >> 16));
        return r;
    }
}

// Where the c-th 16-byte piece of a head's channels lies in the products: in the packed cache's order (a lane group holds a
// quarter of the channels) or the rows' (a step holds neighbouring channels).
template <int NSTEPS, bool QUARTERS>
__device__ __forceinline__ void place_of(int c, int& step, int& group)
{
    if constexpr (QUARTERS) {
        group = c / NSTEPS;
        step = c % NSTEPS;
    } else {
        step = c / 4;
        group = c % 4;
    }
}

// n <= KEYS rows from k, v (stride: bytes from row to row); the tile's other rows become zeros
template <typename CT, typename ST, int HD, bool QUARTERS>
__device__ void stage_rows(const char* k, const char* v, int64_t k_stride, int64_t v_stride, int n, u4* __restrict__ k_tile, u4* __restrict__ v_tile)
{
    constexpr int PIECES = HD * ESIZE<CT> / 16;        // of a row
    constexpr int PB = 16 / ESIZE<CT> * ESIZE<ST>;     // bytes of a piece in memory
    const int tid = threadIdx.x;
#pragma unroll 4
    for (int u = tid; u < KEYS * PIECES; u += 64 * WAVES) {
        const int row = u / PIECES, c = u % PIECES;
        int step, group;
        place_of<STEPS<CT, HD>, QUARTERS>(c, step, group);
        u4 x = {0, 0, 0, 0};
        if (row < n) x = row_piece<CT, ST>(k + row * k_stride + c * PB);
        k_tile[((row >> 4) * STEPS<CT, HD> + step) * 64 + 16 * group + (row & 15)] = x;
    }
    if constexpr (ESIZE<CT> == 2) {
        // 8 keys x 8 channels are transposed in registers
        for (int u = tid; u < KEYS / 8 * PIECES; u += 64 * WAVES) {
            const int c = u % PIECES, jj = u / PIECES % 4, blk = u / PIECES / 4;
            u4 x[8];
#pragma unroll
            for (int t = 0; t < 8; t++) {
                const int row = 32 * blk + 16 * (t >> 2) + 4 * jj + (t & 3);
                x[t] = u4{0, 0, 0, 0};
                if (row < n) x[t] = row_piece<CT, ST>(v + row * v_stride + c * PB);
            }
#pragma unroll
            for (int i = 0; i < 8; i++) {
                u4 y;
#pragma unroll
                for (int w = 0; w < 4; w++)
                    y[w] = __builtin_amdgcn_perm(x[2 * w + 1][i >> 1], x[2 * w][i >> 1], (i & 1) ? 0x07060302 : 0x05040100);
                const int ch = 8 * c + i;
                v_tile[(blk * (HD / 16) + (ch >> 4)) * 64 + 16 * jj + (ch & 15)] = y;
            }
        }
    } else {
        for (int u = tid; u < KEYS / 4 * PIECES; u += 64 * WAVES) {
            const int c = u % PIECES, jj = u / PIECES % 4, t16 = u / PIECES / 4;
            u4 x[4];
#pragma unroll
            for (int t = 0; t < 4; t++) {
                const int row = 16 * t16 + 4 * jj + t;
                x[t] = u4{0, 0, 0, 0};
                if (row < n) x[t] = row_piece<CT, ST>(v + row * v_stride + c * PB);
            }
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int ch = 4 * c + i;
                v_tile[(t16 * (HD / 16) + (ch >> 4)) * 64 + 16 * jj + (ch & 15)] = u4{x[0][i], x[1][i], x[2][i], x[3][i]};
            }
        }
    }
}

// ---- staging: plain rows of a 16-bit type, from memory to LDS without registers between ----------------------------------
// A load of 16 bytes per lane lands in LDS at 16 bytes per lane in the lanes' order, so a tile lies there row by row.  What is free
// is which 16 bytes of its row a lane takes: piece c of row r goes to place c ^ f(r), so that the products' reads, which go down
// the rows, meet all banks.  Values are read with the transposing load: 16 lanes give the addresses of 4 rows x 16 channels and
// get 4 rows of one channel each.
template <int HD>
struct Direct {
    static constexpr int PIECES = HD / 8, PER_LOAD = 64 * WAVES / PIECES, LOADS = KEYS / PER_LOAD;      // rows of one load of the workgroup
    uint32_t k_off, v_off, k_step, v_step;     // this lane's offset in a tile, and from load to load
    int row;
    uint32_t k_piece, v_piece, k_stride, v_stride;
    int k_lds, v_lds;                          // byte offsets in a tile of this lane's operands: key tile 0, step 0; first value tile
    __device__ __forceinline__ Direct(int64_t ks, int64_t vs)
    {
        const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, j = lane >> 4;
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

    // rows from k, v on, n of them (the last one is read again for the rest: its weights are zero)
    __device__ __forceinline__ void load(const char* k, const char* v, int n, char* k_tile, char* v_tile) const
    {
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            uint32_t ko = k_off + i * k_step, vo = v_off + i * v_step;
            if (n < KEYS) {
                const uint32_t at = row + i * PER_LOAD < n ? row + i * PER_LOAD : n - 1;
                ko = at * k_stride + k_piece, vo = at * v_stride + v_piece;
            }
            const int to = (i * 64 * WAVES + wave * 64) * 16;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(k + ko), (__attribute__((address_space(3))) void*)(k_tile + to), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(v + vo), (__attribute__((address_space(3))) void*)(v_tile + to), 16, 0, 0);
        }
    }
    __device__ __forceinline__ u4 keys(const char* k_tile, int t, int st) const
    {
        return *reinterpret_cast<const u4*>(k_tile + ((k_lds + t * 16 * (2 * HD)) ^ (64 * st)));
    }
    __device__ __forceinline__ u4 values(const char* v_tile, int vs, int ct) const
    {
        typedef short s4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s4* lds4;
        const char* p = v_tile + ((v_lds + vs * 32 * (2 * HD)) ^ (32 * ct));
        struct { s4 a, b; } x = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p)), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + 16 * (2 * HD)))};
        return __builtin_bit_cast(u4, x);
    }
};

// ---- staging: a class of the packed cache ------------------------------------------------------------------------------
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

// The 64 token slots from tok0 (a multiple of 32) of class BITS.  Slots from slots_left on (a multiple of 32) are not the sequence's: they become zeros,
// because a weight of zero times whatever lies there need not be zero.
template <typename CT, int HD, int BITS>
__device__ void stage_packed(const wq_packed_kv& kv, int kvh, int64_t tok0, int64_t slots_left, u4* __restrict__ k_tile, u4* __restrict__ v_tile)
{
    constexpr int C = BITS == 2 ? 0 : (BITS == 4 ? 1 : 2);
    constexpr int CT16 = HD / 16;
    const int tid = threadIdx.x, lane = tid & 63, group = kv.group, G = HD / group;
    const int64_t cap = kv.cap[C];
    const uint8_t* kc = static_cast<const uint8_t*>(kv.codes[C]) + (int64_t)kvh * cap * HD * BITS / 8;
    const uint8_t* vc = static_cast<const uint8_t*>(kv.codes[C]) + ((int64_t)kv.Hkv + kvh) * cap * HD * BITS / 8;
    const uint32_t* km = static_cast<const uint32_t*>(kv.meta[C]) + (int64_t)kvh * cap * G;
    const uint32_t* vm = static_cast<const uint32_t*>(kv.meta[C]) + ((int64_t)kv.Hkv + kvh) * cap * G;
    {   // keys: thread = (16-token tile, lane of the product): a quarter of a token's channels
        constexpr int N = HD / 4, BYTES = N * BITS / 8;
        const int t16 = tid >> 6, m = lane & 15, j = lane >> 4;
        uint32_t w[(BYTES + 3) / 4] = {};
        uint32_t meta = 0;                             // (a quarter lies in one group: a group has at least 32 channels)
        if (16 * t16 < slots_left) {
            const int64_t tile = (tok0 >> 4) + t16;
            load_words<BYTES>(kc + (tile * 64 + lane) * BYTES, w);
            meta = km[(tile * G + j * N / group) * 16 + m];
        }
        const float s = wq_f16_bits_to_float(meta & 0xFFFF), mn = wq_f16_bits_to_float(meta >> 16);
#pragma unroll
        for (int st = 0; st < STEPS<CT, HD>; st++) {
            constexpr int E = 16 / ESIZE<CT>;
            float x[E];
#pragma unroll
            for (int e = 0; e < E; e++) x[e] = in_range(fmaf(s, code_of<BITS>(w, E * st + e), mn));
            u4 y;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if constexpr (ESIZE<CT> == 2) y[e] = pack2(x[2 * e], x[2 * e + 1], CT());
                else y[e] = __float_as_uint(x[e]);
            }
            k_tile[(t16 * STEPS<CT, HD> + st) * 64 + lane] = y;
        }
    }
    {   // values: thread = (32-token block, half of the channels, lane of the product): 8 tokens of every 16th channel
        constexpr int N = CT16 / 2, BYTES = N * BITS;
        const int blk = tid >> 7, half = (tid >> 6) & 1, jj = lane >> 4;
        uint32_t w[(BYTES + 3) / 4] = {};
        uint32_t meta[8] = {};
        int have = -1;
        const bool real = 32 * blk < slots_left;
        const int64_t block = (tok0 >> 5) + blk;
        if (real) load_words<BYTES>(vc + (block * 64 + lane) * (CT16 * BITS) + half * BYTES, w);
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int ct = half * N + i, g = ct * 16 / group;
            if (real && g != have) {
                const uint4 a = *reinterpret_cast<const uint4*>(vm + ((2 * block) * G + g) * 16 + 4 * jj);
                const uint4 b = *reinterpret_cast<const uint4*>(vm + ((2 * block + 1) * G + g) * 16 + 4 * jj);
                meta[0] = a.x, meta[1] = a.y, meta[2] = a.z, meta[3] = a.w;
                meta[4] = b.x, meta[5] = b.y, meta[6] = b.z, meta[7] = b.w;
                have = g;
            }
            float x[8];
#pragma unroll
            for (int t = 0; t < 8; t++)
                x[t] = in_range(fmaf(wq_f16_bits_to_float(meta[t] & 0xFFFF), code_of<BITS>(w, 8 * i + t), wq_f16_bits_to_float(meta[t] >> 16)));
            if constexpr (ESIZE<CT> == 2) {
                v_tile[(blk * CT16 + ct) * 64 + lane] = u4{pack2(x[0], x[1], CT()), pack2(x[2], x[3], CT()), pack2(x[4], x[5], CT()), pack2(x[6], x[7], CT())};
            } else {
#pragma unroll
                for (int h = 0; h < 2; h++)
                    v_tile[((2 * blk + h) * CT16 + ct) * 64 + lane] =
                        u4{__float_as_uint(x[4 * h]), __float_as_uint(x[4 * h + 1]), __float_as_uint(x[4 * h + 2]), __float_as_uint(x[4 * h + 3])};
            }
        }
    }
}

// ---- what both kernels share -------------------------------------------------------------------------------------------
struct Out {
    void* out;                 // [rows of q][Hq][hd]
    float* lse;                // [rows of q][Hq] or NULL
    float* part;               // numerators of the splits [row of q * Hq + head][split][hd]
    float* part_ml;            // their references (log2) and sums [..][split][2]
};

// The sequence that workgroup `tile` works for and its first row there.  Sequence b's rows are off[b] * rep .. off[b+1] * rep - 1
// (a row per query head); its tiles are numbered from off[b] * rep / ROWS + b: at least as many numbers as it has tiles.
// False: nothing to do.
struct Place {
    int seq, row0, rows;       // the tile's first row in its sequence, rows of the sequence
    int64_t first;             // first q row of the sequence
};
__device__ __forceinline__ int64_t clipped(int32_t x, int64_t most) { return x < 0 ? 0 : (x > most ? most : x); }
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

template <typename CT, typename ST, int HD, bool QUARTERS>
__device__ __forceinline__ void load_query(Query<CT, HD>& q, int n, const char* row)
{
    const int group = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int st = 0; st < STEPS<CT, HD>; st++) {
        const int c = QUARTERS ? group * STEPS<CT, HD> + st : 4 * st + group;
        q[n][st] = row ? row_piece<CT, ST>(row + c * (16 / ESIZE<CT> * ESIZE<ST>)) : u4{0, 0, 0, 0};
    }
}

// ... a bf16 query as fp16, divided by the power of two above the row's largest entry: exact down to 2^-24 of that power
template <int HD>
__device__ __forceinline__ float query_as_f16(Query<F16, HD>& q, int n)
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

// As a partial for the merge (parts), or as the result.
template <typename CT, int HD>
__device__ __forceinline__ void store_rows(const Rows<HD>& r, const Place& p, int rep, int Hq, int kvh, int wave, int split, int splits, bool parts, const Out& out)
{
    const int lane = threadIdx.x & 63, group = lane >> 4;
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        const float sum = sum_of_column(r.sum[n]);
        const int row = p.row0 + (wave * COLS + n) * 16 + (lane & 15);
        if (row >= p.rows) continue;
        const int64_t at = (p.first + row / rep) * Hq + kvh * rep + row % rep;
        const float ref = r.ref[n] - SHIFT;
        if (parts) {
            float* to = out.part + (at * splits + split) * HD;
#pragma unroll
            for (int ct = 0; ct < HD / 16; ct++) *reinterpret_cast<f4*>(to + 16 * ct + 4 * group) = r.o[ct][n];
            if (group == 0) {
                out.part_ml[(at * splits + split) * 2] = ref;
                out.part_ml[(at * splits + split) * 2 + 1] = sum;
            }
            continue;
        }
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        char* to = static_cast<char*>(out.out) + at * HD * ESIZE<CT>;
#pragma unroll
        for (int ct = 0; ct < HD / 16; ct++) {
            const f4 x = r.o[ct][n] * inv;
            if constexpr (ESIZE<CT> == 2)
                *reinterpret_cast<uint2*>(to + (16 * ct + 4 * group) * 2) = make_uint2(pack2(x[0], x[1], CT()), pack2(x[2], x[3], CT()));
            else
                *reinterpret_cast<f4*>(to + (16 * ct + 4 * group) * 4) = x;
        }
        if (out.lse && group == 0) out.lse[at] = sum > 0.f ? (ref + log2f(sum)) * 0.69314718055994530942f : -INFINITY;
    }
}

// ---- wq_prefill_attention ----------------------------------------------------------------------------------------------
struct PrefillArgs {
    const char *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;      // bytes from row to row
    const int32_t *q_off, *kv_off, *prefix_len;
    int64_t total_q, total_kv;
    int B, Hq, rep, splits;
    float scale;                               // log2(e) * sm_scale
    Out out;
};

template <typename CT, int HD>
__global__ __launch_bounds__(64 * WAVES, 2) void k_prefill(PrefillArgs a)
{
    constexpr bool DIRECT = ESIZE<CT> == 2;                       // two tiles in LDS: one is met while the next one arrives
    __shared__ __align__(16) u4 s_k[1 + DIRECT][K_PIECES<CT, HD>], s_v[1 + DIRECT][V_PIECES<CT, HD>];
    const int Hkv = a.Hq / a.rep, kvh = blockIdx.x % Hkv, split = blockIdx.y;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    Place p;
    if (!find_place(a.q_off, a.B, a.rep, a.total_q, (gridDim.x - 1 - blockIdx.x) / Hkv, p)) return;      // (the last rows see the most keys: they begin first)
    const int64_t kv0 = clipped(a.kv_off[p.seq], a.total_kv), kv1 = clipped(a.kv_off[p.seq + 1], a.total_kv);
    const int len = kv1 > kv0 ? (int)(kv1 - kv0) : 0;
    const int first = len - p.rows / a.rep;                       // position of the sequence's first query row
    int prefix = a.prefix_len ? a.prefix_len[p.seq] : 0;
    prefix = prefix < 0 ? 0 : (prefix > len ? len : prefix);
    // a row sees the keys below max(position + 1, prefix)
    auto limit_of = [&](int row) {
        const int seen = first + row / a.rep + 1;
        return seen > prefix ? seen : prefix;
    };
    const int last_row = (p.row0 + ROWS < p.rows ? p.row0 + ROWS : p.rows) - 1;
    const int tiles = (limit_of(last_row) + KEYS - 1) / KEYS;
    const int lo = (int)((int64_t)split * tiles / a.splits), hi = (int)((int64_t)(split + 1) * tiles / a.splits);

    Rows<HD> r;
    Query<CT, HD> q;
    clear(r);
    const int wrow0 = p.row0 + wave * COLS * 16;
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        const int row = wrow0 + 16 * n + (lane & 15);
        const char* at = nullptr;
        r.limit[n] = 0;
        r.scale[n] = a.scale;
        if (row < p.rows) {
            at = a.q + (p.first + row / a.rep) * a.q_stride + (kvh * a.rep + row % a.rep) * (HD * ESIZE<CT>);
            r.limit[n] = limit_of(row);
        }
        load_query<CT, CT, HD, false>(q, n, at);
    }
    const bool any = wrow0 < p.rows;
    const int wlast = wrow0 + COLS * 16 <= p.rows ? wrow0 + COLS * 16 - 1 : p.rows - 1;
    const int least = any ? limit_of(wrow0) : 0, most = any ? limit_of(wlast) : 0;
    const char* k = a.k + kv0 * a.k_stride + kvh * (HD * ESIZE<CT>);
    const char* v = a.v + kv0 * a.v_stride + kvh * (HD * ESIZE<CT>);
    if constexpr (DIRECT) {
        const Direct<HD> rows(a.k_stride, a.v_stride);
        auto load = [&](int t) {
            const int64_t key0 = (int64_t)t * KEYS;
            rows.load(k + key0 * a.k_stride, v + key0 * a.v_stride, len - (int)key0, reinterpret_cast<char*>(s_k[t & 1]), reinterpret_cast<char*>(s_v[t & 1]));
        };
        if (lo < hi) load(lo);
        __syncthreads();
        for (int t = lo; t < hi; t++) {
            if (t + 1 < hi) load(t + 1);
            __builtin_amdgcn_sched_barrier(0);                     // (the loads go out here)
            const int key0 = t * KEYS;
            const char *k_tile = reinterpret_cast<const char*>(s_k[t & 1]), *v_tile = reinterpret_cast<const char*>(s_v[t & 1]);
            if (key0 < most)
                attend_tile<CT, HD>(r, q, [&](int kt, int st) { return rows.keys(k_tile, kt, st); },
                                    [&](int vs, int ct) { return rows.values(v_tile, vs, ct); }, key0, key0 + KEYS > least);
            __syncthreads();                                       // the next tile is there, this one is free
        }
    } else {
        for (int t = lo; t < hi; t++) {
            const int key0 = t * KEYS;
            __syncthreads();
            stage_rows<CT, CT, HD, false>(k + key0 * a.k_stride, v + key0 * a.v_stride, a.k_stride, a.v_stride, len - key0, s_k[0], s_v[0]);
            __syncthreads();
            if (key0 < most) attend_staged<CT, HD>(r, q, s_k[0], s_v[0], key0, key0 + KEYS > least);
        }
    }
    store_rows<CT, HD>(r, p, a.rep, a.Hq, kvh, wave, split, a.splits, a.splits > 1, a.out);
}

// ---- wq_decode_attention_shared: the shared part --------------------------------------------------------------------------
struct SharedArgs {
    const char* q;                             // [B][Hq][hd]
    const int32_t* req_off;
    int B, P, Hq, rep, splits;
    float scale;
    wq_packed_kv kv;
    Out out;
};

// QT: the query's type; packed tokens are walked in fp16 (fp32 for fp32 queries), 16-bit rows in the cache's own type
template <typename QT, int HD>
__global__ __launch_bounds__(64 * WAVES, 2) void k_shared(SharedArgs a)
{
    using CT = std::conditional_t<std::is_same_v<QT, F32>, F32, F16>;
    using ST = std::conditional_t<std::is_same_v<QT, Bf16>, Bf16, F16>;        // of the 16-bit rows
    __shared__ __align__(16) u4 s_k[K_PIECES<CT, HD>], s_v[V_PIECES<CT, HD>];
    const int Hkv = a.kv.Hkv, kvh = blockIdx.x % Hkv, split = blockIdx.y;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    Place p;
    if (!find_place(a.req_off, a.P, a.rep, a.B, blockIdx.x / Hkv, p)) return;
    int tiles[4], all = 0, len[4];
#pragma unroll
    for (int c = 0; c < 4; c++) {
        const int64_t room = c < 3 ? a.kv.cap[c] - a.kv.cls_off[c][p.seq] : a.kv.cap16 - a.kv.off16[p.seq];
        len[c] = c < 3 ? a.kv.cls_len[c][p.seq] : a.kv.len16[p.seq];
        if (len[c] > room) len[c] = (int)room;
        tiles[c] = len[c] > 0 ? (len[c] + KEYS - 1) / KEYS : 0;
        all += tiles[c];
    }
    const int lo = (int)((int64_t)split * all / a.splits), hi = (int)((int64_t)(split + 1) * all / a.splits);

    Rows<HD> r;
    Query<CT, HD> q;
    clear(r);
    const int wrow0 = p.row0 + wave * COLS * 16;
    const char* at[COLS];
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        const int row = wrow0 + 16 * n + (lane & 15);
        at[n] = row < p.rows ? a.q + ((p.first + row / a.rep) * a.Hq + kvh * a.rep + row % a.rep) * (HD * ESIZE<QT>) : nullptr;
        r.scale[n] = a.scale;
        if constexpr (std::is_same_v<QT, Bf16>) {
            load_query<Bf16, Bf16, HD, true>(q, n, at[n]);
            r.scale[n] = a.scale * query_as_f16<HD>(q, n);
        } else {
            load_query<CT, QT, HD, true>(q, n, at[n]);
        }
    }
    const bool any = wrow0 < p.rows;
    int done = 0;                              // tiles of the classes before
    auto walk = [&](auto bits) __attribute__((always_inline)) {
        constexpr int BITS = decltype(bits)::value, c = BITS == 2 ? 0 : (BITS == 4 ? 1 : 2);
        const int64_t tok0 = a.kv.cls_off[c][p.seq];
        const int64_t slots = (len[c] + 31) / 32 * 32;
        const int t0 = lo > done ? lo - done : 0, t1 = hi - done < tiles[c] ? hi - done : tiles[c];
        for (int t = t0; t < t1; t++) {
            const int key0 = t * KEYS;
            __syncthreads();
            stage_packed<CT, HD, BITS>(a.kv, kvh, tok0 + key0, slots - key0, s_k, s_v);
            __syncthreads();
#pragma unroll
            for (int n = 0; n < COLS; n++) r.limit[n] = len[c];
            if (any) attend_staged<CT, HD>(r, q, s_k, s_v, key0, key0 + KEYS > len[c]);
        }
        done += tiles[c];
    };
    walk(std::integral_constant<int, 2>());
    walk(std::integral_constant<int, 4>());
    walk(std::integral_constant<int, 8>());
    if (hi > done) {
        using CR = std::conditional_t<std::is_same_v<QT, Bf16>, Bf16, CT>;
        if constexpr (std::is_same_v<QT, Bf16>) {
#pragma unroll
            for (int n = 0; n < COLS; n++) {
                load_query<Bf16, Bf16, HD, true>(q, n, at[n]);
                r.scale[n] = a.scale;
            }
        }
        const int64_t row0 = a.kv.off16[p.seq], stride = (int64_t)a.kv.Hkv * HD * 2;
        const char* k = static_cast<const char*>(a.kv.k16) + row0 * stride + kvh * (HD * 2);
        const char* v = static_cast<const char*>(a.kv.v16) + row0 * stride + kvh * (HD * 2);
        const int t0 = lo > done ? lo - done : 0;
        for (int t = t0; t < hi - done; t++) {
            const int key0 = t * KEYS;
            __syncthreads();
            stage_rows<CR, ST, HD, true>(k + key0 * stride, v + key0 * stride, stride, stride, len[3] - key0, s_k, s_v);
            __syncthreads();
#pragma unroll
            for (int n = 0; n < COLS; n++) r.limit[n] = len[3];
            if (any) attend_staged<CR, HD>(r, q, s_k, s_v, key0, key0 + KEYS > len[3]);
        }
    }
    store_rows<QT, HD>(r, p, a.rep, a.Hq, kvh, wave, split, a.splits, true, a.out);
}

// ---- the splits' merge -------------------------------------------------------------------------------------------------
struct CombineArgs {
    int64_t rows;              // (q row, head) pairs
    int Hq, splits, dtype;
    const int32_t* off;        // rows of q outside off[0] .. off[nseq] - 1 have no partials,
    int nseq;
    bool leave;                // ... and are left as they were
    const float* own_out;      // NULL, or one more partial, normalised [rows][hd], with its log-sum-exp
    const float* own_lse;
    Out out;
};

// A wavefront per row; a lane takes one or two channels.
template <int HD>
__global__ __launch_bounds__(256) void k_attend_combine(CombineArgs a)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= a.rows) return;
    const int lane = threadIdx.x & 63;
    int n = a.splits;
    const int64_t b = row / a.Hq;
    if (b < a.off[0] || b >= a.off[a.nseq]) {
        if (a.leave) return;
        n = 0;
    }
    const float* ml = a.out.part_ml + row * a.splits * 2;
    float M = -INFINITY;
    for (int s = 0; s < n; s++) M = fmaxf(M, ml[2 * s]);
    const float own = a.own_lse ? a.own_lse[row] * LOG2E : -INFINITY;
    M = fmaxf(M, own);
    float L = 0.f, x[HD / 64] = {};
    if (M > -INFINITY) {
        for (int s = 0; s < n; s++) {
            const float m = ml[2 * s], w = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
            L = fmaf(ml[2 * s + 1], w, L);
#pragma unroll
            for (int i = 0; i < HD / 64; i++) x[i] = fmaf(a.out.part[(row * a.splits + s) * HD + 64 * i + lane], w, x[i]);
        }
        if (own > -INFINITY) {
            const float w = __builtin_amdgcn_exp2f(own - M);
            L += w;
#pragma unroll
            for (int i = 0; i < HD / 64; i++) x[i] = fmaf(a.own_out[row * HD + 64 * i + lane], w, x[i]);
        }
    }
    const float inv = L > 0.f ? 1.f / L : 0.f;
#pragma unroll
    for (int i = 0; i < HD / 64; i++) {
        const int64_t at = row * HD + 64 * i + lane;
        const float y = x[i] * inv;
        if (a.dtype == WQ_F32) static_cast<float*>(a.out.out)[at] = y;
        else static_cast<uint16_t*>(a.out.out)[at] = a.dtype == WQ_BF16 ? (uint16_t)pack2(y, 0.f, Bf16()) : (uint16_t)pack2(y, 0.f, F16());
    }
    if (a.out.lse && lane == 0) a.out.lse[row] = L > 0.f ? (M + log2f(L)) * 0.69314718055994530942f : -INFINITY;
}

void combine(wq_ctx* ctx, const CombineArgs& c, int hd)
{
    hipLaunchKernelGGL(hd == 128 ? k_attend_combine<128> : k_attend_combine<64>, dim3((unsigned)((c.rows + 3) / 4)), dim3(256), 0, ctx->stream, c);
}

int64_t tiles_of(int64_t total, int rep, int nseq) { return total * rep / ROWS + nseq; }

int auto_splits_of(int64_t workgroups, int64_t max_keys)
{
    int64_t s = workgroups > 0 ? (512 + workgroups - 1) / workgroups : 1;
    const int64_t most = (max_keys + 4 * KEYS - 1) / (4 * KEYS);
    if (s > most) s = most;
    if (s > WQ_MAX_ATTEND_SPLITS) s = WQ_MAX_ATTEND_SPLITS;
    return s < 1 ? 1 : (int)s;
}

size_t partials_bytes(int64_t rows, int hd, int splits) { return wq_align256((size_t)rows * splits * (hd + 2) * sizeof(float)); }

}  // namespace

int wq_prefill_splits(int64_t total_q, int B, int Hq, int Hkv, int64_t max_kv_rows)
{
    return auto_splits_of(tiles_of(total_q, Hq / Hkv, 0) * Hkv + (int64_t)Hkv * (total_q < B ? total_q : B), max_kv_rows);
}
size_t wq_prefill_ws_bytes(int64_t total_q, int Hq, int hd, int splits)
{
    return splits > 1 ? partials_bytes(total_q * Hq, hd, splits) : 0;
}

int wq_shared_splits(int B, int P, int Hq, int Hkv, int64_t max_prefix_tokens)
{
    return auto_splits_of(tiles_of(B, Hq / Hkv, P) * Hkv, max_prefix_tokens);
}
size_t wq_shared_ws_bytes(int B, int Hq, int hd, int splits)
{
    const size_t rows = (size_t)B * Hq;
    return partials_bytes(rows, hd, splits) + wq_align256(rows * hd * sizeof(float)) + wq_align256(rows * sizeof(float));
}

int wq_launch_prefill(wq_ctx* ctx, const WqPrefill& f)
{
    PrefillArgs a;
    const int size = f.dtype == WQ_F32 ? 4 : 2;
    a.q = static_cast<const char*>(f.q), a.k = static_cast<const char*>(f.k), a.v = static_cast<const char*>(f.v);
    a.q_stride = f.q_stride * size, a.k_stride = f.k_stride * size, a.v_stride = f.v_stride * size;
    a.q_off = f.q_off, a.kv_off = f.kv_off, a.prefix_len = f.prefix_len;
    a.total_q = f.total_q, a.total_kv = f.total_kv;
    a.B = f.B, a.Hq = f.Hq, a.rep = f.Hq / f.Hkv, a.splits = f.splits;
    a.scale = f.sm_scale * LOG2E;
    a.out.out = f.out, a.out.lse = f.lse;
    a.out.part = reinterpret_cast<float*>(ctx->ws + WQ_WS_HEADER);
    a.out.part_ml = a.out.part + f.total_q * f.Hq * f.splits * f.hd;
    const dim3 grid((unsigned)(f.Hkv * tiles_of(f.total_q, a.rep, f.B)), (unsigned)f.splits);
    void (*kernel)(PrefillArgs) = f.dtype == WQ_F32 ? (f.hd == 128 ? k_prefill<F32, 128> : k_prefill<F32, 64>)
                                : f.dtype == WQ_BF16 ? (f.hd == 128 ? k_prefill<Bf16, 128> : k_prefill<Bf16, 64>)
                                                     : (f.hd == 128 ? k_prefill<F16, 128> : k_prefill<F16, 64>);
    hipLaunchKernelGGL(kernel, grid, dim3(64 * WAVES), 0, ctx->stream, a);
    if (f.splits > 1) combine(ctx, CombineArgs{f.total_q * f.Hq, f.Hq, f.splits, f.dtype, f.q_off, f.B, true, nullptr, nullptr, a.out}, f.hd);
    WQ_HIP_CHECK(ctx, hipGetLastError());
    return WQ_OK;
}

// Three launches: every request over its own cache (wq_decode_attention's kernels), the shared caches, the merge.
int wq_launch_shared(wq_ctx* ctx, const WqShared& f)
{
    const wq_packed_kv* kv = f.prefix;
    const int64_t rows = (int64_t)f.B * f.Hq;
    SharedArgs a;
    a.q = static_cast<const char*>(f.q);
    a.req_off = f.req_off;
    a.B = f.B, a.P = kv->B, a.Hq = f.Hq, a.rep = f.Hq / kv->Hkv, a.splits = f.splits;
    a.scale = f.sm_scale * LOG2E;
    a.kv = *kv;
    a.out.out = f.out, a.out.lse = f.lse;
    char* at = ctx->ws + WQ_WS_HEADER + f.own_ws_bytes;
    a.out.part = reinterpret_cast<float*>(at);
    a.out.part_ml = a.out.part + rows * f.splits * kv->hd;
    at += partials_bytes(rows, kv->hd, f.splits);
    float* own_out = nullptr;
    float* own_lse = nullptr;
    if (f.own) {
        own_out = reinterpret_cast<float*>(at);
        own_lse = reinterpret_cast<float*>(at + wq_align256(rows * kv->hd * sizeof(float)));
        const int rc = wq_launch_decode(ctx, f.q, f.q_dtype, f.B, f.Hq, f.own, f.sm_scale, f.own_splits, f.own_algo, own_out, own_lse);
        if (rc != WQ_OK) return rc;
    }
    const dim3 grid((unsigned)(kv->Hkv * tiles_of(f.B, a.rep, a.P)), (unsigned)f.splits);
    void (*kernel)(SharedArgs) = f.q_dtype == WQ_F32 ? (kv->hd == 128 ? k_shared<F32, 128> : k_shared<F32, 64>)
                               : f.q_dtype == WQ_BF16 ? (kv->hd == 128 ? k_shared<Bf16, 128> : k_shared<Bf16, 64>)
                                                      : (kv->hd == 128 ? k_shared<F16, 128> : k_shared<F16, 64>);
    hipLaunchKernelGGL(kernel, grid, dim3(64 * WAVES), 0, ctx->stream, a);
    combine(ctx, CombineArgs{rows, f.Hq, f.splits, f.q_dtype, f.req_off, a.P, false, own_out, own_lse, a.out}, kv->hd);
    WQ_HIP_CHECK(ctx, hipGetLastError());
    return WQ_OK;
}
