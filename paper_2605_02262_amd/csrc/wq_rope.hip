// Rotary positions: channel pairs (a, b) of the first rot_dim channels of every query and key head become
//     a' = (a cos t - b sin t) mscale,   b' = (b cos t + a sin t) mscale,   t = position * inv_freq[pair],
// with the pair's channels half a rot_dim apart or next to each other.  k_rope turns a prompt's rows, k_rope_append the new
// token of every sequence and writes its key and value into the cache (the quantizer and the decode calls read rotated keys).
//
// The angle is reduced in fp64: a product of a far position and a frequency has more digits before the point than fp32
// has after it (position 10^6: an fp32 product is off by 0.06 rad).  One lane per frequency takes cosine and sine of a
// row's angle once for all heads, through LDS; with them per (head, pair) the trigonometry alone would cost a
// quarter of the call.
#include "wq_internal.h"

namespace {

struct RopeArgs {
    const void* x[2];          // queries, keys
    void* y[2];
    int64_t x_stride[2], y_stride[2];   // elements from row to row
    int heads[2];
    const int32_t* positions;
    const float* inv_freq;
    float mscale;
    int rot;
    int64_t rows;
};

// cos, sin of position * frequency, times mscale
__device__ __forceinline__ float2 rope_turn(int position, float inv_freq, float mscale)
{
    constexpr double PER_TURN = 0.15915494309189533577;       // 1 / 2 pi
    double t = (double)position * (double)inv_freq * PER_TURN;
    t -= rint(t);                                              // [-1/2, 1/2] turns
    float s, c;
    sincospif((float)(2.0 * t), &s, &c);
    return make_float2(c * mscale, s * mscale);
}

template <typename T>
struct Piece {                 // 8 consecutive elements as they lie in memory
    uint4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Piece<T> load_piece(const T* p)
{
    Piece<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; i++) r.w[i] = reinterpret_cast<const uint4*>(p)[i];
    return r;
}
template <typename T>
__device__ __forceinline__ void store_piece(T* p, const Piece<T>& r)
{
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; i++) reinterpret_cast<uint4*>(p)[i] = r.w[i];
}
template <typename T>
__device__ __forceinline__ void to_floats(const Piece<T>& r, float* x) { wq_ld8(reinterpret_cast<const T*>(&r), x); }

__device__ __forceinline__ uint16_t round16(float x, __hip_bfloat16) { return __bfloat16_as_ushort(__float2bfloat16(x)); }
__device__ __forceinline__ uint16_t round16(float x, __half) { return __half_as_ushort(__float2half_rn(x)); }

template <typename T>
__device__ __forceinline__ Piece<T> from_floats(const float* x)
{
    Piece<T> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; i++)
            r.w[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = round16(x[2 * i], T()) | (uint32_t)round16(x[2 * i + 1], T()) << 16;
        r.w[0] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return r;
}

// One unit of a head's work: two pieces that hold 8 pairs (halves), one that holds 4 (neighbours), or one behind rot_dim,
// which is copied.
template <bool PAIRS>
__device__ __forceinline__ int units_of(int hd, int rot) { return PAIRS ? hd / 8 : rot / 16 + (hd - rot) / 8; }

template <typename T, bool PAIRS>
struct Unit {
    Piece<T> a, b;
    int at;                    // first channel of a
    bool turned;
    __device__ __forceinline__ void place(int u, int rot)
    {
        if constexpr (PAIRS) {
            at = 8 * u;
            turned = at < rot;
        } else {
            const int n = rot / 16;
            turned = u < n;
            at = turned ? 8 * u : rot + 8 * (u - n);
        }
    }
    __device__ __forceinline__ void load(const T* head, int rot)
    {
        a = load_piece(head + at);
        if (!PAIRS && turned) b = load_piece(head + at + rot / 2);
    }
    __device__ __forceinline__ void turn(const float2* cs)
    {
        if (!turned) return;
        float x[8];
        to_floats(a, x);
        if constexpr (PAIRS) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float2 t = cs[at / 2 + i];
                const float p = x[2 * i], q = x[2 * i + 1];
                x[2 * i] = fmaf(p, t.x, -(q * t.y));
                x[2 * i + 1] = fmaf(q, t.x, p * t.y);
            }
            a = from_floats<T>(x);
        } else {
            float z[8];
            to_floats(b, z);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float2 t = cs[at + i];
                const float p = x[i], q = z[i];
                x[i] = fmaf(p, t.x, -(q * t.y));
                z[i] = fmaf(q, t.x, p * t.y);
            }
            a = from_floats<T>(x);
            b = from_floats<T>(z);
        }
    }
};

// A wavefront per row; four units per lane are in flight while the angles are found.
template <typename T, int HD, bool PAIRS>
__global__ __launch_bounds__(256) void k_rope(RopeArgs a)
{
    __shared__ float2 s_cs[4][HD / 2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * 4 + wave;
    const bool real = row < a.rows;
    const int per = units_of<PAIRS>(HD, a.rot), nq = a.heads[0] * per, n = nq + a.heads[1] * per;
    float2* cs = s_cs[wave];
    constexpr int K = 4;
    for (int u0 = 0; u0 < n; u0 += 64 * K) {
        Unit<T, PAIRS> unit[K];
        T* to[K];
#pragma unroll
        for (int k = 0; k < K; k++) {
            const int u = u0 + 64 * k + lane;
            to[k] = nullptr;
            if (!real || u >= n) continue;
            const int which = u >= nq, v = u - (which ? nq : 0), head = v / per;
            unit[k].place(v - head * per, a.rot);
            const T* from = static_cast<const T*>(a.x[which]) + row * a.x_stride[which] + (int64_t)head * HD;
            unit[k].load(from, a.rot);
            to[k] = static_cast<T*>(a.y[which]) + row * a.y_stride[which] + (int64_t)head * HD;
        }
        if (u0 == 0) {
            if (real && lane < a.rot / 2) cs[lane] = rope_turn(a.positions[row], a.inv_freq[lane], a.mscale);
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < K; k++) {
            if (!to[k]) continue;
            unit[k].turn(cs);
            store_piece(to[k] + unit[k].at, unit[k].a);
            if (!PAIRS && unit[k].turned) store_piece(to[k] + unit[k].at + a.rot / 2, unit[k].b);
        }
    }
}

// 8 values of a row in the cache's 16-bit type: raw for the 16-bit types, fp32 to fp16
template <typename T>
__device__ __forceinline__ uint4 cache_piece(const Piece<T>& p)
{
    if constexpr (sizeof(T) == 2) {
        return p.w[0];
    } else {
        float x[8];
        to_floats(p, x);
        return from_floats<__half>(x).w[0];
    }
}

// A workgroup per sequence: its queries are turned, its key is turned into row off16[b] + len16[b] of the cache, its value
// copied there, and len16[b] raised.
template <typename T, int HD, bool PAIRS>
__global__ __launch_bounds__(256) void k_rope_append(RopeArgs a, const T* __restrict__ v, int64_t v_stride, wq_packed_kv kv, uint32_t* __restrict__ status)
{
    __shared__ float2 cs[HD / 2];
    const int b = blockIdx.x, tid = threadIdx.x;
    const int64_t at = (int64_t)kv.off16[b] + kv.len16[b];
    const bool full = at >= kv.off16[b + 1] || at >= kv.cap16;
    if (tid < a.rot / 2) cs[tid] = rope_turn(a.positions[b], a.inv_freq[tid], a.mscale);
    __syncthreads();                       // (also: every lane has read len16[b] before it changes)
    const int per = units_of<PAIRS>(HD, a.rot), nq = a.heads[0] * per, nk = full ? 0 : a.heads[1] * per, nv = full ? 0 : a.heads[1] * (HD / 8);
    for (int u = tid; u < nq + nk; u += 256) {
        const int which = u >= nq, w = u - (which ? nq : 0), head = w / per;
        Unit<T, PAIRS> unit;
        unit.place(w - head * per, a.rot);
        unit.load(static_cast<const T*>(a.x[which]) + b * a.x_stride[which] + (int64_t)head * HD, a.rot);
        unit.turn(cs);
        const bool two = !PAIRS && unit.turned;
        if (!which) {
            T* to = static_cast<T*>(a.y[0]) + b * a.y_stride[0] + (int64_t)head * HD + unit.at;
            store_piece(to, unit.a);
            if (two) store_piece(to + a.rot / 2, unit.b);
        } else {
            uint16_t* to = static_cast<uint16_t*>(kv.k16) + (at * kv.Hkv + head) * HD + unit.at;
            *reinterpret_cast<uint4*>(to) = cache_piece(unit.a);
            if (two) *reinterpret_cast<uint4*>(to + a.rot / 2) = cache_piece(unit.b);
        }
    }
    for (int u = tid; u < nv; u += 256) {
        const int64_t e = 8 * (int64_t)u;
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(kv.v16) + at * kv.Hkv * HD + e) = cache_piece(load_piece(v + b * v_stride + e));
    }
    if (tid == 0) {
        if (full) atomicOr(status, WQ_DEV_SEG16_OVERFLOW);
        else kv.len16[b] += 1;
    }
}

template <typename T, int HD>
void rope(wq_ctx* ctx, const RopeArgs& a, bool pairs)
{
    const int64_t most = 4 * WQ_MOST_GROUPS_256;               // rows of a launch
    for (int64_t done = 0; done < a.rows; done += most) {
        RopeArgs part = a;
        for (int i = 0; i < 2; i++) {
            if (!a.heads[i]) continue;
            part.x[i] = static_cast<const T*>(a.x[i]) + done * a.x_stride[i];
            part.y[i] = static_cast<T*>(a.y[i]) + done * a.y_stride[i];
        }
        part.positions += done;
        part.rows = a.rows - done < most ? a.rows - done : most;
        hipLaunchKernelGGL((pairs ? k_rope<T, HD, true> : k_rope<T, HD, false>), dim3((unsigned)((part.rows + 3) / 4)), dim3(256), 0, ctx->stream, part);
    }
}
template <typename T, int HD>
void append(wq_ctx* ctx, const RopeArgs& a, bool pairs, const void* v, int64_t v_stride, const wq_packed_kv* kv)
{
    hipLaunchKernelGGL((pairs ? k_rope_append<T, HD, true> : k_rope_append<T, HD, false>), dim3((unsigned)a.rows), dim3(256), 0, ctx->stream, a,
                       static_cast<const T*>(v), v_stride, *kv, wq_status_ptr(ctx));
}

RopeArgs rope_args(const WqRope& r)
{
    RopeArgs a;
    a.x[0] = r.q, a.x[1] = r.k, a.y[0] = r.q_out, a.y[1] = r.k_out;
    a.x_stride[0] = r.q_stride, a.x_stride[1] = r.k_stride, a.y_stride[0] = r.q_out_stride, a.y_stride[1] = r.k_out_stride;
    a.heads[0] = r.Hq, a.heads[1] = r.Hkv;
    a.positions = r.positions, a.inv_freq = r.inv_freq, a.mscale = r.mscale, a.rot = r.rot_dim, a.rows = r.rows;
    return a;
}

}  // namespace

#define WQ_BY_TYPE(call, ...)                                                                                                       \
    switch (r.dtype) {                                                                                                              \
        case WQ_F32: r.hd == 128 ? call<float, 128>(__VA_ARGS__) : call<float, 64>(__VA_ARGS__); break;                             \
        case WQ_BF16: r.hd == 128 ? call<__hip_bfloat16, 128>(__VA_ARGS__) : call<__hip_bfloat16, 64>(__VA_ARGS__); break;          \
        default: r.hd == 128 ? call<__half, 128>(__VA_ARGS__) : call<__half, 64>(__VA_ARGS__);                                      \
    }

int wq_launch_rope(wq_ctx* ctx, const WqRope& r)
{
    const RopeArgs a = rope_args(r);
    WQ_BY_TYPE(rope, ctx, a, r.layout == WQ_ROPE_PAIRS)
    WQ_HIP_CHECK(ctx, hipGetLastError());
    return WQ_OK;
}

int wq_launch_rope_append(wq_ctx* ctx, const WqRope& r, const void* v, int64_t v_stride, const wq_packed_kv* kv)
{
    const RopeArgs a = rope_args(r);
    WQ_BY_TYPE(append, ctx, a, r.layout == WQ_ROPE_PAIRS, v, v_stride, kv)
    WQ_HIP_CHECK(ctx, hipGetLastError());
    return WQ_OK;
}
