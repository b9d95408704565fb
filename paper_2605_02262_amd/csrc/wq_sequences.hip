// What a serving program does with a batch's rows and caches between its layers' kernels: wq_tree_accept (which drafted rows stay),
// wq_append_rows (their keys and values into every layer's cache) and wq_copy_sequences (forks, compaction).
#include <type_traits>

#include "wq_internal.h"

namespace {

__device__ __forceinline__ int64_t clipped(int64_t x, int64_t most) { return x < 0 ? 0 : (x > most ? most : x); }

// ---- wq_tree_accept ----------------------------------------------------------------------------------------------------
// A workgroup per sequence.  Every row looks whether its parent's choice is its token, the first such row of a parent is its child, and one
// lane follows the children from row 0.
__global__ __launch_bounds__(256) void k_accept(WqAccept a, uint32_t* status)
{
    __shared__ int32_t s_child[WQ_MAX_TREE], s_token[WQ_MAX_TREE];
    __shared__ int s_count;
    const int b = blockIdx.x;
    const int64_t first = clipped(a.row_off[b], a.total_rows);
    int64_t rows = clipped(a.row_off[b + 1], a.total_rows) - first;
    if (rows > a.max_rows && threadIdx.x == 0) atomicOr(status, WQ_DEV_TOO_MANY_ROWS);
    const int n = rows < 0 ? 0 : (int)(rows > a.max_rows ? a.max_rows : rows);
    for (int i = threadIdx.x; i < n; i += 256) s_child[i] = WQ_MAX_TREE, s_token[i] = a.target[first + i];
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 256) {
        const int up = a.parent ? a.parent[first + i] : i - 1;
        if (up >= 0 && up < i && a.tokens[first + i] == s_token[up]) atomicMin(&s_child[up], i);
    }
    __syncthreads();
    int32_t* path = a.path + (int64_t)b * a.max_path;
    if (threadIdx.x == 0) {
        int count = 0, last = -1;
        for (int at = 0; at < n && count < a.max_path; at = s_child[at]) path[count++] = last = at;
        a.n_path[b] = count;
        a.next_token[b] = last >= 0 ? s_token[last] : -1;
        s_count = count;
    }
    __syncthreads();
    for (int i = s_count + threadIdx.x; i < a.max_path; i += 256) path[i] = -1;
}

// ---- wq_append_rows ----------------------------------------------------------------------------------------------------
constexpr int APPEND_LAYERS = 48;              // of a launch: what its arguments hold
struct AppendArgs {
    const char *k[APPEND_LAYERS], *v[APPEND_LAYERS];
    uint16_t *k16[APPEND_LAYERS], *v16[APPEND_LAYERS];
    int32_t *off16[APPEND_LAYERS], *len16[APPEND_LAYERS];
    int64_t cap16[APPEND_LAYERS];
    int64_t k_stride, v_stride;                // elements from row to row
    const int32_t *row_off, *take, *n_take;
    int64_t total_rows;
    int B, max_take, row_elems, pieces;        // pieces: workgroups that share a sequence's rows of a layer
    uint32_t* status;
};
constexpr int PIECE_ROWS = 16;

// How many rows sequence b gets in this layer; 0 where it is refused (the bits that say why in *bits).  For all threads of a workgroup.
__device__ __forceinline__ int rows_of(const AppendArgs& a, int layer, int b, uint32_t* bits)
{
    const int64_t first = clipped(a.row_off[b], a.total_rows), rows = clipped(a.row_off[b + 1], a.total_rows) - first;
    int64_t n = a.take ? a.n_take[b] : (rows > 0 ? rows : 0);
    uint32_t bad = 0;
    if (n < 0) bad = WQ_DEV_BAD_INDEX;
    else if (n > a.max_take) bad = WQ_DEV_TOO_MANY_ROWS;
    else if (a.take) {
        bool out = false;
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int at = a.take[(int64_t)b * a.max_take + i];
            out = out || at < 0 || at >= rows;
        }
        if (__syncthreads_or(out)) bad = WQ_DEV_BAD_INDEX;
    }
    const int64_t from = a.off16[layer][b], held = a.len16[layer][b], end = a.off16[layer][b + 1] < a.cap16[layer] ? a.off16[layer][b + 1] : a.cap16[layer];
    if (!bad && (from < 0 || held < 0 || (n > 0 && from + held + n > end))) bad = WQ_DEV_SEG16_OVERFLOW;
    *bits = bad;
    return bad ? 0 : (int)n;
}

template <typename T>
__device__ __forceinline__ uint4 as_16bit(const T* p)
{
    if constexpr (sizeof(T) == 2) {
        return *reinterpret_cast<const uint4*>(p);
    } else {
        typedef _Float16 h8 __attribute__((ext_vector_type(8)));
        float x[8];
        wq_ld8(p, x);
        h8 y;
#pragma unroll
        for (int i = 0; i < 8; i++) y[i] = (_Float16)x[i];    // to nearest even
        return __builtin_bit_cast(uint4, y);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_append_rows(AppendArgs a)
{
    const int piece = blockIdx.x % a.pieces, b = blockIdx.x / a.pieces % a.B, layer = blockIdx.x / a.pieces / a.B;
    uint32_t bad;
    const int n = rows_of(a, layer, b, &bad);
    if (bad && piece == 0 && threadIdx.x == 0) atomicOr(a.status, bad);
    const int64_t first = clipped(a.row_off[b], a.total_rows), to = (int64_t)a.off16[layer][b] + a.len16[layer][b];
    __syncthreads();                           // every lane has read len16[b] before it changes
    const int row0 = piece * PIECE_ROWS, rows = a.pieces == 1 ? n : (n - row0 < PIECE_ROWS ? n - row0 : PIECE_ROWS), chunks = a.row_elems / 8;
    for (int u = threadIdx.x; u < rows * 2 * chunks; u += 256) {
        const int row = u / (2 * chunks), c = u % (2 * chunks), at = row0 + row, e = (c < chunks ? c : c - chunks) * 8;
        const int64_t from = first + (a.take ? a.take[(int64_t)b * a.max_take + at] : at);
        const bool value = c >= chunks;
        const T* src = reinterpret_cast<const T*>(value ? a.v[layer] : a.k[layer]) + from * (value ? a.v_stride : a.k_stride) + e;
        uint16_t* dst = (value ? a.v16[layer] : a.k16[layer]) + (to + at) * a.row_elems + e;
        *reinterpret_cast<uint4*>(dst) = as_16bit(src);
    }
    if (a.pieces == 1 && threadIdx.x == 0 && n > 0) a.len16[layer][b] += n;
}

// Where a sequence's rows are copied by several workgroups, its length is raised when all of them are done
__global__ __launch_bounds__(64) void k_raise(AppendArgs a)
{
    const int b = blockIdx.x % a.B, layer = blockIdx.x / a.B;
    uint32_t bad;
    const int n = rows_of(a, layer, b, &bad);
    __syncthreads();
    if (threadIdx.x == 0 && n > 0) a.len16[layer][b] += n;
}

// ---- wq_copy_sequences -------------------------------------------------------------------------------------------------
struct CopyCache {
    char *codes[3], *meta[3], *k16, *v16;
    int32_t *cls_off[3], *cls_len[3], *off16, *len16;
    float* v_scale_max;
    int64_t cap[3], cap16;
};
constexpr int COPY_LAYERS = 10;                // of a launch: what its arguments hold
struct CopyArgs {
    CopyCache src[COPY_LAYERS], dst[COPY_LAYERS];
    const int32_t* from;
    int src_B, dst_B, Hkv, hd, groups;
    int64_t end[4];                            // workgroups of k_copy over a layer: of the classes 0, .. 0 to 2, .. and the 16-bit rows
    uint32_t* status;
};

__device__ __forceinline__ int pad32(int n) { return (n + 31) & ~31; }

// Tokens that a sequence really has room for in its cache (tables that say more are not followed)
__device__ __forceinline__ int tokens_of(const CopyCache& c, int k, int s)
{
    const int64_t off = k < 3 ? c.cls_off[k][s] : c.off16[s], room = (k < 3 ? c.cap[k] : c.cap16) - off;
    const int n = k < 3 ? c.cls_len[k][s] : c.len16[s];
    return off < 0 || n < 0 ? 0 : (n > room ? (int)(room < 0 ? 0 : room) : n);
}

// The copies' tables.  A workgroup per layer; a running sum over the sequences, 1024 at a time.
__global__ __launch_bounds__(1024) void k_copy_plan(CopyArgs a)
{
    __shared__ int64_t s_sum[3][16];
    const CopyCache &src = a.src[blockIdx.x], &dst = a.dst[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t before[3] = {0, 0, 0};             // tokens of the sequences in front of these 1024
    uint32_t bits = 0;
    for (int d0 = 0; d0 < a.dst_B; d0 += 1024) {
        const int d = d0 + threadIdx.x;
        int s = d < a.dst_B ? a.from[d] : -1, len[4] = {0, 0, 0, 0};
        if (s < -1 || s >= a.src_B) bits |= WQ_DEV_BAD_INDEX, s = -1;
        if (s >= 0)
#pragma unroll
            for (int k = 0; k < 4; k++) len[k] = tokens_of(src, k, s);
        int64_t sum[3];
#pragma unroll
        for (int k = 0; k < 3; k++) {
            sum[k] = pad32(len[k]);
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                const int64_t y = __shfl_up(sum[k], o, 64);
                if (lane >= o) sum[k] += y;
            }
            if (lane == 63) s_sum[k][wave] = sum[k];
        }
        __syncthreads();
        bool fits = true;
#pragma unroll
        for (int k = 0; k < 3; k++) {
            int64_t all = 0, front = 0;
            for (int w = 0; w < 16; w++) {
                if (w < wave) front += s_sum[k][w];
                all += s_sum[k][w];
            }
            const int64_t end = before[k] + front + sum[k], begin = end - pad32(len[k]);
            if (len[k] > 0 && end > dst.cap[k]) bits |= WQ_DEV_CLASS_OVERFLOW, fits = false;
            if (d < a.dst_B) dst.cls_off[k][d] = (int32_t)(begin < dst.cap[k] ? begin : dst.cap[k]);
            if (d == a.dst_B - 1) dst.cls_off[k][d + 1] = (int32_t)(end < dst.cap[k] ? end : dst.cap[k]);
            before[k] += all;
        }
        if (d < a.dst_B) {
            const int64_t off = dst.off16[d], end = dst.off16[d + 1] < dst.cap16 ? dst.off16[d + 1] : dst.cap16;
            if (len[3] > 0 && (off < 0 || off + len[3] > end)) bits |= WQ_DEV_SEG16_OVERFLOW, fits = false;
#pragma unroll
            for (int k = 0; k < 3; k++) dst.cls_len[k][d] = fits ? len[k] : 0;
            dst.len16[d] = fits ? len[3] : 0;
            dst.v_scale_max[d] = fits && s >= 0 ? src.v_scale_max[s] : 0.f;
        }
        __syncthreads();
    }
    if (bits) atomicOr(a.status, bits);
}

constexpr int COPY_BYTES = 16384;              // of codes, or of 16-bit rows, that a workgroup copies

// Blocks of 32 tokens of a class (a plane and a KV head), or 16-bit rows, by the tables that k_copy_plan has left
__global__ __launch_bounds__(256) void k_copy(CopyArgs a)
{
    const int64_t unit = blockIdx.x;
    const CopyCache &src = a.src[blockIdx.y], &dst = a.dst[blockIdx.y];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int k = unit < a.end[0] ? 0 : unit < a.end[1] ? 1 : unit < a.end[2] ? 2 : 3;
    const int64_t u = unit - (k > 0 ? a.end[k - 1] : 0);
    if (k < 3) {
        const int bytes = 4 * a.hd * (2 << k), words = 128 * a.groups;         // of a block's codes and metadata
        const int per = COPY_BYTES / bytes, planes = 2 * a.Hkv, plane = (int)(u % planes);
        const int64_t j0 = u / planes * per, used = dst.cls_off[k][a.dst_B] / 32;
        for (int64_t j = j0 + wave; j < j0 + per && j < used; j += 4) {
            const int d = wq_find_seq(dst.cls_off[k], a.dst_B, 32 * j), s = a.from[d];
            const int64_t in = j - dst.cls_off[k][d] / 32;
            if (32 * in >= dst.cls_len[k][d]) continue;
            const int64_t i = src.cls_off[k][s] / 32 + in;
            const uint4* x = reinterpret_cast<const uint4*>(src.codes[k] + (plane * (src.cap[k] / 32) + i) * bytes);
            uint4* y = reinterpret_cast<uint4*>(dst.codes[k] + (plane * (dst.cap[k] / 32) + j) * bytes);
            for (int e = lane; e < bytes / 16; e += 64) y[e] = x[e];
            x = reinterpret_cast<const uint4*>(src.meta[k] + (plane * (src.cap[k] / 32) + i) * words);
            y = reinterpret_cast<uint4*>(dst.meta[k] + (plane * (dst.cap[k] / 32) + j) * words);
            for (int e = lane; e < words / 16; e += 64) y[e] = x[e];
        }
        return;
    }
    const int bytes = a.Hkv * a.hd * 2, per = bytes < COPY_BYTES ? COPY_BYTES / bytes : 1;
    const int64_t row0 = u / 2 * per;
    const char* from = u & 1 ? src.v16 : src.k16;
    char* to = u & 1 ? dst.v16 : dst.k16;
    for (int64_t row = row0 + wave; row < row0 + per && row < dst.cap16; row += 4) {
        if (row < dst.off16[0] || row >= dst.off16[a.dst_B]) continue;
        const int d = wq_find_seq(dst.off16, a.dst_B, row);
        const int64_t in = row - dst.off16[d];
        if (in >= dst.len16[d]) continue;
        const uint4* x = reinterpret_cast<const uint4*>(from + (src.off16[a.from[d]] + in) * bytes);
        uint4* y = reinterpret_cast<uint4*>(to + row * bytes);
        for (int e = lane; e < bytes / 16; e += 64) y[e] = x[e];
    }
}

}  // namespace

int wq_launch_accept(wq_ctx* ctx, const WqAccept& f)
{
    hipLaunchKernelGGL(k_accept, dim3((unsigned)f.B), dim3(256), 0, ctx->stream, f, wq_status_ptr(ctx));
    WQ_HIP_CHECK(ctx, hipGetLastError());
    return WQ_OK;
}

int wq_launch_append_rows(wq_ctx* ctx, const WqAppendRows& f)
{
    AppendArgs a = {};
    a.k_stride = f.k_stride, a.v_stride = f.v_stride;
    a.row_off = f.row_off, a.take = f.take, a.n_take = f.n_take, a.total_rows = f.total_rows;
    a.B = f.B, a.max_take = f.max_take, a.row_elems = f.kv[0].Hkv * f.kv[0].hd;
    a.pieces = (f.max_take + PIECE_ROWS - 1) / PIECE_ROWS;
    a.status = wq_status_ptr(ctx);
    void (*const kernel)(AppendArgs) = f.dtype == WQ_F32 ? k_append_rows<float> : k_append_rows<uint16_t>;
    if ((int64_t)(f.n_layers < APPEND_LAYERS ? f.n_layers : APPEND_LAYERS) * f.B > WQ_MOST_GROUPS_256 / a.pieces)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many rows");
    for (int l0 = 0; l0 < f.n_layers; l0 += APPEND_LAYERS) {
        const int n = f.n_layers - l0 < APPEND_LAYERS ? f.n_layers - l0 : APPEND_LAYERS;
        for (int l = 0; l < n; l++) {
            const wq_packed_kv& kv = f.kv[l0 + l];
            a.k[l] = static_cast<const char*>(f.k[l0 + l]), a.v[l] = static_cast<const char*>(f.v[l0 + l]);
            a.k16[l] = static_cast<uint16_t*>(kv.k16), a.v16[l] = static_cast<uint16_t*>(kv.v16);
            a.off16[l] = kv.off16, a.len16[l] = kv.len16, a.cap16[l] = kv.cap16;
        }
        hipLaunchKernelGGL(kernel, dim3((unsigned)(n * f.B * a.pieces)), dim3(256), 0, ctx->stream, a);
        if (a.pieces > 1) hipLaunchKernelGGL(k_raise, dim3((unsigned)(n * f.B)), dim3(64), 0, ctx->stream, a);
    }
    WQ_HIP_CHECK(ctx, hipGetLastError());
    return WQ_OK;
}

int wq_launch_copy_sequences(wq_ctx* ctx, int n_layers, const wq_packed_kv* src, const wq_packed_kv* dst, const int32_t* from)
{
    CopyArgs a = {};
    a.from = from;
    a.src_B = src->B, a.dst_B = dst->B, a.Hkv = dst->Hkv, a.hd = dst->hd, a.groups = dst->hd / dst->group;
    a.status = wq_status_ptr(ctx);
    auto held = [](const wq_packed_kv& kv) {
        CopyCache c;
        for (int k = 0; k < 3; k++) {
            c.codes[k] = static_cast<char*>(kv.codes[k]), c.meta[k] = static_cast<char*>(kv.meta[k]);
            c.cls_off[k] = kv.cls_off[k], c.cls_len[k] = kv.cls_len[k], c.cap[k] = kv.cap[k];
        }
        c.k16 = static_cast<char*>(kv.k16), c.v16 = static_cast<char*>(kv.v16);
        c.off16 = kv.off16, c.len16 = kv.len16, c.cap16 = kv.cap16, c.v_scale_max = kv.v_scale_max;
        return c;
    };
    const int64_t row_bytes = (int64_t)a.Hkv * a.hd * 2, rows_per = row_bytes < COPY_BYTES ? COPY_BYTES / row_bytes : 1;
    auto count = [&](int l0, int n) {          // of layers l0 .. l0 + n - 1: workgroups over each, for the largest of every class
        int64_t all = 0;
        for (int k = 0; k < 4; k++) {
            int64_t cap = 0;
            for (int l = l0; l < l0 + n; l++) {
                const int64_t c = k < 3 ? dst[l].cap[k] : dst[l].cap16;
                cap = c > cap ? c : cap;
            }
            const int per = COPY_BYTES / (4 * a.hd * (2 << (k & 3)));
            all += k < 3 ? (cap / 32 + per - 1) / per * 2 * a.Hkv : (cap + rows_per - 1) / rows_per * 2;
            a.end[k] = all;
        }
        return all;
    };
    for (int l0 = 0; l0 < n_layers; l0 += COPY_LAYERS) {
        const int n = n_layers - l0 < COPY_LAYERS ? n_layers - l0 : COPY_LAYERS;
        if (count(l0, n) > WQ_MOST_GROUPS_256 / n) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many workgroups");
    }
    for (int l0 = 0; l0 < n_layers; l0 += COPY_LAYERS) {
        const int n = n_layers - l0 < COPY_LAYERS ? n_layers - l0 : COPY_LAYERS;
        const int64_t all = count(l0, n);
        for (int l = 0; l < n; l++) a.src[l] = held(src[l0 + l]), a.dst[l] = held(dst[l0 + l]);
        hipLaunchKernelGGL(k_copy_plan, dim3((unsigned)n), dim3(1024), 0, ctx->stream, a);
        if (all > 0) hipLaunchKernelGGL(k_copy, dim3((unsigned)all, (unsigned)n), dim3(256), 0, ctx->stream, a);
    }
    WQ_HIP_CHECK(ctx, hipGetLastError());
    return WQ_OK;
}
