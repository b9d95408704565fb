// What a serving program does with a batch's rows and caches between its layers' kernels: wq_tree_accept (which drafted rows stay),
// wq_append_rows (their keys and values into every layer's cache) and wq_copy_sequences (forks, compaction).
#include <type_traits>

#include "wq_internal.h"

namespace {

__device__ __forceinline__ int64_t clipped(int64_t x, int64_t most) { return x < 0 ? 0 : (x > most ? most : x); }

// ---- wq_tree_accept ----------------------------------------------------------------------------------------------------
// Bound by its start and three memory round trips (3.1 us of 8 sequences, 3.5 of 512).  A workgroup per sequence.  Every row looks whether its parent's choice is its token, the first such row of a parent is its child, and one
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
// Bound by memory: each row is read and written once (28 layers of 4 x 512 rows, 4 KV heads of 128: 235 MB in 46 us, 5.1 TB/s), a few accepted rows by the launch
// (8 sequences, 5.4 us for all layers: one launch a layer would be 28).  A workgroup copies 16 rows of a sequence and layer, 16 bytes a lane; every one checks the
// sequence's whole selection by itself, so that a refused sequence stays as it was without a second launch.
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
// Bound by memory: each byte is read and written once.  What costs beside it is to know what goes where, since only the device knows the tables.  A
// workgroup reads them for the launch's sequences, sums them up in LDS (a few dependent loads, 3 us, once) and then copies its share of the layer's real
// bytes, whatever the capacities; a launch of its own for the tables would take longer than the copies of a small call.  (23 of 32 sequences of 25500 tokens, 365 MB:
// 72.5 us, 5.0 TB/s, as a copy of that size; 24 layers of 8 sequences of 200 tokens in 3 launches 24 us)
struct CopyCache {
    char *codes[3], *meta[3], *k16, *v16;
    int32_t *cls_off[3], *cls_len[3], *off16, *len16;
    float* v_scale_max;
    int64_t cap[3], cap16;
};
constexpr int COPY_LAYERS = 10;                // of a launch: what its arguments hold
constexpr int COPY_SEQUENCES = 512;            // of a launch: what a workgroup keeps of the tables in LDS
constexpr int COPY_ITEM = 4096;                // bytes that a wavefront copies at a time: four loads of 16 bytes a lane
struct CopyArgs {
    CopyCache src[COPY_LAYERS], dst[COPY_LAYERS];
    const int32_t* from;
    int src_B, dst_B, Hkv, hd, groups;
    int first, end;                            // the copy's sequences of this launch
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

// The launch's sequences: where the blocks of 32 tokens of class k lie in the copy (at[k][i] .. at[k][i+1]-1) and in the source (from[k][i], -1: nothing to copy); the
// 16-bit rows' items (at[3]) and the rows that they begin with
struct CopyTables {
    int at[4][COPY_SEQUENCES + 1], from[4][COPY_SEQUENCES], row[COPY_SEQUENCES], rows[COPY_SEQUENCES];
    int64_t sum[4][4];
};

// Number of the entry of at[0 .. n] that x lies in: at[i] <= x < at[i+1]
__device__ __forceinline__ int entry_of(const int* at, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(256) void k_copy(CopyArgs a)
{
    __shared__ CopyTables t;
    const CopyCache &src = a.src[blockIdx.y], &dst = a.dst[blockIdx.y];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, count = a.end - a.first;
    const int64_t row_bytes = (int64_t)a.Hkv * a.hd * 2;
    const int rows_per = row_bytes < COPY_ITEM ? (int)(COPY_ITEM / row_bytes) : 1;
    // tables; one workgroup writes the copy's
    int64_t before[4] = {0, 0, 0, 0};          // blocks (and items of rows) of the sequences in front
    uint32_t bits = 0;
    for (int d0 = 0; d0 < a.end; d0 += 256) {
        const int d = d0 + threadIdx.x, i = d - a.first;
        int s = d < a.end ? a.from[d] : -1, len[4] = {0, 0, 0, 0};
        if (s < -1 || s >= a.src_B) {
            s = -1;
            if (i >= 0) bits |= WQ_DEV_BAD_INDEX;
        }
        if (s >= 0)
#pragma unroll
            for (int k = 0; k < 4; k++) len[k] = tokens_of(src, k, s);
        bool fits = true;
        int64_t off = 0;
        if (d < a.end && len[3] > 0) {
            const int64_t end = dst.off16[d + 1] < dst.cap16 ? dst.off16[d + 1] : dst.cap16;
            off = dst.off16[d];
            if (off < 0 || off + len[3] > end) {
                fits = false;
                if (i >= 0) bits |= WQ_DEV_SEG16_OVERFLOW;
            }
        }
        int64_t sum[4];
        const int mine[4] = {pad32(len[0]) / 32, pad32(len[1]) / 32, pad32(len[2]) / 32, i >= 0 && fits ? (len[3] + rows_per - 1) / rows_per : 0};
#pragma unroll
        for (int k = 0; k < 4; k++) {
            sum[k] = mine[k];
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                const int64_t y = __shfl_up(sum[k], o, 64);
                if (lane >= o) sum[k] += y;
            }
            if (lane == 63) t.sum[k][wave] = sum[k];
        }
        __syncthreads();
        int64_t begin[4];
#pragma unroll
        for (int k = 0; k < 4; k++) {
            int64_t all = 0, front = 0;
#pragma unroll
            for (int w = 0; w < 4; w++) {
                if (w < wave) front += t.sum[k][w];
                all += t.sum[k][w];
            }
            begin[k] = before[k] + front + sum[k] - mine[k];
            if (k < 3) {
                const int64_t blocks = dst.cap[k] / 32;
                if (len[k] > 0 && begin[k] + mine[k] > blocks) {
                    fits = false;
                    if (i >= 0) bits |= WQ_DEV_CLASS_OVERFLOW;
                }
                begin[k] = begin[k] < blocks ? begin[k] : blocks;
                sum[k] = before[k] + front + sum[k];
                sum[k] = sum[k] < blocks ? sum[k] : blocks;
            } else {
                sum[k] += before[k] + front;
            }
            before[k] += all;
        }
        if (i >= 0 && i < count) {
#pragma unroll
            for (int k = 0; k < 4; k++) {
                t.at[k][i] = (int)begin[k];
                if (i == count - 1) t.at[k][count] = (int)sum[k];
            }
#pragma unroll
            for (int k = 0; k < 3; k++) t.from[k][i] = fits && len[k] > 0 ? src.cls_off[k][s] / 32 : -1;
            t.from[3][i] = fits && len[3] > 0 ? src.off16[s] : -1;
            t.row[i] = (int)off, t.rows[i] = len[3];
            if (blockIdx.x == 0) {
#pragma unroll
                for (int k = 0; k < 3; k++) {
                    dst.cls_off[k][d] = (int)begin[k] * 32;
                    dst.cls_len[k][d] = fits ? len[k] : 0;
                    if (d == a.dst_B - 1) dst.cls_off[k][d + 1] = (int)sum[k] * 32;
                }
                dst.len16[d] = fits ? len[3] : 0;
                dst.v_scale_max[d] = fits && s >= 0 ? src.v_scale_max[s] : 0.f;
            }
        }
        __syncthreads();
    }
    if (blockIdx.x == 0 && bits) atomicOr(a.status, bits);
    // The wavefronts take items in turn, COPY_ITEM bytes of the blocks of a class (a plane and KV head) with their metadata, or as many rows of keys or values,
    // so that at any time all of them are in one stretch of memory.
    const uint32_t step = gridDim.x * 4, id = blockIdx.x * 4 + wave;
    uint32_t done = 0;                         // items of the classes before, modulo step
    auto first = [&] { return id >= done ? id - done : id + step - done; };
    auto copy_class = [&](auto which) __attribute__((always_inline)) {
        constexpr int k = decltype(which)::value;
        const int per = COPY_ITEM / (4 * a.hd * (2 << k));     // blocks of an item
        const uint32_t per_plane = (t.at[k][count] - t.at[k][0] + per - 1) / per;
        const int64_t all = (int64_t)per_plane * (2 * a.Hkv), items = all < INT32_MAX ? all : INT32_MAX;      // (2^31 items would be 8 TB)
        // pieces of 16 bytes: 256 of an item's codes; 8 a group and block of the metadata
        const int code_shift = 8 - (__ffs(per) - 1), meta_shift = 3 + __ffs(a.groups) - 1, metas = per << meta_shift;
        const char *x_codes = src.codes[k], *x_meta = src.meta[k];
        char *y_codes = dst.codes[k], *y_meta = dst.meta[k];
        const int64_t x_blocks = src.cap[k] / 32, y_blocks = dst.cap[k] / 32;
        for (int64_t u = first(); u < items; u += step) {
            const uint32_t plane = (uint32_t)u / per_plane, in = (uint32_t)u - plane * per_plane;
            const int j0 = t.at[k][0] + (int)in * per, mine = j0 + lane;
            int from = -1;                     // lane l: the block that block j0 + l is a copy of
            if (lane < per && mine < t.at[k][count]) {
                const int i = entry_of(t.at[k], count, mine);
                if (t.from[k][i] >= 0) from = t.from[k][i] + mine - t.at[k][i];
            }
            const int64_t x0 = plane * x_blocks, y0 = plane * y_blocks + j0;
            uint4 v[4], w[2];
            int v_at[4], w_at[2];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int f = lane + 64 * i;
                v_at[i] = __shfl(from, f >> code_shift, 64);
                if (v_at[i] >= 0) v[i] = wq_load_once(x_codes + (((x0 + v_at[i]) << code_shift) + (f & ((1 << code_shift) - 1))) * 16);
            }
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const int f = lane + 64 * i;
                w_at[i] = __shfl(from, (f >> meta_shift) & 63, 64);
                if (f >= metas) w_at[i] = -1;
                if (w_at[i] >= 0) w[i] = wq_load_once(x_meta + (((x0 + w_at[i]) << meta_shift) + (f & ((1 << meta_shift) - 1))) * 16);
            }
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (v_at[i] >= 0) wq_store_once(y_codes + ((y0 << code_shift) + lane + 64 * i) * 16, v[i]);
#pragma unroll
            for (int i = 0; i < 2; i++)
                if (w_at[i] >= 0) wq_store_once(y_meta + ((y0 << meta_shift) + lane + 64 * i) * 16, w[i]);
        }
        done = (uint32_t)((done + items) % step);
    };
    copy_class(std::integral_constant<int, 0>());
    copy_class(std::integral_constant<int, 1>());
    copy_class(std::integral_constant<int, 2>());
    for (int64_t u = first(); u < 2 * (int64_t)t.at[3][count]; u += step) {
        const int i = entry_of(t.at[3], count, (int)(u >> 1));
        if (t.from[3][i] < 0) continue;
        const int r0 = ((int)(u >> 1) - t.at[3][i]) * rows_per, rows = t.rows[i] - r0 < rows_per ? t.rows[i] - r0 : rows_per;
        const char* x = (u & 1 ? src.v16 : src.k16) + (t.from[3][i] + (int64_t)r0) * row_bytes;
        char* y = (u & 1 ? dst.v16 : dst.k16) + (t.row[i] + (int64_t)r0) * row_bytes;
        const int chunks = (int)(rows * row_bytes / 16);
        for (int e = lane; e < chunks; e += 256) {
            uint4 v[4];
#pragma unroll
            for (int n = 0; n < 4; n++)
                if (e + 64 * n < chunks) v[n] = wq_load_once(x + (e + 64 * n) * 16);
#pragma unroll
            for (int n = 0; n < 4; n++)
                if (e + 64 * n < chunks) wq_store_once(y + (e + 64 * n) * 16, v[n]);
        }
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
    a.pieces = (f.max_take - 1) / PIECE_ROWS + 1;
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
    for (int l0 = 0; l0 < n_layers; l0 += COPY_LAYERS) {
        const int n = n_layers - l0 < COPY_LAYERS ? n_layers - l0 : COPY_LAYERS;
        int64_t most = 0;                      // bytes that a layer's copy can have
        for (int l = 0; l < n; l++) {
            const wq_packed_kv& kv = dst[l0 + l];
            a.src[l] = held(src[l0 + l]), a.dst[l] = held(kv);
            const int64_t bytes = 2 * kv.Hkv * (kv.cap16 * kv.hd * 2 + (kv.cap[0] * 2 + kv.cap[1] * 4 + kv.cap[2] * 8) * kv.hd / 8);
            most = bytes > most ? bytes : most;
        }
        // Workgroups: an item a wavefront (four: 29.5 us instead of 23.8 for 24 layers of 8 short sequences, 16.1 instead of 8.3 for one of 3), and up to 1024
        // together (four a compute unit: 74.5 us of the 365 MB, with half as many again 89)
        int64_t groups = (most + 4 * COPY_ITEM - 1) / (4 * COPY_ITEM);
        groups = groups < 1 ? 1 : groups > 1024 / n ? 1024 / n : groups;
        for (a.first = 0; a.first < a.dst_B; a.first = a.end) {
            a.end = a.dst_B - a.first < COPY_SEQUENCES ? a.dst_B : a.first + COPY_SEQUENCES;
            hipLaunchKernelGGL(k_copy, dim3((unsigned)groups, (unsigned)n), dim3(256), 0, ctx->stream, a);
        }
    }
    WQ_HIP_CHECK(ctx, hipGetLastError());
    return WQ_OK;
}
