// wq_tree_attention for 16-bit types and many rows: a workgroup's four wavefronts, 32 rows each, expand every tile of 64 keys together.
// A tile's codes are expanded once for 128 rows and read by all four from LDS (two buffers: the next tile is expanded between this one's products of keys and its
// weights).  Bound by matrix and vector phases one after the other: a wavefront and tile are 64 matrix instructions of 16 cycles and 318 vector instructions of 4, and
// two wavefronts share a SIMD, whose phases overlap only by chance.  Of the cycles (no bank conflicts, 2.08 GHz) the matrix cores are busy in 38 %, the vector unit in 61 %,
// its issue of the matrix instructions among them (9 %).  64 rows of 4 sequences of 50688 tokens, 28 + 4 heads of 128: 247 us (floor 136); one workgroup of 256
// rows in two groups that take turns, as in wq_attend.hip, 315.  16 rows of 8 sequences of 12800 tokens 55 us: 32 us of tiles, 5 of start, 10 until the last
// workgroup starts, join 7.
#include "wq_tree.h"

namespace {

// The new rows that a row does not see, a tile of 64 at a time; the tiles of a tree are walked from the last one on, so that a row's walk along its ancestors goes on
// where it was.
struct Unseen {
    uint64_t* words;                           // [2][R] of a tree; NULL: a chain
    const int32_t* parent;
    int node[COLS];                            // of this lane's rows
    int nodes, node0, last;                    // rows of a tree: those from node0 on, of this tile of rows; the last tile of keys of the walk
    int* up;                                   // this thread's row: the ancestor that comes next
    __device__ __forceinline__ int key_tile(int t) const { return words ? last - t : t; }
    // The words of the t-th tile of the walk, for all threads of the workgroup
    __device__ __forceinline__ void ahead(int t) const
    {
        if (!words || (int)threadIdx.x >= nodes) return;
        const int key0 = 64 * key_tile(t);
        uint64_t word = 0;
        int j = *up;
        while (j >= key0) {
            if (j < key0 + 64) word |= uint64_t(1) << (j - key0);
            const int next = parent[j];
            j = next >= 0 && next < j ? next : -1;
        }
        *up = j;
        words[(t & 1) * 128 + threadIdx.x] = word;
    }
    template <typename CT, int HD>
    __device__ __forceinline__ void hide(const Rows<HD>& r, Products<CT>& s, int key0) const
    {
        const int from = 4 * ((threadIdx.x & 63) >> 4);
#pragma unroll
        for (int n = 0; n < COLS; n++) {
            uint64_t word;
            if (words) {
                word = words[(key0 >> 6 & 1) * 128 + node[n]];
            } else {
                const int left = r.limit[n] - key0;
                word = left >= 64 ? ~uint64_t(0) : (left <= 0 ? 0 : (uint64_t(1) << left) - 1);
            }
            word >>= from;
#pragma unroll
            for (int t = 0; t < KEYS<CT> / 16; t++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (!(word >> (16 * t + i) & 1)) s[t][n][i] = -INFINITY;
        }
    }
};

// QT, G: see walk_cache; G > 0 also for bf16, where log-sum-exps are asked for
template <typename QT, int HD, int G>
__global__ __launch_bounds__(256, HD == 64 ? 3 : 2) void k_tree_tiles(TreeArgs a)
{
    constexpr int BYTES = TILE_BYTES<F16, HD>, R = 128, TK = 64;
    __shared__ __align__(16) char s_k[2 * BYTES], s_v[2 * BYTES], s_m[G > 0 ? 2 * 64 * 4 * G : 16];
    __shared__ uint64_t s_words[2 * R];
    __shared__ int32_t s_parent[WQ_MAX_TREE];
    const int Hkv = a.kv.Hkv, wave = this_wave(), lane = threadIdx.x & 63;
    const wq_packed_kv& kv = a.kv;
    const int unit = (int)blockIdx.x % a.units, piece = (int)blockIdx.x / a.units, kvh = unit % Hkv;
    Place p = {};
    const bool there = place_of<R>(a, unit / Hkv, p);
    const Sequence s = sequence_of<TK>(a, p.seq, there ? p.rows : 0);
    if (!there) {
        leave_unit(a, unit, piece, p, 0);
        return;
    }
    clear_rest<R, HD>(a, p, kvh, piece);
    if (piece >= s.pieces) return;
    leave_unit(a, unit, piece, p, s.pieces);
    const int lo = begin_of(s, piece, 1), hi = begin_of(s, piece + 1, 1), cached = s.all - (p.rows / a.rep + TK - 1) / TK;
    const int node0 = p.row0 / a.rep, last_row = (p.row0 + R < p.rows ? p.row0 + R : p.rows) - 1;
    int newest = last_row / a.rep + 1;                         // (no row sees one behind itself)
    if (newest > a.most) newest = a.most;
    if (p.rows / a.rep > a.most && p.row0 == 0 && lo == 0 && threadIdx.x == 0) atomicOr(a.status, WQ_DEV_TOO_MANY_ROWS);

    Rows<HD> r;
    Query<F16, HD> q;
    clear(r);
    const int wrow0 = p.row0 + wave * COLS * 16;
    const char* row_at[COLS];
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        const int row = wrow0 + 16 * n + (lane & 15);
        row_at[n] = row < p.rows ? a.q + (p.first + row / a.rep) * a.q_stride + (kvh * a.rep + row % a.rep) * (HD * 2) : nullptr;
    }
    walk_cache<QT, HD, G>(r, q, row_at, a.scale, kv, p.seq, kvh, s.len, s.blocks, lo, hi, true, (Lds)s_k, (Lds)s_v, (Lds)s_m);
    const int t0 = lo > cached ? lo - cached : 0, t1 = hi - cached < (newest + TK - 1) / TK ? hi - cached : (newest + TK - 1) / TK;
    if (t0 < t1) {
        int up = node0 + threadIdx.x < WQ_MAX_TREE ? node0 + (int)threadIdx.x : -1;
        Unseen unseen;
        unseen.words = a.parent ? s_words : nullptr, unseen.parent = s_parent, unseen.up = &up;
        unseen.nodes = last_row / a.rep + 1 - node0, unseen.last = t1 - 1;
        if (a.parent)
            for (int i = threadIdx.x; i < newest; i += 256) s_parent[i] = a.parent[p.first + i];
#pragma unroll
        for (int n = 0; n < COLS; n++) {
            const int row = wrow0 + 16 * n + (lane & 15);
            r.limit[n] = row < p.rows ? row / a.rep + 1 : 0;
            unseen.node[n] = row <= last_row ? row / a.rep - node0 : 0;
            r.scale[n] = a.scale;
            load_query<F16, HD>(q, n, row_at[n]);
        }
        const char* k = a.k + p.first * a.k_stride + kvh * (HD * 2);
        const char* v = a.v + p.first * a.v_stride + kvh * (HD * 2);
        walk_rows<QT, HD, false, true>(r, q, k, v, a.k_stride, a.v_stride, newest, a.parent ? 0 : t0, a.parent ? t1 - t0 : t1,
                                       a.parent || wrow0 >= p.rows ? 0 : wrow0 / a.rep + 1, (Lds)s_k, (Lds)s_v, unseen);
    }
    float* left = a.part + ((int64_t)unit * a.splits + piece) * PIECE<HD, R>;
    const int j = lane >> 4;
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        const int row = wrow0 + 16 * n + (lane & 15);
        float sum = sum_of_column(r.sum[n]);
        if (row >= p.rows) continue;
        float ref = r.ref[n] - SHIFT<QT>;
        if (row / a.rep >= a.most) {          // refused: as if it saw nothing
            ref = -INFINITY, sum = 0.f;
#pragma unroll
            for (int ct = 0; ct < HD / 16; ct++) r.o[ct][n] = f4{0.f, 0.f, 0.f, 0.f};
        }
        if (s.pieces > 1) {
            const int x = row - p.row0;
#pragma unroll
            for (int ct = 0; ct < HD / 16; ct++) *reinterpret_cast<f4*>(left + x * HD + 16 * ct + 4 * j) = r.o[ct][n];
            if (j == 0) left[R * HD + 2 * x] = ref, left[R * HD + 2 * x + 1] = sum;
            continue;
        }
        const int64_t at = (p.first + row / a.rep) * a.Hq + kvh * a.rep + row % a.rep;
        const float inv = one_over(sum);
        char* to = static_cast<char*>(a.out) + at * HD * 2;
#pragma unroll
        for (int ct = 0; ct < HD / 16; ct++) {
            const f4 x = r.o[ct][n] * inv;
            *reinterpret_cast<uint2*>(to + (16 * ct + 4 * j) * 2) = make_uint2(pack2(x[0], x[1], QT()), pack2(x[2], x[3], QT()));
        }
        if (a.lse && j == 0) a.lse[at] = log_sum_exp(ref, sum);
    }
}

template <typename QT>
TreeKernel of_groups(int hd, int groups)
{
    if (hd == 64) return groups == 1 ? k_tree_tiles<QT, 64, 1> : k_tree_tiles<QT, 64, 2>;
    return groups == 1 ? k_tree_tiles<QT, 128, 1> : groups == 2 ? k_tree_tiles<QT, 128, 2> : k_tree_tiles<QT, 128, 4>;
}

}  // namespace

TreeKernel wq_tree_tiles_kernel(int dtype, int hd, int groups)
{
    if (dtype == WQ_F16) return of_groups<F16>(hd, groups);
    if (groups > 0) return of_groups<Bf16>(hd, groups);
    return hd == 128 ? k_tree_tiles<Bf16, 128, 0> : k_tree_tiles<Bf16, 64, 0>;
}
