// What the kernels of wq_tree_attention share: their arguments, a packed cache's walk, who sees whom in a tree, who does what.
#pragma once
#include "wq_attend.h"

struct TreeArgs {
    const char *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;      // bytes from row to row
    const int32_t *row_off, *parent;
    int64_t total;
    int B, Hq, rep;
    int units, splits;                         // (tile of rows, KV head) pairs, and the parts that each one's keys are cut into
    int most;                                  // new rows of a sequence that count
    int tiles;                                 // 16-bit types: tiles of rows of every sequence, or 0: numbered as in find_place
    float scale;                               // log2(e) * sm_scale
    uint32_t* status;
    wq_packed_kv kv;
    void* out;                                 // as in Out
    float *lse, *part, *part_ml;
    int4* found;                               // 16-bit types: every unit's place and pieces, for the join
    int longest;                               // ... : blocks of keys of the longest sequence, or 0
};

typedef void (*TreeKernel)(TreeArgs);
// The kernel in which every wavefront brings its own keys, for tiles of 16 * columns query rows: see wq_tree_stream.hip
constexpr int WQ_STREAM_WAVES = 4, WQ_STREAM_COLUMNS = 3;
TreeKernel wq_tree_stream_kernel(int dtype, int hd, int columns, bool lse);
// ... and in which a workgroup's four bring tiles of 64 for 128 query rows (groups: of a cache's heads, 0 where keys may be rounded): see wq_tree_tiles.hip
TreeKernel wq_tree_tiles_kernel(int dtype, int hd, int groups);

namespace {

constexpr int WORDS = WQ_MAX_TREE / 64;        // of a row's ancestors

// The tokens of the four segments, and the tiles of TK tokens that they make
template <int TK>
__device__ __forceinline__ int tiles_of_cache(const wq_packed_kv& kv, int seq, int (&len)[4], int (&tiles)[4])
{
    int all = 0;
#pragma unroll
    for (int c = 0; c < 4; c++) {
        const int64_t room = c < 3 ? kv.cap[c] - kv.cls_off[c][seq] : kv.cap16 - kv.off16[seq];
        len[c] = c < 3 ? kv.cls_len[c][seq] : kv.len16[seq];
        if (len[c] > room) len[c] = (int)room;
        tiles[c] = len[c] > 0 ? (len[c] + TK - 1) / TK : 0;
        all += tiles[c];
    }
    return all;
}

// Tiles lo .. hi-1 of a cache, the classes one after the other; hi may lie behind its last tile
template <typename QT, int HD, int G>
__device__ __forceinline__ void walk_cache(Rows<HD>& r, Query<Walked<QT>, HD>& q, const char* const (&row_at)[COLS], float scale, const wq_packed_kv& kv, int seq, int kvh,
                                           const int (&len)[4], const int (&tiles)[4], int lo, int hi, bool any, Lds s_k, Lds s_v, Lds s_m)
{
    int done = 0;                                              // tiles of the classes before
    auto walk = [&](auto bits) __attribute__((always_inline)) {
        constexpr int BITS = decltype(bits)::value, c = BITS == 2 ? 0 : (BITS == 4 ? 1 : 2);
        const int t0 = lo > done ? lo - done : 0, t1 = hi - done < tiles[c] ? hi - done : tiles[c];
        done += tiles[c];
        if (t0 < t1) walk_class<QT, HD, G, true, BITS>(r, q, row_at, scale, kv, seq, kvh, len[c], t0, t1, any, s_k, s_v, s_m);
    };
    largest_instead_of_infinity<QT>(true);
    walk(std::integral_constant<int, 2>());
    walk(std::integral_constant<int, 4>());
    walk(std::integral_constant<int, 8>());
    largest_instead_of_infinity<QT>(false);
    shift_rows<QT>(r);
    const int t0 = lo > done ? lo - done : 0, t1 = hi - done > tiles[3] ? tiles[3] : hi - done;
    if (t0 < t1) walk_rows16<QT, HD, true>(r, q, row_at, scale, kv, seq, kvh, len[3], t0, t1, any, s_k, s_v);      // (of no rows there would be no last one to read again)
}

// Which new rows each of the rows node0 .. node0 + n - 1 sees, a bit each: itself, its parent, its parent's parent ..  (a parent lies in front of its
// child, so every walk ends).  For all threads of a workgroup.
__device__ __forceinline__ void find_ancestors(const int32_t* parent, int node0, int n, uint64_t* seen, int32_t* s_parent, int threads)
{
    const int last = node0 + n < WQ_MAX_TREE ? node0 + n : WQ_MAX_TREE;
    for (int i = threadIdx.x; i < last; i += threads) s_parent[i] = parent[i];
    for (int i = threadIdx.x; i < n * WORDS; i += threads) seen[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += threads) {
        int j = node0 + i;
        if (j >= WQ_MAX_TREE) continue;
        uint64_t word = 0;
        int at = j >> 6;
        while (true) {
            if (j >> 6 != at) seen[i * WORDS + at] = word, word = 0, at = j >> 6;
            word |= uint64_t(1) << (j & 63);
            const int up = s_parent[j];
            if (up < 0 || up >= j) break;
            j = up;
        }
        seen[i * WORDS + at] = word;
    }
    __syncthreads();
}

// ---- who does what -------------------------------------------------------------------------------------------------------
// The rows of tile `tile`: the B sequences' first tiles, then their second ones ..  Numbers without a tile cost more than their start: the dispatcher deals workgroups
// out in turn, and those behind wait for a full engine while others have room.  So they are few here, and at the end.
template <int R>
__device__ __forceinline__ bool place_of(const TreeArgs& a, int tile, Place& p)
{
    if (!a.tiles) return find_place<R>(a.row_off, a.B, a.rep, a.total, tile, p);
    const int b = tile % a.B;                              // (known before the rows are: the cache's tables are read beside them)
    const int64_t first = clipped(a.row_off[b], a.total), end = clipped(a.row_off[b + 1], a.total);
    p.seq = b, p.first = first, p.rows = end > first ? (int)((end - first) * a.rep) : 0, p.row0 = tile / a.B * R;
    return p.row0 < p.rows;
}
// Rows behind a sequence's last tile, which its caller's bound left out: as if they saw nothing (16-bit types; by the last tile's first piece)
template <int R, int HD>
__device__ __forceinline__ void clear_rest(const TreeArgs& a, const Place& p, int kvh, int piece)
{
    if (piece > 0 || !a.tiles || p.row0 / R != a.tiles - 1) return;
    for (int64_t i = threadIdx.x; i < (int64_t)(p.rows - p.row0 - R) * (HD / 8); i += blockDim.x) {
        const int row = p.row0 + R + (int)(i / (HD / 8));
        const int64_t at = (p.first + row / a.rep) * a.Hq + kvh * a.rep + row % a.rep;
        reinterpret_cast<uint4*>(a.out)[at * (HD / 8) + i % (HD / 8)] = make_uint4(0, 0, 0, 0);
        if (a.lse && i % (HD / 8) == 0) a.lse[at] = -INFINITY;
    }
}

// A unit is a tile of R query rows of a sequence under one KV head; its keys are blocks of TK, those of the cache's four segments and then the new
// rows'.  It is cut into a.splits pieces, a workgroup each; where the caller has told the longest sequence's blocks (a.longest), into as many as its own
// length is of that: only the device knows it.
struct Sequence {
    int len[4], blocks[4], rows, all, pieces;  // rows: (new row, query head) pairs; all: blocks
};
template <int TK>
__device__ __forceinline__ Sequence sequence_of(const TreeArgs& a, int b, int rows)
{
    Sequence s;
    s.rows = rows;
    s.all = tiles_of_cache<TK>(a.kv, b, s.len, s.blocks) + (rows / a.rep + TK - 1) / TK;
    int n = a.splits;
    if (a.longest > 0 && s.all < a.longest) n = (int)(((uint32_t)s.all * (uint32_t)n + a.longest - 1) / a.longest);      // (up to 2^23 blocks, 64 pieces)
    s.pieces = n < s.all ? n : s.all;
    return s;
}

// Where piece i of n begins in a unit of a sequence.  Near a class's border it begins there: a start in another class costs a workgroup about as much as `near_class`
// blocks.  (Less than half a piece either way: none is empty.)
__device__ __forceinline__ int begin_of(const Sequence& s, int i, int near_class)
{
    const int n = s.pieces, share = s.all / n, over = s.all - share * n, x = share * i + (i < over ? i : over);
    if (i <= 0 || i >= n) return x;
    const int near = (share - 1) / 2 < near_class ? (share - 1) / 2 : near_class;
    int border = 0, y = x;
#pragma unroll
    for (int c = 0; c < 4; c++) {
        border += s.blocks[c];
        if (abs(x - border) <= near) y = border;
    }
    return y > 0 && y < s.all ? y : x;
}

// What the join has to know of a unit, from its first piece: x, y first new row and first (row, head) pair, z the sequence's pairs, w pieces (0: no such unit)
__device__ __forceinline__ void leave_unit(const TreeArgs& a, int unit, int piece, const Place& p, int pieces)
{
    if (a.splits > 1 && piece == 0 && threadIdx.x == 0) a.found[unit] = pieces ? make_int4((int)p.first, p.row0, p.rows, pieces) : make_int4(0, 0, 0, 0);
}

// A piece's numerators in the workspace: [row][channel], then [row] (reference, sum)
template <int HD, int R> constexpr int PIECE = R * (HD + 2);

}  // namespace
