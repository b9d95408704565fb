// wq_tree_attention: several new rows of every sequence attend to its packed cache and to each other, along a tree of drafted tokens or as a
// chain.  A row is a (new row, query head) pair, as in wq_attend.hip; its sequence's keys are the cache's tiles and, behind them, the new rows'.
//     out = sum_j w_j v_j / sum_j w_j,   w_j = 2^(scale q.k_j - ref),   ref a running reference of the row, lse = ln 2 (ref + log2 sum_j w_j)
// in one pass over the keys; what several workgroups have of a row's sums is brought to a common ref and added (k_tree_join).
// 16-bit types: by the rows that a sequence has under a KV head.  Up to 48 (and 49 to 64 as two tiles): wq_tree_stream.hip, near the cache's bytes for few;
// more: wq_tree_tiles.hip, bound by products and the vector instructions that expand codes and form weights, one after the other.  Here: who gets what, the join, and
// fp32, whose products have a ninth of the 16-bit rate (3 trees of 7 rows over 144 tokens 11.7 us, of that two launches 9).
// Roundings of 16-bit queries: weights to the values' type and packed values to fp16, which the products take, and without lse packed keys for bf16; references, sums of
// weights, numerators, parts and their join stay fp32.  A result is off by 1.7e-3 in bf16 (its own rounding alone: as much) and 2.6e-4 in fp16 (2.1e-4).  Weights in
// two parts of 16 bits would be half as many products again, a fifth of a tile's time.
#include "wq_tree.h"

namespace {

// The new rows that a row does not see
struct Unrelated {
    const uint64_t* seen;                      // NULL: a chain
    int node[COLS];                            // the rows' places in it
    template <typename CT, int HD>
    __device__ __forceinline__ void hide(const Rows<HD>& r, Products<CT>& s, int key0) const
    {
        const int from = 4 * ((threadIdx.x & 63) >> 4) + (key0 & 63);          // this lane's first key in the word
#pragma unroll
        for (int n = 0; n < COLS; n++) {
            uint64_t word;
            if (seen) {
                word = seen[node[n] * WORDS + (key0 >> 6)];
            } else {
                const int left = r.limit[n] - (key0 & ~63);
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

template <int HD>
__global__ __launch_bounds__(64 * WAVES<F32>, 2) void k_tree(TreeArgs a)
{
    constexpr int BYTES = TILE_BYTES<F32, HD>, R = ROWS<F32>, TK = KEYS<F32>;
    __shared__ __align__(16) char s_k[BYTES], s_v[BYTES];
    __shared__ uint64_t s_seen[(R + 1) * WORDS];
    __shared__ int32_t s_parent[WQ_MAX_TREE];
    const int Hkv = a.kv.Hkv, wave = this_wave(), lane = threadIdx.x & 63;
    const wq_packed_kv& kv = a.kv;
    const int unit = (int)blockIdx.x % a.units, split = (int)blockIdx.x / a.units, kvh = unit % Hkv;
    Place p;
    if (!find_place<R>(a.row_off, a.B, a.rep, a.total, unit / Hkv, p)) return;
    const int n = p.rows / a.rep, node0 = p.row0 / a.rep;      // the sequence's new rows; the first one of this tile
    if (n > a.most && p.row0 == 0 && threadIdx.x == 0) atomicOr(a.status, WQ_DEV_TOO_MANY_ROWS);
    const int last_row = (p.row0 + R < p.rows ? p.row0 + R : p.rows) - 1;
    int tiles[4], len[4], newest = last_row / a.rep + 1;       // (no row sees one behind itself)
    if (newest > a.most) newest = a.most;
    const int cached = tiles_of_cache<TK>(kv, p.seq, len, tiles), all = cached + (newest + TK - 1) / TK;
    const int lo = (int)((int64_t)split * all / a.splits), hi = (int)((int64_t)(split + 1) * all / a.splits);

    Rows<HD> r;
    Query<F32, HD> q;
    clear(r);
    const int wrow0 = p.row0 + wave * COLS * 16;
    const char* row_at[COLS];
#pragma unroll
    for (int c = 0; c < COLS; c++) {
        const int row = wrow0 + 16 * c + (lane & 15);
        row_at[c] = row < p.rows ? a.q + (p.first + row / a.rep) * a.q_stride + (kvh * a.rep + row % a.rep) * (HD * 4) : nullptr;
    }
    const bool any = wrow0 < p.rows && wave * COLS * 16 < R;
    walk_cache<F32, HD, 0>(r, q, row_at, a.scale, kv, p.seq, kvh, len, tiles, lo, hi, any, (Lds)s_k, (Lds)s_v, (Lds)s_k);
    if (hi > cached && lo < hi) {
        const int t0 = lo > cached ? lo - cached : 0, t1 = hi - cached;
        Unrelated unrelated;
        unrelated.seen = a.parent ? s_seen : nullptr;
        if (a.parent) find_ancestors(a.parent + p.first, node0, last_row / a.rep + 1 - node0, s_seen, s_parent, 64 * WAVES<F32>);
#pragma unroll
        for (int c = 0; c < COLS; c++) {
            const int row = wrow0 + 16 * c + (lane & 15);
            r.limit[c] = row < p.rows ? row / a.rep + 1 : 0;
            unrelated.node[c] = row <= last_row ? row / a.rep - node0 : 0;
            r.scale[c] = a.scale;
            load_query<F32, HD>(q, c, row_at[c]);
        }
        const int least = a.parent || !any ? 0 : wrow0 / a.rep + 1, most = any ? newest : 0;
        const char* k = a.k + p.first * a.k_stride + kvh * (HD * 4);
        const char* v = a.v + p.first * a.v_stride + kvh * (HD * 4);
        for (int t = t0; t < t1; t++) {
            const int key0 = t * TK;
            __syncthreads();
            stage_rows<F32, HD>(k + key0 * a.k_stride, v + key0 * a.v_stride, a.k_stride, a.v_stride, newest - key0, (Lds4)s_k, (Lds4)s_v);
            __syncthreads();
            attend_f32<HD>(r, q, (Lds4)s_k, (Lds4)s_v, key0, least, most, unrelated);
        }
    }
#pragma unroll
    for (int c = 0; c < COLS; c++)
        if ((wrow0 + 16 * c + (lane & 15)) / a.rep >= a.most) {        // refused: as if it saw nothing
            r.ref[c] = -INFINITY, r.sum[c] = 0.f;
#pragma unroll
            for (int ct = 0; ct < HD / 16; ct++) r.o[ct][c] = f4{0.f, 0.f, 0.f, 0.f};
        }
    if (any) store_rows<F32, HD>(r, p, a.rep, a.Hq, kvh, wave, split, a.splits > 1 ? a.splits : 0, {a.out, a.lse, a.part, a.part_ml});
}

// fp32, in tiles of 32 rows: the four wavefronts take 16 rows and 16 of a tile's 32 keys each, and leave a part for the merge for each half of the keys.  Bound by the
// matrix cores: 28 rows are all one wavefront's in k_tree, and with heads of 128 that one keeps 46 of its registers in scratch, this one none (154).
template <int HD>
__global__ __launch_bounds__(256, 2) void k_tree_few(TreeArgs a)
{
    constexpr int BYTES = TILE_BYTES<F32, HD>, R = 32, TK = KEYS<F32>, ST = STEPS<F32, HD>;
    __shared__ __align__(16) char s_k[BYTES], s_v[BYTES];
    __shared__ uint64_t s_seen[(R + 1) * WORDS];
    __shared__ int32_t s_parent[WQ_MAX_TREE];
    const int Hkv = a.kv.Hkv, wave = this_wave(), lane = threadIdx.x & 63, j = lane >> 4, half = wave >> 1;
    const wq_packed_kv& kv = a.kv;
    const int unit = (int)blockIdx.x % a.units, split = (int)blockIdx.x / a.units, kvh = unit % Hkv;
    Place p;
    if (!find_place<R>(a.row_off, a.B, a.rep, a.total, unit / Hkv, p)) return;
    const int node0 = p.row0 / a.rep;
    if (p.rows / a.rep > a.most && p.row0 == 0 && threadIdx.x == 0) atomicOr(a.status, WQ_DEV_TOO_MANY_ROWS);
    const int last_row = (p.row0 + R < p.rows ? p.row0 + R : p.rows) - 1;
    int tiles[4], len[4], newest = last_row / a.rep + 1;       // (no row sees one behind itself)
    if (newest > a.most) newest = a.most;
    const int cached = tiles_of_cache<TK>(kv, p.seq, len, tiles), all = cached + (newest + TK - 1) / TK;
    const int lo = (int)((int64_t)split * all / a.splits), hi = (int)((int64_t)(split + 1) * all / a.splits);
    const int row = p.row0 + 16 * (wave & 1) + (lane & 15);
    const char* row_at = row < p.rows ? a.q + (p.first + row / a.rep) * a.q_stride + (kvh * a.rep + row % a.rep) * (HD * 4) : nullptr;
    const bool any = p.row0 + 16 * (wave & 1) < p.rows;

    f4 o[HD / 16];
    float ref = -INFINITY, sum = 0.f;
    QueryRows<F32, HD, 1> q;
#pragma unroll
    for (int ct = 0; ct < HD / 16; ct++) o[ct] = f4{0.f, 0.f, 0.f, 0.f};
    // The staged tile's keys from key0 on, of which the row sees those that sees() says
    auto attend = [&](int key0, auto sees) __attribute__((always_inline)) {
        if (!any) return;
        f4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < ST; st++) s = product<F32>(((Lds4)s_k)[(half * ST + st) * 64 + lane], q[0][st], s);
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (!sees(key0 + 16 * half + 4 * j + i)) s[i] = -INFINITY;
        const float most = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])) * a.scale;
        if (__ballot(most > ref + SLACK)) {
            const float to = fmaxf(ref, max_of_column(most)), by = to == ref ? 1.f : __builtin_amdgcn_exp2f(ref - to);
            ref = to;
            sum *= by;
#pragma unroll
            for (int ct = 0; ct < HD / 16; ct++) o[ct] *= by;
        }
        const float shift = ref == -INFINITY ? 0.f : -ref;
        u4 w;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float x = __builtin_amdgcn_exp2f(fmaf(s[i], a.scale, shift));
            sum += x;
            w[i] = __float_as_uint(x);
        }
#pragma unroll
        for (int ct = 0; ct < HD / 16; ct++) o[ct] = product<F32>(((Lds4)s_v)[(half * (HD / 16) + ct) * 64 + lane], w, o[ct]);
    };
    int done = 0;
    auto walk_class = [&](auto bits) __attribute__((always_inline)) {
        constexpr int BITS = decltype(bits)::value, c = BITS == 2 ? 0 : (BITS == 4 ? 1 : 2);
        const int t0 = lo > done ? lo - done : 0, t1 = hi - done < tiles[c] ? hi - done : tiles[c];
        done += tiles[c];
        if (t0 >= t1) return;
        PackedKeys<HD, BITS, 32> keys(kv, kvh, kv.cls_off[c][p.seq], 0);
        PackedValues<HD, BITS, 32> values(kv, kvh, kv.cls_off[c][p.seq], 0);
        const bool brings_keys = wave < 2;
        auto load = [&](int t) {
            if (brings_keys) keys.load(t);
            else values.load(t);
        };
        load(t0);
        load_query_quarter<F32, HD>(q, 0, row_at);
        for (int t = t0; t < t1; t++) {
            __syncthreads();                                   // (the tile before has been read)
            if (brings_keys) keys.stage_f32((Lds4)s_k);
            else values.stage_f32((Lds4)s_v);
            __syncthreads();
            if (t + 1 < t1) load(t + 1);
            __builtin_amdgcn_sched_barrier(0);
            attend(t * TK, [&](int key) { return key < len[c]; });
        }
    };
    walk_class(std::integral_constant<int, 2>());
    walk_class(std::integral_constant<int, 4>());
    walk_class(std::integral_constant<int, 8>());
    if (hi > done && lo < hi) {
        load_query<F32, HD>(q, 0, row_at);
        const int64_t row0 = kv.off16[p.seq], stride = (int64_t)Hkv * HD * 2;
        const char* k16 = static_cast<const char*>(kv.k16) + row0 * stride + kvh * (HD * 2);
        const char* v16 = static_cast<const char*>(kv.v16) + row0 * stride + kvh * (HD * 2);
        for (int t = lo > done ? lo - done : 0; t < tiles[3] && t < hi - done; t++) {
            const int key0 = t * TK;
            __syncthreads();
            stage_rows<F16, HD>(k16 + key0 * stride, v16 + key0 * stride, stride, stride, len[3] - key0, (Lds4)s_k, (Lds4)s_v);
            __syncthreads();
            attend(key0, [&](int key) { return key < len[3]; });
        }
    }
    if (hi > cached && lo < hi) {
        if (a.parent) find_ancestors(a.parent + p.first, node0, last_row / a.rep + 1 - node0, s_seen, s_parent, 256);
        const int limit = row < p.rows ? row / a.rep + 1 : 0;
        const uint64_t* seen = s_seen + (row <= last_row ? row / a.rep - node0 : 0) * WORDS;
        const char* k = a.k + p.first * a.k_stride + kvh * (HD * 4);
        const char* v = a.v + p.first * a.v_stride + kvh * (HD * 4);
        for (int t = lo > cached ? lo - cached : 0; t < hi - cached; t++) {
            const int key0 = t * TK;
            __syncthreads();
            stage_rows<F32, HD>(k + key0 * a.k_stride, v + key0 * a.v_stride, a.k_stride, a.v_stride, newest - key0, (Lds4)s_k, (Lds4)s_v);
            __syncthreads();
            attend(key0, [&](int key) { return a.parent ? (seen[key >> 6] >> (key & 63) & 1) != 0 : key < limit; });
        }
    }
    sum = sum_of_column(sum);
    if (row >= p.rows) return;
    const bool refused = row / a.rep >= a.most;                // as if it saw nothing
    const int64_t slot = ((p.first + row / a.rep) * a.Hq + kvh * a.rep + row % a.rep) * (2 * a.splits) + 2 * split + half;
#pragma unroll
    for (int ct = 0; ct < HD / 16; ct++) *reinterpret_cast<f4*>(a.part + slot * HD + 16 * ct + 4 * j) = refused ? f4{0.f, 0.f, 0.f, 0.f} : o[ct];
    if (j == 0) a.part_ml[2 * slot] = refused ? -INFINITY : ref, a.part_ml[2 * slot + 1] = refused ? 0.f : sum;
}

// The pieces of units that are cut: a wavefront per row; a row's pieces are read by halves of it in turn.  A launch of its own: with the last workgroup of a unit
// joining, 32 pieces of 128 rows (2 MB) would go through one compute unit.  (us: 4.5 of 1000 rows in 4 pieces, 7 of 4096 in 16)
template <int HD, int R>
__global__ __launch_bounds__(256) void k_tree_join(TreeArgs a, int dtype)
{
    const int lane = threadIdx.x & 63, unit = blockIdx.x / (R / 4), in = blockIdx.x % (R / 4) * 4 + this_wave(), kvh = unit % a.kv.Hkv;
    const int4 found = a.found[unit];
    const int row = found.y + in, pieces = found.w;
    if (pieces <= 1 || row >= found.z) return;
    const float* parts = a.part + (int64_t)unit * a.splits * PIECE<HD, R>;
    auto piece = [&](int i) { return parts + (int64_t)i * PIECE<HD, R>; };
    constexpr int LANES = HD / 4, GROUPS = 64 / LANES;
    f4 y[8];
    auto load = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 8; k++) {
            const int i = i0 + k * GROUPS + lane / LANES;
            y[k] = i < pieces ? *reinterpret_cast<const f4*>(piece(i) + in * HD + 4 * (lane % LANES)) : f4{0.f, 0.f, 0.f, 0.f};
        }
    };
    load(0);                                   // (on their way while the weights are found)
    float m = -INFINITY, l = 0.f;              // lane i: piece i
    if (lane < pieces) {
        const float* ml = piece(lane) + R * HD + 2 * in;
        m = ml[0], l = ml[1];
    }
    const float M = wave_max(m), w = __builtin_amdgcn_exp2f(m - (M == -INFINITY ? 0.f : M)), L = wave_sum(l * w);
    f4 x = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < pieces; i0 += 8 * GROUPS) {
        if (i0 > 0) load(i0);
#pragma unroll
        for (int k = 0; k < 8; k++) {
            const int i = i0 + k * GROUPS + lane / LANES;
            const float f = __shfl(w, i & 63, 64);
            x += y[k] * (i < pieces ? f : 0.f);
        }
    }
    store_merged<HD>({a.out, a.lse, nullptr, nullptr}, dtype, ((int64_t)found.x + row / a.rep) * a.Hq + kvh * a.rep + row % a.rep, sum_of_groups<HD>(x), M, L);
}

template <int R>
void launch_pieces(wq_ctx* ctx, const TreeArgs& a, TreeKernel kernel, int dtype)
{
    void (*const join)(TreeArgs, int) = a.kv.hd == 128 ? k_tree_join<128, R> : k_tree_join<64, R>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.units * a.splits)), dim3(256), 0, ctx->stream, a);
    if (a.splits > 1) hipLaunchKernelGGL(join, dim3((unsigned)(a.units * (R / 4))), dim3(256), 0, ctx->stream, a, dtype);
}

}  // namespace

WqTreePlan wq_tree_plan(int64_t total_rows, int B, int Hq, int Hkv, int hd, int dtype, int64_t max_cache_tokens, int64_t slots, int max_rows, int num_splits, size_t room)
{
    const int rep = Hq / Hkv;
    const int64_t used = total_rows < B ? total_rows : B;     // sequences that have rows
    WqTreePlan s = {};
    if (max_cache_tokens > int64_t(1) << 40) max_cache_tokens = int64_t(1) << 40;
    // Units, if the sequences' rows lie evenly about their average up to max_rows
    const double mean = (double)total_rows / used, over = max_rows > mean ? max_rows - mean : 0;
    auto units_of = [&](int rows) {
        double n = 0;
        for (int i = 0; i < 16; i++) n += ceil(fmax(1.0, round(mean + (over > 0 ? over + 0.5 : 0) * (2 * i - 15) / 16)) * rep / rows) / 16;
        return n * used * Hkv;
    };
    if (dtype != WQ_F32) {
        // Columns of a sequence, on the average.  Up to three: every wavefront brings its own keys; four in two tiles; more in tiles of 128 rows.  us of four columns in
        // tiles of 32 rows, of 128: 28 + 4 heads of 128, 8 sequences of 12800 tokens 40, 46, 32 of 4200 50, 60, 4 of 50400 62, 73 (fp16 75, 83), one of 12800 23.8, 23.2;
        // 32 + 8 of 128 64, 75, 79, 104, 115, 127; 14 + 2 of 64 21, 25, 24, 30, 29, 34.  Of five, 8 x 12800: 53, 48 (32 + 8 heads: 94, 76); one sequence 22.8, 24.8, and heads of 64
        // 25.0, 27.8 would be better off in tiles of 32
        const int64_t columns = ((total_rows + used - 1) / used * rep + 15) / 16;
        s.columns = (int)(columns <= WQ_STREAM_COLUMNS ? columns : columns == 4 ? 2 : 8);
        s.rows = 16 * s.columns;
        const int tile = s.columns <= WQ_STREAM_COLUMNS ? 32 : 64;
        s.units = tiles_of(total_rows, rep, B, s.rows) * Hkv;
        if (const int64_t tiles = ((int64_t)max_rows * rep + s.rows - 1) / s.rows; tiles > 0 && tiles * B * Hkv <= s.units) s.tiles = (int)tiles, s.units = tiles * B * Hkv;
        const double real = units_of(s.rows);
        const int64_t blocks = (max_cache_tokens + tile - 1) / tile + ((int64_t)max_rows + tile - 1) / tile;
        // The cache's capacity says how long the sequences are on the average: those that are shorter than the longest have fewer pieces
        const double average = slots > 0 && slots < (int64_t)B * max_cache_tokens ? (double)slots / ((double)B * max_cache_tokens) : 1.0;
        s.longest = num_splits > 0 || blocks > 1 << 23 ? 0 : (int)blocks;
        if (num_splits > 0) {
            s.splits = num_splits;
        } else {
            // Rounds of the workgroups that the card holds at a time: `most` a compute unit, as its registers and LDS have it.  In steps of a workgroup that has a
            // unit for itself (1.2 us: a tile of 64 keys, or a block of 32 of every wavefront): a piece's steps, which take longer where workgroups share a unit (SLOWER), its
            // start and end; the join's launch and what the pieces leave in memory for it (6.6e6 bytes a step: 5.5 TB/s).  (us of 8 x 12800 tokens, 4 rows of 7 heads for each of 4 KV heads: 34 in 8
            // pieces, a workgroup a unit; 35 in 12; 32 in 16, two a unit; 38 in 20.  Where lengths differ, blocks of wavefronts fill in for each other, half a round lost
            // at the end: 32 chains 107 in 3, 110 in 4, 103 in 6, 95 in 8)
            const bool tiles = s.columns > WQ_STREAM_COLUMNS;
            const int most = hd == 128 ? (s.columns == 1 ? 3 : 2) : (s.columns == 1 ? 4 : s.columns == WQ_STREAM_COLUMNS ? 2 : 3);
            constexpr double SLOWER[5] = {1, 1, 1.5, 2.1, 3};
            double best = 0;
            s.splits = 1;
            for (int p = 1; p <= WQ_MAX_ATTEND_SPLITS && p <= (blocks < 4 ? 1 : blocks); p++) {
                const double groups = real * (average < 0.95 ? fmin(p, p * average + 0.5) : p), rounds = average < 0.95 && !tiles ? fmax(1.0, groups / (256 * most) + 0.5) : ceil(groups / (256 * most));
                const double steps = ceil((double)blocks / p / (tiles ? 1 : WQ_STREAM_WAVES)) * SLOWER[(int)fmin(most, ceil(groups / 256))];
                const double time = rounds * (steps + (tiles ? 5 : 6)) + (p > 1 ? 4 + groups * s.rows * hd * 4 / 6.6e6 : 0);
                if (p == 1 || time < best) best = time, s.splits = p;
            }
        }
        auto size = [&] {
            s.groups = s.units * s.splits;
            s.bytes = s.splits > 1 ? wq_align256((size_t)s.groups * s.rows * (hd + 2) * 4) + wq_align256((size_t)s.units * sizeof(int4)) : 0;
        };
        size();
        // (the join has a workgroup for four rows of every unit)
        while (num_splits <= 0 && s.splits > 1 && (s.bytes > room || s.groups > WQ_MOST_GROUPS_256 / 2 || s.units * (s.rows / 4) > WQ_MOST_GROUPS_256)) s.splits--, size();
        return s;
    }
    // fp32: rounds as above, in steps of 32 keys of k_tree with a unit for itself; a workgroup of it whose sequences have few rows multiplies with some of its wavefronts
    // only, and shares the unit at little cost.  k_tree_few where a sequence has up to 640 rows under a KV head, on the average, and its keys are cut anyway (us, beside
    // k_tree, 4 KV heads of 128: 28 rows over 30 x 18700 tokens 450, 802; 8 x 6500 tokens, 91 rows 186, 208, 280 rows 356, 401, 420 rows 524, 492, 595 rows 731, 641, 637 rows
    // 758, 952, 1400 rows as long; 2 heads of 64, 8 x 6800 tokens: 140 rows 89, 90, 630 rows 259, 271, 2100 rows 668, 581; 8 heads of 64 with a query head each, 300 rows
    // 460, 486; 8 of 128 with four, 600 rows 1375, 1257.  Between 400 and 640 either may be the faster one)
    auto fit = [&](bool few) {
        WqTreePlan x = {};
        x.few = few, x.rows = few ? 32 : ROWS<F32>;
        x.units = tiles_of(total_rows, rep, B, x.rows) * Hkv;
        const int top = few ? WQ_MAX_ATTEND_SPLITS / 2 : WQ_MAX_ATTEND_SPLITS;      // (a lane of the merge for every part)
        x.splits = num_splits > 0 ? (num_splits < top ? num_splits : top) : 1;
        if (num_splits <= 0) {
            const int64_t blocks = (max_cache_tokens + 31) / 32 + ((int64_t)max_rows + 31) / 32;
            const int most = few ? (hd == 128 ? 3 : 5) : (hd == 128 ? 2 : 3);
            const double real = units_of(x.rows), active = fmin(4.0, ceil(mean * rep / 32)) / 4, slower = 1 + 0.7 * active;
            constexpr double SHARED[6] = {0.6, 0.6, 0.8, 0.9, 1.05, 1.25};
            double best = 0;
            for (int p = 1; p <= top && p <= (blocks < 4 ? 1 : blocks); p++) {
                const double groups = real * p, rounds = ceil(groups / (256 * most)), share = fmin(most, ceil(groups / 256));
                const double time = rounds * (ceil((double)blocks / p) * (few ? SHARED[(int)share] : pow(slower, share - 1)) + 3) + (p > 1 ? 2 + p * 0.1 : 0);
                if (p == 1 || time < best) best = time, x.splits = p;
            }
        }
        auto bytes = [&]() -> size_t { return x.splits > 1 ? partials_bytes(total_rows * Hq, hd, x.splits * (few ? 2 : 1)) : 0; };
        while (num_splits <= 0 && x.splits > 1 && (bytes() > room || x.units * x.splits > WQ_MOST_GROUPS_256 / 2 || total_rows * Hq > 4 * WQ_MOST_GROUPS_256)) x.splits--;
        x.bytes = bytes();
        x.groups = x.units * x.splits;
        return x;
    };
    if (mean * rep <= 640)
        if (const WqTreePlan x = fit(true); x.splits > 1) return x;
    return fit(false);
}

int wq_launch_tree(wq_ctx* ctx, const WqTree& f)
{
    TreeArgs a = {};
    const int size = f.dtype == WQ_F32 ? 4 : 2, hd = f.kv->hd;
    a.q = static_cast<const char*>(f.q), a.k = static_cast<const char*>(f.k), a.v = static_cast<const char*>(f.v);
    a.q_stride = f.q_stride * size, a.k_stride = f.k_stride * size, a.v_stride = f.v_stride * size;
    a.row_off = f.row_off, a.parent = f.parent;
    a.total = f.total_rows;
    a.most = f.max_rows > 0 ? f.max_rows : INT32_MAX;
    if (f.parent && a.most > WQ_MAX_TREE) a.most = WQ_MAX_TREE;
    a.B = f.B, a.Hq = f.Hq, a.rep = f.Hq / f.kv->Hkv, a.splits = f.plan.splits;
    a.units = (int)f.plan.units;
    a.scale = f.sm_scale * WQ_LOG2E;
    a.status = wq_status_ptr(ctx);
    a.kv = *f.kv;
    a.out = f.out, a.lse = f.lse;
    a.part = reinterpret_cast<float*>(ctx->ws + WQ_WS_HEADER);
    const int parts = a.splits * (f.plan.few ? 2 : 1);
    a.part_ml = a.part + f.total_rows * f.Hq * parts * hd;
    if (f.plan.columns) {
        a.longest = f.plan.longest;
        a.tiles = f.plan.tiles;
        a.found = reinterpret_cast<int4*>(reinterpret_cast<char*>(a.part) + wq_align256((size_t)f.plan.groups * f.plan.rows * (hd + 2) * 4));
        const TreeKernel kernel = f.plan.columns > WQ_STREAM_COLUMNS
                                      ? wq_tree_tiles_kernel(f.dtype, hd, f.dtype == WQ_F16 || f.lse ? hd / f.kv->group : 0)
                                      : wq_tree_stream_kernel(f.dtype, hd, f.plan.columns, f.lse != nullptr);
        switch (f.plan.columns) {
            case 1: launch_pieces<16>(ctx, a, kernel, f.dtype); break;
            case 2: launch_pieces<32>(ctx, a, kernel, f.dtype); break;
            case 3: launch_pieces<48>(ctx, a, kernel, f.dtype); break;
            default: launch_pieces<128>(ctx, a, kernel, f.dtype);
        }
        WQ_HIP_CHECK(ctx, hipGetLastError());
        return WQ_OK;
    }
    hipLaunchKernelGGL(f.plan.few ? (hd == 128 ? k_tree_few<128> : k_tree_few<64>) : (hd == 128 ? k_tree<128> : k_tree<64>), dim3((unsigned)f.plan.groups), dim3(64 * WAVES<F32>), 0, ctx->stream, a);
    if (a.splits > 1) {
        const MergeArgs m = {f.total_rows * f.Hq, f.Hq, parts, f.dtype, f.row_off, f.B, {a.out, a.lse, a.part, a.part_ml}};
        hipLaunchKernelGGL(hd == 128 ? k_merge<128> : k_merge<64>, dim3((unsigned)((m.rows + 3) / 4)), dim3(256), 0, ctx->stream, m);
    }
    WQ_HIP_CHECK(ctx, hipGetLastError());
    return WQ_OK;
}
