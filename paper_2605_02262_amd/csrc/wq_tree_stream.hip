// wq_tree_attention for 16-bit types: every wavefront walks blocks of 32 tokens by itself.
// With up to 48 rows (columns of 16: the matrix instruction's width) under a KV head the cache's bytes and their expansion are what there is to do, and tiles shared
// by a workgroup cost barriers and a way through LDS.  Here a wavefront's codes go from memory to registers, are expanded there into the products' operands and never
// leave; the four of a workgroup take blocks in turn and put their sums together at the end.  A block of 32 tokens is 450 instructions for one column, 580 for two,
// 720 for three (bf16, heads of 128; products of codes as they are 600 for two), so one column is near memory; two and three are bound by
// those instructions, one behind the other in the two wavefronts that a SIMD has registers for (2.1 us for a block each, vector unit 48 % active).
// us of 8 sequences of 12800 tokens, 28 + 4 heads of 128 (91 MB, 17.5 at a copy's rate): one row 25.4, 4 rows 31.0, 6 rows 36.7; a workgroup of the last: starts
// within 7 us, tables and queries 5, walk 15 to 20 (5 TB/s while it lasts), sums together 3; join 5.  Tiles shared by the workgroup: 28 (one row), 41 (6 rows).
#include "wq_tree.h"

namespace {

constexpr int NW = WQ_STREAM_WAVES;

// A wavefront's rows, CW columns of 16: as Rows
template <int HD, int CW>
struct Columns {
    f4 o[HD / 16][CW];
    float ref[CW], sum[CW], scale[CW];
};
template <int CW> using Block = f4[2][CW];                     // products of 32 keys: key 16 t + 4 (lane / 16) + i of row lane % 16

// The weights of a block's 32 keys
template <typename CT, int HD, int CW, typename Order>
__device__ __forceinline__ void weigh(Columns<HD, CW>& r, const Block<CW>& s, u4 (&p)[CW])
{
    float most[CW];
    bool move = false;
#pragma unroll
    for (int n = 0; n < CW; n++) {
        float m = fmaxf(s[0][n][0], s[1][n][0]);
#pragma unroll
        for (int i = 1; i < 4; i++) m = fmaxf(fmaxf(m, s[0][n][i]), s[1][n][i]);
        most[n] = m * r.scale[n];
        move = move || most[n] > r.ref[n] + SLACK;
    }
    if (__ballot(move)) {
#pragma unroll
        for (int n = 0; n < CW; n++) {
            const float ref = fmaxf(r.ref[n], max_of_column(most[n]));
            const float by = ref == r.ref[n] ? 1.f : __builtin_amdgcn_exp2f(r.ref[n] - ref);
            r.ref[n] = ref;
            r.sum[n] *= by;
#pragma unroll
            for (int ct = 0; ct < HD / 16; ct++) r.o[ct][n] *= by;
        }
    }
#pragma unroll
    for (int n = 0; n < CW; n++) {
        const float shift = r.ref[n] == -INFINITY ? 0.f : SHIFT<CT> - r.ref[n];
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            w[e] = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][n][e & 3], r.scale[n], shift));
            r.sum[n] += w[e];
        }
#pragma unroll
        for (int e = 0; e < 4; e++) p[n][e] = pack2(w[Order::first(e)], w[Order::second(e)], CT());
    }
}

// Blocks first, first + NW, .. below end of a class's segment of len tokens.  PRECISE: codes enter the products as they are, a group's at a time, and its
// scale and minimum meet the sums in fp32.
template <int HD, int BITS, int CW, bool PRECISE>
__device__ __forceinline__ void stream_packed(Columns<HD, CW>& r, const char* s_query, const float* s_sum, const wq_packed_kv& kv, int kvh, int64_t tok0, int len,
                                              int first, int end, uint32_t* s_meta)
{
    constexpr int C = BITS == 2 ? 0 : (BITS == 4 ? 1 : 2), ST = STEPS<F16, HD>, KB = HD / 4 * BITS / 8, VB = HD / 16 * BITS;
    using Order = std::conditional_t<BITS == 8, Near, Far>;
    const int lane = threadIdx.x & 63, m = lane & 15, j = lane >> 4, G = HD / kv.group;
    const int64_t k_slot = kvh * kv.cap[C] + tok0, v_slot = (kv.Hkv + kvh) * kv.cap[C] + tok0;
    const uint8_t* k_codes = static_cast<const uint8_t*>(kv.codes[C]) + k_slot * (HD * BITS / 8) + lane * KB;
    const uint8_t* v_codes = static_cast<const uint8_t*>(kv.codes[C]) + v_slot * (HD * BITS / 8) + lane * VB;
    // a block's metadata words, 32 G of the keys and then 32 G of the values: load r takes 64 of them
    const uint32_t* k_meta = static_cast<const uint32_t*>(kv.meta[C]) + k_slot * G + lane;
    const uint32_t* v_meta = static_cast<const uint32_t*>(kv.meta[C]) + v_slot * G + lane;
    const uint32_t* m0 = G == 1 && lane >= 32 ? v_meta - 32 : k_meta;
    const uint32_t* m1 = G == 2 ? v_meta : k_meta + 64;
    uint32_t wk[2][(KB + 3) / 4], wv[(VB + 3) / 4], wm[4] = {0, 0, 0, 0};
    auto load_meta = [&](int b) {
        const int64_t at = (int64_t)b * 32 * G;
        wm[0] = m0[at];
        if (G >= 2) wm[1] = m1[at];
        if (G == 4) wm[2] = v_meta[at], wm[3] = v_meta[at + 64];
    };
    auto load_keys = [&](int b) {
#pragma unroll
        for (int t = 0; t < 2; t++) load_words<KB>(k_codes + (int64_t)b * (4 * HD * BITS) + t * 64 * KB, wk[t]);
    };
    auto load_values = [&](int b) { load_words<VB>(v_codes + (int64_t)b * (4 * HD * BITS), wv); };
    // (one block ahead.  Two cost one column's kernels their third wavefront a SIMD, 31 -> 39 us of 8 x 12800 tokens, and brought two columns' nothing)
    load_meta(first);
    load_keys(first);
    load_values(first);
    // (two columns' queries stay in registers; more are read from LDS at every block, where they would not leave enough of them)
    constexpr bool HELD = CW * ST <= 8;
    u4 held[HELD ? CW : 1][HELD ? ST : 1];
    auto query = [&](int n, int st) -> u4 {
        if constexpr (HELD) return held[n][st];
        else return *reinterpret_cast<const u4*>(s_query + (n * ST + st) * 1024 + lane * 16);
    };
    if constexpr (HELD) {
#pragma unroll
        for (int n = 0; n < CW; n++)
#pragma unroll
            for (int st = 0; st < ST; st++) held[n][st] = *reinterpret_cast<const u4*>(s_query + (n * ST + st) * 1024 + lane * 16);
    }
#pragma unroll 1
    for (int b = first; b < end; b += NW) {
        s_meta[lane] = wm[0];
        if (G >= 2) s_meta[64 + lane] = wm[1];
        if (G == 4) s_meta[128 + lane] = wm[2], s_meta[192 + lane] = wm[3];
        asm volatile("" ::: "memory");                         // (one wavefront's LDS operations keep their order)
        const bool more = b + NW < end;
        if (more) load_meta(b + NW);
        Block<CW> s;
        if constexpr (PRECISE) {
#pragma unroll
            for (int t = 0; t < 2; t++) {
                u4 a[ST];
#pragma unroll
                for (int st = 0; st < ST; st++) a[st] = expanded_keys<BITS>(wk[t], st, Codes(), Codes());
#pragma unroll
                for (int g = 0; g < 4; g++) {
                    if (g >= G) break;
                    const u4 sm = *reinterpret_cast<const u4*>(s_meta + (t * G + g) * 16 + 4 * j);
                    const uint32_t mine = (j * G >> 2) == g ? ~0u : 0u;
                    float q_sum[CW];
#pragma unroll
                    for (int n = 0; n < CW; n++) q_sum[n] = s_sum[(g * 4 / G) * (16 * CW) + 16 * n + m];
                    f4 x[CW];
#pragma unroll
                    for (int st = 0; st < ST; st++) {
                        const u4 y = {a[st][0] & mine, a[st][1] & mine, a[st][2] & mine, a[st][3] & mine};
#pragma unroll
                        for (int n = 0; n < CW; n++) x[n] = product<F16>(y, query(n, st), st ? x[n] : f4{0.f, 0.f, 0.f, 0.f});
                    }
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const uint32_t word = sm[i];
                        const h2 f = __builtin_bit_cast(h2, word);
#pragma unroll
                        for (int n = 0; n < CW; n++) {
                            const float y = g ? fmaf((float)f[1], q_sum[n], s[t][n][i]) : (float)f[1] * q_sum[n];
                            s[t][n][i] = fmaf((float)f[0], x[n][i], y);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        } else {
            u4 a[2][ST];
#pragma unroll
            for (int t = 0; t < 2; t++) {
                const h2 sm = __builtin_bit_cast(h2, s_meta[(t * G + (j * G >> 2)) * 16 + m]);
#pragma unroll
                for (int st = 0; st < ST; st++) a[t][st] = expanded_keys<BITS>(wk[t], st, h2{sm[0], sm[0]}, h2{sm[1], sm[1]});
            }
#pragma unroll
            for (int st = 0; st < ST; st++)
#pragma unroll
                for (int n = 0; n < CW; n++) {
                    const u4 y = query(n, st);
#pragma unroll
                    for (int t = 0; t < 2; t++) s[t][n] = product<F16>(a[t][st], y, st ? s[t][n] : f4{0.f, 0.f, 0.f, 0.f});
                }
        }
        if (more) load_keys(b + NW);
        const int left = len - 32 * b;
        if (left < 32) {
#pragma unroll
            for (int t = 0; t < 2; t++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (16 * t + 4 * j + i >= left)
#pragma unroll
                        for (int n = 0; n < CW; n++) s[t][n][i] = -INFINITY;
        }
        u4 p[CW];
        weigh<F16, HD, CW, Order>(r, s, p);
        h2 vs[4], vm[4];
#pragma unroll
        for (int c = 0; c < HD / 32; c++) {                    // 32 channels are of one group
            if (c == 0 || 32 * c % kv.group == 0) {
                const int g = 32 * c / kv.group;
                const u4 x = *reinterpret_cast<const u4*>(s_meta + (2 * G + g) * 16 + 4 * j), y = *reinterpret_cast<const u4*>(s_meta + (3 * G + g) * 16 + 4 * j);
                const uint32_t t[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    vs[e] = __builtin_bit_cast(h2, low_halves(t[Order::first(e)], t[Order::second(e)]));
                    vm[e] = __builtin_bit_cast(h2, high_halves(t[Order::first(e)], t[Order::second(e)]));
                }
            }
#pragma unroll
            for (int ct = 2 * c; ct < 2 * c + 2; ct++) {
                const u4 x = expanded_values<BITS>(wv, ct, vs, vm);
#pragma unroll
                for (int n = 0; n < CW; n++) r.o[ct][n] = product<F16>(x, p[n], r.o[ct][n]);
            }
        }
        asm volatile("" ::: "memory");                         // (the metadata have been read)
        if (more) load_values(b + NW);
    }
}

// Chunks first, first + NW, .. below end of 32 of the n rows from k, v on: keys straight into registers, values through the wavefront's piece of LDS.
// sees(n, c): this lane's 8 keys of chunk c that its row of column n sees, bits 16 t + i.
template <typename QT, int HD, int CW, typename Sees>
__device__ __forceinline__ void stream_rows(Columns<HD, CW>& r, const QueryRows<QT, HD, CW>& q, const char* k, const char* v, int64_t k_stride, int64_t v_stride, int n,
                                            int first, int end, Lds tile, const Sees& sees)
{
    constexpr int ST = STEPS<QT, HD>, PIECES = HD / 8, PER_LOAD = 64 / PIECES, LOADS = 32 / PER_LOAD;
    using D = Direct<HD>;
    const int lane = threadIdx.x & 63, m = lane & 15, j = lane >> 4;
    const D rows(v_stride, v_stride);
#pragma unroll 1
    for (int c = first; c < end; c += NW) {
        const int64_t key0 = 32 * (int64_t)c;
        const int left = n - 32 * c;                           // (the last row is read again for the rest: its weights are zero)
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int row = i * PER_LOAD + lane / PIECES, piece = (lane % PIECES) ^ (D::swizzle(row) * 2 & (PIECES - 1));
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(v + (key0 + (row < left ? row : left - 1)) * v_stride + 16 * piece),
                                             (__attribute__((address_space(3))) void*)(tile + i * 1024), 16, 0, 0);
        }
        Block<CW> s;
#pragma unroll
        for (int t = 0; t < 2; t++) {
            const int row = 16 * t + m;
            const char* at = k + (key0 + (row < left ? row : left - 1)) * k_stride;
            u4 a[ST];
#pragma unroll
            for (int st = 0; st < ST; st++) a[st] = *reinterpret_cast<const u4*>(at + (4 * st + j) * 16);
#pragma unroll
            for (int st = 0; st < ST; st++)
#pragma unroll
                for (int col = 0; col < CW; col++) s[t][col] = product<QT>(a[st], q[col][st], st ? s[t][col] : f4{0.f, 0.f, 0.f, 0.f});
        }
#pragma unroll
        for (int col = 0; col < CW; col++) {
            const uint32_t bits = sees(col, c);
#pragma unroll
            for (int t = 0; t < 2; t++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (!(bits >> (16 * t + i) & 1)) s[t][col][i] = -INFINITY;
        }
        u4 p[CW];
        weigh<QT, HD, CW, Natural>(r, s, p);
        __builtin_amdgcn_s_waitcnt(0x0F70);                    // vmcnt(0): the values are in LDS
        asm volatile("" ::: "memory");
#pragma unroll
        for (int ct = 0; ct < HD / 16; ct++) {
            const u4 x = rows.values(tile, 0, ct);
#pragma unroll
            for (int col = 0; col < CW; col++) r.o[ct][col] = product<QT>(x, p[col], r.o[ct][col]);
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);                    // lgkmcnt(0): they are out of it again
        asm volatile("" ::: "memory");
    }
}

__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : (n <= 0 ? 0u : (1u << n) - 1); }

// The first of this wavefront's blocks from t0 on, where block t of a segment is the part's (done + t - lo)-th
__device__ __forceinline__ int first_block(int t0, int done, int lo) { return t0 + ((this_wave() - (done + t0 - lo)) & (NW - 1)); }

template <typename QT, int HD, int CW, bool PRECISE>
__global__ __launch_bounds__(64 * NW, 2) void k_tree_stream(TreeArgs a)
{
    static_assert(NW == 4, "a wavefront for each 16 of 64 channels");
    constexpr int R = 16 * CW, ST = STEPS<F16, HD>, TILE = 32 * HD * 2, QUERY = CW * ST * 1024;
    constexpr int ENDS = NW * CW * (4 * 1024 + 128), WALK = 3 * QUERY + NW * TILE, BIG = WALK > ENDS ? WALK : ENDS;
    // the queries as each class's products take them, and the values of 16-bit rows, a piece of each wavefront; in the end numerators, references and
    // sums
    __shared__ __align__(16) char s_big[BIG];
    __shared__ uint64_t s_seen[R * WORDS];
    __shared__ __align__(16) uint32_t s_meta[NW][256];         // (before the walk a tree's parents)
    __shared__ float s_scale[R], s_sum[PRECISE ? 4 : 1][R];
    static_assert(sizeof(s_meta) >= WQ_MAX_TREE * 4, "");
    const int Hkv = a.kv.Hkv, wave = this_wave(), lane = threadIdx.x & 63, j = lane >> 4;
    const wq_packed_kv& kv = a.kv;

    const int unit = (int)blockIdx.x % a.units, piece = (int)blockIdx.x / a.units, kvh = unit % Hkv;
    Place p = {};
    const bool there = place_of<R>(a, unit / Hkv, p);
    const int b = p.seq, row0 = p.row0, rows = there ? p.rows : 0;
    const int64_t first_row = p.first;
    // A wavefront prepares a column's queries (CW <= 4); they are on their way while the cache's tables are
    auto row_at = [&](int n) -> const char* {
        const int row = row0 + 16 * n + (lane & 15);
        return row < rows ? a.q + (first_row + row / a.rep) * a.q_stride + (kvh * a.rep + row % a.rep) * (HD * 2) : nullptr;
    };
    QueryRows<F16, HD, 1> query;
    if (wave < CW) load_query_quarter<F16, HD>(query, 0, row_at(wave));
    const Sequence s = sequence_of<32>(a, b, rows);
    if (!there) {
        leave_unit(a, unit, piece, p, 0);
        return;
    }
    clear_rest<R, HD>(a, p, kvh, piece);
    if (piece >= s.pieces) return;
    leave_unit(a, unit, piece, p, s.pieces);
    const int lo = begin_of(s, piece, 8), hi = begin_of(s, piece + 1, 8);
    const int node0 = row0 / a.rep, last_row = (row0 + R < rows ? row0 + R : rows) - 1;
    int newest = last_row / a.rep + 1;                         // (no row sees one behind itself)
    if (newest > a.most) newest = a.most;
    if (rows / a.rep > a.most && row0 == 0 && lo == 0 && threadIdx.x == 0) atomicOr(a.status, WQ_DEV_TOO_MANY_ROWS);
    const int cached = s.all - (rows / a.rep + 31) / 32;
    if (a.parent && hi > cached) find_ancestors(a.parent + first_row, node0, last_row / a.rep + 1 - node0, s_seen, reinterpret_cast<int32_t*>(s_meta), 64 * NW);

    // Queries in fp16 and in every class's order
    if (wave < CW) {
        QueryRows<F16, HD, 1>&q = query, y;
        const bool bad = not_finite<QT, HD>(q, 0);
        float scale = a.scale;
        if constexpr (std::is_same_v<QT, Bf16>) scale = fminf(fmaxf(a.scale * query_as_f16<HD>(q, 0), FLT_MIN), FLT_MAX);      // (see walk_cache)
        if (bad) scale = NAN;
        if (lane < 16) s_scale[16 * wave + lane] = scale;
        if constexpr (PRECISE) {
            float mine = 0.f;
#pragma unroll
            for (int st = 0; st < ST; st++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const uint32_t word = q[0][st][e];
                    const h2 f = __builtin_bit_cast(h2, word);
                    mine += (float)f[0] + (float)f[1];
                }
            // of the head's groups: a quarter's own (4), two quarters' (2), all (1)
            const int G = HD / kv.group;
            if (G < 4) mine += __shfl_xor(mine, 16, 64);
            if (G < 2) mine += __shfl_xor(mine, 32, 64);
            s_sum[j][16 * wave + (lane & 15)] = mine;      // of the quarter's group
        }
        auto leave = [&](auto bits, int order) __attribute__((always_inline)) {
#pragma unroll
            for (int st = 0; st < ST; st++) y[0][st] = q[0][st];
            order_query<decltype(bits)::value, HD>(y, 0);
#pragma unroll
            for (int st = 0; st < ST; st++) *reinterpret_cast<u4*>(s_big + order * QUERY + (wave * ST + st) * 1024 + lane * 16) = y[0][st];
        };
        leave(std::integral_constant<int, 2>(), 0);
        leave(std::integral_constant<int, 4>(), 1);
        leave(std::integral_constant<int, 8>(), 2);
    }
    __syncthreads();

    Columns<HD, CW> r;
#pragma unroll
    for (int n = 0; n < CW; n++) {
        r.ref[n] = -INFINITY, r.sum[n] = 0.f, r.scale[n] = s_scale[16 * n + (lane & 15)];
#pragma unroll
        for (int ct = 0; ct < HD / 16; ct++) r.o[ct][n] = f4{0.f, 0.f, 0.f, 0.f};
    }
    // (MODE.FP16_OVFL: see walk_cache)
    constexpr int FP16_OVFL = 1 | 23 << 6;
    __builtin_amdgcn_s_setreg(FP16_OVFL, 1);
    int done = 0;
    auto walk_class = [&](auto bits) __attribute__((always_inline)) {
        constexpr int BITS = decltype(bits)::value, c = BITS == 2 ? 0 : (BITS == 4 ? 1 : 2);
        const int t0 = lo > done ? lo - done : 0, t1 = hi - done < s.blocks[c] ? hi - done : s.blocks[c];
        const int first = first_block(t0, done, lo);
        done += s.blocks[c];
        if (first >= t1) return;
        stream_packed<HD, BITS, CW, PRECISE>(r, s_big + c * QUERY, &s_sum[0][0], kv, kvh, kv.cls_off[c][b], s.len[c], first, t1, s_meta[wave]);
    };
    walk_class(std::integral_constant<int, 2>());
    walk_class(std::integral_constant<int, 4>());
    walk_class(std::integral_constant<int, 8>());
    __builtin_amdgcn_s_setreg(FP16_OVFL, 0);
    if constexpr (std::is_same_v<QT, Bf16>) {              // from the packed tokens' shift to the rows', exact
#pragma unroll
        for (int n = 0; n < CW; n++) {
            r.sum[n] *= exp2f(SHIFT<QT> - SHIFT<F16>);
#pragma unroll
            for (int ct = 0; ct < HD / 16; ct++) r.o[ct][n] *= exp2f(SHIFT<QT> - SHIFT<F16>);
        }
    }
    if (hi > done) {
        const Lds tile = (Lds)s_big + 3 * QUERY + wave * TILE;
        int t0 = lo > done ? lo - done : 0, t1 = hi - done < s.blocks[3] ? hi - done : s.blocks[3], first = first_block(t0, done, lo);
        const int done16 = done + s.blocks[3], n0 = lo > done16 ? lo - done16 : 0, first_new = first_block(n0, done16, lo);
        const int n1 = hi - done16 < (newest + 31) / 32 ? hi - done16 : (newest + 31) / 32;
        if (first < t1 || first_new < n1) {
            QueryRows<F16, HD, CW> q;
#pragma unroll
            for (int n = 0; n < CW; n++) {
                r.scale[n] = a.scale;
                load_query<F16, HD>(q, n, row_at(n));
            }
            if (first < t1) {
                const int64_t from = kv.off16[b], stride = (int64_t)Hkv * HD * 2;
                const char* k = static_cast<const char*>(kv.k16) + from * stride + kvh * (HD * 2);
                const char* v = static_cast<const char*>(kv.v16) + from * stride + kvh * (HD * 2);
                stream_rows<QT, HD, CW>(r, q, k, v, stride, stride, s.len[3], first, t1, tile, [&](int, int c) { return low_bits(s.len[3] - 32 * c) >> 4 * j; });
            }
            if (first_new < n1) {
                const char* k = a.k + first_row * a.k_stride + kvh * (HD * 2);
                const char* v = a.v + first_row * a.v_stride + kvh * (HD * 2);
                const uint32_t* seen = reinterpret_cast<const uint32_t*>(s_seen);
                stream_rows<QT, HD, CW>(r, q, k, v, a.k_stride, a.v_stride, newest, first_new, n1, tile, [&](int n, int c) {
                    const int row = row0 + 16 * n + (lane & 15), node = row / a.rep;
                    uint32_t bits = 0;
                    if (row <= last_row) bits = a.parent ? seen[(node - node0) * (2 * WORDS) + c] : low_bits(node + 1 - 32 * c);
                    return bits >> 4 * j;
                });
            }
        }
    }
    // The wavefronts' numerators together, 64 channels at a time: each brings its own to the rows' common reference, and each sums up and stores 16 of them
    float(*s_ml)[CW][2][16] = reinterpret_cast<float(*)[CW][2][16]>(s_big + 4 * NW * CW * 1024);
    __syncthreads();                                           // (everybody has read the queries and its values)
#pragma unroll
    for (int n = 0; n < CW; n++) {
        r.sum[n] = sum_of_column(r.sum[n]);
        r.ref[n] -= SHIFT<QT>;
        if (j == 0) s_ml[wave][n][0][lane] = r.ref[n], s_ml[wave][n][1][lane] = r.sum[n];
    }
    __syncthreads();
    float M[CW], L[CW];
#pragma unroll
    for (int n = 0; n < CW; n++) {
        M[n] = -INFINITY, L[n] = 0.f;
#pragma unroll
        for (int w = 0; w < NW; w++) M[n] = fmaxf(M[n], s_ml[w][n][0][lane & 15]);
        const float base = M[n] == -INFINITY ? 0.f : M[n], by = __builtin_amdgcn_exp2f(r.ref[n] - base);
#pragma unroll
        for (int w = 0; w < NW; w++) L[n] += s_ml[w][n][1][lane & 15] * __builtin_amdgcn_exp2f(s_ml[w][n][0][lane & 15] - base);
#pragma unroll
        for (int ct = 0; ct < HD / 16; ct++) r.o[ct][n] *= by;
    }
    float* left = a.part + ((int64_t)unit * a.splits + piece) * PIECE<HD, R>;
#pragma unroll
    for (int pass = 0; pass < HD / 64; pass++) {
        if (pass > 0) __syncthreads();
#pragma unroll
        for (int n = 0; n < CW; n++)
#pragma unroll
            for (int i = 0; i < 4; i++) *reinterpret_cast<f4*>(s_big + ((wave * CW + n) * 4 + i) * 1024 + lane * 16) = r.o[4 * pass + i][n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < CW; n++) {
            f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; w++) x += *reinterpret_cast<const f4*>(s_big + ((w * CW + n) * 4 + wave) * 1024 + lane * 16);
            const int row = row0 + 16 * n + (lane & 15), channel = 64 * pass + 16 * wave + 4 * j;
            if (row >= rows) continue;
            const bool refused = row / a.rep >= a.most;       // as if it saw nothing
            const float ref = refused ? -INFINITY : M[n], sum = refused ? 0.f : L[n];
            if (refused) x = f4{0.f, 0.f, 0.f, 0.f};
            const bool first = pass == 0 && wave == 0 && j == 0;
            if (s.pieces > 1) {
                const int at = 16 * n + (lane & 15);
                *reinterpret_cast<f4*>(left + at * HD + channel) = x;
                if (first) left[R * HD + 2 * at] = ref, left[R * HD + 2 * at + 1] = sum;
                continue;
            }
            const int64_t to_row = (first_row + row / a.rep) * a.Hq + kvh * a.rep + row % a.rep;
            x *= one_over(sum);
            *reinterpret_cast<uint2*>(static_cast<char*>(a.out) + (to_row * HD + channel) * 2) = make_uint2(pack2(x[0], x[1], QT()), pack2(x[2], x[3], QT()));
            if (a.lse && first) a.lse[to_row] = log_sum_exp(ref, sum);
        }
    }
}

template <typename QT, int HD, bool PRECISE>
TreeKernel of_columns(int columns)
{
    switch (columns) {
        case 1: return k_tree_stream<QT, HD, 1, PRECISE>;
        case 2: return k_tree_stream<QT, HD, 2, PRECISE>;
    }
    return k_tree_stream<QT, HD, 3, PRECISE>;
}

TreeKernel stream_kernel(int dtype, int hd, int columns, bool precise)
{
    if (dtype == WQ_F16) return hd == 128 ? of_columns<F16, 128, true>(columns) : of_columns<F16, 64, true>(columns);
    if (precise) return hd == 128 ? of_columns<Bf16, 128, true>(columns) : of_columns<Bf16, 64, true>(columns);
    return hd == 128 ? of_columns<Bf16, 128, false>(columns) : of_columns<Bf16, 64, false>(columns);
}

}  // namespace

TreeKernel wq_tree_stream_kernel(int dtype, int hd, int columns, bool lse) { return stream_kernel(dtype, hd, columns, dtype == WQ_F16 || lse); }
