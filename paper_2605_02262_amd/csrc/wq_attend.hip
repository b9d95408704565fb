// Attention of many query rows of one KV head over one sequence: wq_prefill_attention (keys and values are plain rows, a
// row sees the keys up to its own position and the sequence's prefix) and the shared part of wq_decode_attention_shared
// (keys and values are a packed cache that the requests of a group all attend to).
//
// A row is a (token, query head) pair or a (request, query head) pair: the rep query heads of a KV head are neighbouring
// rows of one product, so a tile of keys and values is brought once for all of them.  A workgroup walks the keys a tile at a time:
//   S^T = K Q^T    A operand: 16 keys, B operand: 16 rows   -> a lane holds 4 x 4 keys of one row
//   online softmax in the lane's own registers (running reference and sum, fp32)
//   O^T += V^T P^T A operand: 16 channels, B operand: 16 rows: P^T needs no exchange between lanes, because the keys'
//                  order inside a product is free: V's operand takes them in the order in which S^T left them
// 16-bit types: 256 rows (32 per wavefront), 64 keys; two groups of four wavefronts in turn (take_turns), one workgroup per compute unit
// (its accumulators, queries and scores take 220 to 240 registers a lane).  fp32: 128 rows, 32 keys, four wavefronts.
//   k_prefill        keys and values plain rows, from memory into LDS without registers between (Direct)
//   k_prefill_few    the same for so few query rows that the keys are shared out instead
//   k_shared         packed classes, expanded to fp16 on their way into LDS (PackedKeys, PackedValues; fp16 queries meet keys' codes), then 16-bit rows
//   k_shared_finish  a request's own 16-bit rows, and the merge of the parts; k_merge, k_merge_tail: the merges of k_prefill's
// Packed tiles lie in LDS in the operands' own order, [step][lane][16 bytes]: every LDS read of the products is one conflict-free 16-byte
// load per lane.  Plain rows lie as they came, their 16-byte pieces exchanged by row.
//
// What bounds it (28 query heads, 4 KV heads of 128, bf16, one MI355X): the phases of vector instructions.  A tile of 64 keys takes a wavefront 64 matrix
// instructions, 1150 cycles, and 1200 to 1450 cycles of exponents, sums and conversions; the two groups' phases together are 3740
// cycles (matrix cores busy 57 % of them, vector unit active 60 %).  12800 query rows over as many keys: 1.95 ms = 1.18 PFLOP/s with a prefix of 98 %,
// 1.04 ms = 1.13 causal, where a library product of 8192^3 reaches 1.37.  A packed tile also has to be expanded, 16384 codes, 4900 cycles, and the phase in
// which group 1 forms weights and expands values is the longest: neither unit is full (33 %, 48 %), but that wavefront's instructions follow each
// other.  50 700 packed tokens under 64 requests (448 rows per KV head): 72 us of a call's 85 in a series = 0.65 PFLOP/s (81 traced by itself).
// A lone wavefront issues one vector instruction in 6 cycles, two on a SIMD one in 2.7: more of them do not fit the registers.
// Short walks cost what they cannot overlap: 2 us from the launch to the first load, 2 until its first product, 2 for the result.
//
// fp32 queries take the fp32 matrix instruction throughout.  16-bit queries take the 16-bit ones: the weights are rounded to
// the value's type (the sum of weights is not), packed values to fp16 (2^-11 of a value whose own step is its
// scale; below the output's own rounding), and so are packed keys for bf16 queries, whose results are rounded eight times coarser.
#include "wq_attend.h"

namespace {

// ---- wq_prefill_attention ----------------------------------------------------------------------------------------------
struct PrefillArgs {
    const char *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;      // bytes from row to row
    const int32_t *q_off, *kv_off, *prefix_len;
    int64_t total_q, total_kv;
    int B, Hq, rep, splits;
    int units, tail, tail_splits;              // KV heads * tiles; the last so many of them in the order of the launch are cut into so many parts
    float scale;                               // log2(e) * sm_scale
    Out out;
};

template <typename CT, int HD, bool SPLIT>
__global__ __launch_bounds__(64 * WAVES<CT>, 2) void k_prefill(PrefillArgs a)
{
    constexpr int BYTES = TILE_BYTES<CT, HD> * (ESIZE<CT> == 2 ? 2 : 1), R = ROWS<CT, SPLIT>;
    __shared__ __align__(16) char s_k[BYTES], s_v[BYTES];
    const int Hkv = a.Hq / a.rep, wave = this_wave(), lane = threadIdx.x & 63, in_tail = (int)blockIdx.x - (a.units - a.tail);
    int unit = blockIdx.x, split = blockIdx.y, parts = a.splits;
    if (in_tail >= 0 && a.tail > 0) unit = a.units - a.tail + in_tail / a.tail_splits, split = in_tail % a.tail_splits, parts = a.tail_splits;
    const int kvh = unit % Hkv;
    Place p;
    if (!find_place<R>(a.q_off, a.B, a.rep, a.total_q, (a.units - 1 - unit) / Hkv, p)) return;      // (the last rows see the most keys: they begin first)
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
    const int last_row = (p.row0 + R < p.rows ? p.row0 + R : p.rows) - 1;
    const int tiles = (limit_of(last_row) + KEYS<CT> - 1) / KEYS<CT>;
    const int lo = (int)((int64_t)split * tiles / parts), hi = (int)((int64_t)(split + 1) * tiles / parts);

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
        load_query<CT, HD>(q, n, at);
    }
    const bool any = wrow0 < p.rows && wave * COLS * 16 < R;
    const int wlast = wrow0 + COLS * 16 <= p.rows ? wrow0 + COLS * 16 - 1 : p.rows - 1;
    const int least = any ? limit_of(wrow0) : 0, most = any ? limit_of(wlast) : 0;
    const char* k = a.k + kv0 * a.k_stride + kvh * (HD * ESIZE<CT>);
    const char* v = a.v + kv0 * a.v_stride + kvh * (HD * ESIZE<CT>);
    if constexpr (ESIZE<CT> == 2) {
        if (lo < hi) walk_rows<CT, HD, SPLIT>(r, q, k, v, a.k_stride, a.v_stride, len, lo, hi, least, (Lds)s_k, (Lds)s_v);
    } else {
        for (int t = lo; t < hi; t++) {
            const int key0 = t * KEYS<CT>;
            __syncthreads();
            stage_rows<CT, HD>(k + key0 * a.k_stride, v + key0 * a.v_stride, a.k_stride, a.v_stride, len - key0, (Lds4)s_k, (Lds4)s_v);
            __syncthreads();
            attend_f32<HD>(r, q, (Lds4)s_k, (Lds4)s_v, key0, least, most);
        }
    }
    if (any) store_rows<CT, HD>(r, p, a.rep, a.Hq, kvh, wave, split, parts > 1 ? parts : 0, a.out, a.tail > 0 ? (int64_t)(a.units - 1 - unit) * R : -1);
}

// ---- wq_decode_attention_shared ------------------------------------------------------------------------------------------
struct SharedArgs {
    const char* q;                             // [B][Hq][hd]
    const int32_t* req_off;
    int B, P, Hq, rep;
    int units, splits;                         // (tile of rows, KV head) pairs of the shared caches, and the parts that each is cut into
    float scale;
    wq_packed_kv kv;
    Out out;
};

// QT, G: see walk_cache
template <typename QT, int HD, int G>
__global__ __launch_bounds__(64 * WAVES<QT>, 2) void k_shared(SharedArgs a)
{
    using CT = Walked<QT>;
    constexpr bool PIPED = ESIZE<QT> == 2;
    constexpr int BYTES = TILE_BYTES<CT, HD> * (1 + PIPED), R = ROWS<QT>, TK = KEYS<QT>;
    __shared__ __align__(16) char s_k[BYTES], s_v[BYTES], s_m[G > 0 ? 2 * 64 * 4 * G : 16];
    const int Hkv = a.kv.Hkv, wave = this_wave(), lane = threadIdx.x & 63;
    const wq_packed_kv& kv = a.kv;
    const int unit = (int)blockIdx.x % a.units, split = (int)blockIdx.x / a.units, kvh = unit % Hkv;
    Place p;
    if (!find_place<R>(a.req_off, a.P, a.rep, a.B, unit / Hkv, p)) return;
    // (Both loops over the classes stand here, not in functions like the trees' (wq_tree.h): the compiler keeps 36 more scalars in vector registers then, and with fp32 and heads
    // of 128 five more registers in scratch.  us, here and there: 64 requests over 51200 tokens 84.5, 85.2; the configuration's tiers 31.8, 32.3; fp32, 64 over 12800: 152, 155)
    int tiles[4], all = 0, len[4];
#pragma unroll
    for (int c = 0; c < 4; c++) {
        const int64_t room = c < 3 ? kv.cap[c] - kv.cls_off[c][p.seq] : kv.cap16 - kv.off16[p.seq];
        len[c] = c < 3 ? kv.cls_len[c][p.seq] : kv.len16[p.seq];
        if (len[c] > room) len[c] = (int)room;
        tiles[c] = len[c] > 0 ? (len[c] + TK - 1) / TK : 0;
        all += tiles[c];
    }
    const int lo = (int)((int64_t)split * all / a.splits), hi = (int)((int64_t)(split + 1) * all / a.splits);

    Rows<HD> r;
    Query<CT, HD> q;
    clear(r);
    const int wrow0 = p.row0 + wave * COLS * 16;
    const char* row_at[COLS];
#pragma unroll
    for (int n = 0; n < COLS; n++) {
        const int row = wrow0 + 16 * n + (lane & 15);
        row_at[n] = row < p.rows ? a.q + ((p.first + row / a.rep) * a.Hq + kvh * a.rep + row % a.rep) * (HD * ESIZE<QT>) : nullptr;
    }
    const bool any = wrow0 < p.rows;   // (fp32: a wavefront without rows only brings tiles; 16-bit types: it keeps its turns, on zeros)
    int done = 0;                                              // tiles of the classes before
    auto walk = [&](auto bits) __attribute__((always_inline)) {
        constexpr int BITS = decltype(bits)::value, c = BITS == 2 ? 0 : (BITS == 4 ? 1 : 2);
        const int t0 = lo > done ? lo - done : 0, t1 = hi - done < tiles[c] ? hi - done : tiles[c];
        done += tiles[c];
        if (t0 < t1) walk_class<QT, HD, G, false, BITS>(r, q, row_at, a.scale, kv, p.seq, kvh, len[c], t0, t1, any, (Lds)s_k, (Lds)s_v, (Lds)s_m);
    };
    largest_instead_of_infinity<QT>(true);
    walk(std::integral_constant<int, 2>());
    walk(std::integral_constant<int, 4>());
    walk(std::integral_constant<int, 8>());
    largest_instead_of_infinity<QT>(false);
    shift_rows<QT>(r);
    if (hi > done) walk_rows16<QT, HD, false>(r, q, row_at, a.scale, kv, p.seq, kvh, len[3], lo > done ? lo - done : 0, hi - done, any, (Lds)s_k, (Lds)s_v);
    if (any) store_rows<QT, HD>(r, p, a.rep, a.Hq, kvh, wave, split, a.splits, a.out);
}

// The tail's tiles: a wavefront per row, 64 workgroups per tile.  Many rows, few parts: four loads in flight, and twice the wavefronts
template <int HD>
__global__ __launch_bounds__(256) void k_merge_tail(PrefillArgs a, int dtype)
{
    const int Hkv = a.Hq / a.rep, u = blockIdx.x >> 6, in_tile = (blockIdx.x & 63) * 4 + this_wave(), lane = threadIdx.x & 63, parts = a.tail_splits;
    Place p;
    if (!find_place<256>(a.q_off, a.B, a.rep, a.total_q, u / Hkv, p) || p.row0 + in_tile >= p.rows) return;
    const int row = p.row0 + in_tile, kvh = (a.units - 1 - u) % Hkv;
    const int64_t slot = ((int64_t)u * 256 + in_tile) * parts;
    const float m = lane < parts ? a.out.part_ml[(slot + lane) * 2] : -INFINITY;
    const float l = lane < parts ? a.out.part_ml[(slot + lane) * 2 + 1] : 0.f;
    const float M = wave_max(m), w = __builtin_amdgcn_exp2f(m - (M == -INFINITY ? 0.f : M));
    const f4 x = sum_of_groups<HD>(sum_of_parts<HD, 4>(a.out.part + slot * HD, parts, w));
    store_merged<HD>(a.out, dtype, (p.first + row / a.rep) * a.Hq + kvh * a.rep + row % a.rep, x, M, wave_sum(l * w));
}

// wq_prefill_attention over few query rows: a workgroup per 16 of them and part of the keys.  Bound by latencies: 8 single tokens (14 query heads, 2 KV
// heads of 64) over 6400 rows, 26 MB: 13.0 us with the merge (k_prefill: 15.4).
template <typename CT, int HD>
__global__ __launch_bounds__(64 * FEW, 4) void k_prefill_few(PrefillArgs a, int dtype)
{
    __shared__ Few<HD> s;
    const int Hkv = a.Hq / a.rep, kvh = blockIdx.x % Hkv, split = blockIdx.y, wave = this_wave(), lane = threadIdx.x & 63;
    Place p;
    if (!find_place<16>(a.q_off, a.B, a.rep, a.total_q, blockIdx.x / Hkv, p)) return;
    const int64_t kv0 = clipped(a.kv_off[p.seq], a.total_kv), kv1 = clipped(a.kv_off[p.seq + 1], a.total_kv);
    const int len = kv1 > kv0 ? (int)(kv1 - kv0) : 0, first = len - p.rows / a.rep;
    int prefix = a.prefix_len ? a.prefix_len[p.seq] : 0;
    prefix = prefix < 0 ? 0 : (prefix > len ? len : prefix);
    auto limit_of = [&](int row) {
        const int seen = first + row / a.rep + 1;
        return seen > prefix ? seen : prefix;
    };
    const int rows = p.rows - p.row0 < 16 ? p.rows - p.row0 : 16;
    const int most = limit_of(p.row0 + rows - 1), chunks = most > 0 ? (most + 31) / 32 : 0;
    const int lo = (int)((int64_t)split * chunks / a.splits), hi = (int)((int64_t)(split + 1) * chunks / a.splits);
    {
        const int row = p.row0 + (lane & 15);
        const bool there = row < p.rows;
        f4 o[HD / 16];
        float ref, sum;
        walk_few<CT, HD>(there ? a.q + (p.first + row / a.rep) * a.q_stride + (kvh * a.rep + row % a.rep) * (HD * ESIZE<CT>) : nullptr, a.scale,
                         there ? limit_of(row) : 0, a.k + kv0 * a.k_stride + kvh * (HD * ESIZE<CT>), a.v + kv0 * a.v_stride + kvh * (HD * ESIZE<CT>), a.k_stride,
                         a.v_stride, len, lo, hi, (Lds)s.v[wave], o, ref, sum);
        leave_few<HD>(s, o, ref, sum);
    }
    __syncthreads();
    for (int r = wave; r < rows; r += FEW) {
        const float m = lane < FEW ? s.m[lane][r] : -INFINITY, l = lane < FEW ? s.l[lane][r] : 0.f;
        const float M = wave_max(m), w = __builtin_amdgcn_exp2f(m - (M == -INFINITY ? 0.f : M));
        const f4 x = sum_of_groups<HD>(join_few<HD>(s, r, w));
        const float L = wave_sum(l * w);
        const int row = p.row0 + r;
        const int64_t at = (p.first + row / a.rep) * a.Hq + kvh * a.rep + row % a.rep;
        if (a.splits == 1) {
            store_merged<HD>(a.out, dtype, at, x, M, L);
        } else {
            if (lane < HD / 4) reinterpret_cast<f4*>(a.out.part)[(at * a.splits + split) * (HD / 4) + lane] = x;
            if (lane == 0) a.out.part_ml[(at * a.splits + split) * 2] = M, a.out.part_ml[(at * a.splits + split) * 2 + 1] = L;
        }
    }
}

// ---- wq_decode_attention_shared: the requests' own 16-bit rows, and the merge ------------------------------------------------
struct FinishArgs {
    const char* q;
    const int32_t* req_off;
    int P, Hq, rep, parts, dtype;
    float scale;
    const char *k, *v;         // own 16-bit rows [row][Hkv][hd], or NULL
    const int32_t *off16, *len16;
    int64_t cap16;
    const float* own_out;      // or: one more part, normalised [B * Hq][hd], with its log-sum-exp
    const float* own_lse;
    Out out;
};

// Memory-bound where there are many requests: 64 of them with 200 rows each and 32 parts, 80 MB: 12.6 us.  (As further workgroups of k_shared
// they cost the same; the merge alone first and the walk in front of it, one after the other, 3 us more for a few short ones.)
// A workgroup per (request, KV head): eight wavefronts walk the request's own rows, while wavefront 8 + r merges query head r's parts;
// then each of those takes in what the eight have found.
template <typename QT, int HD>
__global__ __launch_bounds__(1024) void k_shared_finish(FinishArgs a)
{
    constexpr int W = FEW, LANES = HD / 4;
    __shared__ Few<HD> s;
    const int Hkv = a.Hq / a.rep, b = blockIdx.x / Hkv, kvh = blockIdx.x % Hkv, wave = this_wave(), lane = threadIdx.x & 63;
    const int64_t row0 = (int64_t)b * a.Hq + kvh * a.rep;
    int len = 0;
    if (a.k) {
        const int64_t room = a.cap16 - a.off16[b];
        len = a.len16[b];
        if (len > room) len = (int)room;
    }
    const int r = wave - W;
    const int64_t row = row0 + r;
    f4 x = {0.f, 0.f, 0.f, 0.f};
    float m2 = -INFINITY, l2 = 0.f;                            // lanes 0 .. 7: the wavefronts' sums; lane 8: an own part from outside; lane 9: the parts
    if (wave < W) {
        if (len > 0) {
            const int64_t stride = (int64_t)Hkv * HD * 2, first = a.off16[b] * stride + kvh * (HD * 2);
            f4 o[HD / 16];
            float ref, sum;
            const int n = lane & 15;
            walk_few<QT, HD>(n < a.rep ? a.q + (row0 + n) * (HD * ESIZE<QT>) : nullptr, a.scale, len, a.k + first, a.v + first, stride, stride, len, 0,
                             (len + 31) / 32, (Lds)s.v[wave], o, ref, sum);
            leave_few<HD>(s, o, ref, sum);
        }
    } else {
        const int parts = b >= a.req_off[0] && b < a.req_off[a.P] ? a.parts : 0;
        float m = -INFINITY, l = 0.f;                          // lane s: part s
        if (lane < parts) {
            m = a.out.part_ml[(row * a.parts + lane) * 2];
            l = a.out.part_ml[(row * a.parts + lane) * 2 + 1];
        }
        const float most = wave_max(m), w = __builtin_amdgcn_exp2f(m - (most == -INFINITY ? 0.f : most));
        x = sum_of_parts<HD>(a.out.part + row * a.parts * HD, parts, w);
        l = wave_sum(l * w);
        if (a.own_lse) {
            // (the decode kernels make zeros and -infinity of a query that is not finite: as if the cache were empty)
            bool bad = false;
#pragma unroll
            for (int c = lane; c < HD; c += 64) {
                const char* at = a.q + (row * HD + c) * ESIZE<QT>;
                if constexpr (std::is_same_v<QT, F32>) bad = bad || !isfinite(*reinterpret_cast<const float*>(at));
                else bad = bad || (*reinterpret_cast<const uint16_t*>(at) & EXPONENT16<QT>) == EXPONENT16<QT>;
            }
            bad = __any(bad);
            if (lane == W) m2 = a.own_lse[row] * WQ_LOG2E, l2 = bad ? NAN : m2 == -INFINITY ? 0.f : 1.f;
        }
        if (lane == W + 1) m2 = most, l2 = l;
    }
    __syncthreads();
    if (wave < W) return;
    if (len > 0 && lane < W) m2 = s.m[lane][r], l2 = s.l[lane][r];
    const float M = wave_max(m2), w2 = __builtin_amdgcn_exp2f(m2 - (M == -INFINITY ? 0.f : M));
    x *= __shfl(w2, W + 1, 64);
    if (len > 0) x += join_few<HD>(s, r, w2);
    x = sum_of_groups<HD>(x);
    if (a.own_out) x += reinterpret_cast<const f4*>(a.own_out)[row * LANES + lane % LANES] * __shfl(w2, W, 64);
    store_merged<HD>(a.out, a.dtype, row, x, M, wave_sum(l2 * w2));
}

// Query rows of a workgroup of the prompt's kernels: 256, or 128 where there are no more (SPLIT).  us per call, 256 -> 128: 9 rows of 7 heads, 64
// sequences of 6400 keys, heads of 64: 206 -> 145; one of 12544, heads of 128: 22.6 -> 19.4.  The shared kernels always take 256: both groups
// expand tiles then, rows or not (112 rows a KV head, 19719 tokens, 128 -> 256: 34.4 -> 32.5).
int rows_of(int64_t q_rows, int rep, int dtype) { return dtype != WQ_F32 && q_rows * rep > 128 ? 256 : 128; }
// Prompt attention over so few that k_prefill_few takes them (on the average: any number is right): two tiles of 16, though each reads the
// keys.  us per call, k_prefill -> k_prefill_few: 4 rows of 7 heads a group, 64 sequences of 6400 keys, heads of 64: 142 -> 79 (5 rows would be three
// tiles: 143), of 128: 412 -> 315; one sequence of 500 keys: 8.8 -> 7.6 and 9.7 -> 11.9.  One kernel for the whole call: 200 rows and 64 single tokens over 6400
// keys each, 28/4 heads of 128, take 331 us, apart 60 + 212.
bool few_rows(int64_t total_q, int B, int rep, int dtype) { return dtype != WQ_F32 && total_q * rep <= (int64_t)B * 32; }

template <typename CT>
auto prefill_kernel(int hd, bool split) -> void (*)(PrefillArgs)
{
    if constexpr (!std::is_same_v<CT, F32>)
        if (split) return hd == 128 ? k_prefill<CT, 128, true> : k_prefill<CT, 64, true>;
    return hd == 128 ? k_prefill<CT, 128, false> : k_prefill<CT, 64, false>;
}
auto shared_kernel(int dtype, int hd, int groups) -> void (*)(SharedArgs)
{
    if (dtype == WQ_F32) return hd == 128 ? k_shared<F32, 128, 0> : k_shared<F32, 64, 0>;
    if (dtype == WQ_BF16) return hd == 128 ? k_shared<Bf16, 128, 0> : k_shared<Bf16, 64, 0>;
    if (hd == 64) return groups == 1 ? k_shared<F16, 64, 1> : k_shared<F16, 64, 2>;
    return groups == 1 ? k_shared<F16, 128, 1> : groups == 2 ? k_shared<F16, 128, 2> : k_shared<F16, 128, 4>;
}

template <typename QT>
auto finish_kernel(int hd) -> void (*)(FinishArgs) { return hd == 128 ? k_shared_finish<QT, 128> : k_shared_finish<QT, 64>; }

// Own caches with room for packed tokens have a decode launch of their own, and longer ones where there are too few requests to fill the
// card: k_shared_finish walks a request's rows with one workgroup per KV head, 256 keys in about 1.1 us.  us per call over 39 000 shared tokens, own
// rows there -> apart, 4 KV heads: 1 request, 512 rows 41 -> 44, 1024: 46 -> 44, 2048: 54 -> 44; 16 requests, 1024: 51 -> 52, 2048: 60 -> 57;
// 64 requests, 512: 78 -> 88, 4000: 168 -> 183.
constexpr int64_t OWN_INSIDE = 1024;
// Below this many keys a tail's merge (15 to 20 us with its launch) costs about what its parts save (half of 32 tiles of 1.8 us, or more)
constexpr int64_t TAIL_KEYS = 2048;

}  // namespace

WqPrefillPlan wq_prefill_plan(int64_t total_q, int B, int Hq, int Hkv, int hd, int dtype, int64_t max_kv_rows, bool prefix, int num_splits, size_t room)
{
    const int rep = Hq / Hkv;
    const int64_t used = total_q < B ? total_q : B;           // sequences that have rows
    WqPrefillPlan s = {};
    s.splits = num_splits;
    s.few = few_rows(total_q, B, rep, dtype);
    const int rows = s.few ? 16 : rows_of((total_q + B - 1) / B, rep, dtype);
    s.rows = rows;
    const int64_t units = tiles_of(total_q, rep, B, rows) * Hkv;
    s.groups = units;
    if (num_splits <= 0) {
        // (few rows: no parts of up to 512 keys, two rounds of every wavefront: a merge costs 3 us, a round one)
        s.splits = s.few ? max_kv_rows <= 512 ? 1 : auto_splits_of((tiles_of(total_q, rep, 0, rows) + used) * Hkv, max_kv_rows, 512, 32 * FEW)
                         : auto_splits_of((tiles_of(total_q, rep, 0, rows) + used) * Hkv, max_kv_rows, 256, dtype == WQ_F32 ? 32 : 64);
        // Tiles of equal length (a prefix) for more than the card's 256 compute units: the last round's, where they are no more than half of
        // them, are cut along the keys to fill it (1404 tiles, 124 of them cut in two: 1950 us, 2050 uncut).  Where there is no prefix a sequence's tiles are
        // launched longest first, and the last ones are short: 12800 causal rows reach 1.13 PFLOP/s uncut, those above 1.18.
        const int64_t rest = units % 256;
        if (rows == 256 && s.splits == 1 && prefix && units > 256 && rest > 0 && rest <= 128 && max_kv_rows >= TAIL_KEYS) {
            s.tail = (int)rest;
            s.tail_splits = (int)(256 / rest < max_kv_rows / 512 ? 256 / rest : max_kv_rows / 512);
            if (s.tail_splits > WQ_MAX_ATTEND_SPLITS) s.tail_splits = WQ_MAX_ATTEND_SPLITS;
        }
    }
    auto bytes = [&]() -> size_t {
        return s.tail > 0 ? partials_bytes((int64_t)s.tail * 256, hd, s.tail_splits) : s.splits > 1 ? partials_bytes(total_q * Hq, hd, s.splits) : 0;
    };
    // A smaller call can want more parts, and more room for them, than the one that the workspace was sized for: it makes do with fewer
    if (num_splits <= 0) {
        while (s.tail > 0 && bytes() > room)
            if (--s.tail_splits < 2) s.tail = s.tail_splits = 0;
        while (s.splits > 1 && bytes() > room) s.splits--;
    }
    s.bytes = bytes();
    return s;
}

WqSharedPlan wq_shared_plan(int B, int P, int Hq, int Hkv, int hd, int q_dtype, int64_t max_prefix_tokens, int64_t max_own_tokens, bool own, bool own_packed,
                            int num_splits, size_t room)
{
    const int rep = Hq / Hkv;
    WqSharedPlan s;
    s.rows = q_dtype == WQ_F32 ? 128 : 256;
    s.splits = num_splits > 0 ? num_splits : auto_splits_of(tiles_of(B, rep, P, s.rows) * Hkv, max_prefix_tokens, 256, q_dtype == WQ_F32 ? 32 : 64);
    s.own_decode = own && (own_packed || (max_own_tokens > OWN_INSIDE && (int64_t)B * Hkv < 256));
    const int64_t rows = (int64_t)B * Hq;
    const int decode_splits = wq_auto_splits(B, Hkv, max_own_tokens);
    int fewer = decode_splits;
    auto size = [&] {
        s.decode_bytes = s.own_decode ? wq_decode_ws_bytes(B, Hq, hd, fewer) : 0;
        s.bytes = s.decode_bytes + partials_bytes(rows, hd, s.splits);
        if (s.own_decode) s.bytes += wq_align256(rows * hd * sizeof(float)) + wq_align256(rows * sizeof(float));
        return s.bytes;
    };
    // (as for prompts; what one part and one split take grows with the requests)
    while (num_splits <= 0 && s.splits > 1 && size() > room) s.splits--;
    while (s.own_decode && fewer > 1 && size() > room) fewer--;
    size();
    s.decode_splits = fewer < decode_splits ? fewer : 0;
    s.groups = tiles_of(B, rep, P, s.rows) * Hkv * s.splits;
    return s;
}

int wq_launch_prefill(wq_ctx* ctx, const WqPrefill& f)
{
    PrefillArgs a;
    const int size = f.dtype == WQ_F32 ? 4 : 2;
    a.q = static_cast<const char*>(f.q), a.k = static_cast<const char*>(f.k), a.v = static_cast<const char*>(f.v);
    a.q_stride = f.q_stride * size, a.k_stride = f.k_stride * size, a.v_stride = f.v_stride * size;
    a.q_off = f.q_off, a.kv_off = f.kv_off, a.prefix_len = f.prefix_len;
    a.total_q = f.total_q, a.total_kv = f.total_kv;
    a.B = f.B, a.Hq = f.Hq, a.rep = f.Hq / f.Hkv, a.splits = f.plan.splits;
    a.scale = f.sm_scale * WQ_LOG2E;
    a.out.out = f.out, a.out.lse = f.lse;
    a.out.part = reinterpret_cast<float*>(ctx->ws + WQ_WS_HEADER);
    a.units = (int)f.plan.groups, a.tail = f.plan.tail, a.tail_splits = f.plan.tail_splits;
    a.out.part_ml = a.out.part + (a.tail > 0 ? (int64_t)a.tail * 256 * a.tail_splits : f.total_q * f.Hq * a.splits) * f.hd;
    const dim3 grid((unsigned)(a.units - a.tail + a.tail * a.tail_splits), (unsigned)a.splits);
    if (f.plan.few) {
        void (*const kernel)(PrefillArgs, int) = f.dtype == WQ_BF16 ? (f.hd == 128 ? k_prefill_few<Bf16, 128> : k_prefill_few<Bf16, 64>)
                                                                    : (f.hd == 128 ? k_prefill_few<F16, 128> : k_prefill_few<F16, 64>);
        hipLaunchKernelGGL(kernel, grid, dim3(64 * FEW), 0, ctx->stream, a, f.dtype);
    } else {
        void (*const kernel)(PrefillArgs) = f.dtype == WQ_F32 ? prefill_kernel<F32>(f.hd, false) : f.dtype == WQ_BF16 ? prefill_kernel<Bf16>(f.hd, f.plan.rows == 128)
                                                                                                              : prefill_kernel<F16>(f.hd, f.plan.rows == 128);
        hipLaunchKernelGGL(kernel, grid, dim3(f.dtype == WQ_F32 ? 256 : 512), 0, ctx->stream, a);
    }
    if (a.tail > 0) {
        hipLaunchKernelGGL(f.hd == 128 ? k_merge_tail<128> : k_merge_tail<64>, dim3((unsigned)a.tail * 64), dim3(256), 0, ctx->stream, a, f.dtype);
    } else if (a.splits > 1) {
        const MergeArgs m = {f.total_q * f.Hq, f.Hq, a.splits, f.dtype, f.q_off, f.B, a.out};
        hipLaunchKernelGGL(f.hd == 128 ? k_merge<128> : k_merge<64>, dim3((unsigned)((m.rows + 3) / 4)), dim3(256), 0, ctx->stream, m);
    }
    WQ_HIP_CHECK(ctx, hipGetLastError());
    return WQ_OK;
}

// The shared caches; then the requests' own rows and the merge.  Own caches that this is not for go first, through
// wq_decode_attention's kernels.
int wq_launch_shared(wq_ctx* ctx, const WqShared& f)
{
    const wq_packed_kv* kv = f.prefix;
    const int64_t rows = (int64_t)f.B * f.Hq;
    SharedArgs a;
    a.q = static_cast<const char*>(f.q);
    a.req_off = f.req_off;
    a.B = f.B, a.P = kv->B, a.Hq = f.Hq, a.rep = f.Hq / kv->Hkv;
    a.units = (int)(f.plan.groups / f.plan.splits);
    a.splits = f.plan.splits;
    a.scale = f.sm_scale * WQ_LOG2E;
    a.kv = *kv;
    a.out.out = f.out, a.out.lse = f.lse;
    const int parts = a.splits;
    char* at = ctx->ws + WQ_WS_HEADER + f.plan.decode_bytes;
    a.out.part = reinterpret_cast<float*>(at);
    a.out.part_ml = a.out.part + rows * parts * kv->hd;
    at += partials_bytes(rows, kv->hd, parts);
    float* own_out = nullptr;
    float* own_lse = nullptr;
    if (f.plan.own_decode) {
        own_out = reinterpret_cast<float*>(at);
        own_lse = reinterpret_cast<float*>(at + wq_align256(rows * kv->hd * sizeof(float)));
        const int rc = wq_launch_decode(ctx, f.q, f.q_dtype, f.B, f.Hq, f.own, f.sm_scale, f.decode_splits, f.decode_algo, own_out, own_lse);
        if (rc != WQ_OK) return rc;
    }
    const dim3 grid((unsigned)f.plan.groups);
    hipLaunchKernelGGL(shared_kernel(f.q_dtype, kv->hd, kv->hd / kv->group), grid,
                       dim3(f.q_dtype == WQ_F32 ? 256 : 512), 0, ctx->stream, a);
    FinishArgs m;
    m.q = a.q, m.req_off = f.req_off;
    m.P = a.P, m.Hq = f.Hq, m.rep = a.rep, m.parts = parts, m.dtype = f.q_dtype;
    m.scale = a.scale;
    const bool inside = f.own && !f.plan.own_decode;
    m.k = inside ? static_cast<const char*>(f.own->k16) : nullptr, m.v = inside ? static_cast<const char*>(f.own->v16) : nullptr;
    m.off16 = inside ? f.own->off16 : nullptr, m.len16 = inside ? f.own->len16 : nullptr;
    m.cap16 = inside ? f.own->cap16 : 0;
    m.own_out = own_out, m.own_lse = own_lse;
    m.out = a.out;
    hipLaunchKernelGGL(f.q_dtype == WQ_F32 ? finish_kernel<F32>(kv->hd) : f.q_dtype == WQ_BF16 ? finish_kernel<Bf16>(kv->hd) : finish_kernel<F16>(kv->hd),
                       dim3((unsigned)(f.B * kv->Hkv)), dim3(64 * (8 + a.rep)), 0, ctx->stream, m);
    WQ_HIP_CHECK(ctx, hipGetLastError());
    return WQ_OK;
}
