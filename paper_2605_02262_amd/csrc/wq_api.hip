// C-ABI entry points of libwq: context handling, host-side argument validation, dispatch.
// Every check that needs only host data happens here, before anything is enqueued.
#include <math.h>
#include <mutex>
#include <new>
#include <string.h>

#include "wq_internal.h"

namespace {

bool shape_ok(int Hkv, int hd, int group)
{
    return Hkv > 0 && (hd == 64 || hd == 128) && (group == 32 || group == 64 || group == 128) && hd % group == 0;
}

// Calls f with the address of every buffer (and table that is a layer's own) that a copy writes, or an append; with those of the classes' tables
template <typename F>
void each_copied(const wq_packed_kv& kv, const F& f)
{
    for (int c = 0; c < 3; c++)
        if (kv.cap[c] > 0) f(kv.codes[c]), f(kv.meta[c]);
    if (kv.cap16 > 0) f(kv.k16), f(kv.v16);
    f(kv.len16), f(kv.v_scale_max);
}
template <typename F>
void each_appended(const wq_packed_kv& kv, const F& f)
{
    if (kv.cap16 > 0) f(kv.k16), f(kv.v16);
    f(kv.len16);
}
template <typename F>
void each_table(const wq_packed_kv& kv, const F& f)
{
    for (int c = 0; c < 3; c++) f(kv.cls_off[c]), f(kv.cls_len[c]);
}
// Does something that is written of a layer of dst begin where something of another of its layers, or of src, does?  (src NULL: an append, whose caches' tables stay.
// Layers whose sequences have the same lengths may share the classes' tables: they are written alike.)  An address leaves a bit at a hash of it, and all of them
// are looked through only where the bit is there already: 600 addresses of 24 layers' copies 1.6 us, 2000 of 80 layers' 5.5.
template <typename Each>
bool shares_memory(int n_layers, const wq_packed_kv* src, const wq_packed_kv* dst, const Each& each)
{
    uint64_t bits[1024] = {};
    bool same = false;
    auto place = [](const void* p) { return (uint32_t)((reinterpret_cast<uintptr_t>(p) >> 2) * UINT64_C(0x9E3779B97F4A7C15) >> 48); };
    auto there = [&](const void* p) { return bits[place(p) >> 6] >> (place(p) & 63) & 1; };
    auto add = [&](const void* p) { bits[place(p) >> 6] |= UINT64_C(1) << (place(p) & 63); };
    auto in_sources = [&](const void* p) {
        auto compare = [&](const void* x) { same = same || x == p; };
        for (int m = 0; m < n_layers; m++) each(src[m], compare), each_table(src[m], compare), compare(src[m].off16);
    };
    if (src) {
        for (int l = 0; l < n_layers; l++) each(src[l], add), each_table(src[l], add), add(src[l].off16);
        for (int l = 0; l < n_layers && !same; l++)
            each_table(dst[l], [&](const void* p) {
                if (there(p)) in_sources(p);
            });
        for (int l = 0; l < n_layers; l++) each_table(dst[l], add);
    }
    for (int l = 0; l < n_layers && !same; l++)
        each(dst[l], [&](const void* p) {
            if (there(p)) {
                if (src) in_sources(p);
                auto compare = [&](const void* x) { same = same || x == p; };
                for (int m = 0; m < n_layers; m++) {
                    if (m == l) continue;
                    each(dst[m], compare);
                    if (src) each_table(dst[m], compare);
                }
            }
            add(p);
        });
    return same;
}

bool dtype_ok(int d) { return d == WQ_F32 || d == WQ_BF16 || d == WQ_F16; }

int check_packed(wq_ctx* ctx, const wq_packed_kv* kv, int B, bool need_tables)
{
    if (!kv) return wq_fail(ctx, WQ_ERR_ARG, "packed cache descriptor is NULL");
    if (kv->B != B) return wq_fail(ctx, WQ_ERR_ARG, "packed cache is for B=%d, call has B=%d", kv->B, B);
    if (!shape_ok(kv->Hkv, kv->hd, kv->group))
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "unsupported shape Hkv=%d hd=%d group=%d", kv->Hkv, kv->hd, kv->group);
    if (kv->dtype16 != WQ_BF16 && kv->dtype16 != WQ_F16)
        return wq_fail(ctx, WQ_ERR_ARG, "dtype16 must be WQ_BF16 or WQ_F16");
    for (int c = 0; c < 3; c++) {
        if (kv->cap[c] < 0 || kv->cap[c] % 32 != 0)
            return wq_fail(ctx, WQ_ERR_ARG, "cap[%d]=%lld is not a non-negative multiple of 32", c, (long long)kv->cap[c]);
        if (kv->cap[c] > (int64_t)1 << 26) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "cap[%d] above 2^26 tokens", c);
        if (kv->cap[c] > 0 && (!kv->codes[c] || !kv->meta[c]))
            return wq_fail(ctx, WQ_ERR_ARG, "class %d has capacity but NULL codes/meta", c);
        if (need_tables && (!kv->cls_off[c] || !kv->cls_len[c]))
            return wq_fail(ctx, WQ_ERR_ARG, "class %d offset/length tables are NULL", c);
    }
    if (kv->cap16 < 0 || kv->cap16 > (int64_t)1 << 26) return wq_fail(ctx, WQ_ERR_ARG, "bad cap16");
    if (kv->cap16 > 0 && (!kv->k16 || !kv->v16)) return wq_fail(ctx, WQ_ERR_ARG, "16-bit segment has capacity but NULL k16/v16");
    if (!kv->off16 || !kv->len16) return wq_fail(ctx, WQ_ERR_ARG, "off16/len16 tables are NULL");
    if (!kv->v_scale_max) return wq_fail(ctx, WQ_ERR_ARG, "v_scale_max table is NULL");
    return WQ_OK;
}

}  // namespace

extern "C" {

int wq_create(wq_ctx** out, void* hip_stream, void* workspace, size_t workspace_bytes)
{
    if (!out) return WQ_ERR_ARG;
    *out = nullptr;
    wq_ctx* ctx = new (std::nothrow) wq_ctx();
    if (!ctx) return WQ_ERR_ARG;
    ctx->stream = static_cast<hipStream_t>(hip_stream);
    ctx->ws = static_cast<char*>(workspace);
    ctx->ws_bytes = workspace_bytes;
    ctx->owns_ws = false;
    ctx->timing = false;
    for (int i = 0; i < 2 * WQ_TIMING_RING; i++) ctx->ev[i] = nullptr;
    ctx->ev_calls = 0;
    ctx->err[0] = 0;
    if (!workspace && workspace_bytes > 0) {
        void* p = nullptr;
        if (hipMalloc(&p, workspace_bytes) != hipSuccess) {
            delete ctx;
            return WQ_ERR_HIP;
        }
        ctx->ws = static_cast<char*>(p);
        ctx->owns_ws = true;
    }
    if (ctx->ws && ctx->ws_bytes >= WQ_WS_HEADER && ctx->owns_ws) {
        if (hipMemset(ctx->ws, 0, WQ_WS_HEADER) != hipSuccess) {
            (void)hipFree(ctx->ws);
            delete ctx;
            return WQ_ERR_HIP;
        }
    }
    *out = ctx;
    return WQ_OK;
}

int wq_destroy(wq_ctx* ctx)
{
    if (!ctx) return WQ_OK;
    if (ctx->owns_ws && ctx->ws) (void)hipFree(ctx->ws);
    for (int i = 0; i < 2 * WQ_TIMING_RING; i++)
        if (ctx->ev[i]) (void)hipEventDestroy(ctx->ev[i]);
    delete ctx;
    return WQ_OK;
}

int wq_set_stream(wq_ctx* ctx, void* hip_stream)
{
    if (!ctx) return WQ_ERR_ARG;
    ctx->stream = static_cast<hipStream_t>(hip_stream);
    return WQ_OK;
}

const char* wq_last_error(const wq_ctx* ctx) { return ctx ? ctx->err : "null context"; }

int wq_device_status(wq_ctx* ctx, uint32_t* bits)
{
    if (!ctx || !bits) return WQ_ERR_ARG;
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER) return wq_fail(ctx, WQ_ERR_WORKSPACE, "no workspace");
    WQ_HIP_CHECK(ctx, hipMemcpyAsync(bits, ctx->ws, sizeof(uint32_t), hipMemcpyDeviceToHost, ctx->stream));
    WQ_HIP_CHECK(ctx, hipStreamSynchronize(ctx->stream));
    WQ_HIP_CHECK(ctx, hipMemsetAsync(ctx->ws, 0, sizeof(uint32_t), ctx->stream));
    return WQ_OK;
}

size_t wq_workspace_bytes(int B, int Hq, int hd, int max_splits, int64_t total_vis, int64_t total_txt, int D)
{
    size_t a = wq_decode_ws_bytes(B, Hq, hd, max_splits);
    size_t b = wq_scores_ws_bytes(B, total_vis, total_txt, D);
    size_t c = wq_align256(sizeof(int32_t) * (size_t)(B > 0 ? B + 1 : 1));   // prefix of 16-bit rows (a3)
    size_t m = a > b ? a : b;
    if (c > m) m = c;
    return WQ_WS_HEADER + m;
}

size_t wq_v_scale_floats(int B, int Hkv, const int64_t cap[3])
{
    if (B < 0 || Hkv <= 0 || !cap) return 0;
    size_t blocks = 0;
    for (int c = 0; c < 3; c++) blocks += (size_t)((cap[c] > 0 ? cap[c] : 0) / 32);
    return (size_t)B + blocks * (size_t)Hkv;
}

size_t wq_packed_bytes(int bits, int64_t cap_tokens, int Hkv, int hd, int group, size_t* meta_bytes)
{
    if (meta_bytes) *meta_bytes = 0;
    if (!(bits == 2 || bits == 4 || bits == 8) || cap_tokens < 0 || !shape_ok(Hkv, hd, group)) return 0;
    int64_t cap = (cap_tokens + 31) / 32 * 32;
    if (meta_bytes) *meta_bytes = (size_t)2 * Hkv * cap * (hd / group) * 4;
    return (size_t)2 * Hkv * cap * hd * bits / 8;
}

// total_tokens well below B * max_seq_tokens: the sequences differ in length, and the launch gives a sequence splits in
// proportion to its length (the longest gets them all): more splits, so that about as many workgroups as for equal
// lengths have work
int wq_auto_splits_ragged(int B, int Hkv, int64_t max_seq_tokens, int64_t total_tokens)
{
    const int s0 = wq_auto_splits(B, Hkv, max_seq_tokens);
    if (B <= 0 || max_seq_tokens <= 0 || total_tokens <= 0) return s0;
    const double fill = (double)total_tokens / ((double)B * (double)max_seq_tokens);
    if (fill >= 0.75) return s0;
    // twice the count that would give as many busy workgroups as equal lengths do: with lengths this uneven the launch is as
    // long as its longest sequences take, and more, smaller workgroups on them end earlier (measured on 32 sequences of
    // 8 to 128 frames: 84.7 us with 2 splits for all, 77.4 with 4 by length, 72.5 with 8 by length, 82.6 with 12)
    int64_t s = (int64_t)(2.0 * (double)s0 / fill + 0.5);
    const int64_t most = (max_seq_tokens + 1023) / 1024;
    if (s > most) s = most;
    if (s > 256) s = 256;
    return s > s0 ? (int)s : s0;
}

int wq_auto_splits(int B, int Hkv, int64_t max_seq_tokens)
{
    if (B <= 0 || Hkv <= 0) return 1;
    // one workgroup of eight wavefronts per compute unit (256 CUs) is what the decode kernel's registers allow;
    // more splits only add per-workgroup set-up.  Keep at least 1024 tokens per workgroup.
    int64_t want = (256 + (int64_t)B * Hkv - 1) / ((int64_t)B * Hkv);
    int64_t most = max_seq_tokens > 0 ? (max_seq_tokens + 1023) / 1024 : 1;
    if (want > most) want = most;
    if (want < 1) want = 1;
    if (want > 256) want = 256;
    return (int)want;
}

int wq_window_scores(wq_ctx* ctx, const void* vis_emb, const void* txt_emb, int dtype, int B, int D,
                     const int32_t* vis_off, const int32_t* txt_off, const int32_t* win_size, const int32_t* win_off,
                     int64_t total_vis, int64_t total_txt, int64_t total_win, int algo, float* scores)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0 || D <= 0 || total_vis < 0 || total_txt < 0 || total_win < 0)
        return wq_fail(ctx, WQ_ERR_ARG, "negative size (B=%d D=%d)", B, D);
    if (!dtype_ok(dtype)) return wq_fail(ctx, WQ_ERR_ARG, "unknown dtype %d", dtype);
    if (algo != WQ_SCORE_AUTO && algo != WQ_SCORE_PAIRWISE_MFMA && algo != WQ_SCORE_POOLED)
        return wq_fail(ctx, WQ_ERR_ARG, "unknown scoring algorithm %d", algo);
    if (total_vis > INT32_MAX || total_txt > INT32_MAX) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many rows");
    if (B == 0 || total_win == 0) return WQ_OK;
    if (!vis_off || !txt_off || !win_size || !win_off || !scores) return wq_fail(ctx, WQ_ERR_ARG, "NULL table or output");
    if ((total_vis > 0 && !vis_emb) || (total_txt > 0 && !txt_emb)) return wq_fail(ctx, WQ_ERR_ARG, "NULL embeddings");
    if (algo == WQ_SCORE_PAIRWISE_MFMA && dtype == WQ_F32)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "the matrix-core scoring path takes bf16 or fp16 embeddings");
    if (algo == WQ_SCORE_PAIRWISE_MFMA && D % 128 != 0)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "the matrix-core scoring path needs D %% 128 == 0");
    if (ctx->ws_bytes < WQ_WS_HEADER + wq_scores_ws_bytes(B, total_vis, total_txt, D))
        return wq_fail(ctx, WQ_ERR_WORKSPACE, "workspace too small for scoring");
    return wq_launch_scores(ctx, vis_emb, txt_emb, dtype, B, D, vis_off, txt_off, win_size, win_off, total_vis,
                            total_txt, total_win, algo, scores);
}

int wq_assign_bits(wq_ctx* ctx, const float* scores, int B, const int32_t* win_off, int max_windows, int mode,
                   const int32_t* quota, const float* thresholds, int top_bits, int pin_first, uint8_t* bits,
                   int32_t* perm, int32_t* seg_windows)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0 || max_windows < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    if (mode != WQ_MODE_QUOTA && mode != WQ_MODE_THRESHOLD) return wq_fail(ctx, WQ_ERR_ARG, "unknown mode %d", mode);
    if (top_bits != 8 && top_bits != 16) return wq_fail(ctx, WQ_ERR_ARG, "top_bits must be 8 or 16, got %d", top_bits);
    if (max_windows > WQ_MAX_WINDOWS)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than %d windows per sequence", WQ_MAX_WINDOWS);
    if (B == 0) return WQ_OK;
    if (!win_off || !seg_windows) return wq_fail(ctx, WQ_ERR_ARG, "NULL table");
    if (max_windows > 0 && (!scores || !bits || !perm)) return wq_fail(ctx, WQ_ERR_ARG, "NULL scores or output");
    if (mode == WQ_MODE_QUOTA && !quota) return wq_fail(ctx, WQ_ERR_ARG, "quota mode without quota table");
    if (mode == WQ_MODE_THRESHOLD && !thresholds) return wq_fail(ctx, WQ_ERR_ARG, "threshold mode without thresholds");
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER) return wq_fail(ctx, WQ_ERR_WORKSPACE, "no workspace");
    return wq_launch_assign(ctx, scores, B, win_off, max_windows, mode, quota, thresholds, top_bits, pin_first != 0,
                            bits, perm, seg_windows);
}

int wq_layer_thresholds(const double* s, int n_layers, double alpha, float* t_low, float* t_high)
{
    if (n_layers < 0 || !isfinite(alpha)) return WQ_ERR_ARG;
    if (n_layers > 0 && (!s || !t_low || !t_high)) return WQ_ERR_ARG;
    for (int i = 0; i < n_layers; i++)
        if (!(s[i] >= 0.0 && s[i] <= 1.0)) return WQ_ERR_ARG;
    for (int i = 0; i < n_layers; i++) {
        // expm1 keeps the quotient accurate where alpha * s is small; alpha = 0 is the limit s
        const double lo = alpha == 0.0 ? s[i] : expm1(alpha * s[i]) / expm1(alpha);
        const double hi = alpha == 0.0 ? s[i] : expm1(-alpha * s[i]) / expm1(-alpha);
        t_low[i] = (float)lo;
        t_high[i] = (float)hi;
    }
    return WQ_OK;
}

int wq_vote_bits(wq_ctx* ctx, const uint8_t* bits_in, int B, const int32_t* win_off, int max_windows, uint8_t* bits_out,
                 int32_t* perm, int32_t* seg_windows)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0 || max_windows < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    if (max_windows > WQ_MAX_WINDOWS)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than %d windows per sequence", WQ_MAX_WINDOWS);
    if (B == 0) return WQ_OK;
    if (!win_off || !seg_windows) return wq_fail(ctx, WQ_ERR_ARG, "NULL table");
    if (max_windows > 0 && (!bits_in || !bits_out || !perm)) return wq_fail(ctx, WQ_ERR_ARG, "NULL widths or output");
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER) return wq_fail(ctx, WQ_ERR_WORKSPACE, "no workspace");
    return wq_launch_vote(ctx, bits_in, B, win_off, max_windows, bits_out, perm, seg_windows);
}

int wq_validate_assignment(wq_ctx* ctx, int B, const int32_t* win_off, int max_windows, const int32_t* perm, const int32_t* seg_windows)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0 || max_windows < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    if (max_windows > WQ_MAX_WINDOWS)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than %d windows per sequence", WQ_MAX_WINDOWS);
    if (B == 0) return WQ_OK;
    if (!win_off || !seg_windows || (max_windows > 0 && !perm)) return wq_fail(ctx, WQ_ERR_ARG, "NULL table");
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER) return wq_fail(ctx, WQ_ERR_WORKSPACE, "no workspace");
    return wq_launch_validate(ctx, B, win_off, max_windows, perm, seg_windows);
}

int wq_reorder_quantize(wq_ctx* ctx, const void* K, const void* V, int dtype, int B, const int32_t* kv_off,
                        const int32_t* win_size, const int32_t* win_off, const int32_t* perm,
                        const int32_t* seg_windows, int64_t total_rows, const wq_packed_kv* out)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0 || total_rows < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    if (!dtype_ok(dtype)) return wq_fail(ctx, WQ_ERR_ARG, "unknown dtype %d", dtype);
    int rc = check_packed(ctx, out, B, true);
    if (rc != WQ_OK) return rc;
    if ((dtype == WQ_BF16) != (out->dtype16 == WQ_BF16))
        return wq_fail(ctx, WQ_ERR_ARG, "dtype16 must be bf16 for bf16 input and fp16 for fp16/fp32 input");
    if (total_rows > INT32_MAX) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many rows");
    if (B == 0) return WQ_OK;
    if (!kv_off || !win_size || !win_off || !seg_windows) return wq_fail(ctx, WQ_ERR_ARG, "NULL table");
    if (total_rows > 0 && (!K || !V || !perm)) return wq_fail(ctx, WQ_ERR_ARG, "NULL K, V or perm");
    if ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) % 16 != 0)
        return wq_fail(ctx, WQ_ERR_ARG, "K and V must be 16-byte aligned");
    if (ctx->ws_bytes < WQ_WS_HEADER + wq_align256(sizeof(int32_t) * (size_t)(B + 1)))
        return wq_fail(ctx, WQ_ERR_WORKSPACE, "workspace too small for reorder_quantize");
    return wq_launch_quantize(ctx, K, V, dtype, B, kv_off, win_size, win_off, perm, seg_windows, total_rows, out);
}

int wq_append_kv(wq_ctx* ctx, const void* k_new, const void* v_new, int dtype, int B, const wq_packed_kv* kv)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    if (!dtype_ok(dtype)) return wq_fail(ctx, WQ_ERR_ARG, "unknown dtype %d", dtype);
    int rc = check_packed(ctx, kv, B, false);
    if (rc != WQ_OK) return rc;
    if ((dtype == WQ_BF16) != (kv->dtype16 == WQ_BF16))
        return wq_fail(ctx, WQ_ERR_ARG, "dtype16 must be bf16 for bf16 input and fp16 for fp16/fp32 input");
    if (B == 0) return WQ_OK;
    if (!k_new || !v_new) return wq_fail(ctx, WQ_ERR_ARG, "NULL k_new or v_new");
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER) return wq_fail(ctx, WQ_ERR_WORKSPACE, "no workspace");
    return wq_launch_append(ctx, k_new, v_new, dtype, B, kv);
}

// What both decode entry points check before anything is enqueued; resolves num_splits == 0.
static int check_decode(wq_ctx* ctx, const void* q, int q_dtype, int B, int Hq, const wq_packed_kv* kv, float sm_scale,
                        int* num_splits, int64_t max_seq_tokens, int algo, const float* out, int64_t* longest)
{
    *longest = 0;
    if (B < 0 || Hq <= 0) return wq_fail(ctx, WQ_ERR_ARG, "bad B or Hq");
    if (B > 65535) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than 65535 sequences in one call");      // a grid dimension
    if (!dtype_ok(q_dtype)) return wq_fail(ctx, WQ_ERR_ARG, "unknown q dtype %d", q_dtype);
    int rc = check_packed(ctx, kv, B, true);
    if (rc != WQ_OK) return rc;
    if (Hq % kv->Hkv != 0 || Hq / kv->Hkv > WQ_MAX_REP)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "Hq=%d must be a multiple of Hkv=%d, at most %d query heads per KV head",
                       Hq, kv->Hkv, WQ_MAX_REP);
    const int balgo = algo & ~WQ_DECODE_FLAGS;
    const bool by_length = (algo & WQ_DECODE_BY_LENGTH) != 0;
    if (by_length && max_seq_tokens <= 0) return wq_fail(ctx, WQ_ERR_ARG, "WQ_DECODE_BY_LENGTH needs max_seq_tokens");
    if (balgo != WQ_DECODE_AUTO && balgo != WQ_DECODE_GENERIC && balgo != WQ_DECODE_MFMA)
        return wq_fail(ctx, WQ_ERR_ARG, "unknown decode algorithm %d", algo);
    if (balgo == WQ_DECODE_MFMA && kv->hd / kv->group != 2)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "the matrix-core decode kernel needs hd/group == 2");
    if (*num_splits < 0 || *num_splits > 1024) return wq_fail(ctx, WQ_ERR_ARG, "num_splits out of range");
    if (!(sm_scale > 0.0f) || sm_scale > 3.0e38f) return wq_fail(ctx, WQ_ERR_ARG, "sm_scale must be positive and finite");
    if (B == 0) return WQ_OK;
    if (!q || !out) return wq_fail(ctx, WQ_ERR_ARG, "NULL q or out");
    if (by_length) *longest = max_seq_tokens;
    const bool automatic = *num_splits == 0;
    if (automatic) {
        *num_splits = wq_auto_splits(B, kv->Hkv, max_seq_tokens);
        if (by_length) {    // more splits (the caches' capacities stand in for the tokens), if the workspace has room for them
            int more = wq_auto_splits_ragged(B, kv->Hkv, max_seq_tokens, kv->cap[0] + kv->cap[1] + kv->cap[2] + kv->cap16);
            if (more > WQ_MAX_FUSED_SPLITS) more = WQ_MAX_FUSED_SPLITS;    // (splits by length need the merge inside the kernel)
            if (more > *num_splits && ctx->ws_bytes >= WQ_WS_HEADER + wq_decode_ws_bytes(B, Hq, kv->hd, more)) *num_splits = more;
        }
    }
    if (ctx->ws_bytes < WQ_WS_HEADER + wq_decode_ws_bytes(B, Hq, kv->hd, *num_splits))
        return wq_fail(ctx, WQ_ERR_WORKSPACE, "workspace too small for %d splits", *num_splits);
    // where the kernel merges the splits itself: what makes the launch shortest, as far as a workspace for this count has room
    const int picked = automatic ? wq_decode_pick_splits(q, q_dtype, B, kv, max_seq_tokens, *num_splits, algo) : 0;
    if (picked > 0) {
        *num_splits = picked;
        *longest = by_length && B > 1 ? -max_seq_tokens : 0;      // (the kernel finds the counts, if it merges the splits)
    }
    return WQ_OK;
}

int wq_decode_append_attention(wq_ctx* ctx, const void* q, int q_dtype, int B, int Hq, const wq_packed_kv* kv,
                               const void* k_new, const void* v_new, int new_dtype, float sm_scale, int num_splits,
                               int64_t max_seq_tokens, int algo, float* out, float* lse)
{
    if (!ctx) return WQ_ERR_ARG;
    if (!dtype_ok(new_dtype)) return wq_fail(ctx, WQ_ERR_ARG, "unknown dtype %d", new_dtype);
    if (kv && (new_dtype == WQ_BF16) != (kv->dtype16 == WQ_BF16))
        return wq_fail(ctx, WQ_ERR_ARG, "dtype16 must be bf16 for bf16 input and fp16 for fp16/fp32 input");
    if (B > 0 && (!k_new || !v_new)) return wq_fail(ctx, WQ_ERR_ARG, "NULL k_new or v_new");
    if (algo & WQ_DECODE_PARTIALS_ONLY) return wq_fail(ctx, WQ_ERR_ARG, "partials-only launches do not append");
    int64_t longest = 0;
    int rc = check_decode(ctx, q, q_dtype, B, Hq, kv, sm_scale, &num_splits, max_seq_tokens, algo, out, &longest);
    if (rc != WQ_OK || B == 0) return rc;
    if (wq_decode_can_append(q, q_dtype, B, Hq, kv, num_splits, algo, k_new, v_new, new_dtype))
        return wq_launch_decode(ctx, q, q_dtype, B, Hq, kv, sm_scale, num_splits, algo, out, lse, k_new, v_new, longest);
    // other kernels, other element types: two launches
    rc = wq_launch_append(ctx, k_new, v_new, new_dtype, B, kv);
    if (rc != WQ_OK) return rc;
    return wq_launch_decode(ctx, q, q_dtype, B, Hq, kv, sm_scale, num_splits, algo, out, lse, nullptr, nullptr, longest);
}

int wq_dequantize(wq_ctx* ctx, int B, const wq_packed_kv* src, const wq_packed_kv* dst)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    int rc = check_packed(ctx, src, B, true);
    if (rc != WQ_OK) return rc;
    rc = check_packed(ctx, dst, B, true);
    if (rc != WQ_OK) return rc;
    if (src->Hkv != dst->Hkv || src->hd != dst->hd || src->dtype16 != dst->dtype16)
        return wq_fail(ctx, WQ_ERR_ARG, "source and destination differ in Hkv, hd or dtype16");
    if (src->k16 == dst->k16 || src->v16 == dst->v16) return wq_fail(ctx, WQ_ERR_ARG, "source and destination share their 16-bit segment");
    if (B == 0) return WQ_OK;
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER) return wq_fail(ctx, WQ_ERR_WORKSPACE, "no workspace");
    return wq_launch_dequantize(ctx, B, src, dst);
}

int wq_decode_attention(wq_ctx* ctx, const void* q, int q_dtype, int B, int Hq, const wq_packed_kv* kv,
                        float sm_scale, int num_splits, int64_t max_seq_tokens, int algo, float* out, float* lse)
{
    if (!ctx) return WQ_ERR_ARG;
    int64_t longest = 0;
    const int rc = check_decode(ctx, q, q_dtype, B, Hq, kv, sm_scale, &num_splits, max_seq_tokens, algo, out, &longest);
    if (rc != WQ_OK || B == 0) return rc;
    return wq_launch_decode(ctx, q, q_dtype, B, Hq, kv, sm_scale, num_splits, algo, out, lse, nullptr, nullptr, longest);
}

// ---- rotary positions, prompt attention, decode over shared caches -----------------------------------------------------
constexpr int64_t MOST_GROUPS_512 = WQ_MOST_GROUPS_256 / 2, MOST_GROUPS_1024 = WQ_MOST_GROUPS_256 / 4;

// (offsets of a head inside a row, and of a row inside a tile of 64 with as many KV heads, have 32 bits)
constexpr int MOST_HEADS = 1 << 18;

// what a context's workspace has behind its header
static size_t room_of(const wq_ctx* ctx) { return ctx->ws && ctx->ws_bytes > WQ_WS_HEADER ? ctx->ws_bytes - WQ_WS_HEADER : 0; }

static bool on_16_bytes(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

static bool aligned_cache(const wq_packed_kv* kv)
{
    bool ok = on_16_bytes(kv->k16) && on_16_bytes(kv->v16);
    for (int c = 0; c < 3; c++) ok = ok && on_16_bytes(kv->codes[c]) && on_16_bytes(kv->meta[c]);
    return ok;
}

// The kernels take exponents of two: their scale, times log2(e), has to be finite too
static int check_scale(wq_ctx* ctx, float sm_scale)
{
    if (sm_scale > 0.0f && isfinite(sm_scale * WQ_LOG2E)) return WQ_OK;
    return wq_fail(ctx, WQ_ERR_ARG, "sm_scale must be positive, and finite times log2(e)");
}

// rows of H heads of hd elements, `stride` elements apart
static int check_rows(wq_ctx* ctx, const char* name, const void* p, int64_t stride, int64_t rows, int H, int hd, int dtype)
{
    if (rows == 0) return WQ_OK;
    if (!p) return wq_fail(ctx, WQ_ERR_ARG, "%s is NULL", name);
    if (stride < (int64_t)H * hd) return wq_fail(ctx, WQ_ERR_ARG, "%s: rows of %d x %d elements are %lld elements apart", name, H, hd, (long long)stride);
    if (!on_16_bytes(p) || stride % (dtype == WQ_F32 ? 4 : 8) != 0)
        return wq_fail(ctx, WQ_ERR_ARG, "%s must be 16-byte aligned, its rows a multiple of 16 bytes apart", name);
    return WQ_OK;
}

static int check_rope(wq_ctx* ctx, const WqRope& r)
{
    if (r.rows < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    if (r.rows > INT32_MAX) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many rows");
    if (!dtype_ok(r.dtype)) return wq_fail(ctx, WQ_ERR_ARG, "unknown dtype %d", r.dtype);
    if (r.hd != 64 && r.hd != 128) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "unsupported head dimension %d", r.hd);
    if (r.Hq <= 0 || r.Hkv < 0) return wq_fail(ctx, WQ_ERR_ARG, "bad head counts %d, %d", r.Hq, r.Hkv);
    if (r.Hq > 65536 || r.Hkv > 65536) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than 65536 heads");
    if (r.rot_dim <= 0 || r.rot_dim > r.hd || r.rot_dim % 16 != 0)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "rot_dim=%d must be a multiple of 16 up to the head dimension %d", r.rot_dim, r.hd);
    if (r.layout != WQ_ROPE_HALF && r.layout != WQ_ROPE_PAIRS) return wq_fail(ctx, WQ_ERR_ARG, "unknown layout %d", r.layout);
    if (!isfinite(r.mscale)) return wq_fail(ctx, WQ_ERR_ARG, "mscale must be finite");
    if (r.rows > 0 && (!r.positions || !r.inv_freq)) return wq_fail(ctx, WQ_ERR_ARG, "NULL positions or frequencies");
    int rc = check_rows(ctx, "q", r.q, r.q_stride, r.rows, r.Hq, r.hd, r.dtype);
    if (rc == WQ_OK) rc = check_rows(ctx, "q_out", r.q_out, r.q_out_stride, r.rows, r.Hq, r.hd, r.dtype);
    if (rc == WQ_OK && r.Hkv > 0) rc = check_rows(ctx, "k", r.k, r.k_stride, r.rows, r.Hkv, r.hd, r.dtype);
    return rc;
}

int wq_rope(wq_ctx* ctx, const void* q, int64_t q_stride, const void* k, int64_t k_stride, int dtype, int64_t rows, int Hq, int Hkv, int hd,
            int rot_dim, int layout, const int32_t* positions, const float* inv_freq, float mscale, void* q_out, int64_t q_out_stride,
            void* k_out, int64_t k_out_stride)
{
    if (!ctx) return WQ_ERR_ARG;
    const WqRope r = {q, k, q_out, k_out, q_stride, k_stride, q_out_stride, k_out_stride, dtype, Hq, Hkv, hd, rot_dim, layout, rows, positions, inv_freq, mscale};
    int rc = check_rope(ctx, r);
    if (rc == WQ_OK && Hkv > 0) rc = check_rows(ctx, "k_out", k_out, k_out_stride, rows, Hkv, hd, dtype);
    if (rc == WQ_OK && q == q_out && q_stride != q_out_stride) rc = wq_fail(ctx, WQ_ERR_ARG, "q in place with another stride");
    if (rc == WQ_OK && Hkv > 0 && k == k_out && k_stride != k_out_stride) rc = wq_fail(ctx, WQ_ERR_ARG, "k in place with another stride");
    if (rc != WQ_OK || rows == 0) return rc;
    return wq_launch_rope(ctx, r);
}

int wq_rope_append_kv(wq_ctx* ctx, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int dtype,
                      int B, int Hq, int rot_dim, int layout, const int32_t* positions, const float* inv_freq, float mscale, void* q_out,
                      int64_t q_out_stride, const wq_packed_kv* kv)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    int rc = check_packed(ctx, kv, B, false);
    if (rc != WQ_OK) return rc;
    const WqRope r = {q, k, q_out, nullptr, q_stride, k_stride, q_out_stride, 0, dtype, Hq, kv->Hkv, kv->hd, rot_dim, layout, B, positions, inv_freq, mscale};
    rc = check_rope(ctx, r);
    if (rc == WQ_OK) rc = check_rows(ctx, "v", v, v_stride, B, kv->Hkv, kv->hd, dtype);
    if (rc != WQ_OK) return rc;
    if (B > WQ_MOST_GROUPS_256) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many sequences");
    if ((dtype == WQ_BF16) != (kv->dtype16 == WQ_BF16))
        return wq_fail(ctx, WQ_ERR_ARG, "dtype16 must be bf16 for bf16 input and fp16 for fp16/fp32 input");
    if (q == q_out && q_stride != q_out_stride) return wq_fail(ctx, WQ_ERR_ARG, "q in place with another stride");
    if (!on_16_bytes(kv->k16) || !on_16_bytes(kv->v16)) return wq_fail(ctx, WQ_ERR_ARG, "k16 and v16 must be 16-byte aligned");
    if (B == 0) return WQ_OK;
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER) return wq_fail(ctx, WQ_ERR_WORKSPACE, "no workspace");
    return wq_launch_rope_append(ctx, r, v, v_stride, kv);
}

int wq_rope_frequencies(int rot_dim, double base, int scaling, double factor, int64_t trained_context, float* inv_freq, float* mscale)
{
    if (!inv_freq || !mscale || rot_dim <= 0 || rot_dim % 16 != 0 || !isfinite(base) || !(base > 1.0)) return WQ_ERR_ARG;
    if (scaling < WQ_ROPE_PLAIN || scaling > WQ_ROPE_PARTS) return WQ_ERR_ARG;
    if (scaling != WQ_ROPE_PLAIN && !(isfinite(factor) && factor >= 1.0)) return WQ_ERR_ARG;
    if (scaling == WQ_ROPE_PARTS && trained_context <= 0) return WQ_ERR_ARG;
    if (scaling == WQ_ROPE_BASE) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
    if (!isfinite(base)) return WQ_ERR_ARG;                    // (would turn every pair but the first by nothing)
    for (int i = 0; i < rot_dim / 2; i++) {
        double f = pow(base, -2.0 * i / rot_dim);
        if (scaling == WQ_ROPE_EVEN) f /= factor;
        if (scaling == WQ_ROPE_PARTS) {
            const double turns = (double)trained_context * f / 6.28318530717958647692;
            const double g = fmin(fmax((turns - 1.0) / (32.0 - 1.0), 0.0), 1.0);
            f = (1.0 - g) * f / factor + g * f;
        }
        inv_freq[i] = (float)f;
    }
    *mscale = scaling == WQ_ROPE_PARTS ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
    return WQ_OK;
}

size_t wq_prefill_workspace_bytes(int64_t total_q, int B, int Hq, int Hkv, int hd, int64_t max_kv_rows, int num_splits)
{
    if (total_q <= 0 || B <= 0 || Hq <= 0 || Hkv <= 0 || hd <= 0 || Hq % Hkv != 0) return WQ_WS_HEADER;
    const size_t a = wq_prefill_plan(total_q, B, Hq, Hkv, hd, WQ_F32, max_kv_rows, true, num_splits).bytes;
    const size_t b = wq_prefill_plan(total_q, B, Hq, Hkv, hd, WQ_BF16, max_kv_rows, true, num_splits).bytes;
    return WQ_WS_HEADER + (a > b ? a : b);
}

int wq_prefill_attention(wq_ctx* ctx, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int dtype,
                         int B, int Hq, int Hkv, int hd, const int32_t* q_off, const int32_t* kv_off, const int32_t* prefix_len, int64_t total_q,
                         int64_t total_kv, int64_t max_kv_rows, float sm_scale, int num_splits, void* out, float* lse)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0 || total_q < 0 || total_kv < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    if (!dtype_ok(dtype)) return wq_fail(ctx, WQ_ERR_ARG, "unknown dtype %d", dtype);
    if (hd != 64 && hd != 128) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "unsupported head dimension %d", hd);
    if (Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || Hq / Hkv > WQ_MAX_REP)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "Hq=%d must be a multiple of Hkv=%d, at most %d query heads per KV head", Hq, Hkv, WQ_MAX_REP);
    if (Hq > MOST_HEADS) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than 2^18 heads");
    const int rep = Hq / Hkv;
    if (total_q > INT32_MAX / rep || total_kv > INT32_MAX - 256 || B > INT32_MAX / 2)       // (positions and tiles' ends have 32 bits)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many rows");
    if (num_splits < 0 || num_splits > WQ_MAX_ATTEND_SPLITS) return wq_fail(ctx, WQ_ERR_ARG, "num_splits out of range");
    int rc = check_scale(ctx, sm_scale);
    if (rc != WQ_OK) return rc;
    if (B == 0 || total_q == 0) return WQ_OK;
    if (!q_off || !kv_off || !out) return wq_fail(ctx, WQ_ERR_ARG, "NULL table or output");
    if (!on_16_bytes(out)) return wq_fail(ctx, WQ_ERR_ARG, "out must be 16-byte aligned");
    rc = check_rows(ctx, "q", q, q_stride, total_q, Hq, hd, dtype);
    if (rc == WQ_OK) rc = check_rows(ctx, "k", k, k_stride, total_kv, Hkv, hd, dtype);
    if (rc == WQ_OK) rc = check_rows(ctx, "v", v, v_stride, total_kv, Hkv, hd, dtype);
    if (rc != WQ_OK) return rc;
    if (total_kv > 0 && (k_stride > 1 << 22 || v_stride > 1 << 22))       // (offsets inside a tile have 32 bits)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "rows of k or v are more than 2^22 elements apart");
    const WqPrefillPlan plan = wq_prefill_plan(total_q, B, Hq, Hkv, hd, dtype, max_kv_rows, prefix_len != nullptr, num_splits, room_of(ctx));
    if (plan.groups > MOST_GROUPS_512 || (plan.splits > 1 && total_q * Hq > 4 * WQ_MOST_GROUPS_256)) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many rows");
    if (ctx->ws_bytes < WQ_WS_HEADER + plan.bytes || !ctx->ws)
        return wq_fail(ctx, WQ_ERR_WORKSPACE, "workspace too small for %d splits of %lld rows", plan.tail > 0 ? plan.tail_splits : plan.splits, (long long)total_q);
    return wq_launch_prefill(ctx, {q, k, v, q_stride, k_stride, v_stride, dtype, B, Hq, Hkv, hd, plan, q_off, kv_off, prefix_len, total_q, total_kv, sm_scale,
                                   out, lse});
}

size_t wq_shared_workspace_bytes(int B, int P, int Hq, int Hkv, int hd, int64_t max_prefix_tokens, int64_t max_own_tokens, int num_splits)
{
    if (B <= 0 || P <= 0 || Hq <= 0 || Hkv <= 0 || hd <= 0 || Hq % Hkv != 0) return WQ_WS_HEADER;
    // (own caches that need a decode launch take the most)
    const size_t a = wq_shared_plan(B, P, Hq, Hkv, hd, WQ_F32, max_prefix_tokens, max_own_tokens, true, true, num_splits).bytes;
    const size_t b = wq_shared_plan(B, P, Hq, Hkv, hd, WQ_BF16, max_prefix_tokens, max_own_tokens, true, true, num_splits).bytes;
    return WQ_WS_HEADER + (a > b ? a : b);
}

int wq_decode_attention_shared(wq_ctx* ctx, const void* q, int q_dtype, int B, int Hq, const wq_packed_kv* prefix, const int32_t* req_off,
                               const wq_packed_kv* own, float sm_scale, int num_splits, int64_t max_prefix_tokens, int64_t max_own_tokens, void* out,
                               float* lse)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0 || Hq <= 0) return wq_fail(ctx, WQ_ERR_ARG, "bad B or Hq");
    if (B > 65535) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than 65535 requests in one call");
    if (!dtype_ok(q_dtype)) return wq_fail(ctx, WQ_ERR_ARG, "unknown q dtype %d", q_dtype);
    if (prefix && prefix->B <= 0) return wq_fail(ctx, WQ_ERR_ARG, "no shared sequence");
    int rc = check_packed(ctx, prefix, prefix ? prefix->B : 0, true);
    if (rc != WQ_OK) return rc;
    if (prefix->B > 65535) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than 65535 shared sequences in one call");
    if (Hq % prefix->Hkv != 0 || Hq / prefix->Hkv > WQ_MAX_REP)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "Hq=%d must be a multiple of Hkv=%d, at most %d query heads per KV head", Hq, prefix->Hkv, WQ_MAX_REP);
    if (Hq > MOST_HEADS) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than 2^18 heads");
    if ((q_dtype == WQ_BF16) != (prefix->dtype16 == WQ_BF16))
        return wq_fail(ctx, WQ_ERR_ARG, "dtype16 must be bf16 for bf16 queries and fp16 for fp16/fp32 queries");
    if (!on_16_bytes(q) || !on_16_bytes(out)) return wq_fail(ctx, WQ_ERR_ARG, "q and out must be 16-byte aligned");
    if (!aligned_cache(prefix)) return wq_fail(ctx, WQ_ERR_ARG, "the shared cache's buffers must be 16-byte aligned");
    if (num_splits < 0 || num_splits > WQ_MAX_ATTEND_SPLITS) return wq_fail(ctx, WQ_ERR_ARG, "num_splits out of range");
    rc = check_scale(ctx, sm_scale);
    if (rc != WQ_OK) return rc;
    if (own) {
        rc = check_packed(ctx, own, B, true);
        if (rc != WQ_OK) return rc;
        if (!aligned_cache(own)) return wq_fail(ctx, WQ_ERR_ARG, "the requests' own cache's buffers must be 16-byte aligned");
        if (own->Hkv != prefix->Hkv || own->hd != prefix->hd || own->dtype16 != prefix->dtype16)
            return wq_fail(ctx, WQ_ERR_ARG, "the shared and the requests' own cache differ in Hkv, hd or dtype16");
    }
    if (B == 0) return WQ_OK;
    if (!q || !out || !req_off) return wq_fail(ctx, WQ_ERR_ARG, "NULL q, out or req_off");
    const WqSharedPlan plan = wq_shared_plan(B, prefix->B, Hq, prefix->Hkv, prefix->hd, q_dtype, max_prefix_tokens, max_own_tokens, own != nullptr,
                                             own && own->cap[0] + own->cap[1] + own->cap[2] > 0, num_splits, room_of(ctx));
    if (plan.groups > MOST_GROUPS_512 || (int64_t)B * prefix->Hkv > MOST_GROUPS_1024)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many workgroups");
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER + plan.bytes)
        return wq_fail(ctx, WQ_ERR_WORKSPACE, "workspace too small for %d splits of %d requests", plan.splits, B);
    // an fp32 query's own cache in fp32 arithmetic, like its shared one
    const int algo = q_dtype == WQ_F32 ? WQ_DECODE_GENERIC : WQ_DECODE_AUTO;
    int decode_splits = plan.decode_splits;
    if (plan.own_decode) {
        int64_t longest = 0;
        rc = check_decode(ctx, q, q_dtype, B, Hq, own, sm_scale, &decode_splits, max_own_tokens, algo, static_cast<const float*>(out), &longest);
        if (rc != WQ_OK) return rc;
    }
    return wq_launch_shared(ctx, {q, q_dtype, B, Hq, prefix, own, req_off, sm_scale, plan, decode_splits, algo, out, lse});
}

// ---- several new rows per sequence, copies of sequences -------------------------------------------------------------------
size_t wq_tree_workspace_bytes(int64_t total_rows, int B, int Hq, int Hkv, int hd, int64_t max_cache_tokens, int max_rows, int num_splits)
{
    if (total_rows <= 0 || B <= 0 || Hq <= 0 || Hkv <= 0 || hd <= 0 || Hq % Hkv != 0) return WQ_WS_HEADER;
    size_t most = 0;
    max_cache_tokens = max_cache_tokens < int64_t(1) << 40 ? max_cache_tokens : int64_t(1) << 40;
    for (const int dtype : {WQ_F32, WQ_BF16})
        for (int quarters = 1; quarters <= 4; quarters++) {    // (of the longest sequence's length, on the average: a ragged batch has more parts)
            const size_t bytes = wq_tree_plan(total_rows, B, Hq, Hkv, hd, dtype, max_cache_tokens, (B < 65536 ? B : 65535) * max_cache_tokens / 4 * quarters, max_rows, num_splits).bytes;
            most = bytes > most ? bytes : most;
        }
    return WQ_WS_HEADER + most;
}

int wq_tree_attention(wq_ctx* ctx, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int dtype, int B, int Hq,
                      const wq_packed_kv* kv, const int32_t* row_off, const int32_t* parent, int64_t total_rows, int max_rows, float sm_scale, int num_splits,
                      int64_t max_cache_tokens, void* out, float* lse)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0 || total_rows < 0 || max_rows < 0 || max_cache_tokens < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    if (!dtype_ok(dtype)) return wq_fail(ctx, WQ_ERR_ARG, "unknown dtype %d", dtype);
    int rc = check_packed(ctx, kv, B, true);
    if (rc != WQ_OK) return rc;
    if (!aligned_cache(kv)) return wq_fail(ctx, WQ_ERR_ARG, "the cache's buffers must be 16-byte aligned");
    if (Hq <= 0 || Hq % kv->Hkv != 0 || Hq / kv->Hkv > WQ_MAX_REP)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "Hq=%d must be a multiple of Hkv=%d, at most %d query heads per KV head", Hq, kv->Hkv, WQ_MAX_REP);
    if (Hq > MOST_HEADS) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than 2^18 heads");
    if ((dtype == WQ_BF16) != (kv->dtype16 == WQ_BF16))
        return wq_fail(ctx, WQ_ERR_ARG, "dtype16 must be bf16 for bf16 rows and fp16 for fp16/fp32 rows");
    if (total_rows > INT32_MAX / WQ_MAX_REP - 256 || B > 65535) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many rows or sequences");
    if (parent && max_rows > WQ_MAX_TREE) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "trees of more than %d rows", WQ_MAX_TREE);
    if (num_splits < 0 || num_splits > WQ_MAX_ATTEND_SPLITS) return wq_fail(ctx, WQ_ERR_ARG, "num_splits out of range");
    rc = check_scale(ctx, sm_scale);
    if (rc != WQ_OK) return rc;
    if (B == 0 || total_rows == 0) return WQ_OK;
    if (!row_off || !out) return wq_fail(ctx, WQ_ERR_ARG, "NULL table or output");
    if (!on_16_bytes(out)) return wq_fail(ctx, WQ_ERR_ARG, "out must be 16-byte aligned");
    rc = check_rows(ctx, "q", q, q_stride, total_rows, Hq, kv->hd, dtype);
    if (rc == WQ_OK) rc = check_rows(ctx, "k", k, k_stride, total_rows, kv->Hkv, kv->hd, dtype);
    if (rc == WQ_OK) rc = check_rows(ctx, "v", v, v_stride, total_rows, kv->Hkv, kv->hd, dtype);
    if (rc != WQ_OK) return rc;
    if (k_stride > 1 << 22 || v_stride > 1 << 22)             // (offsets inside a tile have 32 bits)
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "rows of k or v are more than 2^22 elements apart");
    const WqTreePlan plan = wq_tree_plan(total_rows, B, Hq, kv->Hkv, kv->hd, dtype, max_cache_tokens,
                                         kv->cap[0] + kv->cap[1] + kv->cap[2] + kv->cap16, max_rows, num_splits, room_of(ctx));
    if (plan.groups > MOST_GROUPS_512 || (plan.splits > 1 && (total_rows * Hq > 4 * WQ_MOST_GROUPS_256 || plan.units * (plan.rows / 4) > WQ_MOST_GROUPS_256)))
        return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many rows");
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER + plan.bytes)
        return wq_fail(ctx, WQ_ERR_WORKSPACE, "workspace too small for %d splits of %lld rows", plan.splits, (long long)total_rows);
    return wq_launch_tree(ctx, {q, k, v, q_stride, k_stride, v_stride, dtype, B, Hq, kv, plan, row_off, parent, total_rows, max_rows, sm_scale, out, lse});
}

int wq_tree_accept(wq_ctx* ctx, const int32_t* tokens, const int32_t* target, const int32_t* parent, int B, const int32_t* row_off, int64_t total_rows, int max_rows,
                   int max_path, int32_t* path, int32_t* n_path, int32_t* next_token)
{
    if (!ctx) return WQ_ERR_ARG;
    if (B < 0 || total_rows < 0 || max_rows <= 0 || max_path <= 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size, or no row");
    if (max_rows > WQ_MAX_TREE) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "trees of more than %d rows", WQ_MAX_TREE);
    if (B > WQ_MOST_GROUPS_256) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "too many sequences");
    if (B == 0) return WQ_OK;
    if (!row_off || !path || !n_path || !next_token || (total_rows > 0 && (!tokens || !target))) return wq_fail(ctx, WQ_ERR_ARG, "NULL table or output");
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER) return wq_fail(ctx, WQ_ERR_WORKSPACE, "no workspace");
    return wq_launch_accept(ctx, {tokens, target, parent, row_off, B, max_rows, max_path, total_rows, path, n_path, next_token});
}

int wq_append_rows(wq_ctx* ctx, int n_layers, const void* const* k, int64_t k_stride, const void* const* v, int64_t v_stride, int dtype, int B, const int32_t* row_off,
                   int64_t total_rows, const int32_t* take, const int32_t* n_take, int max_take, const wq_packed_kv* kv)
{
    if (!ctx) return WQ_ERR_ARG;
    if (n_layers < 0 || B < 0 || total_rows < 0 || max_take < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    if (!dtype_ok(dtype)) return wq_fail(ctx, WQ_ERR_ARG, "unknown dtype %d", dtype);
    if (n_layers == 0) return WQ_OK;
    if (!k || !v || !kv) return wq_fail(ctx, WQ_ERR_ARG, "NULL array of layers");
    if (max_take > 0 && !take != !n_take) return wq_fail(ctx, WQ_ERR_ARG, "take and n_take go together");      // (a table of no columns has no address)
    for (int l = 0; l < n_layers; l++) {
        int rc = check_packed(ctx, kv + l, B, false);
        if (rc != WQ_OK) return rc;
        if (kv[l].Hkv != kv[0].Hkv || kv[l].hd != kv[0].hd || kv[l].dtype16 != kv[0].dtype16)
            return wq_fail(ctx, WQ_ERR_ARG, "the layers' caches differ in Hkv, hd or dtype16");
        if (kv[l].Hkv > MOST_HEADS) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than 2^18 heads");
        if (!on_16_bytes(kv[l].k16) || !on_16_bytes(kv[l].v16)) return wq_fail(ctx, WQ_ERR_ARG, "k16 and v16 must be 16-byte aligned");
        rc = check_rows(ctx, "k", k[l], k_stride, total_rows, kv[l].Hkv, kv[l].hd, dtype);
        if (rc == WQ_OK) rc = check_rows(ctx, "v", v[l], v_stride, total_rows, kv[l].Hkv, kv[l].hd, dtype);
        if (rc != WQ_OK) return rc;
    }
    if (shares_memory(n_layers, nullptr, kv, [](const wq_packed_kv& x, const auto& f) { each_appended(x, f); })) return wq_fail(ctx, WQ_ERR_ARG, "two layers share a cache's rows or lengths");
    if ((dtype == WQ_BF16) != (kv[0].dtype16 == WQ_BF16))
        return wq_fail(ctx, WQ_ERR_ARG, "dtype16 must be bf16 for bf16 input and fp16 for fp16/fp32 input");
    if (B == 0 || max_take == 0 || (total_rows == 0 && !take)) return WQ_OK;
    if (!row_off) return wq_fail(ctx, WQ_ERR_ARG, "NULL table");
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER) return wq_fail(ctx, WQ_ERR_WORKSPACE, "no workspace");
    return wq_launch_append_rows(ctx, {n_layers, k, v, k_stride, v_stride, dtype, B, row_off, total_rows, take, n_take, max_take, kv});
}

int wq_copy_sequences(wq_ctx* ctx, int n_layers, const wq_packed_kv* src, const wq_packed_kv* dst, const int32_t* from)
{
    if (!ctx) return WQ_ERR_ARG;
    if (n_layers < 0) return wq_fail(ctx, WQ_ERR_ARG, "negative size");
    if (n_layers == 0) return WQ_OK;
    if (!src || !dst) return wq_fail(ctx, WQ_ERR_ARG, "NULL array of layers");
    for (int l = 0; l < n_layers; l++) {
        for (const wq_packed_kv* kv : {src + l, dst + l}) {
            const int B = kv == src + l ? src->B : dst->B;
            if (B < 0 || B > 65535) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than 65535 sequences");
            const int rc = check_packed(ctx, kv, B, true);
            if (rc != WQ_OK) return rc;
            if (!aligned_cache(kv)) return wq_fail(ctx, WQ_ERR_ARG, "the caches' buffers must be 16-byte aligned");
            if (kv->Hkv != src->Hkv || kv->hd != src->hd || kv->group != src->group || kv->dtype16 != src->dtype16)
                return wq_fail(ctx, WQ_ERR_ARG, "the caches differ in Hkv, hd, group or dtype16");
        }
    }
    if (shares_memory(n_layers, src, dst, [](const wq_packed_kv& x, const auto& f) { each_copied(x, f); })) return wq_fail(ctx, WQ_ERR_ARG, "a cache is copied into memory of another one, or of two layers");
    if (dst->B == 0) return WQ_OK;
    if (!from) return wq_fail(ctx, WQ_ERR_ARG, "from is NULL");
    if (src->Hkv > MOST_HEADS) return wq_fail(ctx, WQ_ERR_UNSUPPORTED, "more than 2^18 heads");
    if (!ctx->ws || ctx->ws_bytes < WQ_WS_HEADER) return wq_fail(ctx, WQ_ERR_WORKSPACE, "no workspace");
    return wq_launch_copy_sequences(ctx, n_layers, src, dst, from);
}

// ---- the entry point that allocates nothing ---------------------------------------------------------------------
// Its workspace is this array, part of the code object: every GPU that loads the library holds its own copy at its own
// address.  The name is a host-side stand-in for the symbol; the device address comes from hipGetSymbolAddress, once per
// device, and only that address is handed to kernels.  Zero-initialised when the code object is loaded, which is the
// state a workspace header has to start in.
static __device__ __align__(256) unsigned char scratch[WQ_STATIC_SCRATCH_BYTES];

namespace {
constexpr int WQ_MAX_DEVICES = 64;
struct StaticSlot {
    bool ready = false;
    wq_ctx ctx;
};
StaticSlot g_static[WQ_MAX_DEVICES];
std::mutex g_static_mu;
char g_static_err[256] = "";
}  // namespace

const char* wq_static_last_error(void)
{
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= WQ_MAX_DEVICES) return g_static_err;
    return g_static[dev].ready ? g_static[dev].ctx.err : g_static_err;
}

int wq_decode_attention_static(void* hip_stream, const void* q, int q_dtype, int B, int Hq, const wq_packed_kv* kv,
                               float sm_scale, int num_splits, int64_t max_seq_tokens, int algo, float* out, float* lse)
{
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess || dev < 0 || dev >= WQ_MAX_DEVICES) {
        snprintf(g_static_err, sizeof(g_static_err), "no current device (%s)", e != hipSuccess ? hipGetErrorString(e) : "index out of range");
        return WQ_ERR_HIP;
    }
    StaticSlot& slot = g_static[dev];
    {
        std::lock_guard<std::mutex> lock(g_static_mu);
        if (!slot.ready) {
            void* ptr = nullptr;
            e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
            if (e != hipSuccess || !ptr) {
                snprintf(g_static_err, sizeof(g_static_err), "hipGetSymbolAddress(scratch): %s", hipGetErrorString(e));
                return WQ_ERR_HIP;
            }
            slot.ctx.stream = nullptr;
            slot.ctx.ws = static_cast<char*>(ptr);
            slot.ctx.ws_bytes = WQ_STATIC_SCRATCH_BYTES;
            slot.ctx.owns_ws = false;
            slot.ctx.timing = false;
            for (int i = 0; i < 2 * WQ_TIMING_RING; i++) slot.ctx.ev[i] = nullptr;
            slot.ctx.ev_calls = 0;
            slot.ctx.err[0] = 0;
            slot.ready = true;
        }
    }
    wq_ctx* ctx = &slot.ctx;
    ctx->stream = static_cast<hipStream_t>(hip_stream);
    int64_t longest = 0;
    int splits = num_splits;
    const int rc = check_decode(ctx, q, q_dtype, B, Hq, kv, sm_scale, &splits, max_seq_tokens, algo, out, &longest);
    if (rc == WQ_ERR_WORKSPACE)
        return wq_fail(ctx, WQ_ERR_WORKSPACE, "B=%d Hq=%d hd=%d with %d splits needs %zu bytes of scratch, the static array holds %u", B, Hq,
                       kv->hd, splits, WQ_WS_HEADER + wq_decode_ws_bytes(B, Hq, kv->hd, splits), (unsigned)WQ_STATIC_SCRATCH_BYTES);
    if (rc != WQ_OK || B == 0) return rc;
    return wq_launch_decode(ctx, q, q_dtype, B, Hq, kv, sm_scale, splits, algo, out, lse, nullptr, nullptr, longest);
}

}  // extern "C"
