"""Plain attention and rotary positions in 64 bits, and packed caches with known logical contents, for the tests of the
operators around the cache.  A cache is laid out here from the storage format's field numbers; what no token owns is
filled with bytes that would show up as NaN."""
import math

import numpy as np
import torch

from paper_2605_02262_amd import binding as W

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}     # of a rounding, relative


def i32(v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32).cuda()


def offsets(v):
    return [sum(v[:i]) for i in range(len(v) + 1)]


def attend(q, k, v, limit, sm_scale):
    """(out, lse, sum of weights times |v|, largest sum of |q_c k_c| * sm_scale) of one sequence: q [n, Hq, hd], k, v [L, Hkv, hd] in fp64,
    query row i sees the keys below limit[i]."""
    n, Hq, hd = q.shape
    rep = Hq // k.shape[1]
    out, lse, spread = torch.zeros_like(q), torch.full((n, Hq), -math.inf, dtype=torch.float64), torch.zeros_like(q)
    terms = 0.0
    if k.shape[0] == 0:
        return out, lse, spread, terms
    hidden = torch.arange(k.shape[0])[None] >= torch.as_tensor(limit)[:, None]
    for h in range(Hq):
        kk, vv = k[:, h // rep], v[:, h // rep]
        s = (q[:, h] @ kk.T) * sm_scale
        terms = max(terms, float((q[:, h].abs() @ kk.abs().T).max()) * sm_scale)
        s[hidden] = -math.inf
        lse[:, h] = torch.logsumexp(s, 1)
        seen = torch.isfinite(lse[:, h])
        p = torch.zeros_like(s)
        p[seen] = torch.exp(s[seen] - lse[seen, h][:, None])
        out[:, h], spread[:, h] = p @ vv, p @ vv.abs()
    return out, lse, spread, terms


def weights_error(n_keys, hd, terms, lse_range):
    """Bound of a weight's relative error in fp32 arithmetic: the logit is a sum of hd exact or once rounded products (2^-24 of the sum of their
    magnitudes for each addition), its exponent is formed by one fused multiply-add and one exponential (a step each of values up to the
    logit and the reference), and the weights are summed one after the other (2^-24 each)."""
    return 2.0 ** -24 * (2 * (hd + 4) * terms + 4 * (lse_range + 16) + 8 + n_keys)


def make_cache(rng, lens, Hkv, hd, group, dtype16, slack=0, scale=1.0):
    """lens[b] = (2-, 4-, 8-bit, 16-bit tokens): (PackedKV, [(K, V) in fp64 [tokens, Hkv, hd] in cache order])."""
    B, G = len(lens), hd // group
    pad = lambda n: -(-n // 32) * 32  # noqa: E731
    cap = [sum(pad(ln[c]) for ln in lens) + 32 for c in range(3)]       # (a block that belongs to nobody)
    rows = [ln[3] + slack for ln in lens]
    kv = W.PackedKV(B, Hkv, hd, group, dtype16, cap, offsets(rows))
    parts = [[] for _ in range(B)]
    largest = np.zeros(B, np.float32)
    for c, b in enumerate((2, 4, 8)):
        code = np.zeros((2, cap[c], Hkv, hd), np.uint8)
        s, m = np.full((2, cap[c], Hkv, G), np.nan, np.float16), np.full((2, cap[c], Hkv, G), np.nan, np.float16)
        off = offsets([pad(ln[c]) for ln in lens])
        code[:, off[-1]:] = 2 ** b - 1
        for i, ln in enumerate(lens):
            a, z = off[i], off[i] + ln[c]
            code[:, a:z] = rng.integers(0, 2 ** b, (2, ln[c], Hkv, hd))
            s[:, a:off[i + 1]], m[:, a:off[i + 1]] = 0, 0
            width = scale * rng.lognormal(0, 0.7, (2, ln[c], Hkv, G)) * 4
            s[:, a:z] = width / (2 ** b - 1)
            m[:, a:z] = -width * rng.uniform(0.2, 0.8, width.shape)
            if ln[c]:
                largest[i] = max(largest[i], float(np.abs(s[1, a:z]).max()))
            x = code[:, a:z].reshape(2, ln[c], Hkv, G, group) * s[:, a:z, ..., None].astype(np.float64) + m[:, a:z, ..., None].astype(np.float64)
            parts[i].append(x.reshape(2, ln[c], Hkv, hd))
        tok, ch = np.arange(cap[c])[:, None], np.arange(hd)[None]
        kn = (tok // 16 * 16 * hd) + ((ch // (hd // 4)) * 16 + tok % 16) * (hd // 4) + ch % (hd // 4)
        u = tok % 32
        vn = (tok // 32 * 32 * hd) + (((u % 16 // 4) * 16 + ch % 16) * (hd // 16) + ch // 16) * 8 + 4 * (u // 16) + u % 4
        for plane, n in ((0, kn), (1, vn)):
            for h in range(Hkv):
                field = np.zeros(cap[c] * hd, np.uint8)
                field[n] = code[plane, :, h]
                packed = (field.reshape(-1, 8 // b).astype(np.int32) << (np.arange(8 // b) * b)).sum(1).astype(np.uint8)
                kv.codes[c][plane, h] = torch.from_numpy(packed).cuda()
                words = s[plane, :, h].view(np.uint16).astype(np.uint32) | m[plane, :, h].view(np.uint16).astype(np.uint32) << 16
                words = words.reshape(cap[c] // 16, 16, G).transpose(0, 2, 1).reshape(-1)
                kv.meta[c][plane, h] = torch.from_numpy(words.view(np.int32).copy()).cuda()
        kv.cls_off[c].copy_(i32(off))
        kv.cls_len[c].copy_(i32([ln[c] for ln in lens]))
    rows16 = torch.full((2, kv.cap16, Hkv, hd), math.nan, dtype=dtype16)
    at = offsets(rows)
    for i, ln in enumerate(lens):
        x = torch.from_numpy(rng.normal(0, scale, (2, ln[3], Hkv, hd))).to(dtype16)
        rows16[:, at[i]:at[i] + ln[3]] = x
        parts[i].append(x.double().numpy())
    if kv.cap16:
        kv.k16.copy_(rows16[0])
        kv.v16.copy_(rows16[1])
    kv.len16.copy_(i32([ln[3] for ln in lens]))
    kv.v_scale_max[:B] = torch.from_numpy(largest).cuda()
    logical = [torch.from_numpy(np.concatenate(p, 1)) for p in parts]
    return kv, [(x[0], x[1]) for x in logical]


def rope(x, positions, inv_freq, layout, mscale):
    """x [rows, H, hd] in fp64: (turned, sum of the magnitudes of an output's two terms)."""
    rot = 2 * inv_freq.numel()
    t = positions.double()[:, None, None] * inv_freq.double()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == W.ROPE_HALF else (slice(0, rot, 2), slice(1, rot, 2))
    y, size = x.clone(), torch.zeros_like(x)
    y[..., a] = (x[..., a] * t.cos() - x[..., b] * t.sin()) * mscale
    y[..., b] = (x[..., b] * t.cos() + x[..., a] * t.sin()) * mscale
    size[..., a] = size[..., b] = (x[..., a].abs() + x[..., b].abs()) * abs(mscale)
    return y, size
