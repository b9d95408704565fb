"""Three operators around the packed cache, as cases that can be timed and compared.

A case is a dict of plain values.  Its `kind` is the operator that one pass runs:

  rope     rotary positions of a prompt's queries and keys, cut out of a fused projection
  append   a decode step's rotary positions, the rotated key and the value written behind the request's 16-bit rows
  prefill  attention of new rows over the 16-bit rows of their own sequence: causal, with a visual prefix that all see
  shared   a decode step of requests that ask about the same videos: one packed cache per video, read once for all of
           them, and each request's own 16-bit rows

Sizes are those of the configurations (14 query / 2 KV heads of 64 and 28 / 4 of 128; frames of 196 tokens, windows of 16,
32 and 196; prompts of 16 to 512 tokens) or generic.
"""
import math
import random

import torch

own = False     # True: the framework's calls instead of their plain form

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SMALL = dict(heads=14, kv_heads=2, head_dim=64)
LARGE = dict(heads=28, kv_heads=4, head_dim=128)
BITS = (2, 4, 8)


def _rope(**more):
    return dict(dict(kind="rope", batch=1, rows=1000, rot_dim=0, layout="half", dtype="bf16", start=0, factor=1, base=1000000, **LARGE), **more)


def _append(**more):
    return dict(dict(kind="append", batch=8, held=500, rot_dim=0, layout="half", dtype="bf16", start=12800, factor=1, base=1000000, **LARGE), **more)


def _prefill(**more):
    return dict(dict(kind="prefill", batch=1, rows=1000, held=0, prefix=0, ragged=0, lse=False, dtype="bf16", **LARGE), **more)


def _shared(**more):
    return dict(dict(kind="shared", prefixes=1, batch=8, windows=64, window=196, text=128, top=20, mid=50, top_bits=8, group=64, own_rows=128, ragged=0,
                     dtype="bf16", **LARGE), **more)


def listed():
    return [
        # a decode step of eight requests: one layer's rotary positions and append (the smallest call, latency)
        _append(name="append_batch8"),
        # the prompts of four long videos (256 frames of 196 tokens and 512 tokens of text), one layer
        _rope(name="rope_long_prompts", batch=4, rows=50688),
        # a small model whose heads are rotated in part, neighbouring channels in pairs, far into a stretched context, odd length
        _rope(name="rope_part_far_f16", rows=6411, rot_dim=32, layout="pairs", dtype="f16", start=1000003, factor=8, base=10000, **SMALL),
        # the tiny configuration in fp32: 8 x 16 visual tokens that see each other, 16 of text
        _prefill(name="prefill_tiny_f32", rows=144, prefix=89, dtype="f32", **SMALL),
        # a batch of short prompts of many lengths, fp16
        _prefill(name="prefill_ragged_f16", batch=16, rows=1389, prefix=80, ragged=515, dtype="f16", **LARGE),
        # one prompt of 64 frames and 256 tokens of text
        _prefill(name="prefill_64_frames", rows=12800, prefix=98),
        # a question of 61 tokens behind a clip whose rows are there already
        _prefill(name="prefill_question", rows=61, held=12544, lse=True),
        # single tokens of eight requests over plain rows of many lengths
        _prefill(name="prefill_single_tokens", batch=8, rows=1, held=6400, ragged=77, lse=True, **SMALL),
        # the tiny configuration in fp32: three questions about one short clip
        _shared(name="shared_tiny_f32", batch=3, windows=8, window=16, text=16, top=25, group=32, own_rows=17, dtype="f32", **SMALL),
        # sixteen questions about one video with a 16-bit top tier and windows of 32
        _shared(name="shared_paper_tiers", batch=16, windows=612, window=32, text=135, top=0.4, mid=35, top_bits=16, own_rows=96),
        # sixty-four questions about one long video
        _shared(name="shared_long_video", batch=64, windows=256, text=512, top=10, mid=40, own_rows=200),
        # four clips of a small model with one to many questions each, fp16
        _shared(name="shared_clips_f16", prefixes=4, batch=37, windows=33, text=77, own_rows=90, ragged=2024, group=64, dtype="f16", **SMALL),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    kind = rng.choice(["rope", "append", "prefill", "prefill", "prefill", "shared", "shared", "shared"])
    model = dict(rng.choice([SMALL, LARGE, LARGE, dict(heads=32, kv_heads=8, head_dim=128), dict(heads=8, kv_heads=8, head_dim=64)]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
    hd = model["head_dim"]
    if kind in ("rope", "append"):
        c = dict(batch=_log(rng, 1, 64), rot_dim=rng.choice([0, 0, 16, hd // 2, hd - 32]), layout=rng.choice(["half", "pairs"]), dtype=dtype,
                 start=rng.choice([0, _log(rng, 1, 2000000)]), factor=rng.choice([1, 1, 2, 8]), base=rng.choice([10000, 1000000]), **model)
        if kind == "rope":
            c["batch"] = rng.choice([1, 1, _log(rng, 1, 16)])
            c = _rope(rows=_log(rng, 1, 150000 // c["batch"]), **c)
        else:
            c = _append(held=_log(rng, 1, 2000), **c)
    elif kind == "prefill":
        c = _prefill(batch=rng.choice([1, _log(rng, 1, 24)]), rows=rng.choice([1, _log(rng, 2, 8000)]), held=rng.choice([0, 0, _log(rng, 1, 20000)]),
                     prefix=rng.choice([0, rng.randrange(1, 101)]), dtype=dtype, lse=rng.random() < 0.3, **model)
        if c["batch"] > 1 and rng.random() < 0.7:
            c["ragged"] = rng.randrange(1, 1 << 20)
    else:
        c = _shared(prefixes=rng.choice([1, 1, 1, rng.randint(2, 6)]), window=rng.choice([16, 32, 98, 196]), text=_log(rng, 1, 600),
                    top=rng.choice([0, 10, 20, 25, 100]), group=rng.choice([hd // 2, hd // 2, hd, 32]), top_bits=rng.choice([8, 8, 8, 16]),
                    own_rows=_log(rng, 1, 500), dtype=dtype, **model)
        c["mid"] = rng.choice([m for m in (0, 20, 40, 50) if m + c["top"] <= 100])
        c["batch"] = max(c["prefixes"], _log(rng, 1, 96))
        c["windows"] = max(1, _log(rng, 100, 60000) // c["window"])
        if rng.random() < 0.4:
            c["ragged"] = rng.randrange(1, 1 << 20)
    while _cost(c) > most:
        if kind == "rope":
            c["rows"] = c["rows"] * 3 // 4
        elif kind == "shared":
            c["windows"] = max(1, c["windows"] * 3 // 4)
        elif c["batch"] > 1:
            c["batch"] -= 1
        elif c["held"] > c["rows"]:
            c["held"] = c["held"] * 3 // 4
        else:
            c["rows"] = c["rows"] * 3 // 4
    return c


# ------------------------------------------------------------------------------------------------------------------------
# sizes
# ------------------------------------------------------------------------------------------------------------------------
def _sum(v):
    return [sum(v[:i]) for i in range(len(v) + 1)]


def _rot(c):
    return c["rot_dim"] or c["head_dim"]


def _prefill_sizes(c):
    """(new rows, all rows, rows of the prefix) of every sequence."""
    rng = random.Random(c["ragged"])
    new = [rng.randint(max(1, c["rows"] // 8), c["rows"]) if c["ragged"] else c["rows"] for _ in range(c["batch"])]
    held = [rng.randint(c["held"] // 8, c["held"]) if c["ragged"] else c["held"] for _ in range(c["batch"])]
    rows = [n + h for n, h in zip(new, held)]
    return new, rows, [r * c["prefix"] // 100 for r in rows]


def _pairs(c):
    """(query, key) pairs that are attended, of one head."""
    total = 0
    for n, r, p in zip(*_prefill_sizes(c)):
        first = r - n                                   # position of the first new row: it sees first + 1 keys, or the prefix
        low = min(max(p - first, 0), n)                 # rows that see the prefix and no more
        total += low * p + _range_sum(first + low + 1, r)
    return total


def _range_sum(a, b):
    return (a + b) * (b - a + 1) // 2 if b >= a else 0


def _shared_sizes(c):
    """Per prefix (2-, 4-, 8-, 16-bit tokens) and the number of its requests; per request its own rows."""
    rng = random.Random(c["ragged"])
    tokens, n = [], []
    for p in range(c["prefixes"]):
        w = rng.randint(max(1, c["windows"] // 8), c["windows"]) if c["ragged"] else c["windows"]
        top, both = int(c["top"] * w / 100 + 0.5), int((c["top"] + c["mid"]) * w / 100 + 0.5)
        t = [(w - both) * c["window"], (both - top) * c["window"], top * c["window"], c["text"]]
        if c["top_bits"] == 16:
            t[3] += t[2]
            t[2] = 0
        tokens.append(t)
        n.append(1)
    for b in range(c["batch"] - c["prefixes"]):
        n[rng.randrange(c["prefixes"]) if c["ragged"] else b % c["prefixes"]] += 1
    rows = [rng.randint(1, c["own_rows"]) if c["ragged"] else c["own_rows"] for _ in range(c["batch"])]
    return tokens, n, rows


def work(c):
    size = 4 if c["dtype"] == "f32" else 2
    H, Hkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    if c["kind"] == "rope":
        n = c["batch"] * c["rows"] * (H + Hkv)
        return dict(bytes=2 * n * hd * size + 4 * c["batch"] * c["rows"], flops=3 * n * _rot(c))
    if c["kind"] == "append":
        n = c["batch"] * (H + Hkv)
        return dict(bytes=c["batch"] * (2 * H + Hkv + Hkv) * hd * size + c["batch"] * 2 * Hkv * hd * 2, flops=3 * n * _rot(c))
    if c["kind"] == "prefill":
        new, rows, _ = _prefill_sizes(c)
        return dict(bytes=(2 * sum(new) * H + 2 * sum(rows) * Hkv) * hd * size, flops=4 * H * hd * _pairs(c))
    tokens, n, rows = _shared_sizes(c)
    G = hd // c["group"]
    packed = sum(t * 2 * Hkv * (hd * b // 8 + 4 * G) for p in tokens for t, b in zip(p, BITS)) + sum(p[3] for p in tokens) * 2 * Hkv * hd * 2
    pairs = sum(k * sum(p) for k, p in zip(n, tokens)) + sum(rows)
    return dict(bytes=packed + sum(rows) * 2 * Hkv * hd * 2 + 2 * c["batch"] * H * hd * size, flops=4 * H * hd * pairs)


def _cost(c):
    """Time of a pass as far as sizes tell it; a padded batch of plain attention is charged for its padding."""
    w = work(c)
    flops = w["flops"]
    if c["kind"] == "prefill":
        flops = max(flops, 2 * c["heads"] * c["head_dim"] * c["batch"] * c["rows"] * (c["rows"] + c["held"]))
    return max(w["bytes"], flops / 50)


# ------------------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------------------
class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def keys(self, c, *rows):
        """Keys with channels of very different size, and the factor that gives queries' scaled products a deviation of 2."""
        scale = torch.exp(self.normal(c["kv_heads"], c["head_dim"]))
        fit = 2 * math.sqrt(c["head_dim"]) / scale.norm(dim=-1)
        return [self.normal(r, c["kv_heads"], c["head_dim"]) * scale for r in rows], fit.repeat_interleave(c["heads"] // c["kv_heads"])[:, None]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _frequencies(c):
    """inv_freq of every pair: base^(-2i/rot), stretched evenly by `factor`, fp32 as programs keep it; the cosines' factor."""
    i = torch.arange(0, _rot(c), 2, dtype=torch.float64, device="cuda")
    return (float(c["base"]) ** (-i / _rot(c)) / c["factor"]).float(), 0.1 * math.log(c["factor"]) + 1.0


def _make(c, seed):
    """The inputs in logical form (before anything is laid out)."""
    g, dt = _Draws(seed), DTYPES[c["dtype"]]
    H, Hkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    if c["kind"] in ("rope", "append"):
        rows = c["batch"] * (c["rows"] if c["kind"] == "rope" else 1)
        x = dict(qkv=g.normal(rows, (H + 2 * Hkv) * hd).to(dt))
        if c["kind"] == "rope":
            x["positions"] = (c["start"] + torch.arange(c["rows"], dtype=torch.int32, device="cuda")).repeat(c["batch"])
        else:
            x["positions"] = c["start"] + torch.randint(0, 1000, (rows,), generator=g.g, device="cuda", dtype=torch.int32)
        return x
    if c["kind"] == "prefill":
        new, rows, prefix = _prefill_sizes(c)
        (k,), fit = g.keys(c, sum(rows))
        return dict(q=(g.normal(sum(new), H, hd) * fit).to(dt), k=k.to(dt), v=g.normal(*k.shape).to(dt))
    t16 = torch.bfloat16 if c["dtype"] == "bf16" else torch.float16
    tokens, n, rows = _shared_sizes(c)
    per_class = [[p[k] for p in tokens] for k in range(4)]
    padded = [sum(-(-t // 32) * 32 for t in per_class[k]) for k in range(3)]
    keys, fit = g.keys(c, *padded, sum(per_class[3]), sum(rows))
    x = dict(q=(g.normal(c["batch"], H, hd) * fit).to(dt), classes=[])
    for k, b in enumerate(BITS):
        both = torch.stack([keys[k], g.normal(*keys[k].shape)]).to(t16).float().unflatten(-1, (-1, c["group"]))
        lo, hi = both.amin(-1), both.amax(-1)
        m = lo.half()
        s = ((hi - m.float()) / (2 ** b - 1)).half()
        s = torch.where(s == 0, torch.ones_like(s), s)
        code = ((both - m.float()[..., None]) * (1.0 / s.float())[..., None]).round().clamp(0, 2 ** b - 1).to(torch.uint8).flatten(-2)
        real = torch.cat([torch.arange(-(-t // 32) * 32, device="cuda") < t for t in per_class[k]]) if padded[k] else torch.zeros(0, dtype=torch.bool, device="cuda")
        x["classes"].append((code * real[None, :, None, None], s * real[None, :, None, None], m * real[None, :, None, None]))
    x["k16"], x["k_own"] = keys[3].to(t16), keys[4].to(t16)
    x["v16"], x["v_own"] = g.normal(*keys[3].shape).to(t16), g.normal(*keys[4].shape).to(t16)
    return x


def _bytes(fields, b):
    f = fields.reshape(-1, 8 // b).int()
    shift = torch.arange(0, 8, b, device="cuda", dtype=torch.int32)
    return (f << shift).sum(-1).to(torch.uint8)


def _packed(c, k, code, s, m):
    """A class in the storage format: bytes [plane][head][...] and metadata words [plane][head][...]."""
    Hkv, hd, b = c["kv_heads"], c["head_dim"], BITS[k]
    cap = code.shape[1]
    if cap == 0:
        return torch.zeros(2, Hkv, 0, dtype=torch.uint8, device="cuda"), torch.zeros(2, Hkv, 0, dtype=torch.int32, device="cuda")
    kk = code[0].view(cap // 16, 16, Hkv, 4, hd // 4).permute(2, 0, 3, 1, 4)
    vv = code[1].view(cap // 32, 2, 4, 4, Hkv, hd // 16, 16).permute(4, 0, 2, 6, 5, 1, 3)
    words = (s.view(torch.int16).int() & 0xFFFF) | (m.view(torch.int16).int() << 16)
    words = words.view(2, cap // 16, 16, Hkv, -1).permute(0, 3, 1, 4, 2)
    return torch.stack([_bytes(kk.reshape(Hkv, -1), b), _bytes(vv.reshape(Hkv, -1), b)]).view(2, Hkv, -1), words.reshape(2, Hkv, -1).contiguous()


def prepare(c, seed):
    x = _make(c, seed)
    H, Hkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    st = dict(case=c, scale=1.0 / math.sqrt(hd))
    if own:
        from paper_2605_02262_amd import binding as W
        st["W"] = W
    if c["kind"] in ("rope", "append"):
        qkv = x["qkv"]
        st["q"], st["k"], st["v"] = (qkv[:, a * hd:z * hd].unflatten(-1, (-1, hd)) for a, z in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
        st["positions"] = x["positions"]
        st["inv_freq"], st["mscale"] = _frequencies(c)
        if own:
            st["ctx"] = W.Context(W.workspace_bytes())
            st["layout"] = W.ROPE_HALF if c["layout"] == "half" else W.ROPE_PAIRS
        if c["kind"] == "append":
            t16 = torch.bfloat16 if c["dtype"] == "bf16" else torch.float16
            room = c["held"] + 16
            st["off16"] = _i32([b * room for b in range(c["batch"] + 1)])
            st["held"] = _i32([c["held"] - b % 3 % c["held"] for b in range(c["batch"])])
            st["len16"] = st["held"].clone()
            st["k16"] = torch.zeros(c["batch"] * room, Hkv, hd, dtype=t16, device="cuda")
            st["v16"] = torch.zeros_like(st["k16"])
            if own:
                st["kv"] = _cache(W, c, c["batch"], hd, [0, 0, 0], [b * room for b in range(c["batch"] + 1)], st["k16"], st["v16"], st["held"].tolist())
        return st
    if c["kind"] == "prefill":
        new, rows, prefix = _prefill_sizes(c)
        st.update(x, q_off=_i32(_sum(new)), kv_off=_i32(_sum(rows)), prefix=_i32(prefix) if c["prefix"] else None, longest_q=max(new), longest=max(rows))
        if own:
            st["ctx"] = W.Context(W.prefill_workspace_bytes(sum(new), c["batch"], H, Hkv, hd, max(rows)))
        return st
    tokens, n, rows = _shared_sizes(c)
    st["q"] = x["q"]
    laid = [_packed(c, k, *x["classes"][k]) for k in range(3)]
    st["codes"], st["meta"] = [p[0] for p in laid], [p[1] for p in laid]
    st["cls_off"] = [_i32(_sum([-(-p[k] // 32) * 32 for p in tokens])) for k in range(3)]
    st["cls_len"] = [_i32([p[k] for p in tokens]) for k in range(3)]
    st["k16"], st["v16"], st["k_own"], st["v_own"] = x["k16"], x["v16"], x["k_own"], x["v_own"]
    off16, off_own = _sum([p[3] for p in tokens]), _sum(rows)
    st["off16"], st["len16"], st["off_own"], st["len_own"] = _i32(off16), _i32([p[3] for p in tokens]), _i32(off_own), _i32(rows)
    st["req_off"] = _i32(_sum(n))
    st["longest"], st["longest_own"], st["most"] = max(sum(p) for p in tokens), max(rows), max(n)
    if own:
        cap = [v.shape[1] for v in (x["classes"][k][0] for k in range(3))]
        kv = _cache(W, c, c["prefixes"], c["group"], cap, off16, st["k16"], st["v16"], [p[3] for p in tokens])
        largest = [0.0] * c["prefixes"]
        for k in range(3):
            kv.codes[k].copy_(st["codes"][k])
            kv.meta[k].copy_(st["meta"][k])
            kv.cls_off[k].copy_(st["cls_off"][k])
            kv.cls_len[k].copy_(st["cls_len"][k])
            at = st["cls_off"][k].tolist()
            for p in range(c["prefixes"]):
                if at[p + 1] > at[p]:
                    largest[p] = max(largest[p], float(x["classes"][k][1][1, at[p]:at[p + 1]].abs().max()))
        kv.v_scale_max[:c["prefixes"]] = torch.tensor(largest, device="cuda")
        st["kv"] = kv
        st["mine"] = _cache(W, c, c["batch"], c["group"], [0, 0, 0], off_own, st["k_own"], st["v_own"], rows)
        st["ctx"] = W.Context(W.shared_workspace_bytes(c["batch"], c["prefixes"], H, Hkv, hd, st["longest"], st["longest_own"]))
    return st


def _cache(W, c, B, group, cap, off16, k16, v16, len16):
    kv = W.PackedKV(B, c["kv_heads"], c["head_dim"], group, k16.dtype, cap, off16)
    kv.k16.copy_(k16)
    kv.v16.copy_(v16)
    kv.len16.copy_(_i32(len16))
    return kv


# ------------------------------------------------------------------------------------------------------------------------
# the operators
# ------------------------------------------------------------------------------------------------------------------------
def run(st):
    return (_own_pass if own else _plain_pass)(st)


def _own_pass(st):
    W, c = st["W"], st["case"]
    if c["kind"] == "rope":
        return W.wq_rope(st["ctx"], st["q"], st["k"], st["positions"], st["inv_freq"], layout=st["layout"], mscale=st["mscale"])
    if c["kind"] == "append":
        kv = st["kv"]
        kv.len16.copy_(st["held"])      # a drafted token that is taken back, so that the pass can be repeated
        q = W.wq_rope_append_kv(st["ctx"], st["q"], st["k"], st["v"], st["positions"], st["inv_freq"], kv, layout=st["layout"], mscale=st["mscale"])
        return q, kv.k16, kv.v16, kv.len16
    if c["kind"] == "prefill":
        lse = torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda") if c["lse"] else None
        out = W.wq_prefill_attention(st["ctx"], st["q"], st["k"], st["v"], st["q_off"], st["kv_off"], st["scale"], prefix_len=st["prefix"],
                                     max_kv_rows=st["longest"], lse=lse)
        return (out, lse) if c["lse"] else out
    return W.wq_decode_attention_shared(st["ctx"], st["q"], st["kv"], st["req_off"], st["mine"], st["scale"], max_prefix_tokens=st["longest"],
                                        max_own_tokens=st["longest_own"])


def _plain_pass(st):
    return {"rope": _plain_rope, "append": _plain_append, "prefill": _plain_prefill, "shared": _plain_shared}[st["case"]["kind"]](st)


def _turned(c, x, cos, sin):
    rot, x = _rot(c), x.float()
    head, rest = x[..., :rot], x[..., rot:]
    if c["layout"] == "half":
        a, b = head.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _plain_angles(st):
    angle = st["positions"].double()[:, None, None] * st["inv_freq"].double()     # far positions: fp32 would lose the angle
    return (angle.cos() * st["mscale"]).float(), (angle.sin() * st["mscale"]).float()


def _plain_rope(st):
    cos, sin = _plain_angles(st)
    return tuple(_turned(st["case"], x, cos, sin).to(x.dtype) for x in (st["q"], st["k"]))


def _plain_append(st):
    st["len16"].copy_(st["held"])
    q, k = _plain_rope(st)
    row = (st["off16"][:-1] + st["len16"]).long()
    st["k16"][row] = k.to(st["k16"].dtype)
    st["v16"][row] = st["v"].to(st["v16"].dtype)
    st["len16"] += 1
    return q, st["k16"], st["v16"], st["len16"]


def _padded(x, off, most):
    """Ragged rows as a padded batch, and which of its rows are real."""
    at = off[:-1, None] + torch.arange(most, device="cuda")
    real = at < off[1:, None]
    return x[at.clamp(max=max(x.shape[0] - 1, 0)).long()].float(), real


def _plain_prefill(st):
    c = st["case"]
    H, Hkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    q, new = _padded(st["q"], st["q_off"], st["longest_q"])
    k, there = _padded(st["k"], st["kv_off"], st["longest"])
    v, _ = _padded(st["v"], st["kv_off"], st["longest"])
    B, Lq, L = q.shape[0], q.shape[1], k.shape[1]
    q = q.view(B, Lq, Hkv, H // Hkv, hd).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, hd)
    s = torch.matmul(q * st["scale"], k.permute(0, 2, 3, 1).contiguous())                       # [B, Hkv, rep * Lq, L]
    first = (st["kv_off"].diff() - st["q_off"].diff())[:, None, None]
    i, j = torch.arange(Lq, device="cuda")[:, None], torch.arange(L, device="cuda")
    seen = j <= first + i
    if st["prefix"] is not None:
        seen = seen | (j < st["prefix"][:, None, None])
    seen = seen & there[:, None, :]
    s.view(B, Hkv, -1, Lq, L).masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    s.sub_(m).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s, v.permute(0, 2, 1, 3).contiguous()) / total.clamp(min=1e-38)
    o = o.view(B, Hkv, -1, Lq, hd).permute(0, 3, 1, 2, 4).reshape(B * Lq, H, hd)
    of = torch.arange(B, device="cuda").repeat_interleave(st["q_off"].diff(), output_size=st["q"].shape[0])     # every row's sequence
    at = of * Lq + torch.arange(st["q"].shape[0], device="cuda") - st["q_off"][of]
    out = o[at].to(st["q"].dtype)
    if not c["lse"]:
        return out
    lse = (m + total.log()).view(B, H, Lq).transpose(1, 2).reshape(B * Lq, H)
    return out, lse[at]


def _fields(b, x):
    shift = torch.arange(0, 8, b, device="cuda", dtype=torch.int32)
    return ((x.int()[..., None] >> shift) & (2 ** b - 1)).flatten(-2)


def _unpacked(c, codes, meta, b):
    """fp32 keys and values [token, head, channel] of one class."""
    Hkv, hd, G = c["kv_heads"], c["head_dim"], c["head_dim"] // c["group"]
    cap = meta.shape[-1] // G
    k = _fields(b, codes[0]).view(Hkv, cap // 16, 4, 16, hd // 4).permute(1, 3, 0, 2, 4).reshape(cap, Hkv, hd)
    v = _fields(b, codes[1]).view(Hkv, cap // 32, 4, 16, hd // 16, 2, 4).permute(1, 5, 2, 6, 0, 4, 3).reshape(cap, Hkv, hd)
    w = meta.view(2, Hkv, cap // 16, G, 16).permute(0, 2, 4, 1, 3).reshape(2, cap, Hkv, G)
    s, m = (w & 0xFFFF).to(torch.int16).view(torch.float16).float(), (w >> 16).to(torch.int16).view(torch.float16).float()
    return [((x.view(cap, Hkv, G, -1) * s[p][..., None]) + m[p][..., None]).view(cap, Hkv, hd) for p, x in ((0, k), (1, v))]


def _plain_shared(st):
    c = st["case"]
    H, Hkv, hd, B = c["heads"], c["kv_heads"], c["head_dim"], c["batch"]
    rep, P = H // Hkv, c["prefixes"]
    parts = [_unpacked(c, st["codes"][k], st["meta"][k], b) for k, b in enumerate(BITS) if st["meta"][k].numel()]
    zero = torch.zeros(1, Hkv, hd, device="cuda")
    k, v = (torch.cat([p[i] for p in parts] + [st[n].float(), zero]) for i, n in ((0, "k16"), (1, "v16")))
    # the row of every token of every prefix: 2-, 4-, 8-, 16-bit tokens one after the other
    lens = torch.stack(st["cls_len"] + [st["len16"]]).long()                                    # [4, P]
    starts = torch.stack([o[:-1] for o in st["cls_off"]] + [st["off16"][:-1]]).long()
    caps = [st["meta"][i].shape[-1] // (hd // c["group"]) for i in range(3)]
    starts = starts + torch.tensor(_sum(caps), device="cuda")[:, None]
    ends = lens.cumsum(0)
    t = torch.arange(st["longest"], device="cuda")
    which = (t >= ends[:3, :, None]).sum(0)                                                     # [P, L]
    row = t + (starts - (ends - lens)).T.gather(1, which)
    there = t < ends[3][:, None]
    row = torch.where(there, row, k.shape[0] - 1)
    kp, vp = k[row].permute(0, 2, 3, 1).contiguous(), v[row].permute(0, 2, 1, 3).contiguous()   # [P, Hkv, hd, L], [P, Hkv, L, hd]
    # requests by prefix
    slot = st["req_off"][:-1, None] + torch.arange(st["most"], device="cuda")
    used = slot < st["req_off"][1:, None]
    slot = slot.clamp(max=B - 1).long()                                                         # [P, n]
    q = st["q"].float().view(B, Hkv, rep, hd) * st["scale"]
    qp = q[slot].transpose(1, 2).reshape(P, Hkv, -1, hd)
    sp = torch.matmul(qp, kp).view(P, Hkv, -1, rep, st["longest"])
    sp.masked_fill_(~there[:, None, None, None], -math.inf)
    ko, real = _padded(st["k_own"], st["off_own"], st["longest_own"])
    vo, _ = _padded(st["v_own"], st["off_own"], st["longest_own"])
    so = torch.matmul(q, ko.permute(0, 2, 3, 1).contiguous())                                   # [B, Hkv, rep, Lo]
    so.masked_fill_(~real[:, None, None], -math.inf)
    so = so[slot].transpose(1, 2)                                                               # [P, Hkv, n, rep, Lo]
    m = torch.maximum(sp.amax(-1), so.amax(-1))[..., None]
    ep, eo = sp.sub_(m).exp_(), (so - m).exp_()
    o = torch.matmul(ep.flatten(2, 3), vp).view(P, Hkv, -1, rep, hd) + torch.matmul(eo, vo.transpose(1, 2).contiguous()[slot].transpose(1, 2))
    o = o / (ep.sum(-1, keepdim=True) + eo.sum(-1, keepdim=True))
    out = torch.zeros(B, Hkv, rep, hd, device="cuda")
    out[slot[used]] = o.transpose(1, 2)[used]
    return out.view(B, H, hd).to(st["q"].dtype)


# ------------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------------------------------
def exact(c, seed):
    x = _make(c, seed)
    H, Hkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    rep = H // Hkv
    if c["kind"] in ("rope", "append"):
        inv, mscale = _frequencies(c)
        turn = torch.polar(torch.tensor(mscale, dtype=torch.float64, device="cuda"), x["positions"].double()[:, None] * inv.double())[:, None]
        heads = x["qkv"].view(-1, H + 2 * Hkv, hd)[:, :H + Hkv].double()
        done = heads.clone()
        rot = _rot(c)
        pairs = (slice(0, rot // 2), slice(rot // 2, rot)) if c["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        z = torch.complex(heads[..., pairs[0]], heads[..., pairs[1]]) * turn
        done[..., pairs[0]], done[..., pairs[1]] = z.real, z.imag
        if c["kind"] == "rope":
            return done[:, :H], done[:, H:]
        room = c["held"] + 16
        k16 = torch.zeros(c["batch"], room, Hkv, hd, dtype=torch.float64, device="cuda")
        v16 = torch.zeros_like(k16)
        for b in range(c["batch"]):
            n = c["held"] - b % 3 % c["held"]
            k16[b, n], v16[b, n] = done[b, H:], x["qkv"].view(-1, H + 2 * Hkv, hd)[b, H + Hkv:].double()
        return done[:, :H], k16.flatten(0, 1), v16.flatten(0, 1), None
    if c["kind"] == "prefill":
        new, rows, prefix = _prefill_sizes(c)
        outs, sums = [], []
        for b in range(c["batch"]):
            qs, ks = slice(sum(new[:b]), sum(new[:b + 1])), slice(sum(rows[:b]), sum(rows[:b + 1]))
            q, k, v = x["q"][qs].double(), x["k"][ks].double(), x["v"][ks].double()
            pos = torch.arange(rows[b] - new[b], rows[b], device="cuda")[:, None]
            key = torch.arange(rows[b], device="cuda")
            hidden = (key > pos) & (key >= prefix[b])
            o, l = torch.empty_like(q), torch.empty(new[b], H, dtype=torch.float64, device="cuda")
            for h in range(H):
                logit = (q[:, h] @ k[:, h // rep].T) / math.sqrt(hd)
                logit[hidden] = -math.inf
                l[:, h] = torch.logsumexp(logit, -1)
                o[:, h] = torch.exp(logit - l[:, h:h + 1]) @ v[:, h // rep]
            outs.append(o)
            sums.append(l)
        return (torch.cat(outs), torch.cat(sums)) if c["lse"] else torch.cat(outs)
    tokens, n, rows = _shared_sizes(c)
    wide = [(code.double().unflatten(-1, (-1, c["group"])) * s.double()[..., None] + m.double()[..., None]).flatten(-2) for code, s, m in x["classes"]]
    at, at16, at_own, b = [0, 0, 0], 0, 0, 0
    outs = []
    for p in range(c["prefixes"]):
        kv = [wide[i][:, at[i]:at[i] + tokens[p][i]] for i in range(3)]
        kv.append(torch.stack([x["k16"], x["v16"]])[:, at16:at16 + tokens[p][3]].double())
        at = [a + -(-t // 32) * 32 for a, t in zip(at, tokens[p])]
        at16 += tokens[p][3]
        kv = torch.cat(kv, 1)
        for _ in range(n[p]):
            mine = torch.stack([x["k_own"], x["v_own"]])[:, at_own:at_own + rows[b]].double()
            at_own += rows[b]
            q = x["q"][b].double().view(Hkv, rep, hd)
            logit = torch.cat([q @ kv[0].permute(1, 2, 0), q @ mine[0].permute(1, 2, 0)], -1) / math.sqrt(hd)
            w = torch.softmax(logit, -1)
            outs.append((w[..., :kv.shape[1]] @ kv[1].transpose(0, 1) + w[..., kv.shape[1]:] @ mine[1].transpose(0, 1)).reshape(H, hd))
            b += 1
    return torch.stack(outs)
