"""Four operators of drafted decoding over the packed cache, and of a batch whose sequences come and go, as cases that can
be timed and compared.

A case is a dict of plain values.  Its `kind` is the operator that one pass runs:

  tree     attention of several new rows per sequence: every row sees its sequence's whole packed cache and, among the new
           rows, itself and its ancestors in a tree of drafted tokens (or, without a tree, all rows before it: a chain of
           drafted tokens, the rows of a further question)
  accept   which drafted tokens the model agrees with: the walk from the tree's first row along the tokens that it chose
  append   the keys and values of the rows that stay, copied behind the 16-bit rows of all layers' caches
  copy     sequences of packed caches copied into other caches of all layers, laid out afresh: the same one several
           times (a fork), some of them (compaction), others left out (freed)

Sizes are those of the configurations (14 query / 2 KV heads of 64 and 28 / 4 of 128; 28 layers; frames of 98 and 196 tokens,
windows of 16 and 32; prompts of 16 to 512 tokens) or generic.
"""
import math
import random

import torch

own = False     # True: the framework's calls instead of their plain form

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SMALL = dict(heads=14, kv_heads=2, head_dim=64)
LARGE = dict(heads=28, kv_heads=4, head_dim=128)
BITS = (2, 4, 8)
VOCABULARY = 1 << 17


def _tree(**more):
    return dict(dict(kind="tree", batch=8, windows=64, window=196, text=256, top=20, mid=50, top_bits=8, group=64, rows=16, tree=True, forest=False, ragged=0,
                     lse=False, dtype="bf16", **LARGE), **more)


def _accept(**more):
    return dict(dict(kind="accept", batch=8, rows=64, tree=True, max_path=16, agree=80, ragged=0), **more)


def _append(**more):
    return dict(dict(kind="append", layers=28, batch=8, rows=64, take=6, held=500, ragged=0, dtype="bf16", **LARGE), **more)


def _copy(**more):
    return dict(dict(kind="copy", layers=1, batch=8, keep=8, fork=False, windows=0, window=196, text=200, top=20, mid=50, top_bits=8, group=64, ragged=0,
                     dtype="bf16", **LARGE), **more)


def listed():
    return [
        # the tiny configuration in fp32: three requests, trees of seven drafted tokens
        _tree(name="tree_tiny_f32", batch=3, windows=8, window=16, text=16, top=25, group=32, rows=7, dtype="f32", **SMALL),
        # one user: a video with a 16-bit top tier and windows of 32, a tree of 26 tokens, fp16
        _tree(name="tree_one_user_f16", batch=1, windows=612, window=32, text=135, top=0.4, mid=35, top_bits=16, rows=26, dtype="f16"),
        # eight requests about 64 frames each, trees of 16 tokens
        _tree(name="tree_batch8"),
        # four long videos, trees of 64 tokens
        _tree(name="tree_long_videos", batch=4, windows=256, text=512, top=10, mid=40, rows=64),
        # a batch of 32 clips of many lengths, five tokens drafted in a row
        _tree(name="chain_ragged32", batch=32, windows=128, window=98, text=77, top=25, mid=40, rows=5, tree=False, ragged=515, lse=True),
        # five conversations of a small model: the rows of a further question, of many lengths, fp16
        _tree(name="question_rows_f16", batch=5, windows=33, text=301, group=32, rows=389, tree=False, ragged=77, dtype="f16", **SMALL),
        # a step of eight requests with trees of 64 tokens (the smallest call, latency)
        _accept(name="accept_batch8"),
        # a large batch with trees of up to 255 tokens
        _accept(name="accept_batch512", batch=512, rows=255, ragged=99, max_path=32, agree=93),
        # eight requests' accepted tokens, up to six each, into 28 layers' caches
        _append(name="append_accepted", ragged=31),
        # a further question of 512 tokens of four requests, into 28 layers' caches
        _append(name="append_question", batch=4, rows=512, take=0, held=900),
        # eight beams of a small model, forked after a step: their 16-bit rows of 24 layers
        _copy(name="copy_fork_beams", layers=24, keep=8, fork=True, ragged=5, **SMALL),
        # 32 ragged videos of which 23 stay, one layer
        _copy(name="copy_compact32", batch=32, keep=23, windows=128, window=196, text=400, ragged=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    kind = rng.choice(["tree"] * 6 + ["accept", "append", "append", "copy", "copy"])
    model = dict(rng.choice([SMALL, LARGE, LARGE, dict(heads=32, kv_heads=8, head_dim=128), dict(heads=8, kv_heads=8, head_dim=64)]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
    hd = model["head_dim"]
    video = dict(window=rng.choice([16, 32, 98, 196]), top=rng.choice([0, 10, 20, 25, 100]), group=rng.choice([hd // 2, hd // 2, hd, 32]),
                 top_bits=rng.choice([8, 8, 8, 16]))
    video["mid"] = rng.choice([m for m in (0, 20, 40, 50) if m + video["top"] <= 100])
    ragged = rng.randrange(1, 1 << 20) if rng.random() < 0.5 else 0
    if kind == "tree":
        c = _tree(batch=_log(rng, 1, 48), rows=rng.choice([1, _log(rng, 2, 100), _log(rng, 2, 100)]), text=_log(rng, 1, 600), tree=rng.random() < 0.65,
                  forest=rng.random() < 0.3, ragged=ragged, lse=rng.random() < 0.3, dtype=dtype, **video, **model)
        if rng.random() < 0.25:
            c["rows"] = _log(rng, 65, 255 if c["tree"] else 1500)
        c["windows"] = max(1, _log(rng, 100, 60000) // c["window"])
    elif kind == "accept":
        c = _accept(batch=_log(rng, 1, 600), rows=_log(rng, 1, 1000), tree=rng.random() < 0.8, max_path=_log(rng, 1, 40), agree=rng.choice([50, 80, 95]), ragged=ragged)
    elif kind == "append":
        c = _append(layers=_log(rng, 1, 80), batch=_log(rng, 1, 64), rows=_log(rng, 1, 600), held=_log(rng, 1, 1000), ragged=ragged, dtype=dtype, **model)
        c["take"] = rng.choice([0, rng.randint(1, min(c["rows"], 24))])
    else:
        c = _copy(layers=rng.choice([1, 1, _log(rng, 1, 32)]), batch=_log(rng, 1, 48), fork=rng.random() < 0.5, text=_log(rng, 1, 600), ragged=ragged,
                  dtype=rng.choice(["bf16", "f16"]), **video, **model)
        c["windows"] = rng.choice([0, max(1, _log(rng, 100, 30000) // c["window"])])
        c["keep"] = _log(rng, 1, 48) if c["fork"] else rng.randint(1, c["batch"])
    while _cost(c) > most:
        if c["kind"] == "append":
            c["layers"], c["rows"] = (c["layers"] * 3 // 4, c["rows"]) if c["layers"] > 4 else (c["layers"], max(c["take"], c["rows"] * 3 // 4))
        elif c["kind"] == "copy" and c["layers"] > 1:
            c["layers"] = c["layers"] * 3 // 4
        elif c["batch"] > 4:
            c["batch"] -= c["batch"] // 4
            if c["kind"] == "copy":
                c["keep"] = min(c["keep"], c["batch"])
        elif c["kind"] == "tree" and c["rows"] > 40:
            c["rows"] = c["rows"] * 3 // 4
        else:
            c["windows"] = c["windows"] * 3 // 4
    return c


# ------------------------------------------------------------------------------------------------------------------------
# sizes
# ------------------------------------------------------------------------------------------------------------------------
def _sum(v):
    return [sum(v[:i]) for i in range(len(v) + 1)]


def _spread(rng, c, most, least=1):
    return rng.randint(max(least, most // 8), most) if c["ragged"] else most


def _cache_sizes(c):
    """Per sequence its 2-, 4-, 8- and 16-bit tokens."""
    rng = random.Random(c["ragged"])
    tokens = []
    for _ in range(c["batch"]):
        w = _spread(rng, c, c["windows"], 0) if c["windows"] else 0
        top, both = int(c["top"] * w / 100 + 0.5), int((c["top"] + c["mid"]) * w / 100 + 0.5)
        t = [(w - both) * c["window"], (both - top) * c["window"], top * c["window"], _spread(rng, c, c["text"])]
        if c["top_bits"] == 16:
            t[3] += t[2]
            t[2] = 0
        tokens.append(t)
    return tokens


def _row_sizes(c):
    rng = random.Random(c["ragged"] + 1)
    return [_spread(rng, c, c["rows"]) for _ in range(c["batch"])]


def _parents(c):
    """Per sequence the row's parent among the sequence's rows, -1 for none."""
    rng = random.Random(c["ragged"] + 2)
    out = []
    for n in _row_sizes(c):
        p = [rng.randrange(i) if i else -1 for i in range(n)]
        if c.get("forest"):                     # the last accepted token is in the cache already: the first level has no parent
            p = [-1 if i < max(1, n // 6) else x for i, x in enumerate(p)]
        out.append(p)
    return out


def _seen(c):
    """Per sequence, over its new rows: how many new rows each sees (of one head), summed."""
    if not c["tree"]:
        return [n * (n + 1) // 2 for n in _row_sizes(c)]
    total = []
    for p in _parents(c):
        depth = []
        for x in p:
            depth.append(1 if x < 0 else depth[x] + 1)
        total.append(sum(depth))
    return total


def _take_sizes(c):
    """Per sequence, how many rows are appended."""
    rows, rng = _row_sizes(c), random.Random(c["ragged"] + 3)
    return [min(n, _spread(rng, c, c["take"])) for n in rows] if c["take"] else rows


def _from(c):
    """The sequence that each sequence of the copy is made of."""
    rng = random.Random(c["ragged"] + 4)
    if c["fork"]:
        return [rng.randrange(c["batch"]) for _ in range(c["keep"])]
    return sorted(rng.sample(range(c["batch"]), c["keep"]))


def _token_bytes(c, t, b):
    return t * 2 * c["kv_heads"] * (c["head_dim"] * b // 8 + (4 * c["head_dim"] // c["group"] if b < 16 else 0))


def work(c):
    if c["kind"] == "accept":
        n = sum(_row_sizes(c))
        return dict(bytes=4 * n * (3 if c["tree"] else 2) + 4 * c["batch"] * (c["max_path"] + 2), flops=n)
    H, Hkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    size = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "append":
        n = sum(_take_sizes(c)) * c["layers"] * 2 * Hkv * hd
        return dict(bytes=n * (size + 2), flops=n)
    tokens = _cache_sizes(c)
    cached = [sum(_token_bytes(c, t, b) for t, b in zip(p, BITS + (16,))) for p in tokens]
    if c["kind"] == "copy":
        n = c["layers"] * sum(cached[s] for s in _from(c))
        return dict(bytes=2 * n, flops=n // 4)
    rows = _row_sizes(c)
    pairs = sum(n * sum(p) for n, p in zip(rows, tokens)) + sum(_seen(c))
    return dict(bytes=sum(cached) + sum(rows) * (2 * H + 2 * Hkv) * hd * size, flops=4 * H * hd * pairs)


def _cost(c):
    """Time of a pass as far as sizes tell it; the plain form's padding is charged for."""
    w = work(c)
    if c["kind"] != "tree":
        return w["bytes"]
    longest, rows = max(sum(p) for p in _cache_sizes(c)), max(_row_sizes(c))
    return max(w["bytes"], w["flops"] / 50, 4 * c["heads"] * c["head_dim"] * c["batch"] * rows * (longest + rows) / 80)


# ------------------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------------------
def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.rng = random.Random(seed)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")


def _cached(g, c, tokens, scale):
    """The packed tokens as codes, scales and minima per class, [plane, token slot, head, ...], and the 16-bit rows [plane, row, head, channel]."""
    t16 = torch.bfloat16 if c["dtype"] == "bf16" else torch.float16
    Hkv, hd = c["kv_heads"], c["head_dim"]
    classes = []
    for k, b in enumerate(BITS):
        padded = [-(-p[k] // 32) * 32 for p in tokens]
        both = g.normal(2, sum(padded), Hkv, hd)
        both[0] *= scale
        both = both.to(t16).float().unflatten(-1, (-1, c["group"]))
        lo, hi = both.amin(-1), both.amax(-1)
        m = lo.half()
        s = ((hi - m.float()) / (2 ** b - 1)).half()
        s = torch.where(s == 0, torch.ones_like(s), s)
        code = ((both - m.float()[..., None]) * (1.0 / s.float())[..., None]).round().clamp(0, 2 ** b - 1).to(torch.uint8).flatten(-2)
        real = torch.cat([torch.arange(n, device="cuda") < p[k] for n, p in zip(padded, tokens)])
        classes.append((code * real[None, :, None, None], s * real[None, :, None, None], m * real[None, :, None, None]))
    rows = g.normal(2, sum(p[3] for p in tokens), Hkv, hd)
    rows[0] *= scale
    return classes, rows.to(t16)


def _make(c, seed):
    """The inputs in logical form (before anything is laid out)."""
    g = _Draws(seed)
    if c["kind"] == "accept":
        tokens, target = [], []
        for n, p in zip(_row_sizes(c), _parents(c) if c["tree"] else [range(-1, k - 1) for k in _row_sizes(c)]):
            tok = [g.rng.randrange(VOCABULARY) for _ in range(n)]
            children = {}
            for i, x in enumerate(p):
                children.setdefault(x, []).append(i)
            tokens += tok
            target += [tok[g.rng.choice(children[i])] if i in children and g.rng.random() * 100 < c["agree"] else g.rng.randrange(VOCABULARY) for i in range(n)]
        return dict(tokens=tokens, target=target)
    H, Hkv, hd, dt = c["heads"], c["kv_heads"], c["head_dim"], DTYPES[c["dtype"]]
    if c["kind"] == "append":
        n = sum(_row_sizes(c))
        take = [sorted(g.rng.sample(range(r), k)) if c["take"] else list(range(r)) for r, k in zip(_row_sizes(c), _take_sizes(c))]
        return dict(qkv=[g.normal(n, (H + 2 * Hkv) * hd).to(dt) for _ in range(c["layers"])], take=take)
    tokens = _cache_sizes(c)
    scale = torch.exp(g.normal(Hkv, hd))        # keys have channels of very different size
    if c["kind"] == "copy":
        return dict(layers=[_cached(g, c, tokens, scale) for _ in range(c["layers"])])
    x = dict(zip(("classes", "rows16"), _cached(g, c, tokens, scale)))
    fit = (2 * math.sqrt(hd) / scale.norm(dim=-1)).repeat_interleave(H // Hkv)[:, None]       # scaled products of deviation 2
    qkv = g.normal(sum(_row_sizes(c)), H + 2 * Hkv, hd)
    qkv[:, :H] *= fit
    qkv[:, H:H + Hkv] *= scale
    x["qkv"] = qkv.to(dt).flatten(1)
    return x


def _split(c, qkv):
    H, Hkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    return [qkv[:, a * hd:z * hd].unflatten(-1, (-1, hd)) for a, z in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv))]


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


class _Cache:
    """One layer's packed cache as a program holds it: its buffers and tables, and the framework's handle of them where `own` is true."""

    def __init__(self, c, tokens, classes=None, rows16=None, cap=None, room=None):
        B, Hkv, hd, G = len(tokens), c["kv_heads"], c["head_dim"], c["head_dim"] // c["group"]
        t16 = torch.bfloat16 if c["dtype"] == "bf16" else torch.float16
        off16 = _sum(room or [p[3] for p in tokens])
        if cap is None:
            cap = [sum(-(-p[k] // 32) * 32 for p in tokens) for k in range(3)]
        if own:
            from paper_2605_02262_amd import binding as W
            self.kv = W.PackedKV(B, Hkv, hd, c["group"], t16, cap, off16, fill=0)
            for n in ("codes", "meta", "cls_off", "cls_len", "off16", "len16", "k16", "v16", "v_scale_max"):
                setattr(self, n, getattr(self.kv, n))
        else:
            self.codes = [torch.zeros(2, Hkv, n * hd * b // 8, dtype=torch.uint8, device="cuda") for n, b in zip(cap, BITS)]
            self.meta = [torch.zeros(2, Hkv, n * G, dtype=torch.int32, device="cuda") for n in cap]
            self.cls_off, self.cls_len = [_i32([0] * (B + 1)) for _ in cap], [_i32([0] * B) for _ in cap]
            self.off16, self.len16 = _i32(off16), _i32([0] * B)
            self.k16, self.v16 = (torch.zeros(off16[-1], Hkv, hd, dtype=t16, device="cuda") for _ in range(2))
            self.v_scale_max = torch.zeros(B, device="cuda")
        if classes is None:
            return
        largest = [0.0] * B
        for k, (code, s, m) in enumerate(classes):
            codes, meta = _packed(c, k, code, s, m)
            self.codes[k].copy_(codes)
            self.meta[k].copy_(meta)
            at = _sum([-(-p[k] // 32) * 32 for p in tokens])
            self.cls_off[k].copy_(_i32(at))
            self.cls_len[k].copy_(_i32([p[k] for p in tokens]))
            for b in range(B):
                if at[b + 1] > at[b]:
                    largest[b] = max(largest[b], float(s[1, at[b]:at[b + 1]].abs().max()))
        self.v_scale_max[:B] = torch.tensor(largest, device="cuda")
        self.len16.copy_(_i32([p[3] for p in tokens]))
        self.k16[:rows16.shape[1]].copy_(rows16[0])
        self.v16[:rows16.shape[1]].copy_(rows16[1])


def _together(caches):
    """The buffers of all layers' caches as one tensor each, as a program allocates them: [layer, ...]."""
    def stacked(name, k=None):
        at = [getattr(y, name) if k is None else getattr(y, name)[k] for y in caches]
        whole = torch.stack(at)
        for y, part in zip(caches, whole):
            for holder in (y, y.kv) if own else (y,):
                if k is None:
                    setattr(holder, name, part)
                else:
                    getattr(holder, name)[k] = part
            if own and k is None:
                setattr(y.kv.desc, name, part.data_ptr() if part.numel() else None)
            elif own:
                getattr(y.kv.desc, name)[k] = part.data_ptr() if part.numel() else None
        return whole

    whole = {name: [stacked(name, k) for k in range(3)] for name in ("codes", "meta", "cls_off", "cls_len")}
    whole.update({name: stacked(name) for name in ("k16", "v16", "len16", "v_scale_max")})
    return whole


def prepare(c, seed):
    x = _make(c, seed)
    st = dict(case=c)
    if own:
        from paper_2605_02262_amd import binding as W
        st["W"] = W
    if c["kind"] != "copy":
        rows = _row_sizes(c)
        st["row_off"], st["rows"] = _i32(_sum(rows)), max(rows)
        st["parent"] = _i32(sum(_parents(c), [])) if c.get("tree") else None
    if c["kind"] == "accept":
        st["tokens"], st["target"] = _i32(x["tokens"]), _i32(x["target"])
        if own:
            st["ctx"] = W.Context(0)
        return st
    if c["kind"] == "tree":
        tokens = _cache_sizes(c)
        st["q"], st["k"], st["v"] = _split(c, x["qkv"])
        st["cache"], st["longest"], st["scale"] = _Cache(c, tokens, x["classes"], x["rows16"]), max(sum(p) for p in tokens), 1.0 / math.sqrt(c["head_dim"])
        if own:
            st["ctx"] = W.Context(W.tree_workspace_bytes(sum(rows), c["batch"], c["heads"], c["kv_heads"], c["head_dim"], st["longest"], st["rows"]))
        return st
    if own:
        st["ctx"] = W.Context(0)
    if c["kind"] == "append":
        c16 = dict(c, group=c["head_dim"])
        st["k"], st["v"] = zip(*(_split(c, y)[1:] for y in x["qkv"]))
        most = max(len(t) for t in x["take"])
        st["take"] = _i32([t + [-1] * (most - len(t)) for t in x["take"]]) if c["take"] else None
        st["n_take"] = _i32([len(t) for t in x["take"]]) if c["take"] else None
        st["most"] = most
        st["held"] = _i32([c["held"] - b % 3 % c["held"] for b in range(c["batch"])])
        st["cache"] = [_Cache(c16, [[0, 0, 0, 0]] * c["batch"], room=[c["held"] + most + 1] * c["batch"]) for _ in range(c["layers"])]
        st["whole"] = _together(st["cache"])
        return st
    tokens, src = _cache_sizes(c), _from(c)
    st["from"] = _i32(src)
    st["cache"] = [_Cache(c, tokens, *layer) for layer in x["layers"]]
    cap = [sum(-(-tokens[s][k] // 32) * 32 for s in src) for k in range(3)]
    st["to"] = [_Cache(c, [tokens[s] for s in src], cap=cap, room=[tokens[s][3] + 16 for s in src]) for _ in range(c["layers"])]
    st["whole"] = _together(st["to"])
    return st


# ------------------------------------------------------------------------------------------------------------------------
# the operators
# ------------------------------------------------------------------------------------------------------------------------
def run(st):
    return (_own_pass if own else _plain_pass)(st)


def _own_pass(st):
    W, c = st["W"], st["case"]
    if c["kind"] == "tree":
        lse = torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda") if c["lse"] else None
        out = W.wq_tree_attention(st["ctx"], st["q"], st["k"], st["v"], st["cache"].kv, st["row_off"], st["scale"], parent=st["parent"], max_rows=st["rows"],
                                  max_cache_tokens=st["longest"], lse=lse)
        return (out, lse) if c["lse"] else out
    if c["kind"] == "accept":
        return W.wq_tree_accept(st["ctx"], st["tokens"], st["target"], st["row_off"], parent=st["parent"], max_rows=st["rows"], max_path=c["max_path"])
    if c["kind"] == "append":
        st["whole"]["len16"].copy_(st["held"])  # (drafted rows that are taken back, so that the pass can be repeated)
        W.wq_append_rows(st["ctx"], st["k"], st["v"], [y.kv for y in st["cache"]], st["row_off"], max_take=st["most"], take=st["take"], n_take=st["n_take"])
        return _appended(st)
    W.wq_copy_sequences(st["ctx"], [y.kv for y in st["cache"]], [y.kv for y in st["to"]], st["from"])
    return _copied(st)


def _appended(st):
    return st["whole"]["k16"], st["whole"]["v16"], st["whole"]["len16"]


def _copied(st):
    x = st["whole"]
    return x["codes"], x["meta"], x["cls_off"], x["cls_len"], x["k16"], x["v16"], x["len16"], x["v_scale_max"][:, :st["case"]["keep"]]


def _plain_pass(st):
    return {"tree": _plain_tree, "accept": _plain_accept, "append": _plain_append, "copy": _plain_copy}[st["case"]["kind"]](st)


def _padded(x, off, most):
    """Ragged rows as a padded batch, and which of its rows are real."""
    at = off[:-1, None] + torch.arange(most, device="cuda")
    real = at < off[1:, None]
    return x[at.clamp(max=x.shape[0] - 1).long()], real


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


def _row_of(st):
    """Every row's sequence and its number there."""
    i = torch.arange(st["total"], device="cuda")
    seq = torch.searchsorted(st["row_off"][1:], i, right=True)
    return seq, i - st["row_off"][seq]


def _plain_tree(st):
    c, y = st["case"], st["cache"]
    H, Hkv, hd, B, n = c["heads"], c["kv_heads"], c["head_dim"], c["batch"], st["rows"]
    rep, L = H // Hkv, st["longest"]
    parts = [_unpacked(c, y.codes[k], y.meta[k], b) for k, b in enumerate(BITS) if y.meta[k].numel()]
    zero = torch.zeros(1, Hkv, hd, device="cuda")
    k, v = (torch.cat([p[i] for p in parts] + [r.float(), zero]) for i, r in ((0, y.k16), (1, y.v16)))
    # the row of every token of every sequence: 2-, 4-, 8-, 16-bit tokens one after the other
    lens = torch.stack(y.cls_len + [y.len16]).long()                                            # [4, B]
    starts = torch.stack([o[:-1] for o in y.cls_off] + [y.off16[:-1]]).long()
    caps = [y.meta[i].shape[-1] // (hd // c["group"]) for i in range(3)]
    starts = starts + torch.tensor(_sum(caps), device="cuda")[:, None]
    ends = lens.cumsum(0)
    t = torch.arange(L, device="cuda")
    which = (t >= ends[:3, :, None]).sum(0)                                                     # [B, L]
    row = t + (starts - (ends - lens)).T.gather(1, which)
    there = t < ends[3][:, None]
    row = torch.where(there, row, k.shape[0] - 1)
    kn, real = _padded(st["k"], st["row_off"], n)
    vn, _ = _padded(st["v"], st["row_off"], n)
    q, _ = _padded(st["q"], st["row_off"], n)
    kk = torch.cat([k[row], kn.float()], 1).permute(0, 2, 3, 1).contiguous()                    # [B, Hkv, hd, L + n]
    vv = torch.cat([v[row], vn.float()], 1).transpose(1, 2).contiguous()
    q = (q.float() * st["scale"]).view(B, n, Hkv, rep, hd).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * rep, hd)
    # which new rows see which
    i = torch.arange(n, device="cuda")
    if st["parent"] is None:
        sees = (i <= i[:, None]).expand(B, n, n)
    else:
        parent, _ = _padded(st["parent"], st["row_off"], n)
        reach = ((i == parent[..., None]) | (i == i[:, None])).float()                          # itself and its parent
        for _ in range(max(1, n - 1).bit_length()):
            reach = (torch.matmul(reach, reach) > 0).float()
        sees = reach > 0
    sees = torch.cat([there[:, None, :].expand(B, n, L), sees & real[:, None, :]], -1)
    s = torch.matmul(q, kk)                                                                     # [B, Hkv, n * rep, L + n]
    s.view(B, Hkv, n, rep, L + n).masked_fill_(~sees[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    s.sub_(m).exp_()
    total = s.sum(-1, keepdim=True)
    o = (torch.matmul(s, vv) / total).view(B, Hkv, n, rep, hd).transpose(1, 2).reshape(B * n, H, hd)
    seq, inside = _row_of(dict(st, total=st["q"].shape[0]))
    at = seq * n + inside
    out = o[at].to(st["q"].dtype)
    if not c["lse"]:
        return out
    return out, (m + total.log()).view(B, Hkv, n, rep).transpose(1, 2).reshape(B * n, H)[at]


def _plain_accept(st):
    c, B, N = st["case"], st["case"]["batch"], st["tokens"].shape[0]
    seq, inside = _row_of(dict(st, total=N))
    first = st["row_off"][:-1].long()
    parent = st["parent"].long() if st["parent"] is not None else inside - 1
    above = first[seq] + parent
    agrees = (parent >= 0) & (st["tokens"] == st["target"][above.clamp(min=0)])
    child = torch.full((N + 1,), N, dtype=torch.long, device="cuda")                            # a row's first child that the model agrees with
    child.scatter_reduce_(0, torch.where(agrees, above, N), torch.where(agrees, torch.arange(N, device="cuda"), N), "amin")
    at, path, count, last = first, [], torch.zeros(B, dtype=torch.int32, device="cuda"), first
    for _ in range(c["max_path"]):
        path.append(torch.where(at < N, at - first, -1).int())
        count += (at < N).int()
        last = torch.where(at < N, at, last)
        at = child[at]
    return torch.stack(path, 1), count, st["target"][last]


def _plain_append(st):
    c = st["case"]
    if st["take"] is None:
        j = torch.arange(st["most"], device="cuda")
        n = st["row_off"].diff()
        take = j.expand(c["batch"], -1)
    else:
        take, n = st["take"], st["n_take"]
        j = torch.arange(st["most"], device="cuda")
    real = j < n[:, None]
    source = torch.where(real, st["row_off"][:-1, None] + take, 0).long()
    st["whole"]["len16"].copy_(st["held"])
    for y, k, v in zip(st["cache"], st["k"], st["v"]):
        last = y.k16.shape[0] - 1                                                               # a row that no sequence fills
        to = torch.where(real, (y.off16[:-1] + y.len16)[:, None] + j, last).long()
        for old, new in ((y.k16, k), (y.v16, v)):
            old[to] = torch.where(real[..., None, None], new[source], 0).to(old.dtype)
        y.len16 += n
    return _appended(st)


def _plain_copy(st):
    c, src = st["case"], st["from"].long()
    G = c["head_dim"] // c["group"]
    for a, z in zip(st["cache"], st["to"]):
        for k in range(3):
            length = a.cls_len[k][src]
            z.cls_len[k].copy_(length)
            z.cls_off[k][1:].copy_(((length + 31) // 32 * 32).cumsum(0))
            blocks = z.meta[k].shape[-1] // G // 32
            if blocks:
                j = torch.arange(blocks, device="cuda")
                d = torch.searchsorted(z.cls_off[k][1:].contiguous(), (32 * j).int(), right=True)
                block = j + (a.cls_off[k][src[d]] - z.cls_off[k][d]) // 32
                for old, new in ((z.codes[k], a.codes[k]), (z.meta[k], a.meta[k])):
                    old.view(2, c["kv_heads"], blocks, -1).copy_(new.unflatten(-1, (a.meta[k].shape[-1] // G // 32, -1))[:, :, block])
        row = torch.arange(z.k16.shape[0], device="cuda")
        d = torch.searchsorted(z.off16[1:], row, right=True)
        inside = row - z.off16[d]
        z.len16.copy_(a.len16[src])
        real = inside < z.len16[d]
        row = torch.where(real, a.off16[src[d]] + inside, 0).long()
        for old, new in ((z.k16, a.k16), (z.v16, a.v16)):
            old.copy_(torch.where(real[:, None, None], new[row], old))
        z.v_scale_max[:len(src)] = a.v_scale_max[src]
    return _copied(st)


# ------------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ------------------------------------------------------------------------------------------------------------------------
def exact(c, seed):
    if c["kind"] == "accept":
        return None                             # whole numbers
    x = _make(c, seed)
    H, Hkv, hd = c["heads"], c["kv_heads"], c["head_dim"]
    rep = H // Hkv
    if c["kind"] == "append":
        first, room, out = _sum(_row_sizes(c)), c["held"] + max(len(t) for t in x["take"]) + 1, []
        for qkv in x["qkv"]:
            k16 = torch.zeros(c["batch"], room, Hkv, hd, dtype=torch.float64, device="cuda")
            v16 = torch.zeros_like(k16)
            for b, take in enumerate(x["take"]):
                at = c["held"] - b % 3 % c["held"]
                chosen = qkv.view(-1, H + 2 * Hkv, hd)[[first[b] + i for i in take], H:].double()
                k16[b, at:at + len(take)], v16[b, at:at + len(take)] = chosen[:, :Hkv], chosen[:, Hkv:]
            out.append((k16.flatten(0, 1), v16.flatten(0, 1)))
        return torch.stack([y[0] for y in out]), torch.stack([y[1] for y in out]), None
    tokens = _cache_sizes(c)
    at16 = _sum([p[3] for p in tokens])
    if c["kind"] == "copy":
        src, out = _from(c), []
        largest = [[float(s[1, a:a + p[k]].abs().max()) if p[k] else 0.0 for a, p in zip(_sum([-(-p[k] // 32) * 32 for p in tokens]), tokens)]
                   for layer in x["layers"] for k, (_, s, _) in enumerate(layer[0])]
        for n, (_, rows16) in enumerate(x["layers"]):
            parts = [torch.cat([rows16[:, at16[s]:at16[s + 1]].double(), torch.zeros(2, 16, Hkv, hd, dtype=torch.float64, device="cuda")], 1) for s in src]
            k16, v16 = torch.cat(parts, 1)
            most = torch.tensor([max(largest[3 * n + k][s] for k in range(3)) for s in src], dtype=torch.float64, device="cuda")
            out.append((k16, v16, most))
        return (*([None] * 3,) * 4, *(torch.stack([y[i] for y in out]) for i in (0, 1)), None, torch.stack([y[2] for y in out]))
    wide = [(code.double().unflatten(-1, (-1, c["group"])) * s.double()[..., None] + m.double()[..., None]).flatten(-2) for code, s, m in x["classes"]]
    qkv, first, parents = x["qkv"].view(-1, H + 2 * Hkv, hd), _sum(_row_sizes(c)), _parents(c)
    at = [0, 0, 0]
    outs, sums = [], []
    for b, p in enumerate(tokens):
        mine = qkv[first[b]:first[b + 1]].double()
        n = mine.shape[0]
        both = [wide[i][:, at[i]:at[i] + p[i]] for i in range(3)] + [x["rows16"][:, at16[b]:at16[b + 1]].double()]
        at = [a + -(-t // 32) * 32 for a, t in zip(at, p)]
        kk = torch.cat([y[0] for y in both] + [mine[:, H:H + Hkv]])
        vv = torch.cat([y[1] for y in both] + [mine[:, H + Hkv:]])
        old = kk.shape[0] - n
        hidden = torch.ones(n, old + n, dtype=torch.bool)
        hidden[:, :old] = False
        for i in range(n):
            j = i
            while j >= 0:
                hidden[i, old + j] = False
                j = parents[b][j] if c["tree"] else j - 1
        hidden = hidden.cuda()
        o, l = torch.empty(n, H, hd, dtype=torch.float64, device="cuda"), torch.empty(n, H, dtype=torch.float64, device="cuda")
        for h in range(H):
            logit = (mine[:, h] @ kk[:, h // rep].T) / math.sqrt(hd)
            logit[hidden] = -math.inf
            l[:, h] = torch.logsumexp(logit, -1)
            o[:, h] = torch.exp(logit - l[:, h:h + 1]) @ vv[:, h // rep]
        outs.append(o)
        sums.append(l)
    return (torch.cat(outs), torch.cat(sums)) if c["lse"] else torch.cat(outs)
