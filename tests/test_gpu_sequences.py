"""Which drafted rows stay, rows appended to all layers' caches, sequences copied into other caches; and a run of them together."""
import math

import numpy as np
import pytest
import torch

from paper_2605_02262_amd import binding as W
from tests import attend_ref as R
from tests import tree_ref as T

pytestmark = pytest.mark.gpu


# ---- wq_tree_accept ----------------------------------------------------------------------------------------------------
def _accept(rng, rows, parents, max_path, max_rows=1024, vocabulary=4, front=0, behind=0):
    """A small vocabulary: siblings with the same token, many agreements."""
    off = [front + x for x in R.offsets(rows)]
    total = off[-1] + behind
    tokens, target = (rng.integers(0, vocabulary, total).tolist() for _ in range(2))
    parent = None if parents is None else R.i32([-1] * front + sum(parents, []) + [-1] * behind)
    ctx = W.Context(0)
    path, n_path, following = W.wq_tree_accept(ctx, R.i32(tokens), R.i32(target), R.i32(off), parent, max_rows, max_path)
    assert ctx.device_status() == (W.DEV_TOO_MANY_ROWS if max(rows + [0]) > max_rows else 0)
    longest = 0
    for b, n in enumerate(rows):
        n = min(n, max_rows)
        s = slice(off[b], off[b] + n)
        want, after = T.accept(tokens[s], target[s], None if parents is None else parents[b], max_path)
        assert path[b].tolist() == want + [-1] * (max_path - len(want)) and int(n_path[b]) == len(want) and int(following[b]) == after, b
        longest = max(longest, len(want))
    return longest


@pytest.mark.parametrize("max_path", [1, 3, 40, 500])
def test_accepted_paths(max_path):
    rng = np.random.default_rng(0)
    rows = [1, 0, 2, 64, 17, 255, 256, 257, 1000, 1024, 5]
    assert _accept(rng, rows, [T.random_tree(rng, n, 1 + n % 3) for n in rows], max_path, front=3, behind=4) >= min(max_path, 2)
    _accept(rng, rows, None, max_path)
    _accept(rng, rows, [[i - 1 for i in range(n)] for n in rows], max_path, vocabulary=1)


def test_a_whole_chain_is_accepted():
    rng = np.random.default_rng(1)
    assert _accept(rng, [1024, 700], None, 1024, vocabulary=1) == 1024
    assert _accept(rng, [5000, 3], None, 1024, max_rows=60, vocabulary=1) == 60


def test_accepts_among_values_that_are_no_parents():
    rng = np.random.default_rng(2)
    bad = [[0, 0, 1 << 30, 1, -(1 << 31), 3, 5, 99, 6], [7, 0, 1]]
    for _ in range(20):
        _accept(rng, [9, 3], bad, 9, vocabulary=2)


def test_many_sequences():
    rng = np.random.default_rng(3)
    rows = [int(x) for x in rng.integers(0, 20, 3000)]
    _accept(rng, rows, [T.random_tree(rng, n) for n in rows], 6)


# ---- wq_append_rows ----------------------------------------------------------------------------------------------------
def _caches(layers, B, Hkv, hd, dtype16, room, held):
    out = []
    for _ in range(layers):
        kv = W.PackedKV(B, Hkv, hd, hd, dtype16, [0, 0, 0], R.offsets(room))
        kv.k16.fill_(7), kv.v16.fill_(9)
        kv.len16.copy_(R.i32(held))
        out.append(kv)
    return out


def _append(rng, dtype, layers, rows, take, room, held, Hkv=2, hd=64, max_take=None, status=0, front=1):
    """take: None, or a list of rows per sequence.  Every layer's cache against a plain copy of the rows."""
    B, t16 = len(rows), torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    off = [front + x for x in R.offsets(rows)]
    x = torch.from_numpy(rng.normal(0, 1, (layers, off[-1] + 2, 3 * Hkv + 1, hd))).to(dtype).cuda()
    k, v = [y[:, :Hkv] for y in x], [y[:, 2 * Hkv:3 * Hkv] for y in x]
    kvs = _caches(layers, B, Hkv, hd, t16, room, held)
    taken = [list(range(n)) for n in rows] if take is None else take
    most = max_take or max(max(len(t) for t in taken), 1)
    tables = [None, None] if take is None else [R.i32(sum([(t + [-9] * most)[:most] for t in take], [])), R.i32([len(t) for t in take])]
    ctx = W.Context(0)
    W.wq_append_rows(ctx, k, v, kvs, R.i32(off), most, *tables)
    assert ctx.device_status() == status
    at = R.offsets(room)
    for l, kv in enumerate(kvs):
        want = [torch.full_like(kv.k16, 7), torch.full_like(kv.v16, 9)]
        for b, t in enumerate(taken):
            fits = held[b] + len(t) <= room[b] and len(t) <= most and all(0 <= i < rows[b] for i in t)
            assert int(kv.len16[b]) == held[b] + (len(t) if fits else 0), (l, b)
            for j, i in enumerate(t if fits else []):
                for w, y in zip(want, (k[l], v[l])):
                    w[at[b] + held[b] + j] = y[off[b] + i].to(t16)
        assert torch.equal(kv.k16, want[0]) and torch.equal(kv.v16, want[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_appended_rows(dtype):
    rng = np.random.default_rng(0)
    _append(rng, dtype, 3, [5, 0, 9, 1], [[0, 2, 4], [], [8, 1, 1, 3, 0], [0]], [9, 3, 6, 1], [4, 2, 1, 0])
    _append(rng, dtype, 2, [5, 0, 33, 1], None, [9, 3, 34, 1], [4, 3, 1, 0], Hkv=4, hd=128)
    _append(rng, dtype, 1, [100, 64], [list(range(0, 100, 2)), [63] * 17], [90, 20], [3, 3], Hkv=3)
    _append(rng, dtype, 2, [1, 1], None, [1, 1], [0, 0], Hkv=1)


def test_more_layers_than_a_launch_takes():
    rng = np.random.default_rng(1)
    _append(rng, torch.bfloat16, 50, [3, 2], [[0, 2], [1]], [4, 4], [1, 2])
    _append(rng, torch.float32, 97, [40, 2], None, [44, 4], [1, 2])


def test_sequences_that_are_refused_stay_as_they_are():
    rng = np.random.default_rng(2)
    for n in (3, 40):                                             # one workgroup, several
        rows, room = [n + 2] * 3, [n + 5] * 3
        every = list(range(n))
        _append(rng, torch.bfloat16, 2, rows, [every, every, every], room, [5, 6, 0], status=W.DEV_SEG16_OVERFLOW)
        _append(rng, torch.bfloat16, 2, rows, [every, every[:-1] + [n + 2], every], room, [5, 5, 0], status=W.DEV_BAD_INDEX)
        _append(rng, torch.bfloat16, 2, rows, [every, [-1] + every[1:], every], room, [5, 5, 0], status=W.DEV_BAD_INDEX)
        _append(rng, torch.bfloat16, 2, rows, [every + [0], every, every[:1]], room, [0, 5, 0], max_take=n, status=W.DEV_TOO_MANY_ROWS)
        _append(rng, torch.bfloat16, 2, [n, n + 1, 0], None, room, [5, 0, 0], max_take=n, status=W.DEV_TOO_MANY_ROWS)
    kvs = _caches(1, 1, 2, 64, torch.float16, [9], [2])
    x = torch.ones(4, 2, 64, device="cuda")
    ctx = W.Context(0)
    W.wq_append_rows(ctx, [x], [x], kvs, R.i32([0, 4]), 4, R.i32([0, 1, 2, 3]), R.i32([-1]))
    assert ctx.device_status() == W.DEV_BAD_INDEX and int(kvs[0].len16) == 2
    W.wq_append_rows(ctx, [x[:0]], [x[:0]], kvs, R.i32([0, 0]), 4, R.i32([0, 1, 2, 3]), R.i32([1]))      # no row at all
    assert ctx.device_status() == W.DEV_BAD_INDEX and int(kvs[0].len16) == 2


def test_appending_rows_one_by_one_or_at_once():
    rng = np.random.default_rng(3)
    for dtype in (torch.bfloat16, torch.float32):
        t16 = torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
        x = torch.from_numpy(rng.normal(0, 1, (2, 2 * 6, 4, 128))).to(dtype).cuda()
        a, b = (_caches(1, 2, 4, 128, t16, [9, 9], [2, 3])[0] for _ in range(2))
        ctx = W.Context(0)
        W.wq_append_rows(ctx, [x[0]], [x[1]], [a], R.i32([0, 6, 12]), 6)
        for i in range(6):
            W.wq_append_kv(ctx, x[0, i::6].contiguous(), x[1, i::6].contiguous(), b)
        assert torch.equal(a.k16, b.k16) and torch.equal(a.v16, b.v16) and torch.equal(a.len16, b.len16)


def test_rows_behind_4_gb():
    """Rows 2^22 elements apart, appended behind 4.3 GB of a cache."""
    n, apart, far = 600, 1 << 22, 1 << 24
    room = torch.empty((n - 1) * apart + 4096, dtype=torch.bfloat16, device="cuda")
    k, v = (room[s:].as_strided((n, 2, 64), (apart, 64, 1)) for s in (0, 1024))
    x = torch.randn(2, n, 2, 64, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).cuda()
    k.copy_(x[0]), v.copy_(x[1])
    kv = W.PackedKV(1, 2, 64, 64, torch.bfloat16, [0, 0, 0], [far, far + n + 3])
    kv.len16.fill_(2)
    W.wq_append_rows(W.Context(0), [k], [v], [kv], R.i32([0, n]), n)
    assert torch.equal(kv.k16[far + 2:far + 2 + n], x[0]) and torch.equal(kv.v16[far + 2:far + 2 + n], x[1])


# ---- wq_copy_sequences -------------------------------------------------------------------------------------------------
def _block(kv, c, b):
    """A sequence's class: codes and metadata, padding included, [plane, head, bytes]."""
    G, bits = kv.hd // kv.group, W.CLASS_BITS[c]
    a, n = int(kv.cls_off[c][b]), -(-int(kv.cls_len[c][b]) // 32) * 32
    per = kv.hd * bits // 8
    return kv.codes[c][:, :, a * per:(a + n) * per], kv.meta[c][:, :, a * G:(a + n) * G]


def _copy(rng, lens, src, Hkv=2, hd=64, group=32, dtype16=torch.bfloat16, layers=1, cap=None, room=None, status=0, empty=()):
    """empty: sequences of the copy that are refused."""
    from_kv = [R.make_cache(rng, lens, Hkv, hd, group, dtype16, slack=2)[0] for _ in range(layers)]
    pad = lambda n: -(-n // 32) * 32  # noqa: E731
    picked = [lens[s] if 0 <= s < len(lens) else (0, 0, 0, 0) for s in src]
    room = room or [p[3] + 1 for p in picked]
    to = [W.PackedKV(len(src), Hkv, hd, group, dtype16, cap or [sum(pad(p[c]) for p in picked) for c in range(3)], [2 + x for x in R.offsets(room)], fill=85)
          for _ in range(layers)]
    for kv in to:
        kv.k16.fill_(7), kv.v16.fill_(9)
    ctx = W.Context(0)
    W.wq_copy_sequences(ctx, from_kv, to, R.i32(src))
    assert ctx.device_status() == status
    for a, z in zip(from_kv, to):
        want_off = [R.offsets([pad(p[c]) for p in picked]) for c in range(3)]
        k16, v16 = torch.full_like(z.k16, 7), torch.full_like(z.v16, 9)
        for c in range(3):
            assert z.cls_off[c].tolist() == [min(x, z.cap[c]) for x in want_off[c]]
        for d, s in enumerate(src):
            there = d not in empty and 0 <= s < len(lens)
            assert [int(z.cls_len[c][d]) for c in range(3)] + [int(z.len16[d])] == (list(lens[s]) if there else [0] * 4), d
            assert float(z.v_scale_max[d]) == (float(a.v_scale_max[s]) if there else 0.0)
            if not there:
                continue
            for c in range(3):
                for x, y in zip(_block(a, c, s), _block(z, c, d)):
                    assert torch.equal(x, y)
            n, i, j = lens[s][3], int(a.off16[s]), int(z.off16[d])
            k16[j:j + n], v16[j:j + n] = a.k16[i:i + n], a.v16[i:i + n]
        assert torch.equal(z.k16, k16) and torch.equal(z.v16, v16)
        # nothing is written where no sequence lies
        for c in range(3):
            per = z.hd * W.CLASS_BITS[c] // 8
            owned = torch.zeros(z.cap[c], dtype=torch.bool)
            for d in range(len(src)):
                owned[int(z.cls_off[c][d]):int(z.cls_off[c][d]) + pad(int(z.cls_len[c][d]))] = True
            assert bool((z.codes[c].view(2, Hkv, -1, per)[:, :, ~owned.cuda()] == 85).all())
            assert bool((z.meta[c].view(2, Hkv, -1, hd // group)[:, :, ~owned.cuda()] == 85).all())
    return from_kv, to


LENS = [(100, 64, 33, 20), (0, 40, 0, 3), (7, 0, 290, 0), (0, 0, 0, 0), (0, 0, 0, 65), (1000, 700, 1, 1)]


@pytest.mark.parametrize("Hkv,hd,group,dtype16", [(2, 64, 32, torch.bfloat16), (4, 128, 64, torch.float16), (1, 128, 32, torch.bfloat16), (3, 128, 128, torch.bfloat16), (8, 64, 64, torch.float16)])
def test_copies(Hkv, hd, group, dtype16):
    rng = np.random.default_rng(0)
    for src in ([0, 1, 2, 3, 4, 5], [5, 0, 0, 4, 0, 2, -1, 5], [2], [3, -1], [1, 4]):
        _copy(rng, LENS, src, Hkv, hd, group, dtype16)


def test_more_sequences_and_layers_than_a_launch_takes():
    rng = np.random.default_rng(1)
    lens = [(int(a), int(b), int(c), int(d)) for a, b, c, d in rng.integers(0, 40, (40, 4))]
    _copy(rng, lens, [int(x) for x in rng.integers(-1, 40, 2100)], 1)
    _copy(rng, LENS[:3], [2, 0, 0], layers=23)


def test_copies_that_do_not_fit():
    rng = np.random.default_rng(2)
    # the class of the sequence in the middle, and of the last one; 16-bit rows; sources that do not exist
    _copy(rng, [(64, 0, 0, 2), (32, 0, 0, 2)], [0, 1, 0], cap=[96, 0, 0], status=W.DEV_CLASS_OVERFLOW, empty=(2,))
    _copy(rng, [(64, 0, 0, 2), (32, 0, 5, 2)], [0, 1, 0, 0], cap=[256, 0, 0], status=W.DEV_CLASS_OVERFLOW, empty=(1,))
    _copy(rng, [(64, 0, 0, 9), (32, 0, 5, 2)], [0, 1, 0], room=[9, 3, 8], status=W.DEV_SEG16_OVERFLOW, empty=(2,))
    _copy(rng, [(64, 0, 0, 9), (32, 0, 5, 2)], [0, 2, -2, 1 << 30, 1], status=W.DEV_BAD_INDEX)
    _copy(rng, [(64, 0, 0, 9), (32, 0, 5, 2)], [0, 2, 1], cap=[64, 0, 0], room=[8, 9, 9], status=W.DEV_BAD_INDEX | W.DEV_CLASS_OVERFLOW | W.DEV_SEG16_OVERFLOW, empty=(0, 2))


def test_a_copy_decodes_like_its_source():
    rng = np.random.default_rng(3)
    src = [5, 0, 0, 4, 2]
    (a,), (z,) = _copy(rng, LENS, src, 4, 128, 64)
    q = torch.randn(len(LENS), 28, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    ctx = W.Context(W.workspace_bytes(6, 28, 128, 8))
    flags = W.DECODE_MFMA | W.DECODE_FIXED_SHARES
    x = W.wq_decode_attention(ctx, q, a, 0.088, 4, algo=flags)
    y = W.wq_decode_attention(ctx, q[src].contiguous(), z, 0.088, 4, algo=flags)
    assert torch.equal(x[src], y)


def test_a_copy_behind_4_gb():
    rng = np.random.default_rng(4)
    near = R.make_cache(rng, [(0, 0, 190, 77)], 2, 64, 32, torch.bfloat16)[0]
    far16, far = 1 << 24, 20480000
    wide = [W.PackedKV(1, 2, 64, 32, torch.bfloat16, [0, 0, far + near.cap[2]], [far16, far16 + 77]) for _ in range(1)][0]
    wide.codes[2][:, :, far * 64:] = near.codes[2]
    wide.meta[2][:, :, far * 2:] = near.meta[2]
    wide.cls_off[2].copy_(near.cls_off[2] + far)
    wide.cls_len[2].copy_(near.cls_len[2])
    wide.k16[far16:], wide.v16[far16:] = near.k16, near.v16
    wide.len16.copy_(near.len16)
    back = W.PackedKV(1, 2, 64, 32, torch.bfloat16, [0, 0, 224], [far16, far16 + 80], fill=0)
    W.wq_copy_sequences(W.Context(0), [wide], [back], R.i32([0]))
    assert torch.equal(back.codes[2][:, :, :192 * 64], near.codes[2][:, :, :192 * 64]) and torch.equal(back.meta[2][:, :, :192 * 2], near.meta[2][:, :, :192 * 2])
    assert torch.equal(back.k16[far16:far16 + 77], near.k16) and torch.equal(back.v16[far16:far16 + 77], near.v16)


# ---- together ----------------------------------------------------------------------------------------------------------
def test_drafted_decoding_as_a_program_runs_it():
    """Two layers, two sequences.  Steps in one graph: rotary positions of a tree's rows, its attention over both layers' caches, the walk, the append to both;
    the caches grow by what was accepted.  Then the batch forks.  Every step against 64 bits; in the end one token against plain decoding."""
    Hq, Hkv, hd, B, n, layers, most = 28, 4, 128, 2, 9, 2, 4
    rng = np.random.default_rng(5)
    lens = [(100, 64, 33, 20), (0, 40, 0, 3)]
    both = [R.make_cache(rng, lens, Hkv, hd, 64, torch.bfloat16, slack=3 * most) for _ in range(layers)]
    kvs, held = [x[0] for x in both], [[list(y) for y in x[1]] for x in both]
    inv_freq = torch.tensor(W.wq_rope_frequencies(hd, 1000000.0)[0]).cuda()
    parents = [T.random_tree(rng, n), T.random_tree(rng, n)]
    off, parent = R.i32([0, n, 2 * n]), R.i32(sum(parents, []))
    depth = [[len([j for j in range(n) if T.seen(p, n)[i, j]]) - 1 for i in range(n)] for p in parents]
    start = torch.tensor([sum(x) for x in lens], dtype=torch.int32, device="cuda")
    depths = R.i32(sum(depth, []))
    qkv = [torch.from_numpy(rng.normal(0, 1, (B * n, Hq + 2 * Hkv, hd))).to(torch.bfloat16).cuda() for _ in range(layers)]
    tokens, target = R.i32(rng.integers(0, 3, B * n)), R.i32(rng.integers(0, 3, B * n))
    stream = torch.cuda.Stream()
    ctx = W.Context(max(W.tree_workspace_bytes(B * n, B, Hq, Hkv, hd, 300, n), W.workspace_bytes(4, Hq, hd, 4)), stream=stream)
    torch.cuda.synchronize()
    sm = 1.0 / math.sqrt(hd)
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        turned = [(torch.empty(B * n, Hq, hd, dtype=torch.bfloat16, device="cuda"), torch.empty(B * n, Hkv, hd, dtype=torch.bfloat16, device="cuda")) for _ in range(layers)]
        outs = [torch.empty_like(t[0]) for t in turned]
        with torch.cuda.graph(graph, stream=stream):
            positions = (start[:, None] + depths.view(B, n)).view(-1)
            for l in range(layers):
                x = qkv[l]
                W.wq_rope(ctx, x[:, :Hq], x[:, Hq:Hq + Hkv], positions, inv_freq, q_out=turned[l][0], k_out=turned[l][1])
                W.wq_tree_attention(ctx, *turned[l], x[:, Hq + Hkv:], kvs[l], off, sm, parent, n, 300, out=outs[l])
            path, n_path, following = W.wq_tree_accept(ctx, tokens, target, off, parent, n, most)
            W.wq_append_rows(ctx, [t[1] for t in turned], [x[:, Hq + Hkv:] for x in qkv], kvs, off, most, path, n_path)
            start.add_(n_path)
        for step in range(3):
            tok, tgt = tokens.tolist(), target.tolist()
            at = start.tolist()
            graph.replay()
            torch.cuda.synchronize()
            for b in range(B):
                s = slice(b * n, (b + 1) * n)
                want, after = T.accept(tok[s], tgt[s], parents[b], most)
                assert path[b].tolist() == want + [-1] * (most - len(want)) and int(following[b]) == after
                assert int(start[b]) == at[b] + len(want)
                sees = torch.cat([torch.ones(n, held[0][b][0].shape[0], dtype=torch.bool), T.seen(parents[b], n)], 1)
                for l in range(layers):
                    q, k, v = turned[l][0][s], turned[l][1][s].double().cpu(), qkv[l][s, Hq + Hkv:].double().cpu()
                    exact = R.rope(qkv[l][s, :Hq].double().cpu(), torch.tensor(depth[b]) + at[b], inv_freq.cpu(), W.ROPE_HALF, 1.0)[0]
                    assert float((q.double().cpu() - exact).norm() / exact.norm()) <= 2.0 ** -8
                    o = T.attend(q.double().cpu(), torch.cat([held[l][b][0], k]), torch.cat([held[l][b][1], v]), sees, sm)[0]
                    assert float((outs[l][s].double().cpu() - o).norm() / o.norm()) <= 1.5 * 2.0 ** -8 + 6 * 2.0 ** -11
                    held[l][b] = [torch.cat([h, y[want]]) for h, y in zip(held[l][b], (k, v))]
                    assert int(kvs[l].len16[b]) == held[l][b][0].shape[0] - sum(lens[b][:3])
            tokens.copy_(R.i32(rng.integers(0, 3, B * n)))
            target.copy_(R.i32(rng.integers(0, 3, B * n)))
        src = [1, 0, 0]
        cap = [sum(-(-lens[s][c] // 32) * 32 for s in src) for c in range(3)]
        forked = [W.PackedKV(3, Hkv, hd, 64, torch.bfloat16, cap, R.offsets([40] * 3)) for _ in range(layers)]
        W.wq_copy_sequences(ctx, kvs, forked, R.i32(src))
        q = torch.from_numpy(rng.normal(0, 1, (3, Hq, hd))).to(torch.bfloat16).cuda()
        for l in range(layers):
            o = W.wq_decode_attention(ctx, q, forked[l], sm, 4).double().cpu()
            for d, s in enumerate(src):
                want = R.attend(q[d:d + 1].double().cpu(), *held[l][s], [held[l][s][0].shape[0]], sm)[0][0]
                assert bool(((o[d] - want).abs() <= 2e-3 * want.abs().amax(-1, keepdim=True)).all())
        assert ctx.device_status() == 0
