"""Batches that a plan made from their average does not fit, tables that name more rows than there are, caches that differ from layer to layer."""
import numpy as np
import pytest
import torch

from paper_2605_02262_amd import binding as W
from tests import attend_ref as R
from tests import tree_ref as T
from tests.test_gpu_sequences import _block
from tests.test_gpu_tree_attention import DTYPES, SMALL, _check, _compare, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,group", [((8, 8, 64), 64), (SMALL, 32), ((16, 2, 128), 128)])
@pytest.mark.parametrize("parents", [None, "random"])
def test_a_long_sequence_among_single_rows(dtype, heads, group, parents):
    """The batch's average chooses the kernel and its tiles: the long sequence has many of them."""
    lens = [(33 * (b % 3), 7 * b, b % 2 * 40, 1 + b % 5) for b in range(32)]
    _check(lens, [1] * 20 + [255] + [1] * 11, heads, group, dtype, parents, hints=True)
    _check(lens, [1] * 31 + [1024 if parents else 1300], heads, group, dtype, parents, hints=False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_long_chain(dtype):
    _check([(64, 0, 33, 5)], [2500], (4, 2, 64), 32, dtype, None)
    _check([(0, 0, 0, 0)], [2100], (2, 2, 128), 64, dtype, None, splits=3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,most", [(5, 0), (60, 60)])
def test_tables_that_name_more_rows_than_there_are(dtype, n, most):
    """row_off ends behind the rows of the tensors: those that are there count, also for the walk and the append."""
    rng = np.random.default_rng(3)
    t16 = torch.bfloat16 if dtype == torch.bfloat16 else torch.float16
    kv, cached = R.make_cache(rng, [(64, 40, 9, 4), (0, 33, 0, 2), (5, 0, 0, 1)], 2, 64, 32, t16, slack=n)
    q, k, v = _inputs(rng, 2 * n, SMALL, dtype)
    parents = [T.random_tree(rng, n), T.random_tree(rng, n)]
    off, parent = R.i32([0, n, 2 * n + 7, 1 << 30]), R.i32(sum(parents, []))
    ctx = W.Context(W.tree_workspace_bytes(2 * n, 3, 14, 2, 64, 117, most))
    lse = torch.full((2 * n, 14), 77.0, device="cuda")
    out = W.wq_tree_attention(ctx, q, k, v, kv, off, 0.125, parent, most, 117, lse=lse)
    for b in range(2):
        s = slice(b * n, (b + 1) * n)
        kk, vv = (torch.cat([c, x[s].double().cpu()]) for c, x in zip(cached[b], (k, v)))
        sees = torch.cat([torch.ones(n, cached[b][0].shape[0], dtype=torch.bool), T.seen(parents[b], n)], 1)
        _compare(out[s], lse[s], q[s], kk, vv, sees, 0.125, dtype)
    tokens, target = (rng.integers(0, 3, 2 * n).tolist() for _ in range(2))
    path, n_path, following = W.wq_tree_accept(ctx, R.i32(tokens), R.i32(target), off, parent, 1024, 9)
    for b in range(2):
        s = slice(b * n, (b + 1) * n)
        want, after = T.accept(tokens[s], target[s], parents[b], 9)
        assert path[b].tolist() == want + [-1] * (9 - len(want)) and int(n_path[b]) == len(want) and int(following[b]) == after
    assert path[2].tolist() == [-1] * 9 and int(n_path[2]) == 0 and int(following[2]) == -1
    W.wq_append_rows(ctx, [k], [v], [kv], off, n)
    assert ctx.device_status() == 0 and kv.len16.tolist() == [4 + n, 2 + n, 1]
    for b in range(2):
        a = int(kv.off16[b]) + (4, 2)[b]
        assert torch.equal(kv.k16[a:a + n], k[b * n:(b + 1) * n].to(t16)) and torch.equal(kv.v16[a:a + n], v[b * n:(b + 1) * n].to(t16))


@pytest.mark.parametrize("n", [3, 40])
def test_layers_with_rooms_of_their_own(n):
    """Rows go behind what each layer holds; a layer without room keeps its sequence as it was, and the others get theirs."""
    held, room = [[2, 0], [5, 1], [0, 7], [1, 1]], [[n + 2, n], [n + 9, n + 1], [n - 1, n + 7], [n + 1, n + 4]]
    x = torch.randn(4, 2 * n, 6, 64, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).cuda()
    kvs = []
    for h, r in zip(held, room):
        kv = W.PackedKV(2, 2, 64, 64, torch.bfloat16, [0, 0, 0], R.offsets(r))
        kv.k16.fill_(7), kv.v16.fill_(9)
        kv.len16.copy_(R.i32(h))
        kvs.append(kv)
    ctx = W.Context(0)
    W.wq_append_rows(ctx, [y[:, :2] for y in x], [y[:, 4:] for y in x], kvs, R.i32([0, n, 2 * n]), n)
    assert ctx.device_status() == W.DEV_SEG16_OVERFLOW
    for l, kv in enumerate(kvs):
        k16, v16 = torch.full_like(kv.k16, 7), torch.full_like(kv.v16, 9)
        for b in range(2):
            fits = held[l][b] + n <= room[l][b]
            assert fits == (l != 2 or b != 0) and int(kv.len16[b]) == held[l][b] + (n if fits else 0)
            if fits:
                a = int(kv.off16[b]) + held[l][b]
                k16[a:a + n], v16[a:a + n] = x[l, b * n:(b + 1) * n, :2], x[l, b * n:(b + 1) * n, 4:]
        assert torch.equal(kv.k16, k16) and torch.equal(kv.v16, v16)


def test_layers_with_lengths_of_their_own():
    """Every layer's classes have their own sizes (bits are chosen layer by layer): thirteen layers, two launches."""
    rng = np.random.default_rng(4)
    lens = [[tuple(int(x) for x in rng.integers(0, 150, 3)) + (int(rng.integers(0, 40)),) for _ in range(5)] for _ in range(13)]
    src = [4, 0, 0, -1, 2, 3, 4]
    from_kv = [R.make_cache(rng, ln, 2, 64, 32, torch.bfloat16, slack=2)[0] for ln in lens]
    pad = lambda n: -(-n // 32) * 32  # noqa: E731
    to = []
    for ln in lens:
        picked = [ln[s] if s >= 0 else (0, 0, 0, 0) for s in src]
        to.append(W.PackedKV(len(src), 2, 64, 32, torch.bfloat16, [sum(pad(p[c]) for p in picked) for c in range(3)], R.offsets([p[3] + 1 for p in picked]), fill=85))
    ctx = W.Context(0)
    W.wq_copy_sequences(ctx, from_kv, to, R.i32(src))
    assert ctx.device_status() == 0
    for ln, a, z in zip(lens, from_kv, to):
        for d, s in enumerate(src):
            assert [int(z.cls_len[c][d]) for c in range(3)] + [int(z.len16[d])] == (list(ln[s]) if s >= 0 else [0] * 4)
            if s < 0:
                continue
            for c in range(3):
                for x, y in zip(_block(a, c, s), _block(z, c, d)):
                    assert torch.equal(x, y)
            n, i, j = ln[s][3], int(a.off16[s]), int(z.off16[d])
            assert torch.equal(z.k16[j:j + n], a.k16[i:i + n]) and torch.equal(z.v16[j:j + n], a.v16[i:i + n])
