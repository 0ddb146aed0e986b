"""Embedding lookup with scaling (chain.embed), plain and pooled, and its gradient
by sorted tokens, against the formulas in 64 bits.

Tolerances.  A sum of n terms in double is off by at most n 2^-53 times the sum of
its terms' sizes, below 1e-10 of it here, and the output is rounded to float (2^-24
of the value) and, in a 16-bit type, once more (2^-9 bfloat16 at its spacing of 2^-8,
2^-12 float16 at 2^-11, counted as half a step: 2^-8 and 2^-11 relative at most;
below its smallest normal number, half of float16's step 2^-24).  In a 16-bit type the
partial sums of a row that crosses chunks are rounded to float on the way: 2^-24 of
each, together at most 2^-24 of the sum of the terms' sizes.
"""
import ctypes

import numpy as np
import pytest

ROUND = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


@pytest.fixture(scope="module")
def chain():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2002_06115_amd import chain
    return chain


def lookup(table, ids):
    """table's rows in float64, zeros for padding, and whether each id is a row."""
    ok = (ids >= 0) & (ids < table.shape[0])
    return np.where(ok[..., None], table[np.where(ok, ids, 0)], 0.0), ok


def bags_of(ids, offsets):
    if offsets is None:
        return [np.arange(g * ids.shape[1], (g + 1) * ids.shape[1]) for g in range(ids.shape[0])]
    o = np.clip(offsets, 0, ids.size)
    return [np.arange(o[g], o[g + 1]) for g in range(o.size - 1)]


def oracle(table, ids, offsets, scale, pool, dout):
    """(out, dtable, per-element sums of the terms' sizes of both), float64."""
    rows, ok = lookup(table, ids)
    dt, dt_abs = np.zeros_like(table), np.zeros_like(table)
    if pool is None:
        flat, d = ids.reshape(-1), dout.reshape(-1, table.shape[1]) * scale
        keep = ok.reshape(-1)
        np.add.at(dt, flat[keep], d[keep])
        np.add.at(dt_abs, flat[keep], np.abs(d[keep]))
        return rows * scale, dt, np.abs(rows * scale), dt_abs
    flat, keep = ids.reshape(-1), ok.reshape(-1)
    rows = rows.reshape(-1, table.shape[1])
    bags = bags_of(ids, offsets)
    out, out_abs = np.zeros((len(bags), table.shape[1])), np.zeros((len(bags), table.shape[1]))
    for g, at in enumerate(bags):
        n = int(keep[at].sum())
        w = scale / n if pool == "mean" and n else scale
        out[g], out_abs[g] = rows[at].sum(0) * w, np.abs(rows[at]).sum(0) * abs(w)
        for t in at[keep[at]]:
            dt[flat[t]] += dout[g] * w
            dt_abs[flat[t]] += np.abs(dout[g] * w)
    return out, dt, out_abs, dt_abs


def close(got, want, sums, dtype, what):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape, what
    least = 2.0 ** -25 if dtype == "float16" else 0.0
    rest = 1e-10 if dtype == "float32" else 1e-10 + 2.0 ** -24
    bound = (ROUND[dtype] + 2.0 ** -23) * np.abs(want) + rest * sums + least
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} values off, first at {np.argwhere(bad)[0]}"


def tensors(g, rows, dim, dtype, ids, lead, int_dtype="int64"):
    import torch
    dt = getattr(torch, dtype)
    table = torch.from_numpy(g.standard_normal((rows, dim)).astype(np.float32)).cuda().to(dt)
    dout = torch.from_numpy(g.standard_normal((*lead, dim)).astype(np.float32)).cuda().to(dt)
    return table, dout, torch.from_numpy(ids.astype(int_dtype)).cuda()


def check(chain, table, ids, offsets, scale, pool, dout, dtype):
    import torch
    out = chain.embed(table, ids, offsets, scale=scale, pool=pool)
    back = chain.embed_backward(dout, ids, table.shape[0], offsets, scale=scale, pool=pool)
    scale = float(np.float32(scale))
    want = oracle(table.double().cpu().numpy(), ids.cpu().numpy(),
                  None if offsets is None else offsets.cpu().numpy(), scale, pool,
                  dout.double().cpu().numpy())
    close(out, want[0], want[2], dtype, "out")
    close(back, want[1], want[3], dtype, "dtable")
    again = chain.embed_backward(dout, ids, table.shape[0], offsets, scale=scale, pool=pool)
    assert torch.equal(back.view(torch.uint8), again.view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("tokens,rows,dim", [(1, 1, 1), (1, 7, 5), (3, 2, 4), (130, 50, 7),
                                             (77, 1000, 9), (500, 30, 65), (1000, 4, 128),
                                             (257, 300, 1001), (8192, 700, 3), (8193, 90, 8),
                                             (20_000, 5000, 12)])
def test_plain(chain, dtype, tokens, rows, dim):
    g = np.random.default_rng(tokens * 7 + dim)
    ids = g.integers(-2, rows + 2, tokens)  # some of them padding
    table, dout, ids = tensors(g, rows, dim, dtype, ids, (tokens,),
                               "int32" if tokens % 2 else "int64")
    check(chain, table, ids, None, 0.75, None, dout, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 255, 256, 511, 512, 1 << 18, (1 << 18) + 1])
def test_sort_takes_every_key_width(chain, rows):
    """Ids at both ends of the range, at row counts where the keys need one bit,
    or one radix pass, more."""
    g = np.random.default_rng(rows)
    ids = np.concatenate([g.integers(0, rows, 9000), [0, rows - 1, rows, -1]])
    table, dout, ids = tensors(g, rows, 2, "float32", ids, (ids.size,))
    check(chain, table, ids, None, 1.0, None, dout, "float32")


@pytest.mark.gpu
@pytest.mark.parametrize("word", ["one", "two", "hub"])
@pytest.mark.parametrize("tokens,dim", [(5000, 40), (40_000, 17), (150_000, 4)])
def test_frequent_words(chain, word, tokens, dim):
    """Rows whose sums cross many chunks, to the whole list."""
    g = np.random.default_rng(tokens)
    rows = 600
    ids = {"one": np.full(tokens, 599), "two": np.arange(tokens) % 2 * 300,
           "hub": np.where(g.random(tokens) < 0.7, 5, g.integers(0, rows, tokens))}[word]
    table, dout, ids = tensors(g, rows, dim, "float32", ids, (tokens,))
    check(chain, table, ids, None, 1.0, None, dout, "float32")


@pytest.mark.gpu
@pytest.mark.parametrize("pool", ["sum", "mean"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("bags,tokens,rows,dim", [
    (1, 9, 40, 128), (1, 0, 3, 5), (5, 0, 3, 5), (128, 1411, 500, 128), (7, 4096, 50, 33),
    (7, 4097, 50, 33), (1, 9000, 20, 6), (3000, 6000, 900, 3), (40, 12_000, 31, 70)])
def test_ragged_bags(chain, pool, dtype, bags, tokens, rows, dim):
    import torch
    g = np.random.default_rng(tokens + bags)
    ids = g.integers(-1, rows + 1, tokens)
    cut = np.sort(g.integers(0, tokens + 1, bags - 1))
    offsets = np.concatenate([[0], cut, [tokens]])
    if tokens > 100:
        ids[offsets[bags // 2]:offsets[bags // 2 + 1]] = -1  # a bag of padding alone
    table, dout, ids = tensors(g, rows, dim, dtype, ids, (bags,))
    check(chain, table, ids, torch.from_numpy(offsets).cuda(), 1.5, pool, dout, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("pool", ["sum", "mean"])
def test_tokens_outside_every_bag(chain, pool):
    """Offsets that begin late and end early, with empty bags in a row."""
    import torch
    g = np.random.default_rng(4)
    for tokens in (60, 9000):
        ids = g.integers(0, 20, tokens)
        offsets = np.array([5, 5, 5, 17, 17, tokens - 9, tokens - 9])
        table, dout, dev = tensors(g, 20, 10, "float32", ids, (6,), "int32")
        check(chain, table, dev, torch.from_numpy(offsets.astype("int32")).cuda(), 1.0, pool,
              dout, "float32")


@pytest.mark.gpu
@pytest.mark.parametrize("pool", ["sum", "mean"])
@pytest.mark.parametrize("bags,length", [(1, 1), (5, 7), (64, 30), (3, 6000), (700, 64), (4, 0)])
def test_padded_bags(chain, pool, bags, length):
    g = np.random.default_rng(bags + length)
    ids = g.integers(0, 90, (bags, length))
    for k in range(bags):
        ids[k, g.integers(0, length + 1):] = -1
    table, dout, ids = tensors(g, 90, 24, "float32", ids, (bags,))
    check(chain, table, ids, None, 1.0, pool, dout, "float32")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("tokens,dim", [(70_000, 3), (70_000, 9), (20_000, 130), (9001, 600)])
def test_rows_that_cross_runs_and_chunks(chain, dtype, tokens, dim):
    """Sums that end inside a lane group's run, inside a workgroup's chunk and behind
    many chunks, in rows of every number of lanes."""
    import torch
    g = np.random.default_rng(tokens + dim)
    lengths = np.concatenate([g.integers(0, 30, 400), g.integers(0, 700, 20), [tokens // 2]])
    g.shuffle(lengths)
    offsets = np.minimum(np.concatenate([[0], lengths.cumsum()]), tokens)
    ids = np.sort(g.integers(-1, 900, tokens) ** 2 // 900)
    table, dout, dev = tensors(g, 900, dim, dtype, ids, (offsets.size - 1,))
    check(chain, table, dev, torch.from_numpy(offsets).cuda(), 1.0, "mean", dout, dtype)


@pytest.mark.gpu
def test_a_long_bag_is_counted(chain):
    """A mean over a bag that a whole workgroup counts, between short ones."""
    import torch
    g = np.random.default_rng(8)
    ids = g.integers(-3, 40, 30_000)
    offsets = np.array([0, 3, 10_000, 10_001, 29_000, 30_000])
    table, dout, ids = tensors(g, 40, 6, "float32", ids, (5,))
    check(chain, table, ids, torch.from_numpy(offsets).cuda(), 1.0, "mean", dout, "float32")


@pytest.mark.gpu
def test_many_empty_bags(chain):
    """More bags than a grid has workgroups, with no token, and with two."""
    import torch
    bags = 20_000_000
    table = torch.ones((3, 2), device="cuda")
    ids = torch.tensor([2, 1], device="cuda")
    offsets = torch.zeros(bags + 1, dtype=torch.int64, device="cuda")
    for pool in ("sum", "mean"):
        assert not chain.embed(table, ids[:0], offsets, pool=pool).any()
        offsets[-1] = 2
        out = chain.embed(table, ids, offsets, pool=pool)
        assert not out[:-1].any() and (out[-1] == (2.0 if pool == "sum" else 1.0)).all()
        back = chain.embed_backward(out, ids, 3, offsets, pool=pool)
        assert torch.equal(back[:, 0], torch.tensor([0.0, 2.0, 2.0] if pool == "sum" else
                                                    [0.0, 0.5, 0.5], device="cuda"))
        offsets[-1] = 0


@pytest.mark.gpu
def test_bad_offsets_read_nothing_outside(chain):
    """Offsets past the tokens, or negative, are taken as the nearer end."""
    import torch
    g = np.random.default_rng(9)
    ids = g.integers(0, 9, 50)
    table, dout, ids = tensors(g, 9, 4, "float32", ids, (3,))
    offsets = torch.tensor([-1 << 40, 20, 50, 1 << 40]).cuda()
    check(chain, table, ids, offsets, 1.0, "sum", dout, "float32")


@pytest.mark.gpu
def test_strided_and_unaligned_tables(chain):
    import torch
    g = np.random.default_rng(1)
    for dtype in ("float32", "bfloat16"):
        wide, dout, ids = tensors(g, 50, 41, dtype, g.integers(0, 50, 64), (64,))
        table, narrow = wide[:, 3:36], dout[:, :33].contiguous()
        check(chain, table, ids, None, 2.0, None, narrow, dtype)
        check(chain, wide[7:8, :33], ids, None, 2.0, None, narrow, dtype)


@pytest.mark.gpu
def test_non_finite_values_stay_in_their_rows(chain):
    import torch
    table = torch.ones((6, 8), device="cuda")
    table[2], table[3] = float("nan"), float("inf")
    ids = torch.tensor([0, -1, 1, 2, 3, 99], device="cuda")
    out = chain.embed(table, ids)
    assert torch.equal(out[[0, 2]], table[[0, 1]]) and torch.isnan(out[3]).all()
    assert torch.isinf(out[4]).all() and not out[[1, 5]].any()
    pooled = chain.embed(table, ids, torch.tensor([0, 3, 3, 6], device="cuda"), pool="sum")
    assert torch.equal(pooled[0], torch.full((8,), 2.0, device="cuda")) and not pooled[1].any()
    dout = torch.ones((6, 8), device="cuda")
    dout[1], dout[5] = float("nan"), float("inf")  # the padding's
    back = chain.embed_backward(dout, ids, 6)
    want = torch.zeros((6, 8), device="cuda")
    want[:4] = 1.0
    assert torch.equal(back, want)


@pytest.mark.gpu
def test_autograd_and_differences(chain):
    """The gradient against central differences of the pooled sum (linear in the
    table, so their error is rounding alone: 2^-24 |out| / h per term, 1e-3 here)."""
    import torch
    g = np.random.default_rng(2)
    ids = torch.from_numpy(g.integers(0, 5, (3, 4))).cuda()
    table = torch.from_numpy(g.standard_normal((5, 6)).astype(np.float32)).cuda().requires_grad_()
    up = torch.from_numpy(g.standard_normal((3, 6)).astype(np.float32)).cuda()
    out = chain.embed(table, ids, scale=1.5, pool="mean")
    (got,) = torch.autograd.grad(out, table, up)
    f = lambda t: float((chain.embed(t, ids, scale=1.5, pool="mean").double() * up).sum())  # noqa: E731
    base = table.detach()
    for v in range(5):
        for c in range(6):
            e = torch.zeros_like(base)
            e[v, c] = 2.0 ** -6
            d = (f(base + e) - f(base - e)) / 2.0 ** -5
            assert abs(d - float(got[v, c])) < 1e-3
    # A transposed upstream gradient, and a bfloat16 table.
    tb = base.bfloat16().requires_grad_()
    o = chain.embed(tb, ids[0])
    (gb,) = torch.autograd.grad(o, tb, torch.ones((6, 4), device="cuda", dtype=torch.bfloat16).t())
    assert gb.dtype == torch.bfloat16
    assert torch.equal(gb.float().sum(1), torch.bincount(ids[0], minlength=5) * 6.0)


@pytest.mark.gpu
def test_captured_and_replayed(chain):
    """Two captured graphs and eager work on another stream between replays."""
    import torch
    g = np.random.default_rng(3)
    graphs = []
    for tokens in (300, 12_000):
        table, dout, ids = tensors(g, 400, 20, "float32", g.integers(-1, 400, (4, tokens // 4)),
                                   (4,))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            chain.embed(table, ids, pool="mean")
            chain.embed_backward(dout, ids, 400, pool="mean")
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = chain.embed(table, ids, pool="mean")
            back = chain.embed_backward(dout, ids, 400, pool="mean")
        graphs.append((graph, table, dout, ids, out, back))
    other = torch.cuda.Stream()
    for k in range(3):
        for graph, table, dout, ids, out, back in graphs:
            table.add_(1.0)
            dout.mul_(-1.5)
            ids.copy_(torch.roll(ids, k + 1, 1))
            graph.replay()
            with torch.cuda.stream(other):
                other.wait_stream(torch.cuda.default_stream())
                want = chain.embed(table, ids, pool="mean")
                want_back = chain.embed_backward(dout, ids, 400, pool="mean")
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(back, want_back), k


@pytest.mark.gpu
def test_large_offsets(chain):
    """A table and an output past 2^31 values: 64-bit places."""
    import torch
    rows, dim = 1_100_000, 2048
    table = torch.zeros((rows, dim), dtype=torch.bfloat16, device="cuda")
    table[-1], table[-2, -1] = 3.0, 5.0
    ids = torch.full((rows + 5,), rows - 1, device="cuda", dtype=torch.int32)
    ids[:-1] = torch.arange(rows + 4, device="cuda", dtype=torch.int32) % rows
    out = chain.embed(table, ids)
    assert (out[-1] == 3.0).all() and out[rows - 2, -1] == 5.0 and (out[rows - 1] == 3.0).all()
    back = chain.embed_backward(out, ids, rows)
    assert (back[-1] == 6.0).all() and back[-2, -1] == 5.0 and not back[5].any()


def test_c_refusals():
    from paper_2002_06115_amd import chain as c
    lib, P = c._lib, ctypes.c_void_p
    d = P(256)  # never dereferenced: arguments are checked first

    def plain(tokens=4, ids=d, width=8, rows=5, dim=6, table=d, stride=6, code=0, out=d):
        return lib.kbc_embed(tokens, ids, width, rows, dim, table, stride, code, 1.0, out, None)

    for bad in (dict(tokens=-1), dict(tokens=(1 << 30) + 1), dict(ids=None), dict(width=2),
                dict(rows=0), dict(rows=(1 << 31) - 1), dict(dim=0), dict(dim=65537),
                dict(table=None), dict(stride=5), dict(code=3), dict(out=None)):
        assert plain(**bad) == 1, bad
    assert plain(tokens=0, ids=None, out=None) == 0

    def pool(tokens=8192, bags=2, offsets=d, code=0, out=d, scratch=d, size=1 << 40):
        return lib.kbc_embed_pool(tokens, d, 8, bags, offsets, 5, 6, d, 6, code, 1.0, 1, out,
                                  scratch, size, None)

    need = lib.kbc_embed_pool_scratch_size(8192, 2, 1, 6, 0, 1)
    assert need > 0
    for bad in (dict(bags=-1), dict(tokens=8191, offsets=None), dict(out=None), dict(code=-1),
                dict(scratch=None), dict(size=need - 1), dict(scratch=P(8))):
        assert pool(**bad) == 1, bad

    def back(tokens=10, bags=0, offsets=None, dout=d, out=d, scratch=d, size=1 << 40, code=1):
        return lib.kbc_embed_backward(tokens, d, 4, bags, offsets, 5, 6, dout, code, 1.0, 0, out,
                                      scratch, size, None)

    need = lib.kbc_embed_backward_scratch_size(10, 0, 6, 1, 0)
    assert need > 0
    for bad in (dict(tokens=-2), dict(bags=3), dict(dout=None), dict(out=None),
                dict(scratch=None), dict(size=need - 1), dict(scratch=P(4)), dict(code=7)):
        assert back(**bad) == 1, bad


def test_python_refusals():
    """What is refused before anything is enqueued, on tensors of any device."""
    import torch
    from paper_2002_06115_amd import chain as c
    t, i = torch.zeros((4, 3)), torch.zeros(5, dtype=torch.int64)
    with pytest.raises(TypeError):
        c.embed(t, i)  # not on a GPU
    with pytest.raises(TypeError):
        c.embed(t.double(), i)
    with pytest.raises(TypeError):
        c.embed_backward(t, i, 4)


@pytest.mark.gpu
def test_python_refusals_on_the_gpu(chain):
    import torch
    t = torch.zeros((4, 6), device="cuda")
    i = torch.zeros(8, dtype=torch.int64, device="cuda")
    o = torch.zeros(3, dtype=torch.int64, device="cuda")
    for error, call in [
            (TypeError, lambda: chain.embed(t.double(), i)),
            (TypeError, lambda: chain.embed(t, i.float())),
            (TypeError, lambda: chain.embed(t, i.cpu())),
            (TypeError, lambda: chain.embed(t, i, o.int(), pool="sum")),
            (ValueError, lambda: chain.embed(t[0], i)),
            (ValueError, lambda: chain.embed(t.t(), i)),
            (ValueError, lambda: chain.embed(t[:1].expand(4, 6), i)),
            (ValueError, lambda: chain.embed(t[:0], i)),
            (ValueError, lambda: chain.embed(t, i[::2])),
            (ValueError, lambda: chain.embed(t, i, o)),
            (ValueError, lambda: chain.embed(t, i, pool="sum")),
            (ValueError, lambda: chain.embed(t, i, o[:0], pool="sum")),
            (ValueError, lambda: chain.embed(t, i.view(2, 4), o, pool="sum")),
            (ValueError, lambda: chain.embed(t, i, o, pool="max")),
            (ValueError, lambda: chain.embed_backward(t, i, 4)),
            (ValueError, lambda: chain.embed_backward(t[:3], i, 4, o, pool="sum"))]:
        with pytest.raises(error):
            call()
    with pytest.raises(ValueError):
        chain.embed_backward(t, i[:4], 0)
    assert chain.embed(t, i[:0]).shape == (0, 6)
    table = t.clone().requires_grad_()
    none = chain.embed(table, i[:0])
    assert not torch.autograd.grad(none, table, torch.ones_like(none))[0].any()
    assert chain.embed(t, i[:0].view(0, 4), pool="mean").shape == (0, 6)
    assert not chain.embed_backward(t[:0], i, 4, o[:1], pool="sum").any()
