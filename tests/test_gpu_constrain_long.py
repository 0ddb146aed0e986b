"""Long and uneven histories of chain.constrain, against the formulas in 64 bits (torch,
on the GPU).

Tolerances: an element of a history is computed in double and rounded to float once, every
other is the logit itself: half a step, 2^-24 of the value, or 2^-150.
"""
import numpy as np
import pytest


@pytest.fixture(scope="module")
def chain():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2002_06115_amd import chain
    return chain


PENALTIES = dict(repeat=1.3, presence=0.5, frequency=0.25)


def check(chain, n, b, history, offsets, seed, **penalties):
    """constrain of random logits [n][b] with this history (numpy, ids in [0, n) and
    -1) against the formula, all elements."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = 3 * torch.randn((n, b), device="cuda", generator=gen)
    h = torch.from_numpy(np.ascontiguousarray(history)).cuda()
    o = None if offsets is None else torch.from_numpy(np.ascontiguousarray(offsets)).cuda()
    got = chain.constrain(z, history=h, offsets=o, **penalties)
    if o is None:
        col = torch.arange(b, device="cuda").repeat_interleave(h.shape[1])
    else:
        col = torch.searchsorted(o, torch.arange(h.numel(), device="cuda", dtype=o.dtype),
                                 right=True) - 1
    h = h.reshape(-1)
    valid = (h >= 0) & (h < n) & (col >= 0) & (col < b)
    at, count = torch.unique(h[valid].long() * b + col[valid], return_counts=True)
    p = {k: float(np.float32(v)) for k, v in {**dict(repeat=1, presence=0, frequency=0),
                                               **penalties}.items()}
    x = z.view(-1)[at].double()
    x = torch.where(x > 0, x / p["repeat"], x * p["repeat"]) - p["presence"] - p["frequency"] * count
    off = (got.view(-1)[at].double() - x).abs()
    assert (off <= 2.0 ** -24 * x.abs() + 2.0 ** -150).all()
    rest = got.clone()
    rest.view(-1)[at] = z.view(-1)[at]
    assert torch.equal(rest, z)


def table(ids, slices):
    """(place, slice) of ids in the table that counts a long column's."""
    h = ids.astype(np.uint32) * np.uint32(0x9E3779B9)
    h = (h ^ h >> np.uint32(15)) * np.uint32(0x9E3779B9)
    return h % 2048, (h.astype(np.uint64) * np.uint64(slices) >> np.uint64(32)).astype(np.int64)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["one slice", "few places of one slice", "any"])
def test_ids_that_a_table_cannot_hold(chain, kind):
    """65,536 ids of one slice of a table with 2048 places, and 512 ids of 16 places."""
    g = np.random.default_rng(5)
    n = 1 << 24
    ids = np.arange(n)
    place, sl = table(ids, 256)  # the slice's upper 8 bits: one slice of up to 256, too
    if kind != "any":
        ids = ids[(sl == 37) & (place < (2048 if kind == "one slice" else 16))]
        assert len(ids) > (50_000 if kind == "one slice" else 400)
    for length in (9000, 140_000):
        history = g.choice(ids, length)
        history[::9] = history[0]
        history[4::17] = -1
        check(chain, n, 1, history[None], None, length, **PENALTIES)


@pytest.mark.gpu
def test_ids_that_only_places_of_their_own_hold(chain):
    """Columns of two slices, 1500 ids of 512 places in one of them, among 16,384 rows:
    an eighth of those is the table's size."""
    g = np.random.default_rng(6)
    n, b, length = 16_384, 520, 2000
    place, sl = table(np.arange(n), 2)
    ids = np.flatnonzero((sl == 1) & (place < 512))
    assert len(ids) > 1500
    history = g.choice(ids, (b, length))
    history[1::3] = g.integers(-1, n, history[1::3].shape)
    check(chain, n, b, history, None, 6, **PENALTIES)


@pytest.mark.gpu
def test_a_column_of_two_million_ids(chain):
    """2,000,000 different ids, 1954 slices of the table."""
    n = 2_000_003
    check(chain, n, 1, np.random.default_rng(7).permutation(n)[None, :2_000_000], None, 7,
          **PENALTIES)


def uneven(g, n, lengths):
    """A history of columns of these lengths, a third of it padding or one id."""
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    history = g.integers(0, n, offsets[-1])
    history[::5] = -1
    history[1::7] = n // 2
    return history, offsets


@pytest.mark.gpu
@pytest.mark.parametrize("at", [0, 9_999, 19_999])
def test_one_column_of_nearly_all_ids(chain, at):
    """20,000 columns of 60 ids on average, 1.2 million of them in one."""
    g = np.random.default_rng(at)
    lengths = g.integers(0, 2, 20_000)
    lengths[at] = 1_200_000
    check(chain, 300, 20_000, *uneven(g, 300, lengths), at, **PENALTIES)
    lengths[at] = 150_000
    lengths[(at + 20) % 20_000] = 90_001
    check(chain, 300, 20_000, *uneven(g, 300, lengths), at, **PENALTIES)


@pytest.mark.gpu
@pytest.mark.parametrize("lengths", [
    [4096, 4097, 4095, 0, 1, 8192, 8193, 4096],      # at the length that is shared
    [16_384], [16_385], [0, 0, 16_384, 0, 1],        # at the number from which any is
    [5000] * 13 + [0] * 2000,                        # 31 a column
    [5000] * 13 + [0] * 800,                         # 80 a column
    [0, 300_000, 0, 0, 250_000, 1, 70_000] + [33] * 90,
    [3] * 600 + [40_000] + [3] * 600])
def test_uneven_columns(chain, lengths):
    g = np.random.default_rng(len(lengths))
    history, offsets = uneven(g, 5000, lengths)
    check(chain, 5000, len(lengths), history, offsets, 8, **PENALTIES)
    check(chain, 5000, len(lengths), history, offsets, 8, repeat=1.5)
    # Ids before the first column and behind the last one are of none.
    check(chain, 5000, len(lengths), np.concatenate([history, history])[:len(history) + 9000],
          offsets + 5003, 8, **PENALTIES)


def test_refused_lengths():
    """More ids in one column than a frequency counts, before anything is enqueued."""
    from paper_2002_06115_amd import chain as c
    import ctypes
    d = ctypes.c_void_p(256)  # never dereferenced

    def forward(b, entries, offsets, **change):
        l = c._Limits(repeat_all=1.0, id_bytes=8, entries=entries, history=256, offsets=offsets)
        for k, v in change.items():
            setattr(l, k, v)
        return c._lib.kbc_constrain(10, b, d, 0, ctypes.byref(l), 0.0, d, None)

    for change in (dict(frequency_all=0.5), dict(frequency=256)):
        assert forward(2, (1 << 26) + 2, 256, **change) == 1
        assert forward(2, (1 << 27) + 2, None, **change) == 1
        assert forward(1, (1 << 26) + 1, None, **change) == 1


@pytest.mark.gpu
def test_uneven_columns_replayed(chain):
    """A captured call whose columns' lengths change between replays."""
    import torch
    g = np.random.default_rng(9)
    n, b, total = 3000, 700, 40_000
    z = torch.from_numpy(g.standard_normal((n, b)).astype(np.float32)).cuda()
    h = torch.from_numpy(g.integers(-1, n, total)).cuda()
    lengths = np.zeros((3, b), np.int64)
    lengths[0, 5] = total
    lengths[1] = total // b
    lengths[2, [0, 350, 699]] = 20_000, 15_000, 5000
    offsets = [torch.from_numpy(np.concatenate([[0], np.cumsum(l)])).cuda() for l in lengths]
    o = offsets[0].clone()
    call = lambda: chain.constrain(z, history=h, offsets=o, **PENALTIES)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for k in (1, 2, 0, 1):
        o.copy_(offsets[k])
        h.copy_(h.roll(777))
        graph.replay()
        want = call()
        torch.cuda.synchronize()
        assert torch.equal(out, want), k
    check(chain, n, b, h.cpu().numpy(), offsets[2].cpu().numpy(), 9, **PENALTIES)
