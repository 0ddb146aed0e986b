"""Penalties, biases and masks on logits (chain.constrain) and their gradients,
against the formulas in 64 bits.

Tolerances.  The output is float: an element of no history is one float addition (half
a step, 2^-24 of the value); one of a history is computed in double and rounded once.
dz is one product or quotient in double, rounded to float and, in a 16-bit type, from
there (2^-8 bfloat16, 2^-11 float16; float16 has half its smallest step, 2^-25, below its
normal numbers).  A shared bias' gradient is a sum in double, rounded once: 2^-24 of it,
and 2^-53 n of the sum of sizes.
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


def counts(history, offsets, n, b):
    c = np.zeros((n, b))
    if history is None:
        return c
    for col in range(b):
        ids = history[col] if offsets is None else history[offsets[col]:offsets[col + 1]]
        for i in ids:
            if 0 <= i < n:
                c[i, col] += 1
    return c


def oracle(z, bias, allowed, c, repeat, presence, frequency, fill, dout):
    v = z.copy()
    slope = np.where(c > 0, np.where(z > 0, 1.0 / repeat, repeat), 1.0)
    with np.errstate(invalid="ignore"):
        v = np.where(c > 0, v * np.where(z > 0, 1.0, repeat) / np.where(z > 0, repeat, 1.0)
                     - (presence + frequency * c), v)
        if bias is not None:
            v = v + (bias if bias.ndim == 2 else bias[:, None])
    ok = np.ones(z.shape, bool)
    if allowed is not None:
        ok = np.broadcast_to(allowed if allowed.ndim == 2 else allowed[:, None], z.shape)
    g = np.where(ok, dout, 0.0)
    return np.where(ok, v, fill), g * slope, g


def words(allowed):
    n = allowed.shape[0]
    pad = np.zeros((-(-n // 32) * 32, *allowed.shape[1:]), np.uint32)
    pad[:n] = allowed
    at = np.arange(32, dtype=np.uint32).reshape(1, 32, *[1] * (allowed.ndim - 1))
    w = (pad.reshape(-1, 32, *allowed.shape[1:]) << at).sum(1, dtype=np.uint32)
    return w.view(np.int32)


def cuda(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def close(got, want, rel, what, least=0.0):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape, what
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        near = np.abs(got - want) <= rel * np.abs(want) + least
    assert (same | near).all(), f"{what}: {np.argwhere(~(same | near))[:3]}"


def run(chain, g, n, b, dtype, bias, mask, ragged, length, scalars=False, fill=-np.inf,
        int_dtype="int64"):
    import torch
    z = torch.from_numpy(3 * g.standard_normal((n, b)).astype(np.float32)).cuda()
    z = z.to(getattr(torch, dtype))
    z64 = z.double().cpu().numpy()
    bias = {"none": None, "row": g.standard_normal(n).astype(np.float32),
            "each": g.standard_normal((n, b)).astype(np.float32)}[bias]
    allowed = None
    if mask != "none":
        allowed = g.random((n,) if mask.endswith("row") else (n, b)) < 0.6
        if allowed.ndim == 2 and b > 2:
            allowed[:, 1] = False  # nothing is left to this column
    history = offsets = None
    if length:
        if ragged:
            offsets = np.sort(g.integers(0, length * b + 1, b + 1))
            offsets[0], offsets[-1] = 0, length * b
            history = g.integers(-1, min(n, 40) + 1, length * b)
        else:
            history = g.integers(-1, min(n, 40) + 1, (b, length))
        history = np.where(history >= min(n, 40), n, history)  # padding on either side
    pen = [g.uniform(lo, hi, b).astype(np.float32) for lo, hi in ((0.7, 1.6), (0, 1), (-0.1, 0.4))]
    if scalars:
        pen = [np.float32(1.3), np.float32(0.5), np.float32(0.25)]
    dout = g.standard_normal((n, b)).astype(np.float32)
    c = counts(history, offsets, n, b)
    want, dz_want, db_want = oracle(z64, bias, allowed, c, *[p.astype(np.float64) for p in pen],
                                    fill, dout.astype(np.float64))
    args = dict(history=cuda(None if history is None else history.astype(int_dtype)),
                offsets=cuda(None if offsets is None else offsets.astype(int_dtype)),
                allowed=cuda(words(allowed) if mask.startswith("bits") else allowed))
    if history is not None:
        for name, p in zip(("repeat", "presence", "frequency"), pen):
            args[name] = float(p) if scalars else cuda(p)
    zg, bg = z.clone().requires_grad_(), cuda(bias)
    if bg is not None:
        bg.requires_grad_()
    out = chain.constrain(zg, bias=bg, fill=fill, **args)
    assert out.dtype == torch.float32
    close(out.detach(), want, 2.0 ** -24, "out", 2.0 ** -149)
    up = cuda(dout)
    grads = torch.autograd.grad(out, (zg,) if bg is None else (zg, bg), up)
    close(grads[0], dz_want, ROUND[dtype] + 2.0 ** -23, "dz",
          2.0 ** -25 if dtype == "float16" else 2.0 ** -149)
    assert grads[0].dtype == z.dtype
    if bg is not None:
        db = db_want if bias.ndim == 2 else db_want.sum(1)
        slack = 0.0 if bias.ndim == 2 else 2.0 ** -53 * b * np.abs(db_want).sum(1).max()
        close(grads[1], db, 2.0 ** -24, "dbias", slack)
    again = torch.autograd.grad(chain.constrain(zg, bias=bg, fill=fill, **args),
                                (zg,) if bg is None else (zg, bg), up)
    for x, y in zip(grads, again):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


SHAPES = [(1, 1), (1, 300), (31, 2), (32, 3), (33, 4), (18, 128), (65, 7), (1000, 17), (700, 64),
          (43, 130), (5, 4097), (3, 9001), (40_000, 1), (9000, 5)]


@pytest.mark.gpu
@pytest.mark.parametrize("mask", ["none", "bool_row", "bool", "bits_row", "bits"])
@pytest.mark.parametrize("n,b", SHAPES)
def test_shapes_and_masks(chain, n, b, mask):
    g = np.random.default_rng(n * 31 + b)
    dtype = ["float32", "bfloat16", "float16"][(n + b) % 3]
    bias = ["none", "row", "each"][(n + len(mask)) % 3]
    run(chain, g, n, b, dtype, bias, mask, ragged=b % 2 == 1, length=min(9, 4000 // b + 1))


@pytest.mark.gpu
@pytest.mark.parametrize("bias", ["none", "row", "each"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_types_and_biases(chain, dtype, bias):
    g = np.random.default_rng(len(dtype) * 3 + len(bias))
    for b in (6, 12, 24, 48, 96, 192, 260):
        run(chain, g, 260, b, dtype, bias, "bits", ragged=True, length=5, int_dtype="int32")


@pytest.mark.gpu
@pytest.mark.parametrize("mask", ["none", "bool", "bits_row"])
@pytest.mark.parametrize("bias", ["none", "row", "each"])
@pytest.mark.parametrize("n,b,length", [(1, 1, 1024), (3, 1, 1025), (2000, 1024, 1), (70, 1025, 1),
                                        (600, 256, 4), (600, 257, 3), (1023, 2, 512), (9, 340, 3)])
def test_few_and_many_ids(chain, n, b, length, bias, mask):
    """At and past the sizes where one launch does both."""
    g = np.random.default_rng(n + b + length)
    run(chain, g, n, b, ["float32", "bfloat16"][n % 2], bias, mask, n % 2 == 0, length)


@pytest.mark.gpu
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("length,b", [(1, 5), (31, 3), (33, 2), (2047, 1), (2049, 2), (5000, 3)])
def test_long_histories(chain, length, b, ragged):
    """Columns' histories within a workgroup's entries, across them, and across the
    blocks of ids that are compared at a time."""
    g = np.random.default_rng(length)
    run(chain, g, 900, b, "float32", "row", "bool", ragged, length)


def spread(ids):
    """The 32 bits that a column's table takes the place (the lower 11) and the slice
    (from bit 19 down) of an id from."""
    h = ids.astype(np.uint32) * np.uint32(0x9E3779B9)
    return (h ^ h >> np.uint32(15)) * np.uint32(0x9E3779B9)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["any", "one place", "one slice", "one id"])
@pytest.mark.parametrize("n,b,length", [(300_000, 1, 1800), (300_000, 3, 2049), (400_000, 2, 9000),
                                        (20_000, 600, 64), (50_000, 9, 130)])
def test_histories_of_many_ids(chain, n, b, length, kind):
    """Columns of up to thousands of different ids, also where their places in a
    table collide, more than it has; a column of one id, an empty one, and padding."""
    import torch
    g = np.random.default_rng(n + b + length)
    ids = np.arange(n)
    if kind == "one place":
        ids = ids[spread(ids) % 2048 < 8]
    elif kind == "one slice":
        ids = ids[spread(ids) >> 14 & 63 == 63]
    elif kind == "one id":
        ids = ids[-1:]
    history = g.choice(ids, b * length)
    history[::7] = history[0]
    history[5::11] = -1
    offsets = np.arange(b + 1) * length
    if b > 2:
        offsets[1] = offsets[2]
    z = torch.from_numpy(g.standard_normal((n, b)).astype(np.float32)).cuda()
    allowed = g.random(n) < 0.9
    c = counts(history, offsets, n, b)
    pen = [g.uniform(lo, hi, b).astype(np.float32) for lo, hi in ((0.7, 1.6), (0, 1), (-0.1, 0.4))]
    want, _, _ = oracle(z.double().cpu().numpy(), None, allowed, c,
                        *[p.astype(np.float64) for p in pen], -1e9, np.zeros((n, b)))
    got = chain.constrain(z, history=cuda(history), offsets=cuda(offsets), allowed=cuda(allowed),
                          repeat=cuda(pen[0]), presence=cuda(pen[1]), frequency=cuda(pen[2]),
                          fill=-1e9)
    close(got, want, 2.0 ** -24, "out", 2.0 ** -149)


@pytest.mark.gpu
@pytest.mark.parametrize("penalty", ["repeat", "presence"])
@pytest.mark.parametrize("n,b,length", [(9000, 7, 900), (400, 130, 21), (60, 900, 3), (4000, 1, 5000)])
def test_histories_that_nothing_counts(chain, n, b, length, penalty):
    """Only whether an id occurs matters: ragged columns, empty ones, one of half the ids."""
    import torch
    g = np.random.default_rng(n + b)
    history = g.integers(-2, n + 2, b * length)
    offsets = np.sort(g.integers(0, b * length + 1, b + 1))
    offsets[0], offsets[-1] = 0, b * length
    offsets[1:b // 2] = min(offsets[1:b // 2], default=0)
    z = torch.from_numpy(g.standard_normal((n, b)).astype(np.float32)).cuda()
    args = dict(repeat=np.ones(b), presence=np.zeros(b))
    args[penalty] = g.uniform(0.5, 2, b).astype(np.float32).astype(np.float64)
    dout = g.standard_normal((n, b)).astype(np.float32)
    want, dz, _ = oracle(z.double().cpu().numpy(), None, None, counts(history, offsets, n, b),
                         args["repeat"], args["presence"], 0.0, 0.0, dout.astype(np.float64))
    zg = z.requires_grad_()
    got = chain.constrain(zg, history=cuda(history), offsets=cuda(offsets),
                          **{penalty: cuda(args[penalty].astype(np.float32))})
    close(got.detach(), want, 2.0 ** -24, "out", 2.0 ** -149)
    got, = torch.autograd.grad(got, zg, cuda(dout))
    close(got, dz, ROUND["float32"] + 2.0 ** -23, "dz", 2.0 ** -149)


@pytest.mark.gpu
def test_numbers_for_all_columns(chain):
    g = np.random.default_rng(11)
    run(chain, g, 200, 9, "float32", "each", "bool_row", True, 12, scalars=True)
    run(chain, g, 200, 9, "bfloat16", "row", "bits_row", False, 12, scalars=True, fill=-1e30)
    run(chain, g, 200, 9, "bfloat16", "none", "none", False, 0)


@pytest.mark.gpu
def test_non_finite_values(chain):
    """Masked places hold the fill whatever stood there; the type's lowest value and
    infinities elsewhere stay what the formula makes of them."""
    import torch
    low = torch.finfo(torch.float32).min
    z = torch.tensor([[float("nan"), float("inf")], [float("-inf"), low], [float("nan"), 1.0],
                      [0.0, -0.0]], device="cuda")
    allowed = torch.tensor([[False, False], [True, True], [True, False], [True, True]],
                           device="cuda")
    history = torch.tensor([[0, 1, 2, 3], [0, 1, 2, 3]], device="cuda")
    out = chain.constrain(z, allowed=allowed, history=history, repeat=2.0, fill=low)
    inf = float("inf")
    want = torch.tensor([[low, low], [-inf, -inf], [float("nan"), low], [0.0, 0.0]], device="cuda")
    assert torch.equal(torch.nan_to_num(out, nan=7.0), torch.nan_to_num(want, nan=7.0))
    dout = torch.tensor([[float("nan"), inf], [1.0, 1.0], [2.0, float("nan")], [3.0, 3.0]],
                        device="cuda")
    dz, db = chain.constrain_backward(dout, z, allowed, history, repeat=2.0, bias_dims=1)
    assert torch.equal(dz, torch.tensor([[0.0, 0.0], [2.0, 2.0], [4.0, 0.0], [6.0, 6.0]],
                                        device="cuda"))
    assert torch.equal(db, torch.tensor([0.0, 2.0, 2.0, 6.0], device="cuda"))


@pytest.mark.gpu
def test_against_differences(chain):
    """Away from z = 0 the output is linear in z: differences of steps of 2^-4 are off
    by rounding alone, at most 2 * 2^-24 * 16 / 2^-4 < 1e-4."""
    import torch
    g = np.random.default_rng(12)
    z = g.choice([-1.0, 1.0], (6, 3)) * g.uniform(1, 4, (6, 3))
    z = torch.from_numpy(z.astype(np.float32)).cuda()
    history = torch.from_numpy(g.integers(0, 6, (3, 4))).cuda()
    up = torch.from_numpy(g.standard_normal((6, 3)).astype(np.float32)).cuda()
    args = dict(history=history, repeat=1.5, presence=0.3, frequency=0.1)
    zg = z.clone().requires_grad_()
    (dz,) = torch.autograd.grad(chain.constrain(zg, **args), zg, up)
    for i in range(6):
        for c in range(3):
            e = torch.zeros_like(z)
            e[i, c] = 2.0 ** -4
            d = ((chain.constrain(z + e, **args).double() - chain.constrain(z - e, **args)) * up).sum()
            assert abs(float(d) * 8 - float(dz[i, c])) < 1e-4


@pytest.mark.gpu
def test_gradients_of_what_was_saved(chain):
    """Two graphs at once, walked twice, after the callers' own references are gone and
    their memory has been used again; saved tensors that hooks have moved."""
    import torch
    g = np.random.default_rng(17)

    def graph(seed):
        gen = np.random.default_rng(seed)
        z = torch.from_numpy(gen.standard_normal((300, 8)).astype(np.float32)).cuda().requires_grad_()
        history = torch.from_numpy(gen.integers(0, 300, (8, 20))).cuda()
        allowed = torch.from_numpy(gen.random((300, 8)) < 0.7).cuda()
        repeat = torch.from_numpy(gen.uniform(1.1, 2.0, 8).astype(np.float32)).cuda()
        out = chain.constrain(z, allowed=allowed, history=history, repeat=repeat,
                              presence=torch.rand(8, device="cuda"))
        table = torch.from_numpy(gen.standard_normal((90, 5)).astype(np.float32)).cuda()
        table.requires_grad_()
        q = chain.embed(table, history % 90, pool="mean")
        return (z, out), (table, q)

    up = torch.from_numpy(g.standard_normal((300, 8)).astype(np.float32)).cuda()
    uq = torch.from_numpy(g.standard_normal((8, 5)).astype(np.float32)).cuda()
    walk = lambda s: [torch.autograd.grad(s[0][1], s[0][0], up, retain_graph=True)[0],  # noqa: E731
                      torch.autograd.grad(s[1][1], s[1][0], uq, retain_graph=True)[0]]
    want = [walk(graph(seed)) for seed in (1, 2)]
    both = [graph(seed) for seed in (1, 2)]
    junk = [torch.full((20_000,), 3, device="cuda") for _ in range(50)]
    for _ in range(2):
        for s, w in zip(both, want):
            assert all(torch.equal(a, b) for a, b in zip(walk(s), w))
    del junk
    with torch.autograd.graph.save_on_cpu():
        s = graph(1)
    assert all(torch.equal(a, b) for a, b in zip(walk(s), want[0]))


@pytest.mark.gpu
def test_unaligned_arrays(chain):
    import torch
    g = np.random.default_rng(13)
    base = torch.from_numpy(g.standard_normal(2001).astype(np.float32)).cuda()
    z, bias = base[1:1 + 40 * 25].view(40, 25), base[3:43]
    assert torch.equal(chain.constrain(z, bias=bias), z + bias[:, None])
    zb = base.bfloat16()[1:1 + 40 * 25].view(40, 25)
    assert torch.equal(chain.constrain(zb), zb.float())


@pytest.mark.gpu
def test_captured_and_replayed(chain):
    import torch
    g = np.random.default_rng(14)
    z = torch.from_numpy(g.standard_normal((500, 20)).astype(np.float32)).cuda()
    history = torch.from_numpy(g.integers(0, 500, (20, 30))).cuda()
    dout, bias = torch.randn_like(z), torch.randn(500, device="cuda")

    def step():
        out = chain.constrain(z, bias=bias, history=history, repeat=1.2, presence=0.1,
                              frequency=0.2)
        return out, *chain.constrain_backward(dout, z, None, history, None, 1.2, 1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(3):
        z.mul_(-1.1)
        dout.add_(0.5)
        history.copy_(torch.roll(history, 1, 0) // (k + 1))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), k


@pytest.mark.gpu
def test_from_words_to_answers(chain):
    """The question's words, their relations' logits, a constrained choice among them
    and a hop that keeps its entity sets in 8 bits, forward and backward, against the
    same step in 64 bits on the CPU.  (k-hot sets, whose halves and ones 8 bits hold.)

    Each stage rounds to float once from sums in double (the product with the weights
    is torch's, in float: 12 terms, 12 * 2^-24 of the sum of sizes); the stages'
    conditions here, logits below 20 in size and sums of positive terms in the hop,
    keep the step within 2e-5 of the largest value of each gradient."""
    import torch
    import paper_2002_06115_amd as kbf
    g = np.random.default_rng(15)
    n_e, n_r, n_t, b, dim = 40, 9, 300, 6, 12
    s, r, o = g.integers(0, n_e, n_t), g.integers(0, n_r, n_t), g.integers(0, n_e, n_t)
    kb = kbf.KB(s, r, o, n_e, n_r)
    words_ = g.integers(0, 30, (b, 5))
    words_[2, 3:] = -1
    used = g.integers(0, n_r, (b, 2))
    allowed = g.random((n_r, b)) < 0.7
    allowed[0] = True
    table = g.standard_normal((30, dim)).astype(np.float32)
    weight = g.standard_normal((n_r, dim)).astype(np.float32)
    bias = g.standard_normal(n_r).astype(np.float32)
    X = g.choice([0.0, 0.5, 1.0], (n_e, b)).astype(np.float32)
    dY = g.random((n_e, b)).astype(np.float32)

    leaves = [cuda(a).requires_grad_() for a in (table, weight, bias)]
    q = chain.embed(leaves[0], cuda(words_), pool="mean")
    rho = chain.constrain(leaves[1] @ q.t(), bias=leaves[2], allowed=cuda(allowed),
                          history=cuda(used), repeat=1.3, presence=0.2, fill=-1e30)
    R = chain.softmax(rho.detach()).requires_grad_()
    Y = kbf.follow(kb, cuda(X), R, pack=True)
    (dR,) = torch.autograd.grad(Y, R, cuda(dY))
    R = R.detach()
    grads = torch.autograd.grad(rho, leaves, chain.softmax_backward(R, dR))

    T, W, B = [torch.from_numpy(a.astype(np.float64)).requires_grad_() for a in (table, weight, bias)]
    ok = torch.from_numpy(words_ >= 0)
    q64 = (T[torch.from_numpy(np.maximum(words_, 0))] * ok[..., None]).sum(1) / ok.sum(1)[:, None]
    z = W @ q64.t()
    c = torch.from_numpy(counts(used, None, n_r, b))
    th = float(np.float32(1.3))
    v = torch.where(c > 0, torch.where(z > 0, z / th, z * th) - float(np.float32(0.2)), z) + B[:, None]
    R64 = torch.softmax(torch.where(torch.from_numpy(allowed), v, torch.tensor(-1e30).double()), 0)
    X64 = torch.from_numpy(X.astype(np.float64))
    Y64 = torch.zeros(n_e, b, dtype=torch.float64).index_add(0, torch.from_numpy(o), X64[s] * R64[r])
    want = torch.autograd.grad(Y64, (T, W, B), torch.from_numpy(dY.astype(np.float64)))
    assert (Y.detach().cpu().double() - Y64).abs().max() <= 2e-5 * Y64.abs().max()
    for got, w in zip(grads, want):
        assert (got.cpu().double() - w).abs().max() <= 2e-5 * w.abs().max()


def test_c_refusals():
    from paper_2002_06115_amd import chain as c
    lib, P = c._lib, ctypes.c_void_p
    d = P(256)  # never dereferenced: arguments are checked first

    def limits(**change):
        l = c._Limits(repeat_all=1.0, id_bytes=8)
        for k, v in change.items():
            setattr(l, k, v)
        return ctypes.byref(l)

    def forward(n=10, b=4, z=d, code=0, out=d, l=None, **change):
        return lib.kbc_constrain(n, b, z, code, l or limits(**change), 0.0, out, None)

    def backward(n=10, b=4, z=d, code=0, dout=d, dz=d, **change):
        return lib.kbc_constrain_backward(n, b, z, code, limits(**change), dout, dz, None, None)

    for bad in (dict(n=0), dict(b=0), dict(z=None), dict(out=None), dict(code=3),
                dict(n=(1 << 31) - 1), dict(n=1 << 30, b=1 << 30)):
        assert forward(**bad) == 1, bad
    for bad in (dict(entries=-1), dict(entries=8), dict(entries=8, history=256, id_bytes=3),
                dict(entries=9, history=256), dict(entries=(1 << 30) + 4, history=256),
                dict(repeat_all=0.0), dict(repeat_all=-1.0), dict(presence_all=float("nan")),
                dict(frequency_all=float("inf"))):
        assert forward(**bad) == 1, bad
        assert backward(**bad) == 1, bad
    for bad in (dict(dout=None), dict(dz=None), dict(code=-1),
                dict(z=None, entries=8, history=256, repeat_all=2.0)):
        assert backward(**bad) == 1, bad


def test_python_refusals():
    import torch
    from paper_2002_06115_amd import chain as c
    with pytest.raises(TypeError):
        c.constrain(torch.zeros((4, 3)))  # not on a GPU
    with pytest.raises(TypeError):
        c.constrain_backward(torch.zeros((4, 3)))


@pytest.mark.gpu
def test_python_refusals_on_the_gpu(chain):
    import torch
    z = torch.zeros((40, 3), device="cuda")
    h = torch.zeros((3, 5), dtype=torch.int64, device="cuda")
    o = torch.zeros(4, dtype=torch.int64, device="cuda")
    for error, call in [
            (TypeError, lambda: chain.constrain(z.double())),
            (ValueError, lambda: chain.constrain(z[0])),
            (ValueError, lambda: chain.constrain(z.t())),
            (ValueError, lambda: chain.constrain(z[:0])),
            (TypeError, lambda: chain.constrain(z, bias=z.half())),
            (ValueError, lambda: chain.constrain(z, bias=z[:39])),
            (ValueError, lambda: chain.constrain(z, bias=z[:1])),
            (TypeError, lambda: chain.constrain(z, allowed=z)),
            (ValueError, lambda: chain.constrain(z, allowed=z[:39] > 0)),
            (ValueError, lambda: chain.constrain(z, allowed=torch.zeros(1, dtype=torch.int32,
                                                                        device="cuda"))),
            (TypeError, lambda: chain.constrain(z, history=h.float())),
            (ValueError, lambda: chain.constrain(z, history=h[:2])),
            (ValueError, lambda: chain.constrain(z, history=h[0])),
            (ValueError, lambda: chain.constrain(z, offsets=o)),
            (ValueError, lambda: chain.constrain(z, history=h[0], offsets=o[:3])),
            (ValueError, lambda: chain.constrain(z, history=h, repeat=0.0)),
            (ValueError, lambda: chain.constrain(z, history=h, presence=float("inf"))),
            (TypeError, lambda: chain.constrain(z, history=h, repeat=z[0].double())),
            (ValueError, lambda: chain.constrain(z, history=h, repeat=z[0, :2])),
            (ValueError, lambda: chain.constrain_backward(z, z[:3])),
            (ValueError, lambda: chain.constrain_backward(z, history=h, repeat=2.0)),
            (ValueError, lambda: chain.constrain_backward(z, bias_dims=3)),
            (TypeError, lambda: chain.constrain_backward(z.half()))]:
        with pytest.raises(error):
            call()


@pytest.mark.gpu
def test_large_offsets(chain):
    """More than 2^31 elements."""
    import torch
    n, b = 33_600_000, 65
    z = torch.zeros((n, b), dtype=torch.bfloat16, device="cuda")
    z[-1, -1], z[-1, 0] = 2.0, -2.0
    history = torch.full((b, 1), n - 1, device="cuda")
    allowed = torch.ones(n, dtype=torch.bool, device="cuda")
    allowed[-2] = False
    out = chain.constrain(z, allowed=allowed, history=history, repeat=4.0, fill=-9.0)
    assert float(out[-1, -1]) == 0.5 and float(out[-1, 0]) == -8.0
    assert (out[-2] == -9.0).all() and not out[:-2].any()
    dz, db = chain.constrain_backward(out, z, allowed, history, repeat=4.0, bias_dims=1)
    assert float(dz[-1, -1]) == 0.125 and float(dz[-1, 0]) == -32.0 and not dz[:-1].any()
    assert float(db[-1]) == -7.5 and not db[:-1].any()


@pytest.mark.gpu
def test_two_streams_at_once(chain):
    """Calls of both operators on two streams, their tensors made on a third."""
    import torch
    g = np.random.default_rng(21)
    table = torch.from_numpy(g.standard_normal((3000, 64)).astype(np.float32)).cuda()
    sets = []
    for k in range(2):
        ids = torch.from_numpy(g.integers(-1, 3000, (40, 300))).cuda()
        z = torch.from_numpy(g.standard_normal((4000, 40)).astype(np.float32)).cuda()
        sets.append((ids, z, torch.cuda.Stream()))

    def step(ids, z):
        q = chain.embed(table, ids, pool="mean")
        out = chain.constrain(z, history=ids, repeat=1.5, frequency=0.1)
        return (q, chain.embed_backward(q, ids, 3000, pool="mean"), out,
                chain.constrain_backward(out, z, None, ids, None, 1.5, 1)[1])

    want = [step(ids, z) for ids, z, _ in sets]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for ids, z, stream in sets:
            stream.wait_stream(torch.cuda.default_stream())
            with torch.cuda.stream(stream):
                got.append(step(ids, z))
    torch.cuda.synchronize()
    for k, outs in enumerate(got):
        for x, y in zip(outs, want[k % 2]):
            assert torch.equal(x, y)
