"""Entity sets kept in 8 bits (kbf.pack) and the backward pass that reads them.

The kept values have no tolerance: they are the nearest e4m3 numbers (ties to even)
times a power of two.  The gradients are sums in double of exact products, rounded
once, like those of float sets: against the oracle's double sums over the kept values
within rtol 1e-5 / atol 1e-7 (gpu_util), and from five columns on, where both take the
same chunks in the same order, bitwise what the kept values give as floats.
"""
import ctypes

import numpy as np
import pytest

import oracle
from gpu_util import assert_bitexact, assert_close, from_em, to_em


@pytest.fixture(scope="module")
def kbf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2002_06115_amd as kbf
    return kbf


def kept(X):
    """(values, exponents) that a row-wise e4m3 with the smallest fitting power of two
    keeps of X [rows][b], in float64."""
    X = X.astype(np.float64)
    finite = np.isfinite(X)
    top = np.where(finite, np.abs(X), 0.0).max(1)
    m, k = np.frexp(top)                       # top = m 2^k, m in [1/2, 1)
    e = np.where(top > 0, k - 9 + (m > 0.875), -126)
    e = np.maximum(e, -126)
    x = np.ldexp(np.where(finite, X, 0.0), -e[:, None])
    _, k = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(k - 1, -6) - 3)
    code = np.rint(x / step) * step
    # 256 * 2^120 is past the largest float: 240 * 2^120 is the last value.
    most = np.where(e == 120, 240.0, 448.0)[:, None]
    return np.where(finite, np.ldexp(np.clip(code, -most, most), e[:, None]), np.nan), e


WIDTHS = [1, 2, 3, 4, 5, 6, 7, 8, 10, 31, 32, 33, 64, 93, 128, 129, 255, 256, 257, 300, 1000]


def check_pack(kbf, X):
    import torch
    P = kbf.pack(torch.from_numpy(X).cuda())
    assert P.shape == X.shape
    got = P.unpack().cpu().numpy().astype(np.float64)
    want, e = kept(X)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])
    # The exponent, where a row keeps it: a byte behind the codes up to 3 values, a
    # float before every eight dwords of them from 4 on.
    data, b = P.data.cpu().numpy(), X.shape[1]
    if b < 4:
        assert np.array_equal(data[:, b].astype(np.int64), e + 127)
    else:
        scale = np.ascontiguousarray(data).view(np.float32)[:, ::9]
        assert scale.shape[1] == -(-b // 32) and (scale == np.exp2(e)[:, None]).all()
    return P


@pytest.mark.gpu
@pytest.mark.parametrize("b", WIDTHS)
def test_kept_values(kbf, b):
    g = np.random.default_rng(b)
    for rows in (1, 2, 63, 777):
        X = g.standard_normal((rows, b)) * np.exp2(g.integers(-12, 5, (rows, b)))
        X[g.random((rows, b)) < 0.3] = 0.0
        X *= np.exp2(g.integers(-140, 126, (rows, 1)))
        X = X.clip(-3e38, 3e38).astype(np.float32)
        check_pack(kbf, X)


@pytest.mark.gpu
def test_every_code_and_every_tie(kbf):
    """All values of the format, the midpoints between neighbours and the floats next
    to those, under the largest of a row: 448."""
    bits = np.arange(128)
    s, m = bits >> 3, bits & 7
    v = np.where(s == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (s - 10.0))[:127]
    mid = (v[1:] + v[:-1]) / 2
    near = np.concatenate([np.nextafter(mid.astype(np.float32), np.float32(a)) for a in (0, 1e9)])
    row = np.concatenate([v, mid, near]).astype(np.float32)
    for scale in (1.0, 2.0 ** -100, 2.0 ** 119):
        X = np.stack([row, -row]) * np.float32(scale)
        check_pack(kbf, X)
    assert v[-1] == 448.0


@pytest.mark.gpu
def test_edges_of_the_exponent(kbf):
    """A row's largest value at, and next to, 1.75 times a power of two; rows of zeros,
    of denormals, of the largest floats."""
    tops = []
    for k in (-126, -120, -3, 0, 7, 127):
        t = np.float32(1.75) * np.exp2(np.float32(k))
        tops += [t, np.nextafter(t, np.float32(0)), np.nextafter(t, np.float32(np.inf)),
                 np.exp2(np.float32(k))]
    tops += [0.0, 1e-45, 1e-40, np.finfo(np.float32).max]
    X = np.zeros((len(tops), 9), np.float32)
    X[:, 4] = tops
    X[:, 7] = -np.float32(0.5) * X[:, 4]
    P = check_pack(kbf, X)
    assert np.signbit(P.unpack().cpu().numpy()[0, 7])
    import torch
    Z = kbf.pack(torch.tensor([[0.0, -0.0]], device="cuda")).unpack().cpu().numpy()
    assert not Z.any() and list(np.signbit(Z[0])) == [False, True]


@pytest.mark.gpu
@pytest.mark.parametrize("b", [1, 3, 6, 40, 300])
def test_infinities_and_nan(kbf, b):
    g = np.random.default_rng(b)
    X = g.standard_normal((50, b)).astype(np.float32)
    X[g.random((50, b)) < 0.2] = np.inf
    X[g.random((50, b)) < 0.2] = -np.inf
    X[g.random((50, b)) < 0.2] = np.nan
    X[3] = np.nan
    check_pack(kbf, X)


@pytest.mark.gpu
def test_error_bound(kbf):
    """Half a step: 2^-4 of the value, or 2^-10 of the row's unit."""
    import torch
    g = np.random.default_rng(2)
    X = (g.standard_normal((4000, 24)) * np.exp2(g.integers(-20, 1, (4000, 24)))).astype(np.float32)
    got = kbf.pack(torch.from_numpy(X).cuda()).unpack().cpu().numpy().astype(np.float64)
    unit = np.abs(X).max(1, keepdims=True) / 224.0
    assert (np.abs(got - X) <= np.maximum(2.0 ** -4 * np.abs(X), 2.0 ** -10 * unit)).all()


@pytest.mark.gpu
def test_past_32_bits(kbf):
    """More than 2^32 values."""
    import torch
    X = torch.zeros((33_600_000, 128), device="cuda")
    X[-1] = 3.0
    X[-2, 5] = 0.1
    U = kbf.pack(X).unpack()
    assert (U[-1] == 3.0).all() and abs(float(U[-2, 5]) - 0.1) <= 0.1 * 2.0 ** -4
    assert not U[0].any() and float(U[-2].sum()) == float(U[-2, 5])


def small_kb(seed, n_e=300, n_r=7, n_t=6000):
    g = np.random.default_rng(seed)
    s = np.where(g.random(n_t) < 0.3, g.integers(0, 3, n_t), g.integers(0, n_e, n_t))
    o = np.where(g.random(n_t) < 0.3, g.integers(0, 3, n_t), g.integers(0, n_e, n_t))
    return s.astype(np.int32), g.integers(0, n_r, n_t).astype(np.int32), o.astype(np.int32), n_e, n_r


def check_backward(kbf, s, r, o, n_e, n_r, b, weight, gamma, seed):
    import torch
    g = np.random.default_rng(seed)
    X = np.exp(2 * g.standard_normal((b, n_e))).astype(np.float32)
    X[g.random(X.shape) < 0.2] = 0.0
    R = g.standard_normal((b, n_r)).astype(np.float32)
    dY = g.standard_normal((b, n_e)).astype(np.float32)
    kb = kbf.KB(s, r, o, n_e, n_r, weight=weight)
    P = kbf.pack(to_em(X))
    dX, dR = kb.follow_backward(P, to_em(R), to_em(dY), residual=gamma)
    U = P.unpack()
    want_dx, want_dr = kb.follow_backward(U, to_em(R), to_em(dY), residual=gamma)
    assert_bitexact(from_em(dX), from_em(want_dx), "dX")
    if b > 4:
        assert_bitexact(from_em(dR), from_em(want_dr), "dR")
    _, ref = oracle.follow_backward(s, r, o, n_e, n_r, from_em(U), R, dY, weight=weight)
    assert_close(from_em(dR), ref, f"dR b={b}")
    # dR alone: no R, no dX.
    none, only = kb.follow_backward(P, None, to_em(dY), want_dx=False, residual=gamma)
    assert none is None and torch.equal(only.view(torch.int32), dR.view(torch.int32))
    kb.close()


@pytest.mark.gpu
@pytest.mark.parametrize("path", ["buffer", "plain", "lanes1", "chunks16"])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("b", [1, 2, 3, 4, 5, 6, 8, 12, 16, 31, 32, 36, 64, 93, 128, 130, 260, 261])
def test_backward(kbf, b, weighted, path, monkeypatch):
    if path == "plain":
        monkeypatch.setenv("KBFOLLOW_PLAIN_LOADS", "1")
    if path == "lanes1":
        monkeypatch.setenv("KBFOLLOW_MAX_LPT", "1")
    if path == "chunks16":
        monkeypatch.setenv("KBFOLLOW_REL_CHUNK", "16")
        monkeypatch.setenv("KBFOLLOW_FAN_IN", "3")
    s, r, o, n_e, n_r = small_kb(b * 7 + weighted)
    w = np.random.default_rng(b).uniform(0.1, 2.0, len(s)).astype(np.float32) if weighted else None
    check_backward(kbf, s, r, o, n_e, n_r, b, w, [None, 0.5][b % 2], b)


@pytest.mark.gpu
@pytest.mark.parametrize("b", [4096, 4101])
def test_backward_wide_rows(kbf, b):
    """Rows past the buffer loads' stride."""
    s, r, o, n_e, n_r = small_kb(b, n_e=40, n_t=500)
    check_backward(kbf, s, r, o, n_e, n_r, b, None, None, b)


@pytest.mark.gpu
@pytest.mark.parametrize("b", [3, 10, 32])
def test_backward_concurrent_passes(kbf, b, monkeypatch):
    """dR on the KB's own stream beside dX."""
    monkeypatch.setenv("KBFOLLOW_OVERLAP_BACKWARD", "1")
    s, r, o, n_e, n_r = small_kb(b, n_e=5000, n_r=40, n_t=60_000)
    check_backward(kbf, s, r, o, n_e, n_r, b, None, None, b)


@pytest.mark.gpu
@pytest.mark.parametrize("n_t", [0, 1, 9])
def test_backward_small_kbs(kbf, n_t):
    s, r, o, n_e, n_r = small_kb(n_t, n_e=5, n_r=4, n_t=n_t)
    check_backward(kbf, s, r, o, n_e, n_r, 6, None, 1.0, n_t)


@pytest.mark.gpu
def test_no_entities(kbf):
    import torch
    none = np.zeros(0, np.int32)
    kb = kbf.KB(none, none, none, 0, 3)
    X = torch.zeros((0, 6), device="cuda").requires_grad_()
    R = torch.ones((3, 6), device="cuda").requires_grad_()
    Y = kbf.follow(kb, X, R, pack=True)
    dX, dR = torch.autograd.grad(Y, (X, R), torch.zeros_like(Y))
    assert dX.shape == (0, 6) and dR.shape == (3, 6) and not dR.any()


@pytest.mark.gpu
@pytest.mark.parametrize("b", [3, 4, 33, 128])
def test_checked_build_counts_nothing(kbf, b):
    import torch
    from paper_2002_06115_amd import build as kbuild
    lib = ctypes.CDLL(kbuild.CHECKED_LIB)
    P, I64, I32, SZ = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t
    lib.kb_create.argtypes = [I64, I64, I64, P, P, P, P, P, ctypes.POINTER(P)]
    lib.kb_destroy.argtypes = [P]
    lib.kb_workspace_size.argtypes = [P, I32]
    lib.kb_workspace_size.restype = SZ
    lib.kb_follow_backward_packed.argtypes = [P, I32, P, P, P, P, P, P, SZ, P]
    lib.kb_checked_violations.argtypes = [ctypes.POINTER(ctypes.c_uint64), I32]
    s, r, o, n_e, n_r = small_kb(b)
    g = np.random.default_rng(b)
    X, R, dY = (to_em(g.random((b, n))) for n in (n_e, n_r, n_e))
    kept_ = kbf.pack(X)
    want = kbf.KB(s, r, o, n_e, n_r).follow_backward(kept_, R, dY)
    h, count = P(), ctypes.c_uint64(1)
    ptr = lambda a: a.ctypes.data_as(P)  # noqa: E731
    assert lib.kb_create(n_e, n_r, len(s), ptr(s), ptr(r), ptr(o), None, None, ctypes.byref(h)) == 0
    assert lib.kb_checked_violations(ctypes.byref(count), 1) == 0
    size = lib.kb_workspace_size(h, b)
    ws = torch.empty(max(1, size), dtype=torch.uint8, device="cuda")
    dX, dR = torch.empty_like(X), torch.empty_like(R)
    p = lambda t: P(t.data_ptr())  # noqa: E731
    assert lib.kb_follow_backward_packed(h, b, p(kept_.data), p(R), p(dY),
                                         p(dX), p(dR), p(ws), size,
                                         P(torch.cuda.current_stream().cuda_stream)) == 0
    torch.cuda.synchronize()
    assert lib.kb_checked_violations(ctypes.byref(count), 1) == 0 and count.value == 0
    lib.kb_destroy(h)
    assert torch.equal(dX, want[0]) and torch.equal(dR, want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("residual", [False, True])
def test_autograd(kbf, residual):
    """follow(pack=True): the same output and dX; dR that of the kept values; a three-hop
    chain of them; X's own memory may go."""
    import torch
    s, r, o, n_e, n_r = small_kb(3)
    kb = kbf.KB(s, r, o, n_e, n_r)
    g = np.random.default_rng(3)
    X = to_em(g.random((12, n_e))).requires_grad_()
    R = to_em(g.random((12, n_r))).requires_grad_()
    up = to_em(g.standard_normal((12, n_e)))
    hop = kbf.follow_residual if residual else kbf.follow
    Y, Yp = hop(kb, X, R), hop(kb, X, R, pack=True)
    assert torch.equal(Y, Yp)
    dX, dR = torch.autograd.grad(Yp, (X, R), up)
    want = kb.follow_backward(kbf.pack(X.detach()), R.detach(), up,
                              residual=1.0 if residual else None)
    assert torch.equal(dX, want[0]) and torch.equal(dR, want[1])
    # One side alone.
    (only,) = torch.autograd.grad(hop(kb, X.detach(), R, pack=True), R, up)
    assert torch.equal(only, dR)
    (only,) = torch.autograd.grad(hop(kb, X, R.detach(), pack=True), X, up)
    assert torch.equal(only, dX)
    # A chain: each hop's dR from its own input, kept.
    x, kept_, hops = X, [], 3
    for _ in range(hops):
        kept_.append(x.detach())
        x = hop(kb, x, R * 0.1, pack=True)
    dX, dR = torch.autograd.grad(x, (X, R), up)
    d, total, gamma = up, torch.zeros_like(R), 1.0 if residual else None
    for k in reversed(range(hops)):
        d, part = kb.follow_backward(kbf.pack(kept_[k]), R.detach() * 0.1, d, residual=gamma)
        total += part * 0.1
    assert torch.equal(dX, d)
    # Three terms of one float sum, in another order: three roundings of 2^-24.
    assert torch.allclose(dR, total, rtol=1e-6, atol=1e-6 * float(total.abs().max()))


@pytest.mark.gpu
def test_captured_and_replayed(kbf):
    import torch
    s, r, o, n_e, n_r = small_kb(5, n_e=2000, n_t=30_000)
    kb = kbf.KB(s, r, o, n_e, n_r)
    X = torch.rand((n_e, 20), device="cuda")
    R = torch.rand((n_r, 20), device="cuda")
    dY = torch.randn((n_e, 20), device="cuda")

    def step():
        P = kbf.pack(X)
        return (*kb.follow_backward(P, R, dY), P.unpack())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(3):
        X.mul_(1.3)
        dY.add_(0.25)
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), k


def test_pitch_and_c_refusals():
    import paper_2002_06115_amd as k
    lib, P = k._lib, ctypes.c_void_p
    assert [lib.kb_packed_pitch(b) for b in (-1, 0, 1, 2, 3, 4, 5, 8, 9, 32, 33, 64, 65)] == \
        [0, 0, 2, 4, 4, 8, 12, 12, 16, 36, 44, 72, 80]
    x, c = P(1 << 20), P(1 << 21)  # never dereferenced: checked first
    assert lib.kb_pack(0, 4, None, None, None) == k.KB_OK
    for args in ((-1, 4, x, c), ((1 << 30) + 1, 4, x, c), (5, 0, x, c), (5, 4, None, c),
                 (5, 4, x, None), (5, 4, P((1 << 20) + 4), c), (5, 5, P((1 << 20) + 2), c),
                 (5, 4, x, P((1 << 21) + 2)), (5, 4, x, P((1 << 20) + 16))):
        assert lib.kb_pack(*args, None) == k.KB_EINVAL, args
        rows, b, X, packed = args
        assert lib.kb_unpack(rows, b, packed, X, None) == k.KB_EINVAL, args
    assert lib.kb_follow_backward_packed(None, 4, c, x, x, x, x, None, 0, None) == k.KB_EINVAL


def test_python_refusals():
    import torch
    import paper_2002_06115_amd as k
    with pytest.raises(TypeError):
        k.pack(torch.zeros((3, 4)))
    with pytest.raises(TypeError):
        k.Packed(torch.zeros((3, 8), dtype=torch.uint8), 4)


@pytest.mark.gpu
def test_python_refusals_on_the_gpu(kbf):
    import torch
    X = torch.zeros((6, 5), device="cuda")
    P = kbf.pack(X)
    kb = kbf.KB(np.array([0]), np.array([0]), np.array([1]), 6, 2)
    R = torch.zeros((2, 5), device="cuda")
    for error, call in [
            (TypeError, lambda: kbf.pack(X.double())),
            (ValueError, lambda: kbf.pack(X[0])),
            (ValueError, lambda: kbf.pack(X.t())),
            (ValueError, lambda: kbf.pack(X[:, :0])),
            (TypeError, lambda: kbf.Packed(P.data.int(), 5)),
            (ValueError, lambda: kbf.Packed(P.data, 9)),
            (ValueError, lambda: kbf.Packed(P.data, 0)),
            (ValueError, lambda: kbf.Packed(P.data[::2], 5)),
            (ValueError, lambda: kb.follow_backward(kbf.pack(X[:5]), R, X)),
            (ValueError, lambda: kb.follow_backward(kbf.pack(torch.zeros((6, 4), device="cuda")),
                                                    R, X)),
            (TypeError, lambda: kb.follow(P, R))]:
        with pytest.raises(error):
            call()
    # Overlaps, and no codes, are refused by the library.
    ws = kb.workspace(5)
    at = (None, 0) if ws is None else (ws.data_ptr(), ws.numel())
    out = torch.zeros((6, 5), device="cuda")
    go = lambda packed, dx: kbf._lib.kb_follow_backward_packed(  # noqa: E731
        kb._handle, 5, packed, R.data_ptr(), X.data_ptr(), dx, None, *at, None)
    assert go(None, out.data_ptr()) == kbf.KB_EINVAL
    assert go(out.data_ptr(), out.data_ptr()) == kbf.KB_EINVAL
    assert kbf.pack(X[:0]).unpack().shape == (0, 5)
