"""chain.embed at the ends of its sizes and of its types' ranges."""
import pytest


@pytest.fixture(scope="module")
def chain():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2002_06115_amd import chain
    return chain


@pytest.mark.gpu
def test_tokens_past_one_grid(chain):
    """2^28 tokens and some, rows of 257 values that take 64 lanes: 138 GB."""
    import torch
    tokens, dim = (1 << 28) + 1000, 257
    need = tokens * (2 * dim + 4)
    if torch.cuda.mem_get_info()[1] < need + (8 << 30):
        pytest.skip("not enough memory")
    table = torch.arange(5 * dim, device="cuda").view(5, dim).half()
    ids = torch.arange(tokens, device="cuda", dtype=torch.int32).remainder_(6)  # 5: padding
    out = chain.embed(table, ids)
    wants = torch.cat([table, torch.zeros_like(table[:1])])
    for at in (0, (1 << 28) - 5000, tokens - 2001):
        assert torch.equal(out[at:at + 2001], wants[ids[at:at + 2001].long()])
    for at in range(0, tokens, 1 << 22):  # every row, by its first value and its last
        part = out[at:at + (1 << 22)]
        want = wants[ids[at:at + (1 << 22)].long()]
        assert torch.equal(part[:, 0], want[:, 0]) and torch.equal(part[:, -1], want[:, -1])
    del out, ids
    torch.cuda.empty_cache()  # for the tests after this one


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [3, 64, 1001])
@pytest.mark.parametrize("tokens", [700, 5000, 70_000])
def test_large_values(chain, tokens, dim):
    """Sums that pass a float's range on the way to a mean, or to a scaled sum, that does
    not: powers of two, so every step is exact."""
    import torch
    top = 2.0 ** 127
    table = torch.full((3, dim), top, dtype=torch.bfloat16, device="cuda")
    table[1] = -top
    ids = torch.zeros(tokens, dtype=torch.int64, device="cuda")
    offsets = torch.tensor([0, tokens], device="cuda")
    mean = chain.embed(table, ids, offsets, pool="mean")
    assert (mean == top).all()
    n = tokens // 64 * 64
    small = chain.embed(table, ids[:n], offsets.clamp(max=n), scale=2.0 ** -20, pool="sum")
    assert (small == torch.tensor(n * 2.0 ** 107).to(torch.bfloat16).item()).all()
    ids[tokens // 2:tokens // 2 * 2] = 1  # as many of the opposite
    ids[tokens // 2 * 2:] = -1
    ids[0] = 2
    table[2] = top / 2
    total = chain.embed(table, ids, offsets, pool="sum")
    assert (total == -top / 2).all()

    dout = torch.full((tokens, dim), top, dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(tokens, dtype=torch.int64, device="cuda")
    back = chain.embed_backward(dout[:n], ids[:n], 2, scale=2.0 ** -20)
    assert (back[0] == torch.tensor(n * 2.0 ** 107).to(torch.bfloat16).item()).all()
    assert not back[1].any()
