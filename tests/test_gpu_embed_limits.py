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
