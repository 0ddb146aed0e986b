"""What chain's operators refuse, beyond what each one's own tests try (CPU where the
checks do not ask for a GPU's tensors)."""
import pytest
import torch

from paper_2002_06115_amd import chain

CPU = torch.device("cpu")
BAD_PENALTIES = [
    (TypeError, lambda like: dict(repeat=like.double())),
    (TypeError, lambda like: dict(frequency=torch.ones(3, dtype=torch.int32, device=like.device))),
    (ValueError, lambda like: dict(presence=like[:2])),
    (ValueError, lambda like: dict(repeat=0.0)),
    (ValueError, lambda like: dict(repeat=-1.5)),
    (ValueError, lambda like: dict(frequency=float("nan"))),
    (ValueError, lambda like: dict(presence=float("inf")))]


@pytest.mark.parametrize("error,penalty", BAD_PENALTIES)
def test_penalties_are_checked_without_a_history(error, penalty):
    p = {**dict(repeat=1.0, presence=0.0, frequency=0.0), **penalty(torch.ones(3))}
    with pytest.raises(error):
        chain._limits(5, 3, CPU, None, None, None, None, p)
    good = chain._limits(5, 3, CPU, None, None, None, None,
                         dict(repeat=torch.ones(3), presence=0.5, frequency=torch.ones(3)))
    assert good.entries == 0


@pytest.mark.gpu
def test_penalties_are_checked_without_a_history_on_the_gpu():
    z = torch.randn(5, 3, device="cuda")
    for error, penalty in BAD_PENALTIES:
        with pytest.raises(error):
            chain.constrain(z, **penalty(z[0].contiguous()))
    zg = z.clone().requires_grad_()
    out = chain.constrain(zg, repeat=z[0].abs() + 1, presence=0.5, frequency=z[1].contiguous())
    assert torch.equal(out, z)  # nothing is in no history
    out.backward(z)
    assert torch.equal(zg.grad, z)
    with pytest.raises(ValueError):
        chain.constrain_backward(z, repeat=0.0)


class OnTheGpu(torch.Tensor):
    """A tensor without memory that says it is on a GPU."""
    is_cuda = True


def without_memory(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="meta").as_subclass(OnTheGpu)


def test_widths_past_32_bits():
    """2^32 + 8 columns are not 8."""
    import paper_2002_06115_amd as kbf
    wide = without_memory(1, 2 ** 32 + 8)
    ids = without_memory(1, dtype=torch.int64)
    codes = without_memory(1, kbf._lib.kb_packed_pitch(8), dtype=torch.uint8)
    for call in (lambda: chain.constrain(wide), lambda: chain.constrain_backward(wide),
                 lambda: chain.constrain_backward(without_memory(1, 8), wide),
                 lambda: chain.softmax(wide), lambda: chain.embed(wide, ids),
                 lambda: chain.embed_backward(wide, ids, 1), lambda: kbf.pack(wide),
                 lambda: kbf.Packed(codes, 2 ** 32 + 8)):
        with pytest.raises(ValueError):
            call()
    assert kbf.Packed(codes, 8).b == 8
