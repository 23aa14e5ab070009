"""The operators beside the plan and autograd: gradients of any layout, and inputs for which there are none."""
import pytest

torch = pytest.importorskip("torch")

import paper_2506_06095_amd as smha  # noqa: E402
from paper_2506_06095_amd import cache, sink  # noqa: E402

WAYS = pytest.mark.parametrize("native", [True, False], ids=["native", "python"])


def general_way(monkeypatch, native):
    if not native:
        for module, name in ((sink, "_call"), (cache, "_attention"), (cache, "_evict")):
            monkeypatch.setattr(module, name, lambda *args: None)


def randn(*shape, seed=1, dtype=torch.float16):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.gpu
@WAYS
@pytest.mark.parametrize("strides", [(0, 0, 1 << 23, 1), (8, 8, 1 << 23, 1), (1 << 24, 8, 8, 1), (8, 12, 64, 1), (0, 0, 0, 0)], ids=str)
def test_gradients_of_any_layout(monkeypatch, native, strides):
    """A gradient comes as what follows leaves it: heads merged by a transpose of 2 GiB and more, expanded, overlapping.  What the kernels cannot read as it
    lies is copied: as with a packed copy."""
    general_way(monkeypatch, native)
    x = [randn(1, h, 3, 64, seed=i).requires_grad_() for i, h in enumerate((2, 1, 1))]
    room = randn(1 + (1 << 24) + 1024, seed=9)
    g = room.as_strided((1, 2, 3, 64), strides)
    want = torch.autograd.grad(smha.sink_attention(*x, 2, 1), x, g.contiguous())
    got = torch.autograd.grad(smha.sink_attention(*x, 2, 1), x, g)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
