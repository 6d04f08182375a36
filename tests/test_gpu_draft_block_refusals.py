"""A refused way back through the draft block: no gradient is added, and a right one after it gives the bits of one alone."""
import pytest
import torch

from paper_2608_12703_amd import ad
from paper_2608_12703_amd.train import DraftBlock

pytestmark = pytest.mark.gpu

D, F, ROWS, KEYS = 64, 128, 12, 30


def _made():
    g = torch.Generator().manual_seed(4)
    shapes = [(D,), (D,), (3 * D, D), (3 * D,), (D, D), (D,), (D,), (D,), (D, D), (D,), (2 * D, D), (2 * D,), (D, D), (D,), (D,), (D,),
              (F, D), (F,), (D, F), (D,)]
    block = DraftBlock([(torch.randn(s, generator=g) * 0.1).to(torch.bfloat16).cuda() for s in shapes], ROWS, KEYS, 2)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    cu, ck = ints([0, 5, ROWS]), ints([0, 11, KEYS])
    batches = (ad.Attention(1, 1, cu, cu, 7, 7, causal=True, covers=True), ad.Attention(1, 1, cu, ck, 7, 19, covers=True))
    rand = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    return block, batches, rand(ROWS, D), rand(KEYS, D).to(torch.bfloat16), rand(ROWS, D), rand(ROWS, D)


def test_a_refused_way_back_adds_nothing():
    block, batches, x, enc, dout, dxq = _made()
    out, dx = torch.empty_like(x), torch.empty_like(x)
    block.forward(x, enc, *batches, out)
    block.backward(dout, dx, dxq)
    want = [g.clone() for g in block.grads]
    block.zero_grads()
    for bad in ((dout[:5], dx[:5], None), (dout, dx, dxq.half()), (dout, dx, dxq[:, :32]), (dout, dx[:, :32], None), (dout.half(), dx, None),
                (dout, dx, dxq.cpu()), (dout, dx.cpu(), None)):
        with pytest.raises(ValueError):
            block.backward(*bad)
        assert not any(bool(g.any()) for g in block.grads)
    block.backward(dout, dx, dxq)
    assert all(torch.equal(a, b) for a, b in zip(want, block.grads))


def test_a_refused_pass_leaves_nothing_to_go_back_from():
    block, batches, x, enc, dout, _ = _made()
    out, dx = torch.empty_like(x), torch.empty_like(x)
    block.forward(x, enc, *batches, out)
    with pytest.raises(ValueError):
        block.forward(x * 2, enc.float(), *batches, out)
    with pytest.raises(ValueError, match="last forward"):
        block.backward(dout, dx)
    assert not any(bool(g.any()) for g in block.grads)
    block.forward(x, enc, *batches, out)
    block.backward(dout, dx)
    assert all(bool(torch.isfinite(g).all()) for g in block.grads) and any(bool(g.any()) for g in block.grads)
