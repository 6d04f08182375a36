"""A refused pass of the draft block leaves nothing to go back from, and a refused way back adds nothing (CPU only: the
sublayers' own calls are refused or replaced)."""
import pytest
import torch

from paper_2608_12703_amd import ad
from paper_2608_12703_amd.train import DraftBlock

BF16 = torch.bfloat16


def _block(d=64, f=128, rows=6, keys=10):
    shapes = [(d,), (d,), (3 * d, d), (3 * d,), (d, d), (d,), (d,), (d,), (d, d), (d,), (2 * d, d), (2 * d,), (d, d), (d,), (d,), (d,),
              (f, d), (f,), (d, f), (d,)]
    block = DraftBlock([torch.zeros(s, dtype=BF16) for s in shapes], rows, keys, 2)
    return block, (block.self_attention, block.cross_attention, block.feed_forward)


def _batch(rows, keys):
    ints = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return ad.Attention(1, 1, ints([0, rows]), ints([0, keys]), rows, keys)


@pytest.mark.parametrize("refused", ["self", "keys", "enc", "xq", "cross", "feed"])
def test_a_refused_pass_leaves_nothing_to_go_back_from(refused, monkeypatch):
    """A pass that ran, and one that a sublayer refuses: the sublayers before it have new rows and the others old ones,
    which do not belong together."""
    block, parts = _block()
    attention, cross, feed = parts
    for s in parts:
        s.rows = 3                                     # as the pass before left them
    def passes(s):
        def run(*a, **kw):
            s.rows = 3
        return run
    no = lambda *a, **kw: (_ for _ in ()).throw(ValueError("refused"))  # noqa: E731
    if refused != "self":
        monkeypatch.setattr(attention, "forward", passes(attention))
    if refused == "feed":
        monkeypatch.setattr(cross, "forward", passes(cross))
        monkeypatch.setattr(feed, "forward", no)
    if refused == "cross":
        monkeypatch.setattr(cross, "_begin", no)
        monkeypatch.setattr(cross, "_check", lambda *a: None)
    x, xq = torch.zeros(3, 64), None
    enc = torch.zeros(11 if refused == "keys" else 5, 64, dtype=torch.float32 if refused == "enc" else BF16)
    if refused == "xq":
        xq = torch.zeros(3, 32)
    with pytest.raises(ValueError):
        block.forward(x, enc, _batch(3, 3), _batch(3, 5), torch.zeros(3, 64), xq)
    with pytest.raises(ValueError, match="last forward pass had None"):
        block.backward(torch.zeros(3, 64), torch.zeros(3, 64))


@pytest.mark.parametrize("bad", ["rows", "cross", "dout", "dx", "dxq"])
def test_a_refused_way_back_reaches_no_sublayer(bad, monkeypatch):
    block, parts = _block()
    for s in parts:
        s.rows = 3
        monkeypatch.setattr(s, "backward", lambda *a, **kw: pytest.fail("a sublayer ran"))
    if bad == "cross":
        block.cross_attention.rows = 2
    # (the tensors' own checks, without a GPU)
    def check(name, t, rows, *dtypes):
        if t.shape != (rows, 64) or t.dtype not in dtypes:
            raise ValueError(name)
    monkeypatch.setattr(block.cross_attention, "_check", check)
    monkeypatch.setattr(block.feed_forward, "_rows", check)
    t = dict(dout=torch.zeros(3, 64), dx=torch.zeros(3, 64), dxq=torch.zeros(3, 64))
    if bad == "rows":
        t["dout"] = torch.zeros(2, 64)
    elif bad in t:
        t[bad] = torch.zeros(3, 32) if bad != "dxq" else torch.zeros(3, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        block.backward(t["dout"], t["dx"], t["dxq"])
