"""Windows of any integers, in every kernel that masks a tile: rows whose window ends before it begins, at the ends of
32 bits, beside rows that see keys of the same tile (bounds: attention_common)."""
import pytest
import torch

from attention_common import Batch, Ref, backward, forward, near

pytestmark = pytest.mark.gpu

LOW, HIGH = -2 ** 31, 2 ** 31 - 1
# (a kernel each of the forward pass and of dq; dk and dv have theirs by the keys)
SHAPES = {
    "keys": dict(ql=[40, 9], kl=[300, 70]),                                  # eight waves with keys of their own
    "few": dict(ql=[40] * 70, kl=[300] * 70, heads=4, kv=4),                 # 32 rows, a tile's keys over four waves
    "parts": dict(ql=[3, 1], kl=[2600, 130], heads=1, kv=1),                 # keys in parts
    "wide": dict(ql=[40] * 64, kl=[150] * 64, heads=16, kv=16),              # four waves of 32 rows
}
ENDS = [(1, LOW), (5, LOW + 7), (HIGH, LOW), (HIGH, HIGH), (HIGH - 1, HIGH), (LOW, LOW), (3, -1), (0, LOW), (60, 59), (-5, HIGH),
        (LOW, HIGH), (LOW, 40), (1, HIGH), (2, 2)]


def _windows(bt):
    """Every third row sees some keys in the middle, the others have one of ENDS."""
    win = torch.zeros(bt.q_rows, 2, dtype=torch.int64)
    for r in range(bt.q_rows):
        win[r] = torch.tensor([r % 11, 20 + r % 50] if r % 3 == 0 else ENDS[(r - r // 3) % len(ENDS)])
    return win.to(torch.int32)


@pytest.mark.parametrize("causal,padded", [(False, False), (True, True)])
@pytest.mark.parametrize("name", SHAPES)
def test_windows_of_any_integers(name, causal, padded):
    bt = Batch(seed=3 + causal, causal=causal, padded=padded, lead=2, **SHAPES[name])
    bt.window = _windows(bt)
    seen = torch.cat([bt.seen(b).any(1) for b in range(bt.batch)])
    assert bool(seen.any()) and not bool(seen.all())
    ref = Ref(bt)
    _, o, rest, lse = forward(bt)
    near(o.get(), ref.o, ref.tol_o, "o")
    near(lse.double().cpu(), ref.lse, ref.tol_lse, "lse")
    dq, dk, dv = backward(bt, ref)
    near(dq, ref.dq, ref.tol_dq, "dq")
    near(dk, ref.dk, ref.tol_dk, "dk")
    near(dv, ref.dv, ref.tol_dv, "dv")
