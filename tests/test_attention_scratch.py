"""The workspace that attention sublayers share holds any batch of the sizes it was made for (CPU only: sizes alone)."""
import random

import pytest
import torch

from paper_2608_12703_amd import ad
from paper_2608_12703_amd.train import AttentionScratch


@pytest.mark.parametrize("d,max_rows,max_keys,max_batch", [(64, 448, 20000, 1), (1280, 448, 3000, 4), (384, 2000, 6000, 16), (1280, 40, 9000, 1)])
def test_a_scratch_holds_every_batch_of_its_sizes(d, max_rows, max_keys, max_batch):
    scratch = AttentionScratch(d, max_rows, max_keys, max_batch, device="cpu")
    rng = random.Random(d + max_rows)
    parts = 0
    for k in range(1500):
        batch, rows, keys = rng.randint(1, max_batch), rng.choice([max_rows, rng.randint(1, max_rows)]), rng.choice([max_keys, rng.randint(1, max_keys)])
        # (a sequence's rows may be few of the matrix's: the others belong to none)
        q_max = rng.choice([1, rng.randint(1, rows), rows, max_rows, 1 << 24])
        k_max = rng.choice([keys, rng.randint(1, keys), 1 << 24])
        ints = lambda n, **kw: torch.zeros(n, dtype=torch.int32)  # noqa: E731
        at = ad.Attention(d // 64, d // 64, ints(batch + 1), ints(batch + 1), q_max, k_max, causal=rng.random() < 0.5,
                          window=torch.zeros(rows, 2, dtype=torch.int32) if rng.random() < 0.3 else None)
        forward, backward = ad.attention_workspace_size(at, rows, keys), ad.attention_backward_workspace_size(at, rows, keys)
        parts += forward > 0
        assert max(forward, backward) <= scratch.workspace.nbytes, (batch, rows, keys, q_max, k_max, forward, backward)
    assert parts > 5
