"""Batches that reach each way through the forward pass, by name, and the way that each is meant to reach."""
import torch


def _wide_windows(rows, keys, most, seed):
    g = torch.Generator().manual_seed(seed)
    lo = torch.randint(-50, keys, (rows,), generator=g)
    win = torch.stack([lo, lo + torch.randint(0, most, (rows,), generator=g)], 1)
    win[::5] = torch.tensor([0, 2 ** 31 - 1])
    win[3::7] = 0
    return win.to(torch.int32)


def _lens(n, most, seed):
    g = torch.Generator().manual_seed(seed)
    return [most] + torch.randint(0, most + 1, (n - 1,), generator=g).tolist()


# name: (way, batch).  A way is the kernel, whether the keys are in parts, and whether a workgroup of 32 queries has one
# tile of 128 keys or several.
ROUTES = {
    "keys": ("keys", dict(ql=[40, 9], kl=[1500, 70])),
    "keys_causal": ("keys", dict(ql=[40, 90], kl=[700, 70], causal=True)),
    "keys_windows": ("keys", dict(ql=[40, 9], kl=[1500, 70], window=_wide_windows(49, 1500, 600, 1))),
    "few_one": ("few one", dict(ql=[9, 20], kl=[100, 128])),
    "few_one_causal": ("few one", dict(ql=[20, 9, 0], kl=[100, 12, 5], causal=True, heads=4, kv=1)),
    "few_several": ("few several", dict(ql=_lens(300, 8, 2), kl=_lens(300, 700, 3), heads=1, kv=1)),
    "few_several_causal": ("few several", dict(ql=_lens(300, 30, 4), kl=_lens(300, 300, 5), heads=1, kv=1, causal=True)),
    "few_several_padded": ("few several", dict(ql=_lens(150, 5, 6), kl=_lens(150, 600, 7), heads=4, kv=2, padded=True)),
    "few_several_windows": ("few several", dict(ql=[6] * 300, kl=_lens(300, 500, 8), heads=1, kv=1,
                                                window=_wide_windows(1800, 500, 400, 9))),
    "parts_one": ("few parts one", dict(ql=[17, 65, 3], kl=[2600, 217, 64], heads=2, kv=1)),
    "parts_outside": ("few parts one", dict(ql=[3, 1, 2], kl=[2600, 130, 700], heads=2, kv=1, lead=300)),
    "parts_outside_padded": ("few parts several", dict(ql=[30, 1], kl=[9000, 130], heads=1, kv=1, lead=300, padded=True)),
    "parts_several": ("few parts several", dict(ql=[1], kl=[10000], heads=1, kv=1)),
    "parts_several_heads": ("few parts several", dict(ql=[3, 1, 20], kl=[3000, 2700, 0], heads=20, kv=5)),
    "parts_several_causal": ("few parts several", dict(ql=[40, 3], kl=[9000, 8300], heads=1, kv=1, causal=True)),
    "parts_several_longer": ("few parts several", dict(ql=[300], kl=[9000], heads=1, kv=1, causal=True)),
    "parts_several_padded": ("few parts several", dict(ql=[5, 2], kl=[9000, 100], heads=1, kv=1, padded=True)),
    "parts_several_windows": ("few parts several", dict(ql=[40, 3], kl=[9000, 8300], heads=2, kv=2,
                                                        window=_wide_windows(43, 9000, 4000, 10))),
    "wide": ("wide", dict(ql=[140, 97] * 8, kl=[150, 64] * 8, heads=4, kv=4)),
}
