"""What takes the training objective's gradients to new weights, as measurable cases.

Four calls, each through the public entry points:
  attention           o = softmax(q k^T / 8) v over 64-wide heads, and its rows' log-sum-exp
  attention_backward  dq, dk, dv from what the forward pass was given and what it kept
  adamw               one AdamW step over all tensors of a draft block, states in float32 or in 8 bits
  grad_norm           the norm of all gradients together, and the factor that clips it

Attention works on the matrices that projections write: sequence b owns the query rows cu_q[b] ..
cu_q[b+1] - 1 and the key rows cu_k[b] .. cu_k[b+1] - 1, of which the first q_len[b] and k_len[b] hold
something where rows are padded (outputs of the others are 0).  Key j is visible to query i if
j < k_len, with `causal` if j <= i + k_len - q_len, and with a window if lo_i <= j < hi_i.  A row that sees
nothing gives 0.  o_rest is what o's rounding to bf16 took away, in bf16.

The 8-bit states: 128 consecutive elements of a tensor share a scale s.  m = q s with s = max|m| / 127;
v = q^2 s with s = max v / 65025, q at least 1 where v > 0.  Between two codes the upper one is taken with the
probability that keeps the value's mean, from 16 bits each of a hash of seed, step, tensor and
element.  A bf16 parameter is rounded likewise.

Queries, keys and values are N(0, 1) with a few channels three times as large, as projections of a
LayerNorm have them; weights are N(0, 0.02), gradients and states small.
"""
import math
import random

import torch

own = False

BF16, F32 = torch.bfloat16, torch.float32
FULL = 448           # positions of a full transcript
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.01


def listed():
    return [
        # one position of one utterance over its audio: the smallest call, latency counts
        dict(name="attention_token", op="attention", batch=1, heads=20, kv=20, q=1, k=1500, spread=0, padded=False,
             causal=False, window=0, same=False, pad=0),
        # the draft block's self-attention over a batch of 32 full transcripts, from one q | k | v matrix
        dict(name="attention_self_train", op="attention", batch=32, heads=20, kv=20, q=FULL, k=FULL, spread=0, padded=True,
             causal=True, window=0, same=True, pad=0),
        # cross-attention over ragged transcripts and audio, packed
        dict(name="attention_cross_ragged", op="attention", batch=32, heads=20, kv=20, q=FULL, k=1500, spread=11,
             padded=False, causal=False, window=0, same=False, pad=0),
        # the paper's training batch: 12 utterances, 128 positions each, padded
        dict(name="backward_self_batch", op="attention_backward", batch=12, heads=20, kv=20, q=128, k=128, spread=7,
             padded=True, causal=True, window=0, same=True, pad=0),
        # cross-attention of 32 full transcripts over full audio: the largest call
        dict(name="backward_cross_train", op="attention_backward", batch=32, heads=20, kv=20, q=FULL, k=1500, spread=0,
             padded=False, causal=False, window=0, same=False, pad=0),
        # one long causal sequence at the small width
        dict(name="backward_long", op="attention_backward", batch=1, heads=12, kv=12, q=5000, k=5000, spread=0,
             padded=False, causal=True, window=0, same=True, pad=0),
        # frames around each position's anchor, some positions without any; shared key heads, rows
        # that no 16-byte vector divides
        dict(name="backward_window_ragged", op="attention_backward", batch=12, heads=20, kv=5, q=131, k=1500, spread=5,
             padded=True, causal=False, window=20, same=False, pad=3),
        # the vectors of one block at the tiny width: launch latency
        dict(name="adamw_vectors", op="adamw", d=384, f=768, what="vectors", state="f32", param="f32", copy=False,
             grad="f32", clip=False, step=3),
        # the draft block, float32 parameters with their bf16 copies, states in float32
        dict(name="adamw_block", op="adamw", d=1280, f=2560, what="block", state="f32", param="f32", copy=True,
             grad="f32", clip=True, step=1000),
        # the same with states in 8 bits, read back as a checkpoint of the training run reads them
        dict(name="adamw_block_8bit", op="adamw", d=1280, f=2560, what="block", state="8bit", param="f32", copy=True,
             grad="f32", clip=True, step=1000),
        # the norm of the draft block's gradients
        dict(name="grad_norm_block", op="grad_norm", d=1280, f=2560, what="block", grad="f32"),
        # an odd block's vectors, bf16 gradients
        dict(name="grad_norm_vectors", op="grad_norm", d=381, f=767, what="vectors", grad="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention_backward", "attention_backward", "adamw", "grad_norm"])
    if op == "adamw":
        state, param = rng.choice(["f32", "8bit"]), rng.choice(["f32", "f32", "bf16"])
        return dict(op=op, d=_log(rng, 33, 1280), f=_log(rng, 65, 2560), what=rng.choice(["vectors", "block", "block"]),
                    state=state, param=param, copy=param == "f32" and rng.random() < 0.5,
                    grad=rng.choice(["f32", "bf16"]), clip=rng.random() < 0.5, step=_log(rng, 1, 20000))
    if op == "grad_norm":
        return dict(op=op, d=_log(rng, 33, 1280), f=_log(rng, 65, 2560), what=rng.choice(["vectors", "block"]),
                    grad=rng.choice(["f32", "bf16"]))
    heads = rng.choice([1, 2, 6, 12, 20])
    kv = heads if rng.random() < 0.7 else rng.choice([n for n in range(1, heads + 1) if heads % n == 0])
    same = rng.random() < 0.5
    q = _log(rng, 1, 2000)
    k = q if same else _log(rng, 1, 1500)
    most = 32 * 20 * FULL * 1500
    batch = max(1, min(_log(rng, 1, 64), most // (heads * q * k)))
    return dict(op=op, batch=batch, heads=heads, kv=kv, q=q, k=k, spread=rng.choice([0, rng.randint(1, 1000)]),
                padded=rng.random() < 0.4, causal=rng.random() < (0.7 if same else 0.2),
                window=rng.choice([0, 0, 20, _log(rng, 1, 300)]), same=same, pad=rng.choice([0, 0, 8, 3]))


# ---------------------------------------------------------------------------- inputs

def _type(name):
    return BF16 if name == "bf16" else F32


def _lengths(c):
    """Query and key rows of every sequence."""
    rng = random.Random(c["spread"])
    lens = lambda n: [rng.randint(n // 4, n) if c["spread"] else n for _ in range(c["batch"])]  # noqa: E731
    q = lens(c["q"])
    return q, (q if c["same"] else lens(c["k"]))


def _tensors(c):
    """The sizes of a draft block's parameters, and which of them are decayed."""
    d, f = c["d"], c["f"]
    vectors = [d, d, 3 * d, d] + [d, d, d, 2 * d, d] + [d, d, f, d] + [d, d, d, d]
    matrices = [3 * d * d, d * d] + [d * d, 2 * d * d, d * d] + [f * d, f * d] + [4 * d * d, 2 * d * d]
    sizes = vectors if c["what"] == "vectors" else vectors + matrices
    return sizes, [0.0] * len(vectors) + [DECAY] * (len(sizes) - len(vectors))


class _Draw:
    """Draws on the GPU from one seed, in call order."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def __call__(self, *shape, scale=1.0, dtype=F32):
        return torch.randn(*shape, generator=self.g, device="cuda").mul_(scale).to(dtype)

    def ints(self, n, lo, hi):
        return torch.randint(lo, hi, (n,), generator=self.g, device="cuda")

    def rows(self, rows, cols, pad):
        """bf16 rows `pad` elements apart, one channel in 16 three times as large."""
        x = torch.randn(rows, cols, generator=self.g, device="cuda")
        x[:, ::16] *= 3.0
        wide = torch.zeros(rows, cols + pad, dtype=BF16, device="cuda")
        wide[:, :cols] = x
        return wide[:, :cols]


def _prepare_attention(c, seed):
    rnd, heads, kv = _Draw(seed), c["heads"], c["kv"]
    ql, kl = _lengths(c)
    s = dict(case=c)

    def layout(lens, most):
        own_rows = [most] * len(lens) if c["padded"] else lens
        cu = [0]
        for n in own_rows:
            cu.append(cu[-1] + n)
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        return cu[-1], ints(cu), ints(lens) if c["padded"] else None

    rows_q, s["cu_q"], s["q_len"] = layout(ql, c["q"])
    rows_k, s["cu_k"], s["k_len"] = layout(kl, c["k"])
    wq, wk = 64 * heads, 64 * kv
    if c["same"]:
        both = rnd.rows(rows_q, wq + 2 * wk, c["pad"])
        s["q"], s["k"], s["v"] = both[:, :wq], both[:, wq:wq + wk], both[:, wq + wk:]
    else:
        s["q"], kv_rows = rnd.rows(rows_q, wq, c["pad"]), rnd.rows(rows_k, 2 * wk, c["pad"])
        s["k"], s["v"] = kv_rows[:, :wk], kv_rows[:, wk:]
    if c["window"]:
        # anchors that walk along the audio, and every seventh position without one
        at = torch.cat([torch.arange(n, device="cuda") * kn // max(n, 1) for n, kn in
                        zip([c["q"]] * len(ql) if c["padded"] else ql, kl)])
        at = at + rnd.ints(rows_q, -8, 9)
        win = torch.stack([at - c["window"], at + c["window"] + 1], 1).to(torch.int32)
        win[::7] = 0
        s["window"] = win.contiguous()
    empty = lambda *shape, dtype=BF16: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    s["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if c["op"] == "attention":
        s.update(o=empty(rows_q, wq), lse=empty(heads, rows_q, dtype=F32))
        return s
    o, lse = _attention(s)
    s.update(o=o.to(BF16), lse=lse.contiguous(), dout=rnd(rows_q, wq, scale=1e-3, dtype=BF16))
    s["o_rest"] = (o - s["o"].float()).to(BF16)
    if c["same"]:
        grads = empty(rows_q, wq + 2 * wk)
        s.update(dq=grads[:, :wq], dk=grads[:, wq:wq + wk], dv=grads[:, wq + wk:])
    else:
        grads = empty(rows_k, 2 * wk)
        s.update(dq=empty(rows_q, wq), dk=grads[:, :wk], dv=grads[:, wk:])
    return s


def prepare(case, seed):
    c = case
    if c["op"] in ("attention", "attention_backward"):
        return _prepare_attention(c, seed)
    rnd = _Draw(seed)
    sizes, decay = _tensors(c)
    n = sum(sizes)
    groups = sum(-(-z // 128) for z in sizes)
    s = dict(case=c, g=rnd(n, scale=2e-4, dtype=_type(c["grad"])))
    s["out"] = torch.empty(2, device="cuda")
    if c["op"] == "grad_norm":
        return s
    s["p"] = rnd(n, scale=0.02, dtype=_type(c["param"]))
    s["seed"] = seed % (1 << 32)
    if c["copy"]:
        s["copy"] = s["p"].to(BF16)
    if c["clip"]:
        s["grad_scale"] = rnd(1).abs().clamp(0.1, 1.0)
    if c["state"] == "f32":
        s["m"], s["v"] = rnd(n, scale=1e-4), rnd(n, scale=1e-4).square()
    else:
        s["m"] = rnd(n, scale=40.0).round().clamp(-127, 127).to(torch.int8)
        s["v"] = rnd(n, scale=90.0).abs().round().clamp(1, 255).to(torch.uint8)
        s["m_scale"] = rnd(groups).abs().add(0.5).mul(1e-6)
        s["v_scale"] = rnd(groups).abs().add(0.5).mul(1e-12)
        s["m_value"], s["v_value"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    return s


# ---------------------------------------------------------------------------- one pass

def _handle(s):
    """The call's handle and workspace, which a program keeps from one call to the next."""
    from paper_2608_12703_amd import ad
    c = s["case"]
    if c["op"] in ("attention", "attention_backward"):
        at = ad.Attention(c["heads"], c["kv"], s["cu_q"], s["cu_k"], c["q"], c["k"], q_len=s["q_len"], k_len=s["k_len"],
                          causal=c["causal"], window=s.get("window"), err_flag=s["err"])
        size = ad.attention_workspace_size if c["op"] == "attention" else ad.attention_backward_workspace_size
        return at, torch.empty(size(at, s["q"].shape[0], s["k"].shape[0]), dtype=torch.uint8, device="cuda")
    sizes, decay = _tensors(c)
    cut = lambda name: list(s[name].split(sizes)) if name in s else None  # noqa: E731
    if c["op"] == "grad_norm":
        opt = ad.OptTensors(grads=cut("g"))
        return opt, torch.empty(ad.grad_norm_workspace_size(opt), dtype=torch.uint8, device="cuda")
    scales = [-(-z // 128) for z in sizes]
    more = {name: list(s[name].split(scales)) for name in ("m_scale", "v_scale") if name in s}
    return ad.OptTensors(params=cut("p"), grads=cut("g"), m=cut("m"), v=cut("v"), copies=cut("copy"),
                         weight_decay=decay, **more), None


def _run_own(s):
    from paper_2608_12703_amd import ad
    c = s["case"]
    if "handle" not in s:
        s["handle"] = _handle(s)
    h, space = s["handle"]
    if c["op"] == "attention":
        ad.attention(h, s["q"], s["k"], s["v"], s["o"], s["lse"], None, space)
        return dict(o=s["o"], lse=s["lse"])
    if c["op"] == "attention_backward":
        ad.attention_backward(h, s["q"], s["k"], s["v"], s["o"], s["o_rest"], s["lse"], s["dout"], None, s["dq"], s["dk"],
                              s["dv"], space)
        return dict(dq=s["dq"], dk=s["dk"], dv=s["dv"])
    if c["op"] == "grad_norm":
        ad.grad_norm(h, 1.0, s["out"], space)
        return s["out"]
    ad.adamw(h, LR, c["step"], beta1=BETA1, beta2=BETA2, eps=EPS, seed=s["seed"], grad_scale=s.get("grad_scale"))
    out = dict(p=s["p"])
    if c["copy"]:
        out["copy"] = s["copy"]
    if c["state"] == "8bit":
        ad.opt_state(h, s["m_value"], s["v_value"])
        return dict(out, m=s["m_value"], v=s["v_value"])
    return dict(out, m=s["m"], v=s["v"])


def _spread(s, side, most):
    """Where the padded rows [batch][most] of one side lie, which of them hold something, and the padded
    place of every row."""
    cu = s["cu_" + side].long()
    at = torch.arange(most, device="cuda")
    lens = s[side + "_len"].long() if s[side + "_len"] is not None else cu[1:] - cu[:-1]
    rows = s[side].shape[0]
    index = (cu[:-1, None] + at).clamp(max=max(rows - 1, 0))
    row = torch.arange(rows, device="cuda")
    b = torch.searchsorted(cu, row, right=True) - 1
    return index, at < lens[:, None], b, row - cu[b], lens


def _attention(s):
    """o, lse or dq, dk, dv of the state's inputs in float32."""
    c = s["case"]
    heads, kv = c["heads"], c["kv"]
    n = heads // kv
    iq, live_q, bq, pq, ql = _spread(s, "q", c["q"])
    ik, live_k, bk, pk, kl = _spread(s, "k", c["k"])
    pad = lambda x, i, g, m: x.float()[i].unflatten(2, (g, m, 64)).permute(0, 2, 3, 1, 4)  # noqa: E731
    q, k, v = pad(s["q"], iq, kv, n), pad(s["k"], ik, kv, 1), pad(s["v"], ik, kv, 1)
    i, j = torch.arange(c["q"], device="cuda")[:, None], torch.arange(c["k"], device="cuda")
    seen = live_q[:, :, None] & live_k[:, None, :]
    if c["causal"]:
        seen = seen & (j <= i + (kl - ql)[:, None, None])
    if c["window"]:
        w = s["window"][iq]
        seen = seen & (j >= w[:, :, :1]) & (j < w[:, :, 1:])
    hidden = ~seen[:, None, None]
    x = (q @ k.transpose(-1, -2)).mul_(0.125).masked_fill_(hidden, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(total.masked_fill(total == 0.0, 1.0))
    rows = lambda y, b, at: y.permute(0, 3, 1, 2, 4)[b, at].flatten(1)  # noqa: E731
    if c["op"] == "attention" or "dout" not in s:
        lse = (top + total.log())[..., 0]
        return rows(p @ v, bq, pq), lse.permute(1, 2, 0, 3).flatten(0, 1)[:, bq, pq]
    do = pad(s["dout"], iq, kv, n) * live_q[:, None, None, :, None]
    dp = do @ v.transpose(-1, -2)
    dv = p.transpose(-1, -2) @ do
    delta = (p * dp).sum(-1, keepdim=True)
    ds = dp.sub_(delta).mul_(p).mul_(0.125)
    dq, dk = ds @ k, ds.transpose(-1, -2) @ q
    return rows(dq, bq, pq), rows(dk.sum(2, keepdim=True), bk, pk), rows(dv.sum(2, keepdim=True), bk, pk)


def _mix(x):
    """32 bits from 32 bits: exclusive-ors of shifts between products with odd constants (the fractions
    of the square roots of 2 and 3)."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


GOLDEN = 0x9E3779B9


def _adamw(s):
    """The step on whole buffers; sums and products round in the order written, roots and quotients where a
    code hangs on them in 64 bits."""
    c = s["case"]
    sizes, decay = _tensors(c)
    n, step = sum(sizes), c["step"]
    size = torch.tensor(sizes, device="cuda")
    each = lambda v: torch.repeat_interleave(v, size, output_size=n)  # noqa: E731
    g = s["g"].float()
    if c["clip"]:
        g = g * s["grad_scale"]
    first = torch.cumsum(size, 0) - size
    local = torch.arange(n, device="cuda") - each(first)
    if c["state"] == "8bit":
        groups = (size + 127) // 128
        group = each(torch.cumsum(groups, 0) - groups) + local // 128
        m0 = s["m"].float() * s["m_scale"][group]
        v0 = s["v"].float().square() * s["v_scale"][group]
    else:
        m0, v0 = s["m"], s["v"]
    m = m0 * BETA1 + g * (1.0 - BETA1)
    v = v0 * BETA2 + (g * g) * (1.0 - BETA2)
    keep = each(torch.tensor([1.0 - LR * w for w in decay], device="cuda"))
    root = v.sqrt() * (1.0 / math.sqrt(1.0 - BETA2 ** step)) + EPS
    p = s["p"].float() * keep - (m / root) * (LR / (1.0 - BETA1 ** step))
    if c["state"] == "8bit" or c["param"] == "bf16":
        key = _mix((s["seed"] + GOLDEN * step) & 0xFFFFFFFF)
        keys = _mix((torch.arange(len(sizes), device="cuda") + key) & 0xFFFFFFFF)
        bits = _mix((each(keys) + local * GOLDEN) & 0xFFFFFFFF)
    if c["param"] == "bf16":
        more = _mix((bits + GOLDEN) & 0xFFFFFFFF) & 0xFFFF
        s["p"].copy_(((p.view(torch.int32) + more.int()) & -65536).view(F32))
    else:
        s["p"].copy_(p)
    out = dict(p=s["p"])
    if c["copy"]:
        out["copy"] = s["copy"].copy_(p)
    if c["state"] == "f32":
        return dict(out, m=s["m"].copy_(m), v=s["v"].copy_(v))
    most = lambda x: torch.zeros(s["m_scale"].numel(), device="cuda").scatter_reduce_(0, group, x, "amax")  # noqa: E731
    ratio = lambda a, b: (a.double() / b).float()  # noqa: E731
    mm, vm = most(m.abs()), most(v)
    up = lambda r: ((r.double() + 0.5) / 65536.0).float()  # noqa: E731
    x = m * ratio(torch.full_like(mm, 127.0), mm)[group]
    low = x.floor()
    qm = (low + (x - low > up(bits & 0xFFFF))).clamp(-127, 127)
    y = v * ratio(torch.full_like(vm, 65025.0), vm)[group]
    low = y.double().sqrt().floor().float()
    qv = (low + (y - low * low > up(bits >> 16) * (2.0 * low + 1.0))).clamp(max=255.0)
    qv = torch.where(v > 0.0, qv.clamp(min=1.0), 0.0)
    s["m"].copy_(qm)
    s["v"].copy_(qv)
    s["m_scale"].copy_((mm.double() / 127.0).float())
    s["v_scale"].copy_((vm.double() / 65025.0).float())
    return dict(out, m=qm * s["m_scale"][group], v=qv.square() * s["v_scale"][group])


def run(state):
    if own:
        return _run_own(state)
    s, c = state, state["case"]
    if c["op"] == "attention":
        o, lse = _attention(s)
        return dict(o=o.to(BF16), lse=lse)
    if c["op"] == "attention_backward":
        dq, dk, dv = _attention(s)
        return dict(dq=dq.to(BF16), dk=dk.to(BF16), dv=dv.to(BF16))
    if c["op"] == "adamw":
        return _adamw(s)
    norm = s["g"].double().square().sum().sqrt()
    return torch.stack([norm, (1.0 / norm).clamp(max=1.0)]).float()


# ---------------------------------------------------------------------------- 64 bits

def _exact_attention(s, c):
    ql, kl = _lengths(c)
    heads, kv = c["heads"], c["kv"]
    back = c["op"] == "attention_backward"
    wide = lambda x: x.double().unflatten(1, (-1, 64)).transpose(0, 1)  # noqa: E731  [heads][rows][64]
    q, k, v = wide(s["q"]), wide(s["k"]), wide(s["v"])
    do = wide(s["dout"]) if back else None
    first, second, third = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    lse = q.new_full(q.shape[:2], -math.inf)
    at_q, at_k = s["cu_q"].tolist(), s["cu_k"].tolist()
    for b in range(c["batch"]):
        a, e, nq, nk = at_q[b], at_k[b], ql[b], kl[b]
        if not nq or not nk:
            continue
        shut = torch.zeros(nq, nk, dtype=torch.bool, device="cuda")
        if c["causal"]:
            shut |= torch.ones_like(shut).triu(1 + nk - nq)
        if c["window"]:
            w, col = s["window"][a:a + nq].long(), torch.arange(nk, device="cuda")[None]
            shut |= (col < w[:, 0:1]) | (col >= w[:, 1:2])
        dead = shut.all(1)
        for h in range(heads):
            g = h // (heads // kv)
            qs, ks, vs = q[h, a:a + nq], k[g, e:e + nk], v[g, e:e + nk]
            x = torch.where(shut, -math.inf, qs.mm(ks.t()) / 8.0)
            z = torch.logsumexp(x, 1)
            p = torch.where(dead[:, None], 0.0, torch.exp(x - torch.where(dead, 0.0, z)[:, None]))
            if not back:
                first[h, a:a + nq], lse[h, a:a + nq] = p.mm(vs), z
                continue
            dos = do[h, a:a + nq]
            dp = dos.mm(vs.t())
            ds = p * (dp - (dos * p.mm(vs)).sum(1, keepdim=True)) / 8.0
            first[h, a:a + nq] = ds.mm(ks)
            second[g, e:e + nk] += ds.t().mm(qs)
            third[g, e:e + nk] += p.t().mm(dos)
    flat = lambda x: x.transpose(0, 1).flatten(1)  # noqa: E731
    if not back:
        return dict(o=flat(first), lse=lse)
    return dict(dq=flat(first), dk=flat(second), dv=flat(third))


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] in ("attention", "attention_backward"):
        return _exact_attention(s, c)
    if c["op"] == "grad_norm":
        norm = torch.linalg.vector_norm(s["g"].double())
        return torch.stack([norm, torch.minimum(1.0 / norm, torch.ones_like(norm))])
    sizes, decay = _tensors(c)
    if c["state"] == "8bit":
        spread = lambda t: torch.cat([x.repeat_interleave(128)[:z] for x, z in  # noqa: E731
                                      zip(t.double().split([-(-z // 128) for z in sizes]), sizes)])
        m, v = s["m"].double() * spread(s["m_scale"]), s["v"].double() ** 2 * spread(s["v_scale"])
    else:
        m, v = s["m"].double(), s["v"].double()
    g = s["g"].double() * (s["grad_scale"].double() if c["clip"] else 1.0)
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g.square(), v, BETA2)
    hat_m, hat_v = m / (1.0 - BETA1 ** c["step"]), v / (1.0 - BETA2 ** c["step"])
    rate = torch.cat([torch.full((z,), LR * w, dtype=torch.float64, device="cuda") for z, w in zip(sizes, decay)])
    p = s["p"].double()
    p = p - rate * p - LR * hat_m / (hat_v.sqrt() + EPS)
    # (a parameter or a state rounded by random bits has no value of its own here)
    kept = c["state"] == "f32"
    return dict(p=p if c["param"] == "f32" else None, **(dict(copy=p) if c["copy"] else {}), m=m if kept else None,
                v=v if kept else None)


# ---------------------------------------------------------------------------- work

def work(case):
    c = case
    if c["op"] in ("adamw", "grad_norm"):
        sizes, _ = _tensors(c)
        n = float(sum(sizes))
        g = 4.0 if c["grad"] == "f32" else 2.0
        if c["op"] == "grad_norm":
            return dict(bytes=n * g + 8, flops=2 * n)
        p = 8.0 if c["param"] == "f32" else 4.0
        states = 16.0 if c["state"] == "f32" else 4.0 + 16.0 / 128.0 + 8.0    # (8 bits: their values are written too)
        return dict(bytes=n * (g + p + states + (2.0 if c["copy"] else 0.0)), flops=14 * n)
    ql, kl = _lengths(c)
    pairs = 0
    for nq, nk in zip(ql, kl):
        if c["window"]:
            pairs += nq * min(nk, 2 * c["window"] + 1) * 6 // 7 // (2 if c["causal"] else 1)
        elif c["causal"]:
            short = max(0, nq - nk)                # rows that see nothing
            n = nq - short
            pairs += n * (nk - n) + n * (n + 1) // 2
        else:
            pairs += nq * nk
    rows_q, rows_k, wq, wk = sum(ql), sum(kl), 64.0 * c["heads"], 64.0 * c["kv"]
    if c["op"] == "attention":
        cells = rows_q * (wq * 4 + c["heads"] * 4) + rows_k * wk * 4
        return dict(bytes=cells, flops=4.0 * 64 * c["heads"] * pairs)
    # read: q, o and its rest, dout; k, v.  written: dq, dk, dv
    cells = rows_q * (wq * 10 + c["heads"] * 4) + rows_k * wk * 8
    return dict(bytes=cells, flops=10.0 * 64 * c["heads"] * pairs)
