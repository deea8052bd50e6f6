"""The sequence operators as cases that can be timed and checked.

Two operators of a sequence-mixing block: the gated linear recurrence along
the tokens, and the norms before and after a block with its gate and scaled
residual.  ``run`` is one call of a program that has its inputs on the GPU: a
single-token step, a forward pass, or a forward and backward pass.  With
``own`` it goes through ``paper_2609_32237_amd.seq_api``; without, it computes
the same from elementary torch operations in 32 bits.  ``exact`` gives the
results in 64 bits from the definitions, token by token.
"""
import math

import torch

own = False

EPS = 1e-5
DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one new token for each of a few sequences, as an interactive server steps them: latency counts
        dict(name="scan_step_8x1024_bf16", kind="scan", batch=8, tokens=1, channels=1024, dtype="bf16", train=False, packed=True, ragged=False),
        # one new token for a full serving batch
        dict(name="scan_step_512x4096_fp16", kind="scan", batch=512, tokens=1, channels=4096, dtype="fp16", train=False, packed=True, ragged=False),
        # prompts of different lengths taken in together, one of them empty; the rows are slices of one projection
        dict(name="scan_prompts_6x1501x2048_bf16", kind="scan", batch=6, tokens=1501, channels=2048, dtype="bf16", train=False, packed=True, ragged=True),
        # one very long document: a single sequence, so the work has to be split along the tokens
        dict(name="scan_long_1x65536x1024_bf16", kind="scan", batch=1, tokens=65536, channels=1024, dtype="bf16", train=False, packed=False, ragged=False),
        # training: an ordinary batch, the largest case; an odd, ragged one in 32 bits; few long sequences
        dict(name="scan_train_8x4096x2048_bf16", kind="scan", batch=8, tokens=4096, channels=2048, dtype="bf16", train=True, packed=True, ragged=False),
        dict(name="scan_train_3x777x1023_fp32", kind="scan", batch=3, tokens=777, channels=1023, dtype="fp32", train=True, packed=False, ragged=True),
        dict(name="scan_train_2x16384x1024_fp16", kind="scan", batch=2, tokens=16384, channels=1024, dtype="fp16", train=True, packed=False, ragged=False),
        # the block's end for one token of a few sequences
        dict(name="norm_8x1024_bf16", kind="norm", rows=8, channels=1024, dtype="bf16", train=False, packed=False),
        # the block's end over a prompt, the gate a slice of a wider projection
        dict(name="norm_8192x4096_fp16", kind="norm", rows=8192, channels=4096, dtype="fp16", train=False, packed=True),
        # training: rows of an odd length in 32 bits, an ordinary batch, the widest rows
        dict(name="norm_train_1501x2047_fp32", kind="norm", rows=1501, channels=2047, dtype="fp32", train=True, packed=False),
        dict(name="norm_train_32768x2048_bf16", kind="norm", rows=32768, channels=2048, dtype="bf16", train=True, packed=True),
        dict(name="norm_train_3001x16384_bf16", kind="norm", rows=3001, channels=16384, dtype="bf16", train=True, packed=False),
    ]


def _size(rng, lo, hi):
    """A size spread over the logarithm, on a multiple of 64, of 8, or anywhere."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    m = rng.choice([1, 8, 64, 64])
    n = min(hi, max(lo, n // m * m))
    return n + m if n == 3072 else n


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    most = 1 << (25 if dtype == "fp32" else 26)
    if rng.random() < 0.4:
        channels = _size(rng, 256, 16384)
        rows = min(_size(rng, 1, 65536), most // channels)
        return dict(kind="norm", rows=rows, channels=channels, dtype=dtype, train=rng.random() < 0.6, packed=rng.random() < 0.5)
    if rng.random() < 0.25:
        return dict(kind="scan", batch=_size(rng, 1, 512), tokens=1, channels=_size(rng, 256, 8192), dtype=dtype, train=False,
                    packed=rng.random() < 0.5, ragged=False)
    channels, batch = _size(rng, 128, 8192), rng.choice([1, 1, 2, 3, 4, 8, 16])
    tokens = min(_size(rng, 16, 65536), most // (channels * batch))
    return dict(kind="scan", batch=batch, tokens=tokens, channels=channels, dtype=dtype, train=rng.random() < 0.6,
                packed=rng.random() < 0.5, ragged=rng.random() < 0.4)


# ---------------------------------------------------------------- inputs


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype, d = DTYPES[case["dtype"]], case["channels"]

    def normal(*shape, std=1.0, dtype=dtype):
        return torch.empty(*shape, device="cuda", dtype=dtype).normal_(0.0, std, generator=gen)

    def uniform(n, lo, hi):
        return torch.empty(n, device="cuda").uniform_(lo, hi, generator=gen)

    s = dict(case)
    if case["kind"] == "norm":
        shape = (case["rows"], d)
        # residual streams grow with depth; a block's output starts on another scale than the stream
        s["x"], s["y"] = normal(*shape, std=2.0), normal(*shape, std=0.5)
        s["z"] = normal(case["rows"], 2 * d)[:, d:] if case["packed"] else normal(*shape)
        s["post"], s["pre"], s["scale"] = uniform(d, 0.8, 1.2), uniform(d, 0.8, 1.2), uniform(d, 0.1, 1.0)
        if case["train"]:
            s["grad_out"], s["grad_normed"] = normal(*shape), normal(*shape)
        return s
    b, t = case["batch"], case["tokens"]
    if case["packed"]:  # the three inputs side by side in one projection's output
        x, r, g = normal(b, t, 3 * d).split(d, dim=-1)
    else:
        x, r, g = normal(b, t, d), normal(b, t, d), normal(b, t, d)
    # a channel's memory reaches over 1 to 500 tokens at the gate's middle
    rate = torch.exp(uniform(d, math.log(0.004), 0.0))
    s.update(x=x, r=r, g=g, rate=rate, state=normal(b, d, std=0.3, dtype=torch.float32), lengths=None)
    if case["ragged"]:
        n = torch.randint(1, t + 1, (b,), device="cuda", generator=gen, dtype=torch.int32)
        n[0] = t
        if b > 1:
            n[b - 1] = 0
        s["lengths"] = n
    if case["train"]:
        s["grad_out"], s["grad_state"] = normal(b, t, d), normal(b, d, dtype=torch.float32)
    return s


# ---------------------------------------------------------------- one pass


def run(s):
    if own:
        return _run_own(s)
    return _plain_norm(s) if s["kind"] == "norm" else _plain_scan(s)


def _run_own(s):
    from paper_2609_32237_amd import seq_api as sq

    if s["kind"] == "norm":
        w = s["post"], s["scale"], s["pre"]
        if not s["train"]:
            out, normed = sq.residual_norm(s["x"], s["y"], s["z"], *w, eps=EPS)
            return dict(out=out, normed=normed)
        stats = sq.residual_norm_stats(s["x"])
        out, normed = sq.residual_norm(s["x"], s["y"], s["z"], *w, eps=EPS, stats=stats)
        dx, dy, dz, dpost, dscale, dpre = sq.residual_norm_backward(s["grad_out"], s["grad_normed"], s["x"], s["y"], s["z"], *w, stats,
                                                                  eps=EPS)
        return dict(out=out, normed=normed, dx=dx, dy=dy, dz=dz, dpost=dpost, dscale=dscale, dpre=dpre)
    if not s["train"]:
        y, state = sq.gated_scan(s["x"], s["r"], s["g"], s["rate"], s["state"], s["lengths"])
        return dict(y=y, state=state)
    saved = sq.gated_scan_saved(s["x"])
    y, state = sq.gated_scan(s["x"], s["r"], s["g"], s["rate"], s["state"], s["lengths"], saved=saved)
    dx, dr, dg, drate, dstate = sq.gated_scan_backward(s["grad_out"], s["x"], s["r"], s["g"], s["rate"], saved, s["lengths"],
                                                       grad_state=s["grad_state"])
    return dict(y=y, state=state, dx=dx, dr=dr, dg=dg, drate=drate, dstate=dstate)


def _recur(a, b):
    """h_t = a_t h_(t-1) + b_t from h = 0 along axis 1: neighbours joined in pairs, the half as long
    recurrence of the pairs, and its states carried to the tokens between."""
    t = a.shape[1]
    if t == 1:
        return b
    m = t // 2
    a0, a1, b0, b1 = a[:, 0:2 * m:2], a[:, 1::2], b[:, 0:2 * m:2], b[:, 1::2]
    odd = _recur(a0 * a1, torch.addcmul(b1, a1, b0))
    h = torch.empty_like(b)
    h[:, 0] = b[:, 0]
    h[:, 1::2] = odd
    h[:, 2::2] = torch.addcmul(b[:, 2::2], a[:, 2::2], odd[:, :(t - 1) // 2])
    return h


def _plain_scan(s):
    kind = s["x"].dtype
    x, p, h0 = s["x"].float(), s["rate"], s["state"]
    sr, sg = torch.sigmoid(s["r"].float()), torch.sigmoid(s["g"].float())
    q, c = p * sr, sg * x
    if s["lengths"] is not None:
        live = (torch.arange(x.shape[1], device="cuda") < s["lengths"][:, None])[..., None]
        q, c = q * live, c * live
    a, b = 1.0 - q, q * c
    b[:, 0] = torch.addcmul(b[:, 0], a[:, 0], h0)
    h = _recur(a, b)
    y = h if s["lengths"] is None else h * live
    out = dict(y=y.to(kind), state=h[:, -1].clone())
    if not s["train"]:
        return out
    # the same recurrence from the last token to the first
    dy = s["grad_out"].to(torch.float32, copy=True)
    if s["lengths"] is not None:
        dy *= live
    dy[:, -1] += s["grad_state"]
    back = torch.zeros_like(a)
    back[:, :-1] = a[:, 1:]
    d = _recur(back.flip(1), dy.flip(1)).flip(1)
    before = torch.cat([h0[:, None], h[:, :-1]], dim=1)
    de = d * (c - before)
    if s["lengths"] is not None:
        de = de * live
    dx = d * q * sg
    out.update(dx=dx.to(kind), dr=(de * q * (1.0 - sr)).to(kind), dg=(dx * x * (1.0 - sg)).to(kind), drate=(de * sr).sum((0, 1)),
               dstate=a[:, 0] * d[:, 0])
    return out


def _plain_norm(s):
    kind = s["x"].dtype
    x, y, z, post, scale, pre = s["x"].float(), s["y"].float(), s["z"].float(), s["post"], s["scale"], s["pre"]
    iy = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
    m, sz = y * iy, torch.sigmoid(z)
    gate, w = z * sz, scale * post
    o = x + w * m * gate
    io = torch.rsqrt(o.square().mean(-1, keepdim=True) + EPS)
    oh = o * io
    out = dict(out=o.to(kind), normed=(pre * oh).to(kind))
    if not s["train"]:
        return out
    dn = s["grad_normed"].float()
    v = dn * pre
    t = s["grad_out"].float() + io * (v - oh * (v * oh).mean(-1, keepdim=True))
    u = t * w * gate
    dy = iy * (u - m * (u * m).mean(-1, keepdim=True))
    part = (t * gate * m).sum(0)
    out.update(dx=t.to(kind), dy=dy.to(kind), dz=(t * w * m * (sz + gate * (1.0 - sz))).to(kind), dpost=scale * part,
               dscale=post * part, dpre=(dn * oh).sum(0))
    return out


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    e, d = (4 if case["dtype"] == "fp32" else 2), case["channels"]
    if case["kind"] == "norm":
        n = case["rows"] * d
        return dict(bytes=n * e * (10 if case["train"] else 5) + 4 * d * (6 if case["train"] else 3), flops=n * (55 if case["train"] else 18))
    n, rows = case["batch"] * case["tokens"] * d, case["batch"] * d
    # the lengths of a ragged batch: one whole, one empty, the rest half on average
    live = n if not case["ragged"] else int(n * (1 + max(0, case["batch"] - 2) / 2) / case["batch"])
    if case["train"]:
        return dict(bytes=e * (4 * live + 4 * n) + 16 * rows + 8 * d, flops=live * 45)
    return dict(bytes=e * (3 * live + n) + 8 * rows + 4 * d, flops=live * 15)


# ---------------------------------------------------------------- the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    s = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for k, v in s.items()}
    return _exact_norm(s) if case["kind"] == "norm" else _exact_scan(s)


def _exact_norm(s):
    """The definition, and its gradients by reverse accumulation through it."""
    names = ("x", "y", "z", "post", "scale", "pre")
    x, y, z, post, scale, pre = (s[k].detach().clone().requires_grad_(s["train"]) for k in names)
    m = y / ((y * y).mean(1, keepdim=True) + EPS).sqrt()
    o = x + scale * (post * m) * (z / (1 + torch.exp(-z)))
    n = pre * (o / ((o * o).mean(1, keepdim=True) + EPS).sqrt())
    out = dict(out=o.detach(), normed=n.detach())
    if s["train"]:
        grads = torch.autograd.grad((o, n), (x, y, z, post, scale, pre), (s["grad_out"], s["grad_normed"]))
        out.update(zip(("dx", "dy", "dz", "dpost", "dscale", "dpre"), grads))
    return out


def _exact_scan(s):
    b, t, d = s["x"].shape
    end = torch.full((b,), t, device="cuda") if s["lengths"] is None else s["lengths"].long()
    live = torch.arange(t, device="cuda")[:, None, None] < end[None, :, None]  # tokens first from here on
    x, r, g = (s[k].transpose(0, 1) for k in ("x", "r", "g"))
    keep = torch.where(live, 1 - s["rate"] / (1 + torch.exp(-r)), 1.0)
    add = torch.where(live, (1 - keep) * x / (1 + torch.exp(-g)), 0.0)
    h = torch.empty(t + 1, b, d, dtype=torch.float64, device="cuda")
    h[0] = s["state"]
    for k in range(t):
        torch.addcmul(add[k], keep[k], h[k], out=h[k + 1])
    del add
    out = dict(y=torch.where(live, h[1:], 0.0).transpose(0, 1), state=h[t].clone())
    if not s["train"]:
        return out
    reach = torch.where(live, s["grad_out"].transpose(0, 1), 0.0)  # becomes the whole gradient of h_t
    reach[t - 1] += s["grad_state"]
    for k in range(t - 1, 0, -1):
        reach[k - 1].addcmul_(keep[k], reach[k])
    sr, sg = 1 / (1 + torch.exp(-r)), 1 / (1 + torch.exp(-g))
    dkeep = torch.where(live, reach * (h[:t] - sg * x), 0.0)
    dadd = torch.where(live, reach * (s["rate"] * sr), 0.0)
    out.update(dx=(dadd * sg).transpose(0, 1), dr=(-dkeep * s["rate"] * sr * (1 - sr)).transpose(0, 1),
               dg=(dadd * x * sg * (1 - sg)).transpose(0, 1), drate=(-dkeep * sr).sum((0, 1)), dstate=keep[0] * reach[0])
    return out
