"""The sequence operators in 64 bits on the CPU, from their definitions: the
recurrence token by token, the norms as written, and gradients by reverse
accumulation through both.  Shares no code with the kernels."""
import torch

# half a unit in the last place of a stored activation, relative
UNIT = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}
# half the smallest subnormal: below it rounding is absolute
TINY = {torch.float32: 2.0**-150, torch.float16: 2.0**-25, torch.bfloat16: 2.0**-134}

# FP32 arithmetic against 64 bits, relative to the largest value of the output.
# A sigmoid's relative error is below (|v| + 5) 2^-24, so q and c are within
# about 1e-6 for gates up to 10; a state is an average of c with weights that
# sum to one, and its own roundings add up over a memory of at most a few
# hundred tokens like a random walk (20 x 2^-24 x 2): 3e-6 altogether.  Sums
# over rows and norms over a row stay below that.
FP32_ERROR = 1e-5


def sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def scan(x, r, g, rate, state=None, lengths=None):
    b, t, d = x.shape
    h = torch.zeros(b, d, dtype=torch.float64) if state is None else state
    n = torch.full((b,), t) if lengths is None else lengths.long().clamp(0, t)
    q, c = rate * sigmoid(r), sigmoid(g) * x
    ys = []
    for k in range(t):
        live = (k < n)[:, None]
        h = torch.where(live, (1 - q[:, k]) * h + q[:, k] * c[:, k], h)
        ys.append(torch.where(live, h, torch.zeros_like(h)))
    return (torch.stack(ys, 1) if t else torch.zeros(b, 0, d, dtype=torch.float64)), h


def norm(x, y, z, post, scale, pre, eps):
    o = x
    if y is not None:
        add = post * y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
        if z is not None:
            add = add * z * sigmoid(z)
        if scale is not None:
            add = add * scale
        o = x + add
    return o, None if pre is None else pre * o / torch.sqrt((o * o).mean(-1, keepdim=True) + eps)


def leaf(t):
    """A tensor's values in 64 bits on the CPU, as the start of a gradient."""
    return None if t is None else t.detach().cpu().double().requires_grad_(True)


def check(got, want, what, slack=1.0):
    """Every value within its storage's rounding and FP32_ERROR of the largest."""
    kind = got.dtype
    got, want = got.detach().cpu().double(), want.detach()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    if not want.numel():
        return
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    off = (got - want).nan_to_num(0.0).abs()
    allowed = UNIT[kind] * 1.001 * want.abs() + TINY[kind] + slack * FP32_ERROR * want.nan_to_num(0.0).abs().max()
    worst = (off / allowed.nan_to_num(1.0).clamp_min(1e-300)).max().item()
    assert worst <= 1.0, f"{what}: {worst:.2f} times the allowed error"
