"""Plain implementations in 64 bits of the layer operators, and the inputs of their tests.

Shared by the test_gpu_layer_* files.  Nothing here uses the library."""
import math

import torch

U24 = 2.0 ** -24       # relative rounding of fp32
U23 = 2.0 ** -23       # the same where a sum may truncate instead of round
BF16 = 2.0 ** -8       # half a bf16 step is at most this share of the value
ACT_LIP = 1.2          # largest slope of relu, silu (1.10) and gelu (1.13)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(shape, g, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


def within(got, want, bound, what=""):
    """|got - want| <= bound, element by element; NaN and infinities at the same places."""
    got, want = got.double(), want.double()
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN at other places"
    assert torch.equal(got[~finite & ~torch.isnan(want)], want[~finite & ~torch.isnan(want)]), f"{what}: infinities"
    over = ((got - want).abs() - bound)[finite]
    assert over.numel() == 0 or over.max() <= 0, f"{what}: {over.max():.3g} over the bound"


# ---------------------------------------------------------------------------- norm

def norm(x, residual, weight, eps):
    s = x.double() if residual is None else x.double() + residual.double()
    w = torch.ones(s.shape[1], dtype=torch.float64, device=s.device) if weight is None else weight.double()
    return s, s / (s.square().mean(1, keepdim=True) + eps).sqrt() * w


def norm_grad(total, weight, d_out, d_total, eps):
    """dx, the size of what dx is summed from, d_weight, the size of its terms."""
    s, d = total.double(), d_out.double()
    w = torch.ones(s.shape[1], dtype=torch.float64, device=s.device) if weight is None else weight.double()
    r = 1 / (s.square().mean(1, keepdim=True) + eps).sqrt()
    n, g = s * r, d * w
    t = torch.zeros_like(s) if d_total is None else d_total.double()
    dx = r * (g - n * (g * n).mean(1, keepdim=True)) + t
    size = r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True)) + t.abs()
    return dx, size, (d * n).sum(0), (d * n).abs().sum(0)


# --------------------------------------------------------------------------- router

def softmax(z):
    """softmax over dim 1 in which rows of -inf alone are zero."""
    top = z.amax(1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(1, keepdim=True)
    return p / torch.where(total == 0, torch.ones_like(total), total)


def route(logits, k, mask=None, normalize=True, balance=0.0):
    """idx, gates, counts, prob_sums, loss in 64 bits (CPU)."""
    z = logits.double().cpu()
    T, E = z.shape
    live = torch.ones(T, dtype=torch.bool) if mask is None else mask.cpu().bool()
    order = z.clone()
    order[torch.isnan(z)] = -math.inf
    # among -inf and NaN: -inf first; the sort is stable, so the lowest index among equals
    rank = torch.where(torch.isnan(z), 1, 0)
    idx = torch.empty((T, k), dtype=torch.int64)
    for t in range(T):
        idx[t] = torch.tensor(sorted(range(E), key=lambda e: (-float(order[t, e]), int(rank[t, e]), e))[:k])
    idx[~live] = ((torch.arange(T)[:, None] * k + torch.arange(k)) % E)[~live]
    p = softmax(z)
    gates = softmax(z.gather(1, idx)) if normalize else p.gather(1, idx)
    if normalize:  # a NaN anywhere in a row makes the row's largest logit's exponential no less valid
        gates = gates.clone()
    gates[~live] = 0
    counts = torch.bincount(idx[live].reshape(-1), minlength=E)
    sums = p[live].sum(0)
    n = int(live.sum())
    loss = balance * E * float((counts.double() * sums).sum()) / (n * k * n) if n else 0.0
    return idx, gates, counts, sums, loss


def route_grad(logits, idx, k, mask, normalize, balance, d_gates, d_loss, counts):
    z = logits.double().cpu()
    T, E = z.shape
    live = torch.ones(T, dtype=torch.bool) if mask is None else mask.cpu().bool()
    p = softmax(z)
    dz = torch.zeros_like(z)
    size = torch.zeros_like(z)
    if d_gates is not None:
        d = d_gates.double().cpu()
        if normalize:
            q = torch.zeros_like(z).scatter(1, idx, softmax(z.gather(1, idx)))
        else:
            q = p
        full = torch.zeros_like(z).scatter(1, idx, d)
        mean = (q * full).sum(1, keepdim=True)
        dz += q * (full - mean)
        size += q * (full.abs() + (q * full).abs().sum(1, keepdim=True))
    if d_loss is not None:
        n = int(counts.sum()) // k
        g = d_loss * balance * E * counts.double().cpu() / (n * k * n) if n else torch.zeros(E, dtype=torch.float64)
        dz += p * (g - (p @ g)[:, None])
        size += p * (g.abs() + (p @ g.abs())[:, None])
    dz[~live] = 0
    size[~live] = 0
    return dz, size


# -------------------------------------------------------------------------- product

def rows8_of(values, scales):
    """8-bit rows from e4m3 values [n, H] and fp32 scales [n]."""
    n, h = values.shape
    rows = torch.zeros((n, h + 16), dtype=torch.uint8, device=values.device)
    rows[:, :h] = values.view(torch.uint8)
    rows[:, h:h + 4] = scales.view(torch.uint8).view(n, 4)
    return rows


def offsets_of(counts, first=0):
    return torch.tensor([first] + [first + sum(counts[:i + 1]) for i in range(len(counts))], dtype=torch.int32, device="cuda")


def act(z, name):
    if name == "swiglu":
        g, u = z.chunk(2, 1)
        return g * torch.sigmoid(g) * u
    return {"none": lambda: z, "relu": lambda: z.clamp_min(0), "silu": lambda: z * torch.sigmoid(z),
            "gelu": lambda: z * torch.special.ndtr(z)}[name]()


def act_error(z, dz, name):
    """How far act(z) may be off for z off by dz and the activation evaluated in fp32."""
    if name == "swiglu":
        g, u = z.chunk(2, 1)
        dg, du = dz.chunk(2, 1)
        s = g * torch.sigmoid(g)
        return ACT_LIP * dg * (u.abs() + du) + s.abs() * du + (s * u).abs() * 2.0 ** -18
    if name == "none":
        return dz
    return ACT_LIP * dz + z.abs() * 2.0 ** -18


def act_grad(z, d, name):
    if name == "swiglu":
        g, u = z.chunk(2, 1)
        s = torch.sigmoid(g)
        return torch.cat([d * u * (s + g * s * (1 - s)), d * g * s], 1)
    s = torch.sigmoid(z)
    return d * {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(), "silu": lambda: s + z * s * (1 - s),
                "gelu": lambda: torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[name]()


def product_z(x, w, offsets, bias=None):
    """z and the sum of the magnitudes of its terms, in 64 bits; rows outside the offsets are 0."""
    ends = offsets.tolist()
    z = torch.zeros((x.shape[0], w.shape[1]), dtype=torch.float64, device=x.device)
    size = torch.zeros_like(z)
    for e in range(w.shape[0]):
        at = slice(ends[e], ends[e + 1])
        z[at] = x[at] @ w[e].t()
        size[at] = x[at].abs() @ w[e].abs().t()
        if bias is not None:
            z[at] += bias[e].double()
            size[at] += bias[e].double().abs()
    return z, size
