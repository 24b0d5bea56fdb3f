"""Dropout, alone and in the norm, against plain implementations in 64 bits with the generator in numpy.

Bounds: the mask is exact.  A value takes a product and a sum in fp32 (2^-24 each) and one rounding to bf16;
the norm's bounds are test_gpu_layer_norm.py's, of sums of H terms, on top of that."""
import math

import numpy as np
import pytest
import torch

import dropout_ref as dr
import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say

pytestmark = pytest.mark.gpu
EPS = 1e-6


def rng_of(seed, step=0):
    return torch.tensor([seed, step], dtype=torch.int64, device="cuda")


def check(x, p, rng, site, residual=None, **more):
    got = ep.dropout(x, p, rng, site=site, residual=residual, **more)
    y = x.double() * dr.factor(x.shape, p, rng, site)
    off = y.abs() * ref.U23
    if residual is not None:
        y = y + residual.double()
        off = off + y.abs() * ref.U24
    ref.within(got, y, off + ref.BF16 * (y.abs() + off), "dropout")
    assert residual is not None or torch.equal(got == 0, (y == 0))
    return got


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("shape", [(8,), (1, 16), (3, 5, 24), (7, 2888), (1023, 8), (1024, 8), (1025, 8), (1000, 7168)])
def test_dropout(shape, residual):
    g = ref.gen(sum(shape))
    x = ref.normal(shape, g)
    r = ref.normal(shape, g) if residual else None
    for p in (0.0, 0.1, 0.5, 1.0):
        say(f"dropout {shape} p={p}")
        check(x, p, rng_of(12345, 7), 3, r)


@pytest.mark.parametrize("seed,step,site", [(0, 0, 0), (-1, -1, 2 ** 32 - 1), (2 ** 63 - 1, 2 ** 40 + 5, 1), (-2 ** 63, 2 ** 32, 9)])
def test_seeds_steps_and_sites(seed, step, site):
    say(f"dropout seed={seed} step={step} site={site}")
    x = ref.normal((40, 520), ref.gen(1))
    got = check(x, 0.3, rng_of(seed, step), site)
    assert torch.equal(got, ep.dropout(x, 0.3, rng_of(seed, step), site=site))
    for other in (ep.dropout(x, 0.3, rng_of(seed, step), site=site ^ 1), ep.dropout(x, 0.3, rng_of(seed, step ^ 1), site=site),
                  ep.dropout(x, 0.3, rng_of(seed ^ 1, step), site=site), ep.dropout(x, 0.3, rng_of(seed ^ 1 << 32, step), site=site)):
        share = ((other == 0) == (got == 0)).double().mean()  # independent: 0.3 0.3 + 0.7 0.7
        assert abs(float(share) - 0.58) < 6 * math.sqrt(0.58 * 0.42 / x.numel())


def test_shares_and_neighbours():
    """The dropped share, and how often neighbours at many distances agree, as independent values would."""
    say("dropout: shares")
    x = torch.ones((1 << 22,), dtype=torch.bfloat16, device="cuda")
    for p in (0.05, 0.1, 0.5):
        dropped = (ep.dropout(x, p, rng_of(99)) == 0).double()
        n, q = x.numel(), dr.cut_of(p) / 65536
        assert abs(float(dropped.mean()) - q) < 5 * math.sqrt(q * (1 - q) / n)
        for d in (1, 2, 3, 4, 7, 8, 9, 64, 4096, 65536):
            both = float((dropped[d:] * dropped[:-d]).mean())
            assert abs(both - q * q) < 5 * math.sqrt(q * q * (1 - q * q) / (n - d)) + 5e-9, (p, d)


def test_dropped_values_are_zero_whatever_they_were():
    say("dropout of infinities and NaN")
    x = ref.normal((64, 64), ref.gen(2))
    x[3], x[5] = float("nan"), float("inf")
    got, f = ep.dropout(x, 0.5, rng_of(5)), dr.factor(x.shape, 0.5, rng_of(5), 0)
    assert torch.isnan(got[3][f[3] > 0]).all() and (got[3][f[3] == 0] == 0).all()
    assert torch.isinf(got[5][f[5] > 0]).all() and (got[5][f[5] == 0] == 0).all()
    assert torch.isfinite(got[[i for i in range(64) if i not in (3, 5)]]).all()


def test_in_place_and_no_values():
    say("dropout in place")
    g = ref.gen(3)
    x, r = ref.normal((50, 264), g), ref.normal((50, 264), g)
    want = ep.dropout(x, 0.2, rng_of(1), residual=r)
    for into in ("x", "r"):
        xx, rr = x.clone(), r.clone()
        out = xx if into == "x" else rr
        assert ep.dropout(xx, 0.2, rng_of(1), residual=rr, out=out) is out and torch.equal(out, want)
    assert ep.dropout(x[:0], 0.2, rng_of(1)).shape == (0, 264)


def test_it_is_its_own_gradient():
    """<dropout(x), d> is linear in x with the gradient dropout(d)."""
    say("dropout: gradient")
    g = ref.gen(4)
    x, d = ref.normal((30, 512), g), ref.normal((30, 512), g)
    rng = rng_of(77, 3)
    f = dr.factor(x.shape, 0.25, rng, 2)
    leaf = x.double().requires_grad_()
    ((leaf * f) * d.double()).sum().backward()
    got = ep.dropout(d, 0.25, rng, site=2)
    ref.within(got, leaf.grad, leaf.grad.abs() * (ref.U23 + ref.BF16 * (1 + ref.U23)), "gradient")


def test_values_past_4_gib():
    """Counters and offsets of more than 32 bits' worth of bytes."""
    say("dropout of 4.4 GB")
    n = (2 ** 31 + 2 ** 27) // 8 * 8
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    rng = rng_of(2024, 1)
    got = ep.dropout(x, 0.5, rng, out=x)
    for first in (0, 2 ** 30, 2 ** 31 - 4096, 2 ** 31, n - 8192):
        want = torch.from_numpy(dr.bits(8192, rng, 0, first) >= 32768).cuda()
        want = want[:min(8192, n - first)]
        assert torch.equal(got[first:first + 8192] != 0, want), first
    del x, got


@pytest.mark.parametrize("H", [8, 16, 520, 528, 1024, 2048, 2888, 4096, 7168, 8192, 9000, 20000, 40000])
@pytest.mark.parametrize("T", [1, 3, 70])
def test_norm(T, H):
    say(f"dropout_rmsnorm T={T} H={H}")
    g = ref.gen(T + H)
    x, w = ref.normal((T, H), g), ref.normal(H, g)
    for r in (None, ref.normal((T, H), g)):
        rng = rng_of(T, H)
        got = ep.dropout_rmsnorm(x, 0.2, rng, w, site=4, residual=r, eps=EPS, total=True, rows8=H % 16 == 0)
        s = x.double() * dr.factor(x.shape, 0.2, rng, 4)
        s_off = s.abs() * ref.U23
        if r is not None:
            s = s + r.double()
            s_off = s_off + s.abs() * ref.U24
        ref.within(got.total, s, s_off + ref.BF16 * (s.abs() + s_off), "total")
        y = s / (s.square().mean(1, keepdim=True) + EPS).sqrt() * w.double()
        # s is off by s_off; 1 / rms by the sum of H squares (a product, a sum each: (H + 4) 2^-24 / 2, and the
        # values' own 2^-23) and its root and quotient, then two products
        y_off = y.abs() * ((H / 2 + 16) * ref.U24) + s_off / (s.square().mean(1, keepdim=True) + EPS).sqrt() * w.double().abs()
        ref.within(got.out, y, y_off + ref.BF16 * (y.abs() + y_off), "out")
        if got.rows8 is not None:  # as the norm of the same sums makes them
            q, scale = ep.rows8_values(got.rows8)
            most = y.abs().amax(1, keepdim=True)
            ref.within(scale, most / 448, (y_off.amax(1, keepdim=True) + most * ref.U23) / 448, "scale")
            ref.within(q.double() * scale.double(), y, y.abs() * 2.0 ** -4 + y_off * 1.1 + scale.double() * 2.0 ** -10
                       + y.abs() * 2.0 ** -20, "rows8")


def test_norm_without_dropping_is_the_norm():
    say("dropout_rmsnorm p=0")
    g = ref.gen(1)
    x, r, w, d = (ref.normal(s, g) for s in ((37, 2896), (37, 2896), 2896, (37, 2896)))
    one, two = ep.dropout_rmsnorm(x, 0.0, rng_of(1), w, residual=r, rows8=True), ep.rmsnorm(x, w, residual=r, rows8=True)
    assert torch.equal(one.total, two.total) and torch.equal(one.out, two.out) and torch.equal(one.rows8, two.rows8)
    dx, dr_, dw = ep.dropout_rmsnorm_grad(one.total, w, d, 0.0, rng_of(1), d_total=r)
    want, want_dw = ep.rmsnorm_grad(two.total, w, d, d_total=r)
    assert torch.equal(dx, want) and torch.equal(dr_, want) and torch.equal(dw, want_dw)


@pytest.mark.parametrize("H", [8, 520, 1024, 2048, 2888, 7168, 9000, 20000, 40000])
@pytest.mark.parametrize("T", [1, 5, 600])
def test_norm_gradient(T, H):
    say(f"dropout_rmsnorm_grad T={T} H={H}")
    g = ref.gen(T + H)
    s, d, w, t = ref.normal((T, H), g, 2.0), ref.normal((T, H), g), ref.normal(H, g), ref.normal((T, H), g)
    rng = rng_of(H, T)
    f = dr.factor((T, H), 0.3, rng, 1)
    for dt in (None, t):
        dx, dres, dw = ep.dropout_rmsnorm_grad(s, w, d, 0.3, rng, site=1, d_total=dt, eps=EPS)
        want, want_dw = ep.rmsnorm_grad(s, w, d, d_total=dt, eps=EPS)
        assert torch.equal(dres, want) and torch.equal(dw, want_dw)  # without dropout's part: the norm's gradient
        exact, size, _, _ = ref.norm_grad(s, w, d, dt, EPS)
        off = size * (H + 16) * ref.U24 + exact.abs() * ref.U23
        ref.within(dx, exact * f, f * off + ref.BF16 * f * (exact.abs() + off), "dx")
        only = ep.dropout_rmsnorm_grad(s, w, d, 0.3, rng, site=1, d_total=dt, eps=EPS, d_residual=False, d_weight=False)
        assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
        only = ep.dropout_rmsnorm_grad(s, w, d, 0.3, rng, site=1, d_total=dt, eps=EPS, dx=False)
        assert only[0] is None and torch.equal(only[1], dres) and torch.equal(only[2], dw)


def test_norm_gradient_in_place():
    say("dropout_rmsnorm_grad in place")
    g = ref.gen(8)
    s, d, w, t = ref.normal((90, 2888), g), ref.normal((90, 2888), g), ref.normal(2888, g), ref.normal((90, 2888), g)
    dx, dres, dw = ep.dropout_rmsnorm_grad(s, w, d, 0.3, rng_of(3), d_total=t)
    dd, tt = d.clone(), t.clone()
    got = ep.dropout_rmsnorm_grad(s, w, dd, 0.3, rng_of(3), d_total=tt, dx=dd, d_residual=tt)
    assert torch.equal(dd, dx) and torch.equal(tt, dres) and torch.equal(got[2], dw)


def test_norm_against_differences():
    """Central differences of the loss in 64 bits along random directions of x and of the residual."""
    say("dropout_rmsnorm: differences")
    g = ref.gen(6)
    x, r, w, d, t = (ref.normal(s, g) for s in ((9, 136), (9, 136), 136, (9, 136), (9, 136)))
    rng = rng_of(4, 2)
    f = dr.factor(x.shape, 0.25, rng, 0)
    kept = ep.dropout_rmsnorm(x, 0.25, rng, w, residual=r)
    grads = ep.dropout_rmsnorm_grad(kept.total, w, d, 0.25, rng, d_total=t)

    def loss(xx, rr):
        s = xx * f + rr
        y = s / (s.square().mean(1, keepdim=True) + EPS).sqrt() * w.double()
        return float((y * d.double()).sum() + (s * t.double()).sum())

    for i, have in enumerate(grads[:2]):
        for _ in range(4):
            v = torch.randn(x.shape, dtype=torch.float64, device="cuda", generator=g)
            h = 1e-5
            at = [x.double(), r.double()]
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * v, at[i] - h * v
            along = (loss(*up) - loss(*down)) / (2 * h)
            terms = have.double() * v
            # the total and the result are rounded to bf16; a gradient's terms may be larger than their sum by 4
            assert abs(terms.sum() - along) <= 4 * 2 * ref.BF16 * float(terms.abs().sum()), i


def test_side_stream_and_graph():
    """A captured call draws a new mask where the program advances the step between replays."""
    say("dropout on a side stream and in a graph")
    g = ref.gen(7)
    x, r, w = ref.normal((64, 1024), g), ref.normal((64, 1024), g), ref.normal(1024, g)
    rng = rng_of(31, 0)
    want = ep.dropout(x, 0.1, rng, residual=r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ep.dropout(x, 0.1, rng, residual=r, stream=side)
    n = ep.dropout_rmsnorm(x, 0.1, rng, w, residual=r, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(n.total, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ep.dropout(x, 0.1, rng, residual=r)
        n = ep.dropout_rmsnorm(x, 0.1, rng, w, residual=r)
        back = ep.dropout_rmsnorm_grad(n.total, w, x, 0.1, rng)
        rng[1].add_(1)
    seen = []
    for i in range(4):
        now = rng.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert int(rng[1]) == i + 1
        assert torch.equal(out, ep.dropout(x, 0.1, now, residual=r)) and torch.equal(n.total, out)
        want = ep.dropout_rmsnorm_grad(n.total, w, x, 0.1, now)
        assert all(torch.equal(a, b) for a, b in zip(back, want))
        seen.append(out.clone())
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


def test_nothing_beside_the_outputs():
    say("dropout: what lies beside the outputs")
    for T, H in ((1, 16), (5, 2896), (33, 7168)):
        x, w = ref.normal((T, H), ref.gen(T)), ref.normal(H, ref.gen(H))
        held = [torch.full((3, T, H), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(5)]
        ep.dropout(x, 0.5, rng_of(1), out=held[0][1])
        ep.dropout_rmsnorm(x, 0.5, rng_of(1), w, total=held[1][1], out=held[2][1])
        ep.dropout_rmsnorm_grad(x, w, x, 0.5, rng_of(1), dx=held[3][1], d_residual=held[4][1])
        for t in held:
            assert (t[0] == 7.0).all() and (t[2] == 7.0).all() and not (t[1] == 7.0).all()


def test_binding_refusals():
    say("dropout: refusals of the binding")
    x, rng, w = ref.normal((4, 64), ref.gen(1)), rng_of(1), ref.normal(64, ref.gen(2))
    for bad in (x.cpu(), x.float(), x.t()):
        with pytest.raises(ValueError):
            ep.dropout(bad, 0.1, rng)
    for bad in (dict(rng=None), dict(rng=rng.cpu()), dict(rng=rng.int()), dict(rng=rng[:1]), dict(site=-1), dict(site=2 ** 32),
                dict(residual=x[:2]), dict(out=x.float())):
        with pytest.raises(ValueError):
            ep.dropout(**{"x": x, "p": 0.1, "rng": rng, **bad})
        bad.pop("out", None)
        if bad:
            with pytest.raises(ValueError):
                ep.dropout_rmsnorm(**{"x": x, "p": 0.1, "rng": rng, **bad})
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(ep.EPError):
            ep.dropout(x, p, rng)
        with pytest.raises(ep.EPError):
            ep.dropout_rmsnorm(x, p, rng)
        with pytest.raises(ep.EPError):
            ep.dropout_rmsnorm_grad(x, w, x, p, rng)
    with pytest.raises(ep.EPError):
        ep.dropout(x.view(-1)[:4], 0.1, rng)
    with pytest.raises(ep.EPError):
        ep.dropout_rmsnorm_grad(x, w, x, 0.1, rng, dx=False, d_residual=False)
    into = torch.empty_like(x)
    with pytest.raises(ep.EPError):
        ep.dropout_rmsnorm_grad(x, w, x, 0.1, rng, dx=into, d_residual=into)
    for bad in (dict(d_out=None), dict(d_out=x[:2]), dict(d_total=x[:2]), dict(rng=rng.int())):
        with pytest.raises(ValueError):
            ep.dropout_rmsnorm_grad(**{"total": x, "weight": w, "d_out": x, "p": 0.1, "rng": rng, **bad})
