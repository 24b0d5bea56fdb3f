"""Infinite weights and rows of an adapter's own: the formula's infinities, signs and NaN.

Inputs are whole numbers, so every sum is exact in fp32, and so are the low-rank values (below 2^16) as the sum of two bf16
values: what is left is the result's own rounding, and infinities have the signs of the formula's."""
import pytest
import torch

import adapter_ref as ar
import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say

pytestmark = pytest.mark.gpu
INF = float("inf")


def whole(shape, most, g):
    return torch.randint(-most, most + 1, shape, device="cuda", generator=g).bfloat16()


def inputs(rows, A, R, K, N, seed, act="none", base=True):
    s = ar.make(ar.random_ids(rows, A, seed), A, R, K, N, seed, act, base)
    g, wide = ref.gen(seed), s["b"].shape[1]
    s["x"], s["a"], s["b"] = whole((rows, K), 100, g), whole((A, R, K), 1, g), whole((A, wide, R), 1, g)
    s["w"] = whole((wide, K), 1, g) if base else None
    s["scale"] = torch.tensor([1.0, 0.5, 2.0, 1.0, 0.25], device="cuda")[:A]
    return s, wide, g


def equal(got, want, what):
    """The formula's value rounded once, NaN and infinities at the same places."""
    ref.within(got, want.bfloat16(), torch.zeros_like(want), what)


def forward(s):
    """low and z in 64 bits."""
    of, order, _ = ar.sorted_ids(s["ids"], s["A"])
    x = s["x"].double()
    low = ar.by_adapter(x[order], of, s["a"].double().transpose(1, 2))[0] * ar.scales(s, of)
    z = torch.zeros((x.shape[0], s["b"].shape[1]), dtype=torch.float64, device="cuda")
    z[order] = ar.by_adapter(low, of, s["b"].double().transpose(1, 2))[0]
    return low, z if s["w"] is None else z + x @ s["w"].double().t()


# few results, with and without W; one pass over the contraction; the contraction in two parts, gated too, and in eight
SIZES = [(70, 264, 136, True), (300, 136, 264, False), (5000, 136, 1032, True), (5000, 72, 1032, False), (4500, 5632, 1024, True),
         (141, 1736, 8432, True), (5883, 5576, 144, True)]


@pytest.mark.parametrize("rows,K,N,base", SIZES)
@pytest.mark.parametrize("act", ["none", "relu", "swiglu"])
def test_product(rows, K, N, base, act):
    say(f"adapter_product, infinite weights rows={rows} K={K} N={N} base={base} {act}")
    for R in (8, 40):
        s, wide, _ = inputs(rows, 5, R, K, N, rows + R, act, base)
        s["b"][1, N // 2, 3], s["b"][1, wide - 1, 5], s["b"][2, 0, 0] = INF, -INF, -INF
        s["b"][2, 9, 1], s["b"][2, 9, 2] = INF, INF  # two of them: NaN where their rows' signs differ
        s["a"][3, 2, 7] = INF
        low, z = forward(s)
        assert (z.isinf().sum(0) > 0).sum() >= 4 and z[s["ids"] == 4].isfinite().all()
        got = ep.adapter_product(s["x"], s["a"], s["b"], ar.rows_of(s), w=s["w"], scale=s["scale"], act=act, keep_pre=True,
                                 keep_low=True)
        equal(got.low, low, "low")
        equal(got.pre, z, "pre")
        y = ref.act(z, act)
        if act == "swiglu":  # where exp(-gate) is past 2^126 (e^87.3) its reciprocal is below fp32's normal numbers, and 0
            gate, up = z.chunk(2, 1)
            y = torch.where(gate < -87.3, gate * 0 * up, y)
        ref.within(got.out, y, ref.act_error(z, torch.zeros_like(z), act) + ref.BF16 * y.abs() * 1.01, "y")


@pytest.mark.parametrize("rows,K,N,base", SIZES)
@pytest.mark.parametrize("act", ["none", "relu"])
def test_gradient(rows, K, N, base, act):
    """dz is exact: the derivative is 0 or 1.  x keeps infinities to rows of adapters 0 and 4, a and b to others."""
    say(f"adapter_product_grad, infinite weights and rows, rows={rows} K={K} N={N} base={base} {act}")
    for R in (8, 40):
        s, wide, g = inputs(rows, 5, R, N, K, rows + R, act, base)  # the long contraction is dz's
        d, low = whole((rows, K), 50, g), whole((rows, R), 9, g)
        pre = None if act == "none" else whole((rows, wide), 3, g)
        s["a"][1, 3, N // 2], s["a"][2, 0, 0], s["a"][1, 5, 1], s["b"][3, 7, 2] = INF, -INF, -INF, INF
        for e, column, value in ((0, 4, INF), (4, N - 1, -INF)):
            s["x"][torch.nonzero(s["ids"] == e)[0, 0], column] = value
        of, order, _ = ar.sorted_ids(s["ids"], 5)
        dz = d.double() if pre is None else d.double() * (pre > 0)
        v = ar.by_adapter(dz[order], of, s["b"].double())[0] * ar.scales(s, of)
        dx = torch.zeros((rows, N), dtype=torch.float64, device="cuda")
        dx[order] = ar.by_adapter(v, of, s["a"].double())[0]
        if base:
            dx += dz @ s["w"].double()
        assert (dx.isinf().sum(0) > 0).sum() >= 3
        got = ep.adapter_product_grad(s["x"], s["a"], s["b"], low, d, ar.rows_of(s), w=s["w"], scale=s["scale"], pre=pre, act=act)
        equal(got.dx, dx, "dx")
        for e in range(5):
            at = of == e
            x, n = s["x"][order][at].double(), int(at.sum())
            want = v[at].t() @ x
            # sums past 2^24 are rounded: the formula's bound, and the result's rounding
            off = v[at].abs().t() @ x.abs() * ((2 * n + 8) * ref.U23 + ar.TWO)
            ref.within(got.da[e], want, off + ref.BF16 * (want.abs() + off), f"da {e}")
            assert e not in (0, 4) or want.isinf().any()
            want, off = dz[order][at].t() @ low[at].double(), dz[order][at].abs().t() @ low[at].double().abs() * (n + 8) * ref.U23
            ref.within(got.db[e], want, off + ref.BF16 * (want.abs() + off), f"db {e}")
