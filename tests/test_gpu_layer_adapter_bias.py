"""The gradients of a bias and of W that are trained beside the adapters: ep_expert_product_grad of one expert, over the same
pre and d_y, against 64 bits and against differences."""
import pytest
import torch

import adapter_ref as ar
import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say

pytestmark = pytest.mark.gpu


def step(s, d_y):
    by = ar.rows_of(s)
    got = ep.adapter_product(s["x"], s["a"], s["b"], by, w=s["w"], scale=s["scale"], bias=s["bias"], act=s["act"], keep_pre=True,
                             keep_low=True)
    pre = None if s["act"] == "none" else got.pre
    grad = ep.adapter_product_grad(s["x"], s["a"], s["b"], got.low, d_y, by, w=s["w"], scale=s["scale"], pre=pre, act=s["act"])
    base = ep.expert_product_grad(s["x"], s["w"][None], d_y, pre=pre, act=s["act"], dx=False, dw=False, with_bias=True)
    assert base.dx is None and base.dw is None
    return got, grad, base.dbias[0]


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "swiglu"])
@pytest.mark.parametrize("rows,N", [(1, 8), (130, 136), (5000, 264)])
def test_bias_gradient(rows, N, act):
    say(f"adapters beside a trained bias rows={rows} N={N} {act}")
    s = ar.make(ar.random_ids(rows, 4, rows), 4, 16, 136, N, rows, act, bias=True)
    d_y = ref.normal((rows, N), ref.gen(3))
    got, _, dbias = step(s, d_y)
    pre, d = got.pre.double(), d_y.double()
    dz = ref.act_grad(pre, d, act)
    # the slope is within 2^-17 (adapter_ref), dz is summed unrounded in fp32
    if act == "swiglu":
        gate, up = pre.chunk(2, 1)
        off = torch.cat([d.abs() * up.abs() * (gate.abs() + 1.2), d.abs() * gate.abs()], 1) * 2.0 ** -17
    else:
        off = d.abs() * (pre.abs() + 1.2) * 2.0 ** -17
    ref.within(dbias, dz.sum(0), (off + (dz.abs() + off) * (rows + 8) * ref.U23).sum(0), "dbias")


@pytest.mark.parametrize("act", ["none", "silu", "swiglu"])
def test_against_differences(act):
    """Central differences of <y, d_y> in 64 bits along random directions of the bias."""
    say(f"adapters beside a trained bias, differences {act}")
    rows, A, R, K, N = 50, 3, 16, 72, 40
    s = ar.make(ar.random_ids(rows, A, 3), A, R, K, N, 2, act, bias=True)
    of, order, _ = ar.sorted_ids(s["ids"], A)
    g = ref.gen(9)
    d_y = ref.normal((rows, N), g)
    got, _, dbias = step(s, d_y)
    low = ar.by_adapter(s["x"].double()[order], of, s["a"].double().transpose(1, 2))[0] * ar.scales(s, of)
    z = s["x"].double() @ s["w"].double().t()
    z = z.index_add(0, order, ar.by_adapter(low, of, s["b"].double().transpose(1, 2))[0])

    def loss(bias):
        return float((ref.act(z + bias, act) * d_y.double()).sum())

    # what dbias may be off: pre is rounded to bf16, and the slope changes by at most 1.1 (silu'' is below 0.5, gelu'' below 1) of
    # what its place is off, times the other factor; swiglu's second factor is rounded as well
    pre = got.pre.double()
    step_of = ref.BF16 * pre.abs()
    if act == "swiglu":
        gate, up = pre.chunk(2, 1)
        step_gate, step_up = step_of.chunk(2, 1)
        slack = torch.cat([d_y.double().abs() * (1.1 * up.abs() * step_gate + 1.2 * step_up), d_y.double().abs() * 1.2 * step_gate], 1)
    else:
        slack = d_y.double().abs() * 1.1 * step_of
    for t in range(4):
        v = torch.randn(s["bias"].shape, dtype=torch.float64, device="cuda", generator=g)
        h = 1e-5
        bias = s["bias"].double()
        along = (loss(bias + h * v) - loss(bias - h * v)) / (2 * h)
        # and 2^-10 of the terms for the sums in fp32 and the differences' own error
        off = float((slack.sum(0) * v.abs()).sum()) + 2.0 ** -10 * float((dbias.double() * v).abs().sum())
        assert abs(float((dbias.double() * v).sum()) - along) <= off, t
