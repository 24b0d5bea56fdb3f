"""The router and its gradient against plain implementations in 64 bits.

The ids are compared exactly.  Bounds of the rest: an exponential of z - max, |z - max| <= 64
here, has a relative error of (|z - max| + 4) 2^-24 <= 2^-17; a softmax sums E of them in fp32,
so probabilities and gates are within 2^-16 of themselves, their sums over T tokens within
2^-16 + T 2^-24, and the gradient's terms within 2^-15 of their sizes."""
import math

import pytest
import torch

import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say

pytestmark = pytest.mark.gpu


def check(z, k, mask=None, normalize=True, balance=0.01, grad=True):
    T, E = z.shape
    got = ep.route(z, k, mask=mask, normalize=normalize, balance=balance)
    idx, w, counts, sums, loss = ref.route(z, k, mask, normalize, balance)
    assert torch.equal(got.topk_idx.cpu().long(), idx)
    assert torch.equal(got.expert_counts.cpu().long(), counts)
    ref.within(got.topk_w.cpu(), w, w * 2.0 ** -16, "gates")
    ref.within(got.prob_sums.cpu(), sums, sums * (2.0 ** -16 + T * ref.U24) + 1e-37, "prob_sums")
    assert abs(float(got.loss) - loss) <= abs(loss) * (2.0 ** -15 + T * ref.U24) + 1e-37
    bare = ep.route(z, k, mask=mask, normalize=normalize, counts=False)
    assert bare.expert_counts is None
    assert torch.equal(bare.topk_idx, got.topk_idx) and torch.equal(bare.topk_w, got.topk_w)
    if not grad:
        return got
    g = ref.gen(T + E)
    d = torch.randn((T, k), device="cuda", generator=g)
    dl = torch.tensor([float(T) * 3], device="cuda")
    step = ref.BF16 if z.dtype == torch.bfloat16 else 2.0 ** -20
    for dg, dloss in ((d, dl), (d, None), (None, dl)):
        dz = ep.route_grad(z, got, dg, dloss)
        assert dz.dtype == z.dtype
        want, size = ref.route_grad(z, idx, k, mask, normalize, balance, dg, None if dloss is None else float(dloss), counts)
        ref.within(dz.cpu(), want, want.abs() * step + size * 2.0 ** -14 + 1e-36, "d_logits")
    return got


@pytest.mark.parametrize("E", [1, 2, 7, 8, 16, 17, 60, 64, 65, 128, 129, 200, 256, 257, 500, 512, 513, 1000, 1025, 2048])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_experts(E, dtype):
    for k in sorted({1, min(2, E), min(8, E)}):
        say(f"route E={E} k={k} {dtype}")
        g = ref.gen(E * 10 + k)
        z = ref.normal((33, E), g, 3.0, dtype)
        check(z, k, normalize=True)
        check(z, k, mask=torch.rand(33, device="cuda", generator=g) > 0.3, normalize=False)


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 64, 65, 257, 1000])
@pytest.mark.parametrize("k", [1, 3, 6])
def test_tokens(T, k):
    say(f"route T={T} k={k}")
    g = ref.gen(T)
    check(ref.normal((T, 60), g, 2.0, torch.float32), k)


@pytest.mark.parametrize("E,k", [(64, 64), (96, 96), (130, 100), (2048, 70)])
def test_many_experts_per_token(E, k):
    say(f"route E={E} k={k}")
    g = ref.gen(E)
    z = ref.normal((9, E), g, 2.0, torch.float32)
    check(z, k)
    check(z, k, normalize=False)


def test_ties_and_masked_experts():
    say("route: ties, masked experts")
    E = 70
    z = torch.zeros((8, E), device="cuda")
    z[1] = -0.0
    z[1, 5] = 0.0                               # +0 and -0 are equal
    z[2, 3::2] = -math.inf                      # masked experts
    z[3] = -math.inf
    z[3, 69] = 2.0                              # one expert left
    z[4] = -math.inf                            # none left
    z[5] = torch.finfo(torch.float32).min       # the type's lowest value in every place
    z[6, 10:] = torch.finfo(torch.float32).min
    z[7] = torch.arange(E, device="cuda") % 3
    for dtype in (torch.float32, torch.bfloat16):
        for normalize in (True, False):
            got = check(z.to(dtype), 4, normalize=normalize)
            assert got.topk_idx[0].tolist() == [0, 1, 2, 3] and got.topk_idx[1].tolist() == [0, 1, 2, 3]
            assert got.topk_idx[3].tolist() == [69, 0, 1, 2] and got.topk_w[3].tolist() == [1.0, 0.0, 0.0, 0.0]
            assert not got.topk_w[4].any()
            assert got.topk_idx[7].tolist() == [2, 5, 8, 11]


def test_masked_tokens_are_not_looked_at():
    """Whatever stands in a padding token's logits: no gates, no counts, no gradient, valid ids."""
    say("route: masked tokens")
    T, E, k = 40, 24, 4
    g = ref.gen(2)
    z = ref.normal((T, E), g, 1.0, torch.float32)
    mask = torch.arange(T, device="cuda") % 3 != 1
    z[~mask] = float("nan")
    z[4] = math.inf
    for m in (mask, mask.to(torch.uint8)):
        got = ep.route(z, k, mask=m, balance=1.0)
        assert torch.isfinite(got.prob_sums).all() and torch.isfinite(got.loss)
        assert not got.topk_w[~mask].any() and int(got.expert_counts.sum()) == int(mask.sum()) * k
        want = (torch.arange(T, device="cuda")[:, None] * k + torch.arange(k, device="cuda")) % E
        assert torch.equal(got.topk_idx[~mask].long(), want[~mask])
        dz = ep.route_grad(z, got, torch.randn((T, k), device="cuda"), torch.ones(1, device="cuda"))
        assert not dz[~mask].any() and torch.isfinite(dz).all()
    none = ep.route(z, k, mask=torch.zeros(T, dtype=torch.bool, device="cuda"), balance=1.0)
    assert float(none.loss) == 0 and not none.expert_counts.any() and not none.prob_sums.any()
    lay = ep.dispatch_layout(none.topk_idx, E, 4)   # the layout takes the ids of masked tokens
    ep.layout_validate(lay)


def test_nan_and_infinity_stay_in_their_rows():
    say("route: NaN and +inf")
    T, E, k = 20, 40, 4
    z = ref.normal((T, E), ref.gen(9), 1.0, torch.float32)
    clean = ep.route(z, k)
    z[3, 7] = float("nan")
    z[5] = float("nan")
    z[9, 2] = math.inf
    got = ep.route(z, k)
    keep = torch.tensor([t for t in range(T) if t not in (3, 5, 9)], device="cuda")
    assert torch.equal(got.topk_idx[keep], clean.topk_idx[keep]) and torch.equal(got.topk_w[keep], clean.topk_w[keep])
    assert 7 not in got.topk_idx[3].tolist() and got.topk_idx[5].tolist() == [0, 1, 2, 3] and got.topk_idx[9, 0] == 2
    assert got.topk_w[9].isnan().any() and got.loss.isnan()
    ep.layout_validate(ep.dispatch_layout(got.topk_idx, E, 4))
    unnormalized = ep.route(z, k, normalize=False)
    assert unnormalized.topk_w[[3, 5, 9]].isnan().any(dim=1).all()


def test_no_tokens():
    z = torch.empty((0, 12), device="cuda")
    got = ep.route(z, 3, balance=1.0)
    assert got.topk_idx.shape == (0, 3) and not got.expert_counts.any() and float(got.loss) == 0
    assert ep.route_grad(z, got, torch.empty((0, 3), device="cuda"), torch.ones(1, device="cuda")).shape == (0, 12)


def test_large_repeats_and_reuses_outputs():
    say("route: 20000 tokens, repeated")
    g = ref.gen(4)
    z = ref.normal((20000, 256), g, 1.5, torch.float32)
    mask = torch.rand(20000, device="cuda", generator=g) > 0.1
    got = ep.route(z, 8, mask=mask, balance=0.1)
    order = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :8]
    assert torch.equal(got.topk_idx[mask].long(), order[mask])
    p = torch.softmax(z.double(), 1)[mask]
    ref.within(got.prob_sums, p.sum(0), p.sum(0) * (2.0 ** -16 + 20000 * ref.U24), "prob_sums")
    d = torch.randn((20000, 8), device="cuda", generator=g)
    one = torch.ones(1, device="cuda")
    dz = ep.route_grad(z, got, d, one)
    first = {n: getattr(got, n).clone() for n in ("topk_idx", "topk_w", "expert_counts", "prob_sums", "loss")}
    for _ in range(3):
        again = ep.route(z, 8, mask=mask, balance=0.1, out=got)
        assert again is got and all(torch.equal(getattr(again, n), v) for n, v in first.items())
        assert torch.equal(ep.route_grad(z, got, d, one), dz)
    assert torch.equal(ep.route_grad(z.clone(), got, d, one, out=z), dz)


def test_counts_of_a_group():
    """Counts summed over ranks: the same gradient as of the whole batch's loss."""
    say("route_grad with a group's counts")
    g = ref.gen(6)
    z = ref.normal((64, 30), g, 1.0, torch.float32)
    whole = ep.route(z, 2, balance=1.0)
    one = torch.ones(1, device="cuda")
    want = ep.route_grad(z, whole, None, one)
    for part in (slice(0, 24), slice(24, 64)):
        zp = z[part].contiguous()
        r = ep.route(zp, 2, balance=1.0)
        torch.testing.assert_close(ep.route_grad(zp, r, None, one, counts=whole.expert_counts), want[part], rtol=1e-6, atol=0)


@pytest.mark.parametrize("normalize", [True, False])
def test_gradient_against_differences(normalize):
    """Against central differences of sum(d * gates) + loss in 64 bits, whose choice of experts and
    counts stay as they are along the step."""
    say("route_grad against differences")
    T, E, k = 12, 20, 3
    g = ref.gen(8)
    z = ref.normal((T, E), g, 1.0, torch.float32)
    d = torch.randn((T, k), device="cuda", generator=g)
    got = ep.route(z, k, normalize=normalize, balance=0.7)
    dz = ep.route_grad(z, got, d, torch.full((1,), 5.0, device="cuda"))
    idx, counts = got.topk_idx.cpu().long(), got.expert_counts.cpu().double()

    def loss(a):
        p = torch.softmax(a, 1)
        w = torch.softmax(a.gather(1, idx), 1) if normalize else p.gather(1, idx)
        return (w * d.cpu().double()).sum() + 5.0 * 0.7 * E * (counts / (T * k) * p.sum(0) / T).sum()

    v = torch.randn((T, E), dtype=torch.float64)
    h = 1e-4
    along = (loss(z.cpu().double() + h * v) - loss(z.cpu().double() - h * v)) / (2 * h)
    assert abs((dz.cpu().double() * v).sum() - along) <= 1e-4 * (1 + float(d.abs().sum()) * 1e-2)


def test_binding_refusals():
    """Wrong devices, types, layouts and shapes raise before anything is enqueued."""
    say("route: refusals of the binding")
    z = torch.randn((6, 16), device="cuda")
    got = ep.route(z, 2)
    for bad in (z.cpu(), z.double(), z.t(), z[:, ::2], z[0]):
        with pytest.raises(ValueError):
            ep.route(bad, 2)
    for k in (0, 17):
        with pytest.raises((ep.EPError, RuntimeError)):
            ep.route(z, k)
    with pytest.raises(ValueError):
        ep.route(z, 2, mask=torch.ones(5, dtype=torch.bool, device="cuda"))
    with pytest.raises(ValueError):
        ep.route(z, 3, out=got)
    for bad in (torch.zeros((6, 3), device="cuda"), torch.zeros((6, 2), device="cuda", dtype=torch.float64), torch.zeros((6, 2))):
        with pytest.raises(ValueError):
            ep.route_grad(z, got, bad)
    with pytest.raises(ValueError):
        ep.route_grad(z, got, None, torch.zeros((), device="cuda"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_of_normalized_gates_looks_at_the_chosen_alone(dtype):
    """Without the loss's gradient a NaN that was not chosen is no part of the gates: the row's gradient
    is the one without it.  A NaN or +inf among the chosen is their gradient's, and no other expert's."""
    say(f"route_grad: NaN beside the chosen {dtype}")
    for E, k in ((40, 4), (7, 3), (130, 3), (700, 5), (300, 70)):
        T = 12
        g = ref.gen(E)
        z = ref.normal((T, E), g, 1.0, dtype)
        low = z.float().argmin(1)                   # never among the k largest
        z[3, low[3]] = float("nan")
        z[8, low[8]] = float("nan")
        z[10, 2] = math.inf
        d = torch.randn((T, k), device="cuda", generator=g)
        got = ep.route(z, k)
        assert low[3] not in got.topk_idx[3] and torch.isfinite(got.topk_w[[3, 8]]).all()
        dz = ep.route_grad(z, got, d)
        rest = [t for t in range(T) if t != 10]
        want, size = ref.route_grad(z[rest], got.topk_idx[rest].cpu().long(), k, None, True, 0.0, d[rest], None, None)
        step = ref.BF16 if dtype == torch.bfloat16 else 2.0 ** -20
        ref.within(dz[rest].cpu(), want, want.abs() * step + size * 2.0 ** -14 + 1e-36, "d_logits")
        chosen = torch.zeros(E, dtype=torch.bool, device="cuda")
        chosen[got.topk_idx[10].long()] = True
        assert dz[10][chosen].isnan().all() and not dz[10][~chosen].any()
        whole = ep.route_grad(z, got, d, torch.ones(1, device="cuda"))     # the loss's goes through every p
        assert whole[[3, 8, 10]].isnan().all()


def test_counts_of_a_large_group():
    """A group's counts may add up to more than 32 bits hold."""
    say("route_grad with a large group's counts")
    k, balance, d_loss = 2, 0.5, 3e9
    for E, counts in ((4, [2 ** 31 - 8, 2 ** 31 - 100, 2 ** 30, 2 ** 31 - 2]), (600, [2 ** 24 + 3 * e for e in range(600)])):
        z = ref.normal((20, E), ref.gen(E), 1.0, torch.float32)
        total = torch.tensor(counts, dtype=torch.int32, device="cuda")
        got = ep.route(z, k, balance=balance)
        dz = ep.route_grad(z, got, None, torch.tensor([d_loss], device="cuda"), counts=total)
        n = sum(counts) // k
        g = torch.tensor([d_loss * balance * E * c / (n * k * n) for c in counts], dtype=torch.float64)
        p = torch.softmax(z.double().cpu(), 1)
        want, size = p * (g - (p @ g)[:, None]), p * (g + (p @ g)[:, None])
        ref.within(dz.cpu(), want, want.abs() * 2.0 ** -20 + size * 2.0 ** -14 + 1e-36, "d_logits")
