"""The RMS norm and its gradient against plain implementations in 64 bits.

Bounds, derived from the kernel's arithmetic (fp32): s = x + r has one rounding; the sum of
squares adds at most 128 terms per lane and 22 partial sums, all positive, so it is within
2^-16 of itself; with the root, the division and the products y is within 2^-15 of itself
before its rounding to bf16 (half a step, at most 2^-8 of the value) or e4m3 (half a step, at
most 2^-4 of the value, or 2^-10 scales below e4m3's smallest normal number).  The gradient's
terms carry the same 2^-14; the weight's gradient adds T terms one after the other at most.
"""
import pytest
import torch

import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say

pytestmark = pytest.mark.gpu

# one row length or more for every row geometry, at its ends, and lengths that fill no lane evenly
LENGTHS = [8, 16, 72, 512, 520, 1024, 1032, 2048, 2056, 2888, 4096, 4104, 7168, 8192, 8200, 16384, 16400, 32768, 40008, 65536]


def check(x, r, w, eps, want8=True):
    T, H = x.shape
    want8 = want8 and H % 16 == 0
    got = ep.rmsnorm(x, w, residual=r, eps=eps, total=True, out=True, rows8=want8)
    s, y = ref.norm(x, r, w, eps)
    ref.within(got.total, s, s.abs() * ref.BF16, "total")
    ref.within(got.out, y, y.abs() * (ref.BF16 + 2.0 ** -15), "out")
    if want8:
        q, scale = ep.rows8_values(got.rows8)
        top = y.abs().amax(1, keepdim=True).clamp_min(2.0 ** -100) / 448
        ref.within(scale, top, top * 2.0 ** -14, "scale")
        ref.within(q.float().double() * scale.double(), y, torch.maximum(y.abs() * 2.0 ** -4, top * 2.0 ** -10) * (1 + 2.0 ** -8),
                   "rows8")
        assert not got.rows8[:, H + 4:].any()
    return got


@pytest.mark.parametrize("H", LENGTHS)
@pytest.mark.parametrize("T", [1, 3, 37])
def test_norm(T, H):
    say(f"rmsnorm T={T} H={H}")
    g = ref.gen(T * 100003 + H)
    check(ref.normal((T, H), g), ref.normal((T, H), g, 2.0), ref.normal(H, g), 1e-6)


@pytest.mark.parametrize("T", [256, 1023, 9001])
def test_many_rows(T):
    say(f"rmsnorm T={T}")
    g = ref.gen(T)
    check(ref.normal((T, 1040), g), None, ref.normal(1040, g), 1e-5)
    check(ref.normal((T, 2064), g, 30.0), ref.normal((T, 2064), g), None, 0.0)


def test_no_rows_and_each_output():
    g = ref.gen(1)
    x, w = ref.normal((5, 64), g), ref.normal(64, g)
    empty = ep.rmsnorm(x[:0], w, rows8=True)
    assert empty.out.shape == (0, 64) and empty.rows8.shape == (0, 80) and empty.total is None
    whole = ep.rmsnorm(x, w, residual=x, rows8=True)
    for out, rows8, total in ((True, False, False), (False, True, False), (False, False, True)):
        one = ep.rmsnorm(x, w, residual=x, out=out, rows8=rows8, total=total)
        for name in ("total", "out", "rows8"):
            got = getattr(one, name)
            assert (got is not None) == {"total": total, "out": out, "rows8": rows8}[name]
            assert got is None or torch.equal(got.view(torch.uint8), getattr(whole, name).view(torch.uint8))


def test_extremes_stay_in_their_rows():
    """Zeros, the smallest and largest magnitudes, infinities and NaN, each in a row of its own."""
    say("rmsnorm extremes")
    H = 2064
    g = ref.gen(7)
    x = ref.normal((8, H), g)
    x[0] = 0
    x[1] = 1e-38
    x[2] = 3e18
    x[3, 5] = float("inf")
    x[4, 2063] = float("nan")
    x[5] = 0
    x[5, 9] = -2.0 ** -130     # a subnormal
    clean = ep.rmsnorm(x[6:], None, rows8=True)
    got = check(x[[0, 1, 2, 5, 6, 7]].contiguous(), None, None, 1e-6)
    q, scale = ep.rows8_values(got.rows8)
    assert not got.out[0].any() and not q.view(torch.uint8)[0].any() and scale[0] > 0
    both = ep.rmsnorm(x, None, rows8=True)
    assert torch.equal(both.out[6:], clean.out) and torch.equal(both.rows8[6:], clean.rows8)
    assert both.out[3].isnan()[5] and both.out[4].isnan().all()
    scale = ep.rows8_values(both.rows8)[1]
    assert scale[3].isnan() and scale[4].isnan() and not scale[[0, 1, 2, 5, 6, 7]].isnan().any()


def test_rows_past_4_gib():
    """Rows whose byte offsets pass 32 bits, and the traffic that goes non-temporally."""
    say("rmsnorm past 4 GiB")
    H = 7168
    T = (1 << 32) // (2 * H) + 400
    g = ref.gen(21)
    x = torch.zeros((T, H), dtype=torch.bfloat16, device="cuda")
    w = ref.normal(H, g)
    x[:200], x[-200:] = ref.normal((200, H), g), ref.normal((200, H), g)
    ends = torch.cat([torch.arange(200), torch.arange(T - 200, T)]).cuda()
    got = ep.rmsnorm(x, w, residual=x, rows8=True)
    want = ep.rmsnorm(x[ends], w, residual=x[ends], rows8=True)
    for name in ("total", "out", "rows8"):
        assert torch.equal(getattr(got, name)[ends], getattr(want, name))
    assert not got.out[200:-200].any()
    dx, dw = ep.rmsnorm_grad(got.total, w, got.out, d_total=x)
    dx2, dw2 = ep.rmsnorm_grad(want.total, w, want.out, d_total=x[ends])
    assert torch.equal(dx[ends], dx2)
    size = ref.norm_grad(want.total, w, want.out, x[ends], 1e-6)[3]
    ref.within(dw, dw2.double(), size * (2.0 ** -13 + T * ref.U24), "dw")   # rows of zeros add nothing


def test_graph():
    """The norm, its gradient, the router's and the combine's in one captured graph, replayed with
    new inputs against eager calls."""
    say("layer operators in a graph")
    T, H, E, k = 300, 1040, 24, 3
    g = ref.gen(17)
    x, w, d = ref.normal((T, H), g), ref.normal(H, g), ref.normal((T, H), g)
    z, dg = torch.randn((T, E), device="cuda", generator=g), torch.randn((T, k), device="cuda", generator=g)
    y, pos = ref.normal((T * k, H), g), torch.randperm(T * k, device="cuda", generator=g).int()
    one = torch.ones(1, device="cuda")

    def step():
        n = ep.rmsnorm(x, w, residual=d, rows8=True)
        r = ep.route(z, k, balance=0.5)
        dy, dw = ep.combine_grad(d, y, pos, r.topk_w)
        return [n.total, n.out, n.rows8, *ep.rmsnorm_grad(n.total, w, d, d_total=x), r.topk_idx, r.topk_w, r.expert_counts,
                r.prob_sums, r.loss, ep.route_grad(z, r, dg, one), dy, dw]

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        x.mul_(-1.5), z.mul_(0.5).add_(0.1), y.neg_()
        want = step()
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.uint8) if a.dtype == torch.uint8 else a, b) for a, b in zip(held, want)), i


def test_total_in_place_and_side_stream():
    say("rmsnorm in place, on a stream of its own")
    g = ref.gen(3)
    x, r, w = ref.normal((777, 2048), g), ref.normal((777, 2048), g), ref.normal(2048, g)
    want = ep.rmsnorm(x, w, residual=r)
    for into in (0, 1):
        a, b = x.clone(), r.clone()
        got = ep.rmsnorm(a, w, residual=b, total=(a, b)[into])
        assert torch.equal(got.total, want.total) and torch.equal(got.out, want.out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):  # fresh outputs of the side stream, freed and allocated again while it works
        got = ep.rmsnorm(x, w, residual=r, stream=side)
        torch.empty_like(x).fill_(7.0)
    side.synchronize()
    assert torch.equal(got.out, want.out)


@pytest.mark.parametrize("H", LENGTHS)
@pytest.mark.parametrize("T", [1, 38])
def test_gradient(T, H):
    say(f"rmsnorm_grad T={T} H={H}")
    g = ref.gen(T * 7 + H)
    s, d, w = ref.normal((T, H), g, 3.0), ref.normal((T, H), g), ref.normal(H, g)
    for dt, wt in ((ref.normal((T, H), g), w), (None, None)):
        dx, dw = ep.rmsnorm_grad(s, wt, d, d_total=dt, eps=1e-6)
        want, size, want_w, size_w = ref.norm_grad(s, wt, d, dt, 1e-6)
        ref.within(dx, want, want.abs() * ref.BF16 + size * 2.0 ** -14, "dx")
        ref.within(dw, want_w, size_w * (2.0 ** -14 + T * ref.U24), "dw")


def test_gradient_over_many_rows_repeats():
    say("rmsnorm_grad over many rows")
    T, H = 5003, 1032
    g = ref.gen(11)
    s, d, w = ref.normal((T, H), g), ref.normal((T, H), g), ref.normal(H, g)
    dx, dw = ep.rmsnorm_grad(s, w, d, d_total=d)
    want, size, want_w, size_w = ref.norm_grad(s, w, d, d, 1e-6)
    ref.within(dx, want, want.abs() * ref.BF16 + size * 2.0 ** -14, "dx")
    ref.within(dw, want_w, size_w * (2.0 ** -14 + T * ref.U24), "dw")
    for _ in range(3):
        again = ep.rmsnorm_grad(s, w, d, d_total=d)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    only = ep.rmsnorm_grad(s, w, d, d_total=d.clone(), d_weight=False)
    assert only[1] is None and torch.equal(only[0], dx)
    a = d.clone()
    assert torch.equal(ep.rmsnorm_grad(s, w, a, d_total=a, dx=a, d_weight=False)[0], dx)
    dx0, dw0 = ep.rmsnorm_grad(s[:0], w, d[:0])
    assert dx0.shape == (0, H) and not dw0.any()


def test_gradient_against_differences():
    """<dx, v> and <dw, u> against central differences of sum(d * y) in 64 bits along v and u:
    the difference's own error is of third order in a step of 1e-4."""
    say("rmsnorm_grad against differences")
    T, H, eps = 9, 264, 1e-3
    g = ref.gen(5)
    s, d, w = ref.normal((T, H), g), ref.normal((T, H), g), ref.normal(H, g)
    v, u = torch.randn((T, H), device="cuda", dtype=torch.float64), torch.randn(H, device="cuda", dtype=torch.float64)
    dx, dw = ep.rmsnorm_grad(s, w, d, eps=eps)

    def loss(a, b):
        return (d.double() * ref.norm(a, None, b, eps)[1]).sum()

    h = 1e-4
    along = (loss(s.double() + h * v, w) - loss(s.double() - h * v, w)) / (2 * h)
    size = ref.norm_grad(s, w, d, None, eps)
    assert abs((dx.double() * v).sum() - along) <= (v.abs() * (dx.double().abs() * 2 * ref.BF16 + size[1] * 2.0 ** -14)).sum() + 1e-4
    along = (loss(s, w.double() + h * u) - loss(s, w.double() - h * u)) / (2 * h)
    assert abs((dw.double() * u).sum() - along) <= (u.abs() * size[3]).sum() * 2.0 ** -13 + 1e-4


def test_binding_refusals():
    """Wrong devices, types, layouts and shapes raise before anything is enqueued."""
    say("rmsnorm: refusals of the binding")
    g = ref.gen(1)
    x, w = ref.normal((6, 64), g), ref.normal(64, g)
    for bad in (x.cpu(), x.float(), x.t(), x[:, ::2], x[0], x[:, 8:]):
        with pytest.raises(ValueError):
            ep.rmsnorm(bad, None)
    for bad in (w[:32], w.float(), w.cpu()):
        with pytest.raises(ValueError):
            ep.rmsnorm(x, bad)
    with pytest.raises(ValueError):
        ep.rmsnorm(x, w, residual=x[:5])
    with pytest.raises(ValueError):
        ep.rmsnorm(x, w, out=x.float())
    with pytest.raises(ep.EPError):
        ep.rmsnorm(x, w, out=False)
    with pytest.raises(ep.EPError):
        ep.rmsnorm(ref.normal((6, 72), g), rows8=True)
    with pytest.raises(ValueError):
        ep.rmsnorm_grad(x, w, None)
    with pytest.raises(ValueError):
        ep.rmsnorm_grad(x, w, x[:3])
    with pytest.raises(ValueError):
        ep.rmsnorm_grad(x, w, x, d_weight=torch.zeros(64, device="cuda", dtype=torch.bfloat16))


# Row lengths of every number of waves per row.
WAVES = [80, 1040, 2064, 7168, 16400, 65536]


def rows_at(exponents, H, seed):
    """Rows of values of random sign in [1/2, 1) 2^e, one for each e."""
    g = ref.gen(seed)
    x = (torch.rand((len(exponents), H), device="cuda", generator=g, dtype=torch.float64) * 0.5 + 0.5)
    x = x * torch.where(torch.rand(x.shape, device="cuda", generator=g) < 0.5, -1.0, 1.0)
    return (x * 2.0 ** torch.tensor(exponents, device="cuda", dtype=torch.float64)[:, None]).clamp(-3.3e38, 3.3e38).bfloat16()


@pytest.mark.parametrize("H", WAVES)
def test_largest_values(H):
    """Rows whose squares, and sums of squares, leave fp32 at the top: y is of the size of the weight."""
    say(f"rmsnorm of the largest values H={H}")
    exponents = [59, 60, 61, 64, 100, 116, 120, 122, 123, 124, 125, 126, 127, 128]
    x = rows_at(exponents, H, H)
    x[-1] = 3.3895313892515355e38                   # bf16's largest
    for eps in (0.0, 1e-6):
        check(x, None, None, eps)
    check(x[:-2], x[:-2], None, 1e-6)               # sums of them, up to 2^127
    one = torch.full((1, H), 5e36, dtype=torch.bfloat16, device="cuda")
    assert (ep.rmsnorm(one, None).out == 1).all()


@pytest.mark.parametrize("H", WAVES)
def test_smallest_values(H):
    """The same at the bottom, without eps, down to the subnormals."""
    say(f"rmsnorm of the smallest values H={H}")
    x = rows_at([-39, -40, -41, -44, -64, -100, -120, -126, -128, -130, -132], H, H)
    check(x, None, None, 0.0)
    check(x[:8], x[:8], None, 0.0)


@pytest.mark.parametrize("H", WAVES)
def test_8bit_scale_of_large_and_small_products(H):
    """Values times weights that leave fp32 where y, their product over the row's size, does not."""
    say(f"rmsnorm, 8-bit rows of large and small products H={H}")
    for value, weight, eps in ((50, 100, 1e-6), (100, 30, 1e-6), (3, 126, 1e-6), (126, 60, 0.0), (-100, -40, 0.0), (-40, -95, 0.0),
                               (-120, -20, 0.0), (-60, 120, 0.0), (-10, -115, 0.0)):
        x = rows_at([value - 1, value, value + 1], H, H + value + 200)
        check(x, None, rows_at([weight], H, H)[0].contiguous(), eps)
    x = rows_at([3, 3], H, 1)
    x[0] = 0                                        # zeros beside ordinary rows, whatever the weight
    for weight in (120, -120):
        got = check(x, None, rows_at([weight], H, H)[0].contiguous(), 1e-6)
        assert not ep.rows8_values(got.rows8)[0][0].float().any()    # a zero times a negative weight is -0


@pytest.mark.parametrize("H", WAVES)
def test_gradient_of_large_and_small_values(H):
    """The gradient where the row's values, the rows' gradients or their products are near the ends
    of fp32.  bf16's subnormals are 2^-133 apart, so that a result that small is half of that off."""
    say(f"rmsnorm_grad of large and small values H={H}")
    for value, slope, weight, eps in ((64, 0, 0, 1e-6), (100, 0, 0, 1e-6), (122, 0, 0, 0.0), (127, 0, 0, 0.0), (60, 80, 10, 0.0),
                                      (100, 60, 40, 0.0), (20, 110, 5, 1e-6), (-64, 0, 0, 0.0), (-100, -20, -10, 0.0),
                                      (-126, -6, 0, 0.0), (-130, -12, 0, 0.0), (-20, -90, -20, 0.0), (-38, -60, -40, 0.0)):
        s = rows_at([value - 1, value, value - 2], H, H + value + 300)
        d, w = rows_at([slope, slope, slope - 3], H, H + slope + 700), rows_at([weight], H, H)[0].contiguous()
        for dt in (None, rows_at([0, 3, -20], H, H + 5)):
            dx, dw = ep.rmsnorm_grad(s, w, d, d_total=dt, eps=eps)
            want, size, want_w, size_w = ref.norm_grad(s, w, d, dt, eps)
            ref.within(dx, want, want.abs() * ref.BF16 + size * 2.0 ** -14 + 2.0 ** -133, "dx")
            ref.within(dw, want_w, size_w * (2.0 ** -14 + 3 * ref.U24) + 2.0 ** -147, "dw")


def test_gradient_of_zeros_nan_and_infinity_stays_in_their_rows():
    say("rmsnorm_grad: zeros, NaN and infinities")
    for H in (1032, 7168):
        g = ref.gen(H)
        s, d, w = ref.normal((9, H), g), ref.normal((9, H), g), ref.normal(H, g)
        d[1] = 0
        clean, _ = ep.rmsnorm_grad(s, w, d, d_total=d)
        s[3, 7], d[5, 9] = float("nan"), float("inf")
        d[6, 4] = float("nan")
        dx, _ = ep.rmsnorm_grad(s, w, d, d_total=d)
        keep = [0, 1, 2, 4, 7, 8]
        assert torch.equal(dx[keep], clean[keep]) and not dx[1].any()
        assert dx[3].isnan().all() and dx[6].isnan().all() and not torch.isfinite(dx[5]).any()
