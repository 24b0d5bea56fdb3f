"""The adapters' operators write what is theirs and nothing beside it, in a workspace of just the bytes they name,
on a stream of the caller's, and reach rows past 4 GiB."""
import ctypes

import pytest
import torch

import adapter_ref as ar
import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say
from paper_2609_40093_amd import _lib
from test_gpu_layer_bounds import Guarded, run

pytestmark = pytest.mark.gpu

# rows, adapters, ranks, K, N; packed: each size once by every path, few results and many
SIZES = [(1, 1, 8, 8, 8), (5, 3, 16, 72, 40), (70, 4, 40, 264, 520), (333, 7, 24, 1448, 136), (900, 2, 72, 136, 4104),
         (2600, 60, 8, 200, 1448), (4200, 3, 128, 72, 776)]


@pytest.mark.parametrize("streamed", [False, True])
@pytest.mark.parametrize("rows,A,R,K,N", SIZES)
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_outputs(rows, A, R, K, N, act, streamed):
    say(f"adapters beside their outputs rows={rows} A={A} R={R} K={K} N={N} {act}")
    s, at = ar.make(ar.random_ids(rows, A, rows), A, R, K, N, rows, act, bias=True, residual=True), Guarded()
    wide = s["b"].shape[1]
    order = run(streamed, lambda st: ep.adapter_rows(s["ids"].int(), A, stream=st, out=ep.AdapterRows(
        at((rows,), torch.int32), at((A + 1,), torch.int32))))
    want_order = ar.rows_of(s)
    d = ref.normal((rows, N), ref.gen(1))
    for base in (True, False):
        w = s["w"] if base else None
        more = {"w": w, "scale": s["scale"], "bias": s["bias"], "act": act, "residual": s["res"]}
        got = run(streamed, lambda st: ep.adapter_product(s["x"], s["a"], s["b"], order, keep_pre=at((rows, wide)),
                                                          keep_low=at((rows, R)), out=at((rows, N)), stream=st, **more))
        pre = None if act == "none" else got.pre
        grad = run(streamed, lambda st: ep.adapter_product_grad(
            s["x"], s["a"], s["b"], got.low, d, order, w=w, scale=s["scale"], pre=pre, act=act, dx=at((rows, K)),
            da=at((A, R, K)), db=at((A, wide, R)), stream=st))
        at.check()
        assert torch.equal(order.order, want_order.order) and torch.equal(order.offsets, want_order.offsets)
        want = ep.adapter_product(s["x"], s["a"], s["b"], want_order, keep_pre=True, keep_low=True, **more)
        for name in ("out", "pre", "low"):
            assert torch.equal(getattr(got, name), getattr(want, name)), name
        want = ep.adapter_product_grad(s["x"], s["a"], s["b"], want.low, d, want_order, w=w, scale=s["scale"], pre=pre, act=act)
        for name in ("dx", "da", "db"):
            assert torch.equal(getattr(grad, name), getattr(want, name)), name


@pytest.mark.parametrize("rows,A,R,K,N", SIZES)
@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
def test_workspaces(rows, A, R, K, N, act):
    """Every choice of results, in a workspace of just the bytes that the query names for it."""
    say(f"adapters in their own workspace rows={rows} A={A} R={R} K={K} N={N} {act}")
    lib, code = _lib.load(), _lib.EP_ACTIVATIONS[act]
    s = ar.make(ar.random_ids(rows, A, rows), A, R, K, N, rows, act)
    wide, by = s["b"].shape[1], ar.rows_of(s)
    d, low = ref.normal((rows, N), ref.gen(1)), ref.normal((rows, R), ref.gen(2))
    pre = None if act == "none" else ref.normal((rows, wide), ref.gen(3))
    stream = torch.cuda.current_stream().cuda_stream
    n = ctypes.c_size_t()

    def ptr(*tensors):
        return [t.data_ptr() if t is not None else None for t in tensors]

    for w in (s["w"], None):
        at = Guarded()
        assert lib.ep_adapter_product_workspace_bytes(rows, A, R, K, N, w is not None, code, ctypes.byref(n)) == _lib.EP_OK
        y, work = at((rows, N)), at((n.value,), torch.uint8)
        p = ptr(s["x"], by.order, by.offsets, s["a"], s["b"], s["scale"], w, y, work)
        assert lib.ep_adapter_product(p[0], rows, p[1], p[2], A, R, p[3], p[4], p[5], p[6], K, N, None, code, None, None, None,
                                      p[7], p[8], n.value, stream) == _lib.EP_OK
        at.check()
        assert torch.equal(y, ep.adapter_product(s["x"], s["a"], s["b"], by, w=w, scale=s["scale"], act=act).out)
        want = ep.adapter_product_grad(s["x"], s["a"], s["b"], low, d, by, w=w, scale=s["scale"], pre=pre, act=act)
        for dx, da, db in ((1, 1, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)):
            at = Guarded()
            flags = dx * _lib.EP_ADAPTER_DX + da * _lib.EP_ADAPTER_DA + db * _lib.EP_ADAPTER_DB
            assert lib.ep_adapter_product_grad_workspace_bytes(rows, A, R, K, N, w is not None, code, 1, flags,
                                                               ctypes.byref(n)) == _lib.EP_OK
            outs = [at((rows, K)) if dx else None, at((A, R, K)) if da else None, at((A, wide, R)) if db else None]
            work = at((n.value,), torch.uint8)
            p = ptr(s["x"], by.order, by.offsets, s["a"], s["b"], s["scale"], w, low, pre, d, *outs, work)
            assert lib.ep_adapter_product_grad(p[0], rows, p[1], p[2], A, R, p[3], p[4], p[5], p[6], K, N, p[7], code, p[8], p[9],
                                               p[10], p[11], p[12], p[13], n.value, stream) == _lib.EP_OK
            at.check()
            for got, name in zip(outs, ("dx", "da", "db")):
                assert got is None or torch.equal(got, getattr(want, name)), (dx, da, db, name)


@pytest.mark.parametrize("rows,A,R,K", [(9000, 3, 16, 72), (17000, 5, 32, 136), (9000, 2, 72, 72), (17000, 3, 40, 136),
                                        (33000, 4, 64, 72), (40000, 1, 200, 72), (2100, 80, 40, 72)])
def test_heights_of_the_low_rank_tiles(rows, A, R, K):
    """Rows enough for every height that the low-rank values' tiles have, most of them one adapter's."""
    say(f"adapters' low-rank values rows={rows} A={A} R={R} K={K}")
    ids = ar.random_ids(rows, A, rows)
    ids[rows // 3:] = torch.where(ids[rows // 3:] < 0, -1, A - 1)
    ar.check(ar.make(ids, A, R, K, 520, rows), keep=False)
    ar.check_grad(ar.make(ids, A, R, 136, K, rows))


def test_rows_past_4_gib():
    """Rows in the adapters' order, of x and of y: the places of the last ones are past 32 bits."""
    say("adapters: rows past 4 GiB")
    rows, K, A, R = 600000, 4096, 3, 8  # 4.9 GB
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    s = ar.make([0], A, R, K, 16, 3, base=False)
    back = torch.randperm(rows, device="cuda", generator=ref.gen(4))[:500].sort()[0]
    back = torch.cat([back, torch.arange(rows - 300, rows, device="cuda")])
    x[back] = ref.normal((len(back), K), ref.gen(1))
    ends = [0, 100000, 550000, rows - 7]
    of = torch.bucketize(back, torch.tensor(ends[1:], device="cuda"), right=True)
    by = ep.AdapterRows(None, torch.tensor(ends, dtype=torch.int32, device="cuda"))
    got = ep.adapter_product(x, s["a"], s["b"], by, scale=s["scale"], keep_low=True)
    d = torch.zeros((rows, 16), dtype=torch.bfloat16, device="cuda")
    d[back] = ref.normal((len(back), 16), ref.gen(2))
    grad = ep.adapter_product_grad(x, s["a"], s["b"], got.low, d, by, scale=s["scale"])
    # the same rows alone: other tiles, the same values to their rounding
    some = torch.bincount(of, minlength=A + 1)[:A].cumsum(0)
    alone = ep.AdapterRows(None, torch.cat([some.new_zeros(1), some]).int())
    want = ep.adapter_product(x[back], s["a"], s["b"], alone, scale=s["scale"], keep_low=True)
    small = ep.adapter_product_grad(x[back], s["a"], s["b"], want.low, d[back], alone, scale=s["scale"])
    for a, b, what in ((got.out[back], want.out, "y"), (got.low[back], want.low, "low"), (grad.dx[back], small.dx, "dx"),
                       (grad.da, small.da, "da"), (grad.db, small.db, "db")):
        # each side: half a step of its result and, of its low-rank values, of what they are made of; sums of 4096 terms
        ref.within(a, b.double(), 4 * ref.BF16 * b.double().abs() + 2.0 ** -8 * float(b.double().abs().mean()), what)
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[back] = False
    assert not got.out[rest].any() and not got.low[rest].any() and not grad.dx[rest].any()


def test_an_order_over_more_than_2_gib():
    """Without W a forward's rows are gathered from anywhere; a gradient copies rows that it cannot gather."""
    say("adapters: an order over more than 2 GiB")
    rows, K, A, R = 300000, 4096, 3, 8  # 2.5 GB
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    ids = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    back = torch.cat([torch.arange(0, rows, 997, device="cuda"), torch.arange(rows - 200, rows, device="cuda")]).unique()
    x[back] = ref.normal((len(back), K), ref.gen(1))
    ids[back] = (torch.arange(len(back), device="cuda") % A).int()
    s = ar.make(ids[back], A, R, K, 16, 3, base=False)
    s["x"] = x[back]
    by = ep.adapter_rows(ids, A)
    got = ep.adapter_product(x, s["a"], s["b"], by, scale=s["scale"], keep_low=True)
    d = torch.zeros((rows, 16), dtype=torch.bfloat16, device="cuda")
    d[back] = ref.normal((len(back), 16), ref.gen(2))
    grad = ep.adapter_product_grad(x, s["a"], s["b"], got.low, d, by, scale=s["scale"])
    alone = ar.rows_of(s)
    want = ep.adapter_product(s["x"], s["a"], s["b"], alone, scale=s["scale"], keep_low=True)
    small = ep.adapter_product_grad(s["x"], s["a"], s["b"], want.low, d[back], alone, scale=s["scale"])
    for a, b, what in ((got.out[back], want.out, "y"), (got.low[:len(back)], want.low, "low"), (grad.dx[back], small.dx, "dx"),
                       (grad.da, small.da, "da"), (grad.db, small.db, "db")):
        ref.within(a, b.double(), 4 * ref.BF16 * b.double().abs() + 2.0 ** -8 * float(b.double().abs().mean()), what)
    with pytest.raises(ep.EPError):
        ep.adapter_product(x, s["a"], s["b"], by, w=torch.zeros((16, K), dtype=torch.bfloat16, device="cuda"))


# few results; one pass over the contraction; the contraction in parts
@pytest.mark.parametrize("rows,K,N", [(300, 264, 136), (5000, 136, 1032), (2600, 6000, 1032), (4500, 5632, 1024)])
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_broken_rows_and_adapters_of_every_path(rows, K, N, act):
    """NaN rows (a padded batch's) and adapters with infinities: the other rows keep their values."""
    say(f"adapters: NaN rows and broken adapters rows={rows} K={K} N={N} {act}")
    A, R = 6, 16
    s = ar.make(ar.random_ids(rows, A, rows), A, R, K, N, rows, act)
    by, wide = ar.rows_of(s), s["b"].shape[1]
    d, low = ref.normal((rows, N), ref.gen(1)), ref.normal((rows, R), ref.gen(2))
    pre = None if act == "none" else ref.normal((rows, wide), ref.gen(3))
    more = {"w": s["w"], "scale": s["scale"], "act": act}
    clean = ep.adapter_product(s["x"], s["a"], s["b"], by, **more).out
    dx = ep.adapter_product_grad(s["x"], s["a"], s["b"], low, d, by, pre=pre, **more).dx
    none = s["ids"] < 0
    s["x"][none], d[none] = float("nan"), float("nan")
    whole = ~none
    got = ep.adapter_product(s["x"], s["a"], s["b"], by, **more).out
    grad = ep.adapter_product_grad(s["x"], s["a"], s["b"], low, d, by, pre=pre, **more)
    assert torch.equal(got[whole], clean[whole]) and torch.equal(grad.dx[whole], dx[whole])
    assert torch.isnan(got[none]).all() and torch.isnan(grad.dx[none]).all()
    assert torch.isfinite(grad.da).all() and torch.isfinite(grad.db).all()
    a, b = s["a"].clone(), s["b"].clone()
    a[2, 1], b[4, :, 3] = float("inf"), float("nan")
    got = ep.adapter_product(s["x"], a, b, by, **more).out
    grad = ep.adapter_product_grad(s["x"], a, b, low, d, by, pre=pre, **more)
    assert torch.isnan(got[none | (s["ids"] == 4)]).all() and torch.isnan(grad.dx[none | (s["ids"] == 4)]).all()
    for bad, what, want in ((got, "y", clean), (grad.dx, "dx", dx)):
        whole = ~none & (s["ids"] != 2) & (s["ids"] != 4)
        # summed again in another order: the result's rounding, and sums of up to 6000 terms of about 1 / sqrt(6000)
        ref.within(bad[whole], want[whole].double(), want[whole].double().abs() * 2 * ref.BF16 + 1e-2, what)
