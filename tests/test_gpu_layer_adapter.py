"""The adapters' product against plain implementations in 64 bits (bounds: adapter_ref.py)."""
import pytest
import torch

import adapter_ref as ar
import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "silu", "gelu", "swiglu"]


@pytest.mark.parametrize("A", [1, 15, 16, 63, 64, 255, 256, 1000, 2047])
@pytest.mark.parametrize("rows", [0, 1, 63, 64, 65, 1000, 1025, 20000])
def test_rows_by_adapter(rows, A):
    say(f"adapter_rows rows={rows} A={A}")
    ids = torch.randint(-2, A + 2, (rows,), device="cuda", generator=ref.gen(rows + A)).int()
    if rows > 2:
        ids[0], ids[1] = -2 ** 31, 2 ** 31 - 1
    got = ep.adapter_rows(ids, A)
    _, order, offsets = ar.sorted_ids(ids, A)
    assert torch.equal(got.order.long(), order) and torch.equal(got.offsets.long(), offsets)
    again = ep.AdapterRows(torch.full_like(got.order, -7), torch.full_like(got.offsets, -7))
    assert ep.adapter_rows(ids, A, out=again) is again
    assert torch.equal(again.order, got.order) and torch.equal(again.offsets, got.offsets)


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 64, 129, 300, 1000])
@pytest.mark.parametrize("A", [1, 3, 40])
def test_row_counts(rows, A):
    for K, N, R, act in ((208, 136, 8, "silu"), (128, 264, 24, "swiglu"), (1040, 520, 64, "none")):
        say(f"adapter_product rows={rows} A={A} K={K} N={N} R={R} {act}")
        ar.check(ar.make(ar.random_ids(rows, A, rows + A), A, R, K, N, K + N, act))


@pytest.mark.parametrize("counts,none", [([1], 0), ([0, 5, 0], 0), ([0, 0], 7), ([17, 0, 1, 64], 3), ([128, 127, 300], 0),
                                         ([256, 257, 255], 100), ([1024, 0, 3], 1)], ids=str)
def test_rows_in_the_adapters_order(counts, none):
    say(f"adapter_product packed {counts} and {none}")
    for R, act in ((16, "none"), (40, "swiglu")):
        ar.check(ar.make(ar.packed_ids(counts, none), len(counts), R, 264, 136, 3, act), packed=True)


@pytest.mark.parametrize("R", [8, 16, 24, 32, 40, 64, 72, 120, 128, 136, 200, 256])
@pytest.mark.parametrize("rows", [5, 70, 600])
def test_ranks(rows, R):
    say(f"adapter_product rows={rows} R={R}")
    for base in (True, False):
        ar.check(ar.make(ar.random_ids(rows, 6, R), 6, R, 200, 72, R, base=base))


@pytest.mark.parametrize("K", [8, 16, 56, 64, 72, 136, 512, 1448, 4104])
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_inner_lengths(rows, K):
    say(f"adapter_product rows={rows} K={K}")
    for base in (True, False):
        ar.check(ar.make(ar.random_ids(rows, 4, K), 4, 16, K, 72, K, base=base))


@pytest.mark.parametrize("N", [8, 16, 24, 120, 136, 256, 264, 1032])
@pytest.mark.parametrize("rows", [2, 33, 260])
def test_output_lengths(rows, N):
    say(f"adapter_product rows={rows} N={N}")
    for act in ("none", "swiglu"):
        for base in (True, False):
            ar.check(ar.make(ar.random_ids(rows, 5, N), 5, 24, 200, N, N, act, base=base))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [3, 70, 500])
def test_epilogues(rows, act):
    say(f"adapter_product {act} rows={rows}")
    for bias in (False, True):
        for residual in (False, True):
            for base in (False, True):
                s = ar.make(ar.random_ids(rows, 5, rows), 5, 16, 144, 88, rows, act, base, bias, residual, scaled=bias)
                ar.check(s, keep=bias != residual)


@pytest.mark.parametrize("rows,A,R,K,N", [(1, 1, 16, 7168, 256), (64, 32, 16, 7168, 2048), (64, 64, 128, 2048, 4096),
                                          (256, 200, 32, 4096, 1024), (100, 7, 8, 8192, 64)])
def test_decode_sizes(rows, A, R, K, N):
    """Few rows, with adapters of their own: the contraction is split over workgroups."""
    say(f"adapter_product decode rows={rows} A={A} R={R} K={K} N={N}")
    for act in ("none", "swiglu"):
        s = ar.make(ar.random_ids(rows, A, rows, 0.1), A, R, K, N, rows, act)
        one = ar.check(s)
        two = ep.adapter_product(s["x"], s["a"], s["b"], ar.rows_of(s), w=s["w"], scale=s["scale"], act=act)
        assert torch.equal(one.out, two.out) and two.pre is None and two.low is None


@pytest.mark.parametrize("act", ["none", "swiglu"])
@pytest.mark.parametrize("rows,N", [(4100, 4096), (2600, 6000), (16500, 1032)])
def test_large_tiles(rows, N, act):
    say(f"adapter_product large rows={rows} N={N} {act}")
    ar.check(ar.make(ar.random_ids(rows, 9, rows), 9, 16, 264, N, rows, act, residual=True))
    ar.check(ar.make(sorted(ar.random_ids(rows, 300, rows, 0.0).tolist()), 300, 40, 136, N, rows, act), packed=True)


@pytest.mark.parametrize("A,rows", [(2047, 500), (2047, 5000), (700, 1400)])
def test_many_adapters(A, rows):
    say(f"adapter_product A={A} rows={rows}")
    ar.check(ar.make(ar.random_ids(rows, A, A), A, 8, 72, 136, A))


def test_no_rows_and_no_adapter():
    say("adapter_product without rows, and rows without adapters")
    s = ar.make([], 3, 16, 64, 32, 1)
    got = ep.adapter_product(s["x"], s["a"], s["b"], ar.rows_of(s), w=s["w"], keep_low=True)
    assert got.out.shape == (0, 32) and got.low.shape == (0, 16)
    ar.check(ar.make([-1] * 37, 3, 16, 64, 32, 2))
    ar.check(ar.make([-1] * 37, 3, 16, 64, 32, 2, base=False, residual=True))
    s = ar.make([0] * 37, 1, 16, 64, 32, 3)
    want = ar.check(s)
    got = ep.adapter_product(s["x"], s["a"], s["b"], w=s["w"], scale=s["scale"])  # one adapter has every row
    assert torch.equal(got.out, want.out)


def test_permuted_rows_give_permuted_results():
    """The order is a matter of where rows lie: bits do not depend on it."""
    say("adapter_product: permuted rows")
    s = ar.make(ar.packed_ids([100, 30, 0, 70], 20), 4, 24, 264, 136, 4, "silu", bias=True, residual=True)
    want = ar.check(s, packed=True)
    at = torch.randperm(220, device="cuda", generator=ref.gen(1))
    order = torch.empty_like(at)
    order[at] = torch.arange(220, device="cuda")  # the old batch's row i is row order[i] now
    rows = ep.AdapterRows(order.int(), ar.rows_of(s).offsets)
    got = ep.adapter_product(s["x"][at], s["a"], s["b"], rows, w=s["w"], scale=s["scale"], bias=s["bias"], act="silu",
                             residual=s["res"][at], keep_pre=True, keep_low=True)
    assert torch.equal(got.out, want.out[at]) and torch.equal(got.pre, want.pre[at]) and torch.equal(got.low, want.low)


def test_into_the_residual():
    say("adapter_product into its residual")
    for rows, N in ((40, 520), (700, 1032)):
        s = ar.make(ar.random_ids(rows, 4, rows), 4, 16, 264, N, rows, base=False, residual=True)
        want = ar.check(s).out
        y = s["res"].clone()
        got = ep.adapter_product(s["x"], s["a"], s["b"], ar.rows_of(s), scale=s["scale"], residual=y, out=y)
        assert got.out is y and torch.equal(y, want)


@pytest.mark.parametrize("rows,K,N", [(90, 4096, 264), (600, 136, 264)])
def test_broken_adapters_and_rows_stay_their_own(rows, K, N):
    """Infinities and NaN of one adapter's weights or of one row reach that adapter's rows or that row."""
    say(f"adapter_product: infinities and NaN, rows={rows}")
    for act in ("none", "swiglu"):
        s = ar.make(ar.random_ids(rows, 5, rows), 5, 16, K, N, rows, act, bias=True)
        clean = ep.adapter_product(s["x"], s["a"], s["b"], ar.rows_of(s), w=s["w"], scale=s["scale"], bias=s["bias"], act=act,
                                   keep_pre=True, keep_low=True)
        s["a"][1, 3, 5], s["a"][2, 0, 0] = float("nan"), float("inf")
        s["b"][3, 7, 2], s["b"][0, N - 1, 15] = float("nan"), -float("inf")
        s["x"][7, 1] = float("nan")
        got = ep.adapter_product(s["x"], s["a"], s["b"], ar.rows_of(s), w=s["w"], scale=s["scale"], bias=s["bias"], act=act,
                                 keep_pre=True, keep_low=True)
        whole = (s["ids"] == 4) | (s["ids"] < 0)
        whole[7] = False
        ref.within(got.out[whole], clean.out[whole].double(), clean.out[whole].double().abs() * 2 * ref.BF16 + 1e-2, "rows")
        assert torch.isfinite(got.out[whole]).all()
        assert torch.isnan(got.pre[7]).all()
        for e, col in ((3, 7), (0, N - 1)):  # one broken weight of b: one column of the adapter's rows
            mine = s["ids"] == e
            mine[7] = False
            bad = ~torch.isfinite(got.pre[mine])
            assert bad[:, col].all() and not bad[:, :col].any() and not bad[:, col + 1:].any()
        assert torch.isnan(got.pre[s["ids"] == 1]).all()
        mine = s["ids"] == 2  # an infinite low[., 0]: infinities with the signs of the terms
        mine[7] = False
        want = torch.sign(s["x"][mine, :1].float() * s["b"][2, :, 0].float()) * float("inf")
        some = want.isinf()
        assert torch.equal(got.pre[mine].float()[some], want[some]) and some.float().mean() > 0.9


def test_zero_weight_rows_of_infinite_places():
    """An infinite row beside others: only itself."""
    say("adapter_product: an infinite row")
    s = ar.make(ar.random_ids(200, 3, 1), 3, 8, 72, 40, 1)
    want = ar.check(s).out
    s["x"][11] = float("inf")
    got = ep.adapter_product(s["x"], s["a"], s["b"], ar.rows_of(s), w=s["w"], scale=s["scale"]).out
    keep = torch.arange(200, device="cuda") != 11
    assert torch.equal(got[keep], want[keep]) and not torch.isfinite(got[11]).any()


def test_side_stream_and_graph():
    say("adapter_rows and adapter_product on a side stream and in a graph")
    rows, A = 64, 9
    s = ar.make(ar.random_ids(rows, A, 0), A, 16, 2048, 264, 5, bias=True)
    out = torch.empty((rows, 264), dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()

    def step(stream=None):
        at = ep.adapter_rows(s["ids"], A, stream=stream)
        return ep.adapter_product(s["x"], s["a"], s["b"], at, w=s["w"], scale=s["scale"], bias=s["bias"], out=out,
                                  stream=stream)

    want = step().out.clone()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(4):
        s["ids"].copy_(ar.random_ids(rows, A, seed + 10))
        s["x"].copy_(ref.normal((rows, 2048), ref.gen(seed)))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step().out), seed


@pytest.mark.parametrize("offsets", [[0, 400, 100, 300], [-5, 2 ** 30, 7, 1], [300, 200, 100, 0], [50, 50, 10 ** 9, 10 ** 9]])
def test_offsets_and_orders_that_are_none_stay_in_bounds(offsets):
    """Offsets that decrease or leave the rows, and orders with entries outside: some results, nothing beside them."""
    say(f"adapter_product offsets={offsets}")
    rows = 300
    s = ar.make([0] * rows, 3, 16, 136, 72, 1)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    order = torch.randint(-rows, 2 * rows, (rows,), device="cuda", generator=ref.gen(2)).int()
    order[:3] = torch.tensor([2 ** 31 - 1, -2 ** 31, rows], dtype=torch.int32)
    for o in (None, order):
        for base in (True, False):
            whole = torch.full((3, rows, 72), 7.0, dtype=torch.bfloat16, device="cuda")
            low = torch.full((3, rows, 16), 7.0, dtype=torch.bfloat16, device="cuda")
            ep.adapter_product(s["x"], s["a"], s["b"], ep.AdapterRows(o, off), w=s["w"] if base else None, out=whole[1],
                               keep_low=low[1])
            grad = ep.adapter_product_grad(s["x"], s["a"], s["b"], low[1], whole[1], ep.AdapterRows(o, off),
                                           w=s["w"] if base else None)
            torch.cuda.synchronize()
            assert grad.dx.shape == (rows, 136)
            for t in (whole, low):
                assert (t[0] == 7.0).all() and (t[2] == 7.0).all()


def test_binding_refusals():
    say("adapters: refusals of the binding")
    s = ar.make(ar.random_ids(20, 3, 1), 3, 16, 64, 32, 1)
    rows, x, a, b, w = ar.rows_of(s), s["x"], s["a"], s["b"], s["w"]
    low, d = ref.normal((20, 16), ref.gen(1)), ref.normal((20, 32), ref.gen(2))
    for bad in (x.cpu(), x.float(), x.t(), x[0], x[:, :32]):
        with pytest.raises(ValueError):
            ep.adapter_product(bad, a, b, rows, w=w)
    for bad in (a.float(), a[:2], a[:, :8], a[0], a.transpose(1, 2)):
        with pytest.raises(ValueError):
            ep.adapter_product(x, bad, b, rows, w=w)
    for bad in (b.cpu(), b[0], b.float()):
        with pytest.raises(ValueError):
            ep.adapter_product(x, a, bad, rows, w=w)
    for bad in (dict(w=w[:16]), dict(w=w.float()), dict(scale=torch.ones(2, device="cuda")), dict(bias=w[0, :16].contiguous()),
                dict(residual=d[:3]), dict(act="tanh"), dict(out=d.float()), dict(keep_low=d), dict(keep_pre=low)):
        with pytest.raises(ValueError):
            ep.adapter_product(x, a, b, rows, **{"w": w, **bad})
    with pytest.raises(ValueError):
        ep.adapter_product(x, a, b, w=w)  # three adapters, no offsets
    for bad in (ep.AdapterRows(rows.order[:5], rows.offsets), ep.AdapterRows(rows.order.long(), rows.offsets),
                ep.AdapterRows(rows.order, rows.offsets[:2])):
        with pytest.raises(ValueError):
            ep.adapter_product(x, a, b, bad, w=w)
    with pytest.raises(ep.EPError):
        ep.adapter_product(x, a[:, :12].contiguous(), b[:, :, :12].contiguous(), rows, w=w)  # a rank of 12
    for bad in (dict(low=None), dict(low=low[:4]), dict(d_y=None), dict(d_y=low), dict(act="silu")):
        with pytest.raises(ValueError):
            ep.adapter_product_grad(x, a, b, **{"low": low, "d_y": d, "rows": rows, "w": w, **bad})
    with pytest.raises(ep.EPError):
        ep.adapter_product_grad(x, a, b, low, d, rows, dx=False, da=False, db=False)
    for bad in (s["ids"].long(), s["ids"].cpu(), s["ids"].view(4, 5)):
        with pytest.raises(ValueError):
            ep.adapter_rows(bad, 3)
    for A in (0, -1, 2048):
        with pytest.raises(ep.EPError):
            ep.adapter_rows(s["ids"], A)
    with pytest.raises(ValueError):
        ep.adapter_rows(s["ids"], 3, out=ep.AdapterRows(None, rows.offsets))


@pytest.mark.parametrize("R", [16, 40, 72])
@pytest.mark.parametrize("K", [8, 72, 200, 264, 328])
def test_short_contractions_of_single_rows(K, R):
    """Tiles of one row, whose contraction has fewer steps than a workgroup has groups of waves for them."""
    say(f"adapter_product tiles of one row K={K} R={R}")
    s = ar.make(ar.packed_ids([65] * 40, 1), 40, R, K, 136, K)
    ar.check(s, packed=True)
    ar.check_grad(ar.make(ar.packed_ids([65] * 40, 1), 40, R, 136, K, K), packed=True)
