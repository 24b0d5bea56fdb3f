"""The adapters' gradient against plain implementations in 64 bits (bounds: adapter_ref.py) and
against differences."""
import pytest
import torch

import adapter_ref as ar
import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "silu", "gelu", "swiglu"]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [1, 17, 64, 130, 600])
def test_gradient(rows, act):
    for A, R, K, N in ((1, 8, 72, 40), (3, 16, 264, 136), (20, 40, 136, 264)):
        say(f"adapter_product_grad rows={rows} A={A} R={R} K={K} N={N} {act}")
        for base in (True, False):
            ar.check_grad(ar.make(ar.random_ids(rows, A, rows), A, R, K, N, K, act, base))


@pytest.mark.parametrize("counts,none", [([1], 0), ([0, 5, 0], 0), ([0, 0], 7), ([63, 64, 65, 0], 3), ([300, 257], 90)], ids=str)
def test_rows_in_the_adapters_order(counts, none):
    say(f"adapter_product_grad packed {counts} and {none}")
    for act in ("none", "gelu"):
        ar.check_grad(ar.make(ar.packed_ids(counts, none), len(counts), 24, 264, 136, 3, act), packed=True)


@pytest.mark.parametrize("R", [8, 24, 32, 64, 72, 128, 136, 256])
@pytest.mark.parametrize("rows", [5, 300])
def test_ranks(rows, R):
    say(f"adapter_product_grad rows={rows} R={R}")
    ar.check_grad(ar.make(ar.random_ids(rows, 4, R), 4, R, 136, 200, R))


@pytest.mark.parametrize("K,N", [(8, 8), (8, 520), (520, 8), (64, 64), (72, 1448), (1448, 72), (264, 4104), (4104, 264)])
def test_lengths(K, N):
    say(f"adapter_product_grad K={K} N={N}")
    for act in ("none", "swiglu"):
        ar.check_grad(ar.make(ar.random_ids(150, 3, K), 3, 16, K, N, K + N, act))


@pytest.mark.parametrize("A,rows", [(1, 9000), (1, 40000), (300, 3000), (2047, 900)])
def test_many_rows_and_adapters(A, rows):
    say(f"adapter_product_grad A={A} rows={rows}")
    s = ar.make(sorted(ar.random_ids(rows, A, rows, 0.0).tolist()), A, 16, 136, 264, rows, scaled=A > 1)
    one, two = ar.check_grad(s, packed=True), ar.check_grad(s, packed=True)
    for name in ("dx", "da", "db"):
        assert torch.equal(getattr(one, name), getattr(two, name)), name


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_parts(act, packed):
    """Each result alone, in the workspace of just its bytes."""
    say(f"adapter_product_grad parts {act}")
    s = ar.make(ar.packed_ids([40, 0, 60], 5), 3, 16, 264, 136, 7, act)
    whole = ar.check_grad(s, packed=packed)
    for want in ("dx", "da", "db"):
        got = ar.check_grad(s, packed=packed, **{n: n == want for n in ("dx", "da", "db")})
        for n in ("dx", "da", "db"):
            assert (getattr(got, n) is None) == (n != want)
        assert torch.equal(getattr(got, want), getattr(whole, want)), want


def test_no_rows():
    say("adapter_product_grad without rows")
    s = ar.make([], 3, 16, 64, 32, 1)
    got = ep.adapter_product_grad(s["x"], s["a"], s["b"], torch.empty((0, 16), dtype=torch.bfloat16, device="cuda"),
                                  torch.empty((0, 32), dtype=torch.bfloat16, device="cuda"), ar.rows_of(s), w=s["w"])
    assert got.dx.shape == (0, 64) and not got.da.any() and not got.db.any()


@pytest.mark.parametrize("act", ["none", "silu", "swiglu"])
def test_against_differences(act):
    """Central differences of <y, d_y> in 64 bits along random directions of x, a and b."""
    say(f"adapter_product_grad differences {act}")
    rows, A, R, K, N = 50, 3, 16, 72, 40
    s = ar.make(ar.random_ids(rows, A, 3), A, R, K, N, 2, act)
    of, order, _ = ar.sorted_ids(s["ids"], A)
    g = ref.gen(9)
    d_y = ref.normal((rows, N), g)
    got = ep.adapter_product(s["x"], s["a"], s["b"], ar.rows_of(s), w=s["w"], scale=s["scale"], act=act, keep_pre=True,
                             keep_low=True)
    grad = ep.adapter_product_grad(s["x"], s["a"], s["b"], got.low, d_y, ar.rows_of(s), w=s["w"], scale=s["scale"],
                                   pre=got.pre if act != "none" else None, act=act)

    def loss(x, a, b):
        low = ar.by_adapter(x[order], of, a.transpose(1, 2))[0] * ar.scales(s, of)
        z = x @ s["w"].double().t()
        z = z.index_add(0, order, ar.by_adapter(low, of, b.transpose(1, 2))[0])
        return float((ref.act(z, act) * d_y.double()).sum())

    at = [s[n].double() for n in ("x", "a", "b")]
    for i, have in enumerate((grad.dx, grad.da, grad.db)):
        for t in range(4):
            v = torch.randn(at[i].shape, dtype=torch.float64, device="cuda", generator=g)
            h = 1e-5
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * v, at[i] - h * v
            along = (loss(*up) - loss(*down)) / (2 * h)
            terms = have.double() * v
            # every factor of a term is rounded to bf16 at most four times (pre and its slope, dz, v or low,
            # the result): 4 2^-8 of each term
            assert abs(terms.sum() - along) <= 0.016 * float(terms.abs().sum()), (i, t)


def test_broken_adapters_stay_their_own():
    say("adapter_product_grad: infinities and NaN")
    for rows, K, N in ((90, 264, 136), (700, 520, 264)):
        s = ar.make(ar.random_ids(rows, 4, rows), 4, 16, K, N, rows)
        clean = ar.check_grad(s)
        s["a"][1, 3, 5], s["b"][2, 0, 0] = float("nan"), float("inf")
        g = ref.gen(5)
        d_y, low = ref.normal((rows, N), g), ref.normal((rows, 16), g)
        got = ep.adapter_product_grad(s["x"], s["a"], s["b"], low, d_y, ar.rows_of(s), w=s["w"], scale=s["scale"])
        whole = (s["ids"] != 1) & (s["ids"] != 2)
        ref.within(got.dx[whole], clean.dx[whole].double(), clean.dx[whole].double().abs() * 2 * ref.BF16 + 1e-2, "dx")
        one = s["ids"] == 1
        bad = ~torch.isfinite(got.dx[one])
        assert bad[:, 5].all() and not bad[:, :5].any() and not bad[:, 6:].any()
        for e in (0, 1, 3):
            assert torch.equal(got.da[e], clean.da[e])
        assert torch.equal(got.db, clean.db) and not torch.isfinite(got.da[2]).all()


def test_side_stream_and_graph():
    say("adapter_product_grad on a side stream and in a graph")
    s = ar.make(ar.random_ids(200, 4, 0), 4, 16, 264, 136, 5, "silu")
    rows = ar.rows_of(s)
    g = ref.gen(1)
    d_y, low, pre = ref.normal((200, 136), g), ref.normal((200, 16), g), ref.normal((200, 136), g)

    def step(stream=None):
        return ep.adapter_product_grad(s["x"], s["a"], s["b"], low, d_y, rows, w=s["w"], scale=s["scale"], pre=pre, act="silu",
                                       stream=stream)

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    side.synchronize()
    assert all(torch.equal(getattr(got, n), getattr(want, n)) for n in ("dx", "da", "db"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for seed in range(4):
        d_y.copy_(ref.normal((200, 136), ref.gen(seed + 20)))
        s["x"].copy_(ref.normal((200, 264), ref.gen(seed + 30)))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        assert all(torch.equal(getattr(kept, n), getattr(want, n)) for n in ("dx", "da", "db")), seed
