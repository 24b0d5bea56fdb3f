"""The adapters' kernels by the path that a size takes, against 64 bits (bounds: adapter_ref.py): the kernels that ran are read
from the trace, so that a size that another rule sends elsewhere is found here.

Sizes past the few results' limit go through adapter_low and adapter_product, in one of seven tile shapes, in one pass over the
contraction or in parts that adapter_product_join adds up; dx likewise in five shapes, da and db in parts or not."""
import pytest
import torch

import adapter_ref as ar
import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "silu", "gelu", "swiglu"]
FEW = {"adapter_few", "adapter_few_low", "adapter_few_join"}


def kernels(call):
    """What call() gives, and the kernels that it ran."""
    ep.trace_reset()
    ep.trace_enable(True)
    try:
        got = call()
    finally:
        ep.trace_enable(False)
    torch.cuda.synchronize()
    ran = set(ep.trace_read())
    ep.trace_reset()
    return got, ran


def many(N, act="none", base=True):
    """An odd number of rows a little past the limit of few results."""
    return int(1.03 * (2300000 if base else 4000000) / ((2 * N if act == "swiglu" else N) + 256)) | 1


def check(s, parts=False, **more):
    got, ran = kernels(lambda: ar.check(s, **more))
    assert ran == {"adapter_low", "adapter_product"} | ({"adapter_product_join"} if parts else set()), ran
    return got


@pytest.mark.parametrize("base", [True, False])
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_the_limit(act, base):
    """The last row count of the one path and the first of the other."""
    N = 264
    wide = 2 * N if act == "swiglu" else N
    rows = (2300000 if base else 4000000) // (wide + 256)
    say(f"adapter_product round rows={rows} N={N} {act} base={base}")
    few = kernels(lambda: ar.check(ar.make(ar.random_ids(rows, 5, 1), 5, 16, 136, N, 1, act, base)))[1]
    assert few and few <= FEW, few
    check(ar.make(ar.random_ids(rows + 1, 5, 1), 5, 16, 136, N, 1, act, base))


@pytest.mark.parametrize("base", [True, False])
@pytest.mark.parametrize("R,K,N,rows", [(256, 1448, 72, 611), (64, 7168, 64, 1373), (128, 264, 1032, 1472)])
def test_the_limit_of_low_rank_values(R, K, N, rows, base):
    """The same where the low-rank values' bytes set it."""
    say(f"adapter_product round rows={rows} R={R} K={K} N={N} base={base}")
    few = kernels(lambda: ar.check(ar.make(ar.random_ids(rows, 5, 1), 5, R, K, N, 1, base=base)))[1]
    assert few and few <= FEW, few
    ran = kernels(lambda: ar.check(ar.make(ar.random_ids(rows + 1, 5, 1), 5, R, K, N, 1, base=base)))[1]
    assert {"adapter_low", "adapter_product"} <= ran and not ran & FEW, ran


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("base", [True, False])
def test_epilogues(act, base):
    N = 136
    rows = many(N, act, base)
    say(f"adapter_product {act} rows={rows} base={base}")
    for bias in (False, True):
        for residual in (False, True):
            s = ar.make(ar.random_ids(rows, 5, rows), 5, 16, 144, N, rows, act, base, bias, residual, scaled=bias)
            check(s, keep=bias != residual)


@pytest.mark.parametrize("R", [8, 16, 24, 32, 40, 64, 72, 120, 128, 136, 200, 256])
def test_ranks(R):
    for base in (True, False):
        rows = many(264, base=base)
        say(f"adapter_product rows={rows} R={R} base={base}")
        check(ar.make(ar.random_ids(rows, 6, R), 6, R, 200, 264, R, base=base))


@pytest.mark.parametrize("K", [8, 16, 56, 64, 72, 136, 328, 512, 1448, 4104])
def test_inner_lengths(K):
    for base in (True, False):
        rows = many(520, base=base)
        say(f"adapter_product rows={rows} K={K} base={base}")
        check(ar.make(ar.random_ids(rows, 4, K), 4, 16, K, 520, K, base=base), parts=base and K == 4104)


@pytest.mark.parametrize("N", [8, 16, 24, 120, 136, 256, 264, 1032])
def test_output_lengths(N):
    for act in ("none", "swiglu"):
        for base in (True, False):
            rows = many(N, act, base)
            say(f"adapter_product rows={rows} N={N} {act} base={base}")
            check(ar.make(ar.random_ids(rows, 5, N), 5, 24, 200, N, N, act, base=base))


@pytest.mark.parametrize("counts,none", [([5000], 0), ([0, 4997, 0], 7), ([0, 0], 5000), ([17, 0, 1, 4900, 64], 30),
                                         ([2000, 3, 2600, 1], 500)], ids=str)
def test_rows_in_the_adapters_order(counts, none):
    say(f"adapter_product packed {counts} and {none}")
    for R, act in ((16, "none"), (40, "swiglu")):
        check(ar.make(ar.packed_ids(counts, none), len(counts), R, 264, 264, 3, act), packed=True)


@pytest.mark.parametrize("A,R", [(2047, 8), (2047, 48), (700, 136)])
def test_many_adapters(A, R):
    rows = many(264)
    say(f"adapter_product A={A} R={R} rows={rows}")
    check(ar.make(ar.random_ids(rows, A, A), A, R, 72, 264, A))


def test_permuted_rows_and_the_residual_itself():
    """Bits depend neither on where rows lie nor on whether the results take the residual's place."""
    N = 264
    rows = many(N)
    say(f"adapter_product: permuted rows={rows}, into the residual")
    counts = [rows - 1200, 30, 0, 1000]
    s = ar.make(ar.packed_ids(counts, 170), 4, 24, 264, N, 4, "silu", bias=True, residual=True)
    want = check(s, packed=True)
    at = torch.randperm(rows, device="cuda", generator=ref.gen(1))
    order = torch.empty_like(at)
    order[at] = torch.arange(rows, device="cuda")  # the old batch's row i is row order[i] now
    by = ep.AdapterRows(order.int(), ar.rows_of(s).offsets)
    y = s["res"][at]
    got, ran = kernels(lambda: ep.adapter_product(s["x"][at], s["a"], s["b"], by, w=s["w"], scale=s["scale"], bias=s["bias"],
                                                  act="silu", residual=y, out=y, keep_pre=True, keep_low=True))
    assert ran == {"adapter_low", "adapter_product"}, ran
    assert got.out is y
    assert torch.equal(got.out, want.out[at]) and torch.equal(got.pre, want.pre[at]) and torch.equal(got.low, want.low)


@pytest.mark.parametrize("offsets", [[0, 4000, 100, 3000], [-5, 2 ** 30, 7, 1], [5001, 2000, 100, 0], [50, 50, 10 ** 9, 10 ** 9]])
def test_offsets_and_orders_that_are_none_stay_in_bounds(offsets):
    """Offsets that decrease or leave the rows, and orders with entries outside: some results, nothing beside them."""
    say(f"adapter_product offsets={offsets}")
    rows, K, N, R = 5001, 136, 616, 16  # past both limits
    s = ar.make([0] * rows, 3, R, K, N, 1)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    order = torch.randint(-rows, 2 * rows, (rows,), device="cuda", generator=ref.gen(2)).int()
    order[:3] = torch.tensor([2 ** 31 - 1, -2 ** 31, rows], dtype=torch.int32)
    for o in (None, order):
        for base in (True, False):
            y, low, dx = (torch.full((3, rows, n), 7.0, dtype=torch.bfloat16, device="cuda") for n in (N, R, K))
            _, ran = kernels(lambda: ep.adapter_product(s["x"], s["a"], s["b"], ep.AdapterRows(o, off),
                                                        w=s["w"] if base else None, out=y[1], keep_low=low[1]))
            assert ran == {"adapter_low", "adapter_product"}, ran
            ep.adapter_product_grad(s["x"], s["a"], s["b"], low[1], y[1], ep.AdapterRows(o, off), w=s["w"] if base else None,
                                    dx=dx[1])
            torch.cuda.synchronize()
            for t in (y, low, dx):
                assert (t[0] == 7.0).all() and (t[2] == 7.0).all()


# rows, A, R, K (0: without W, rows of 48), N, activation, parts; by the tile shape
ONE, PARTS = False, True
SHAPES = [
    # 256 x 256
    (8189, 9, 16, 72, 4096, "none", ONE), (4089, 9, 40, 72, 4096, "swiglu", ONE), (218, 2, 240, 6360, 10352, "none", PARTS), (197, 1, 48, 4832, 8456, "swiglu", PARTS),
    (6285, 38, 40, 20184, 136, "none", PARTS), (6194, 17, 112, 21560, 72, "swiglu", PARTS),
    # 256 x 192
    (4100, 9, 16, 72, 4096, "swiglu", ONE), (49034, 2, 128, 0, 8, "none", ONE), (49029, 6, 16, 0, 8, "swiglu", ONE), (146, 1, 224, 1672, 16712, "none", PARTS), (141, 1, 232, 1736, 8432, "swiglu", PARTS),
    (5883, 1, 160, 5576, 144, "none", PARTS), (5807, 1, 144, 6104, 72, "swiglu", PARTS),
    # 256 x 128
    (129, 3, 8, 192, 33208, "none", ONE), (100, 7, 16, 136, 65536, "none", ONE), (129, 2, 16, 0, 17184, "swiglu", ONE),
    # 256 x 64
    (72, 1, 24, 8, 32880, "none", ONE), (64, 5, 40, 136, 131072, "none", ONE), (65, 1, 48, 8, 18072, "swiglu", ONE),
    # 128 x 128
    (20, 3, 16, 72, 131072, "none", ONE), (20, 3, 24, 72, 65536, "swiglu", ONE), (16494, 1, 64, 0, 72, "none", ONE),
    (8464, 3, 208, 1448, 72, "none", PARTS), (8239, 2, 240, 1528, 40, "swiglu", PARTS), (9018, 123, 152, 1544, 8, "none", PARTS),
    (8519, 309, 48, 1728, 8, "swiglu", PARTS),
    # 64 x 64
    (8713, 1, 112, 8, 8, "none", ONE), (8457, 1, 168, 8, 8, "swiglu", ONE), (33475, 575, 240, 8, 8, "none", PARTS),
    (12820, 1710, 208, 8, 8, "swiglu", PARTS), (8839, 708, 168, 8, 8, "none", PARTS), (8804, 670, 200, 8, 8, "swiglu", PARTS),
    # 128 x 32
    (9, 2, 16, 72, 262144, "none", ONE), (9069, 158, 160, 8, 8, "none", ONE), (8483, 222, 128, 8, 8, "swiglu", ONE),
    (16771, 1557, 256, 0, 24, "none", PARTS), (17479, 2021, 216, 8, 16, "swiglu", PARTS), (8835, 1214, 216, 8, 8, "none", PARTS),
    (9344, 1550, 168, 8, 8, "swiglu", PARTS)]


@pytest.mark.parametrize("rows,A,R,K,N,act,parts", SHAPES)
def test_shapes(rows, A, R, K, N, act, parts):
    say(f"adapter_product shape rows={rows} A={A} R={R} K={K} N={N} {act}")
    s = ar.make(ar.random_ids(rows, A, rows), A, R, K or 48, N, rows, act, K > 0, bias=True)
    check(s, parts=parts, keep=rows * N < 10 ** 7)


# few results: rows, A, R, K, N, activation; x W^T in tiles of 128 x 128, 64 x 64 and 128 x 32, each in one part, a few and many
FEW_SHAPES = [(66, 5, 16, 8, 21808, "none"), (66, 5, 40, 2048, 2776, "none"), (66, 5, 72, 17248, 272, "none"),
              (65, 5, 136, 8, 10944, "swiglu"), (67, 5, 16, 2080, 1368, "swiglu"), (65, 5, 256, 4176, 656, "swiglu"),
              (130, 9, 24, 264, 72, "none"), (130, 9, 24, 1448, 136, "swiglu"), (40, 3, 8, 8192, 200, "none"),
              (3, 2, 16, 8, 16392, "none"), (1, 2, 64, 968, 4112, "none"), (17, 4, 128, 4104, 1056, "none"),
              (3, 2, 256, 8, 8200, "swiglu"), (1, 2, 32, 968, 2096, "swiglu"), (17, 4, 8, 4104, 520, "swiglu"),
              (1, 1, 16, 262144, 8, "none"), (5, 2, 256, 32768, 24, "swiglu")]


@pytest.mark.parametrize("rows,A,R,K,N,act", FEW_SHAPES)
def test_few_shapes(rows, A, R, K, N, act):
    say(f"adapter_product few rows={rows} A={A} R={R} K={K} N={N} {act}")
    for base in (True, False):
        s = ar.make(ar.random_ids(rows, A, rows, 0.1), A, R, K, N, rows, act, base, bias=True, residual=base)
        _, ran = kernels(lambda: ar.check(s))
        assert ran == {"adapter_few" if base else "adapter_few_low", "adapter_few_join"}, ran


# rows, A, R, K, N, W; dx in parts, da in parts, db in parts; dx by the tile shape
GRADS = [
    (196, 1, 8, 33128, 24, False, 0, 0, 0), (229, 2, 184, 8424, 1848, True, 1, 0, 0), (195, 1, 248, 2152, 8600, True, 1, 0, 0),
    (135, 1, 24, 33112, 56, False, 0, 0, 0), (137, 5, 112, 13376, 880, True, 1, 0, 0), (133, 2, 192, 1032, 7384, True, 1, 0, 0),
    (32812, 1, 72, 8, 8, False, 0, 1, 1), (33, 12, 112, 8824, 8, True, 1, 0, 0), (71, 25, 80, 8, 8, True, 1, 0, 0),
    (1, 1, 8, 8, 8, False, 0, 0, 0), (1, 3, 152, 8, 8, True, 1, 0, 0), (1, 11, 88, 8, 8, True, 1, 0, 0),
    (2, 33, 8, 8, 8, True, 0, 0, 0), (1, 38, 16, 8, 8, False, 1, 0, 0), (1, 33, 32, 8, 8, False, 1, 0, 0),
    (459, 1, 24, 136, 72, True, None, 1, 1), (2003, 1, 32, 72, 136, True, None, 1, 1), (450, 1, 40, 264, 8, True, None, 1, 1),
    (1987, 1, 200, 72, 520, False, None, 1, 1), (6000, 3, 72, 136, 264, True, None, 1, 1)]


@pytest.mark.parametrize("rows,A,R,K,N,base,dx,da,db", GRADS)
def test_gradient_shapes(rows, A, R, K, N, base, dx, da, db):
    say(f"adapter_product_grad shape rows={rows} A={A} R={R} K={K} N={N} W={base}")
    for act in ("none", "silu"):
        for packed in (False, True):
            ids = ar.random_ids(rows, A, rows, 0.2 if rows > 9 else 0.0)
            if packed:
                ids = torch.where(ids < 0, A, ids).sort()[0]
                ids = torch.where(ids == A, -1, ids)
            s = ar.make(ids, A, R, K, N, rows, act, base)
            _, ran = kernels(lambda: ar.check_grad(s, packed=packed))
            want = {"adapter_low", "adapter_dx", "adapter_weights"} | ({"adapter_dz"} if act != "none" else set())
            want |= {"adapter_weights_join"} if da or db else set()
            if dx is not None:
                want |= {"adapter_dx_join"} if dx else set()
                assert ran == want, ran
            else:
                assert ran - {"adapter_dx_join"} == want, ran


@pytest.mark.parametrize("rows,first,none,base", [(90, 17, 5, True), (300, 40, 0, False), (5000, 700, 31, True), (9000, 300, 0, False)])
@pytest.mark.parametrize("ordered", [False, True])
def test_rows_before_the_first_adapter(rows, first, none, base, ordered):
    """offsets[0] above 0: the places before it have no adapter, as those behind offsets[A].  Whole numbers: every sum is exact."""
    say(f"adapter_product: {first} rows before the first adapter of {rows}, W={base} ordered={ordered}")
    A, R, K, N = 4, 24, 136, 264
    g = ref.gen(rows)

    def whole(shape, most):
        return torch.randint(-most, most + 1, shape, device="cuda", generator=g).bfloat16()

    x, d = whole((rows, K), 50), whole((rows, N), 50)
    a, b, w = whole((A, R, K), 1), whole((A, N, R), 1), whole((N, K), 1) if base else None
    inner = torch.randint(0, A, (rows - first - none,), device="cuda", generator=g).sort()[0]
    of = torch.cat([inner.new_full((first,), A), inner, inner.new_full((none,), A)])
    offsets = torch.searchsorted(inner, torch.arange(A + 1, device="cuda")) + first
    order = torch.randperm(rows, device="cuda", generator=g) if ordered else torch.arange(rows, device="cuda")
    by = ep.AdapterRows(order.int() if ordered else None, offsets.int())
    out, pre = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda"), True
    got = ep.adapter_product(x, a, b, by, w=w, out=out, keep_pre=pre, keep_low=True)
    low = ar.by_adapter(x.double()[order], of, a.double().transpose(1, 2))[0]
    z = torch.zeros((rows, N), dtype=torch.float64, device="cuda")
    z[order] = ar.by_adapter(low, of, b.double().transpose(1, 2))[0]
    if base:
        z += x.double() @ w.double().t()
    assert torch.equal(got.low, low.bfloat16()) and torch.equal(got.out, z.bfloat16()) and torch.equal(got.pre, z.bfloat16())
    grad = ep.adapter_product_grad(x, a, b, got.low, d, by, w=w)
    v = ar.by_adapter(d.double()[order], of, b.double())[0]
    dx = torch.zeros((rows, K), dtype=torch.float64, device="cuda")
    dx[order] = ar.by_adapter(v, of, a.double())[0]
    if base:
        dx += d.double() @ w.double()
    assert torch.equal(grad.dx, dx.bfloat16())
    for e in range(A):
        at = of == e
        for have, long, short, what in ((grad.da[e].t(), x, v, "da"), (grad.db[e], d, got.low.double(), "db")):
            want = long.double()[order][at].t() @ short[at]
            off = long.double()[order][at].abs().t() @ short[at].abs() * (2 * rows + 8) * ref.U23  # past 2^24 sums are rounded
            ref.within(have, want, off + ref.BF16 * (want.abs() + off), f"{what} {e}")
