"""The experts' product and its gradient against plain implementations in 64 bits.

Bounds: products of bf16 or of e4m3 values are exact in fp32; a sum of n terms in any order,
each addition rounded or truncated, is within (n + 8) 2^-23 of the sum of magnitudes (8 more
for the bias, the two scales, the residual and the join of partial sums).  An activation
stretches that by at most 1.2 (layer_ref.act_error) and is itself within 2^-18.  The
gradient's dz is rounded to bf16 before the two products (2^-8 of each term) and its
activation's slope is within 2^-17."""
import math

import pytest
import torch

import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "silu", "gelu", "swiglu"]


def make(counts, K, N, act, seed, first=0, past=0, bits8=False, bias=False, residual=False):
    g = ref.gen(seed)
    E, rows = len(counts), first + sum(counts) + past
    wide = 2 * N if act == "swiglu" else N
    s = {"offsets": ref.offsets_of(counts, first), "N": N, "act": act, "w_scale": None}
    x, w = ref.normal((rows, K), g), ref.normal((E, wide, K), g, K ** -0.5)
    if bits8:
        xs = torch.rand(rows, device="cuda", generator=g) * 0.1 + 1e-3
        s["w_scale"] = torch.rand((E, wide), device="cuda", generator=g) * 0.01 + 1e-4
        xq, wq = (x.float() * 30).to(torch.float8_e4m3fn), (w.float() * 100).to(torch.float8_e4m3fn)
        s["x"], s["w"] = ref.rows8_of(xq, xs), wq
        s["xd"], s["wd"] = xq.double() * xs.double()[:, None], wq.double() * s["w_scale"].double()[:, :, None]
    else:
        s["x"], s["w"], s["xd"], s["wd"] = x, w, x.double(), w.double()
    s["bias"] = ref.normal((E, wide), g) if bias else None
    s["res"] = ref.normal((rows, N), g) if residual else None
    s["range"] = slice(first, first + sum(counts))
    return s


def check(s, f32=False, pre=True):
    K = s["wd"].shape[2]
    z, size = ref.product_z(s["xd"], s["wd"], s["offsets"], s["bias"])
    dz = size * (K + 8) * ref.U23
    y, dy = ref.act(z, s["act"]), ref.act_error(z, dz, s["act"])
    if s["res"] is not None:
        y = y + s["res"].double()
        dy = dy + (y.abs() + s["res"].double().abs()) * ref.U23
    dtype = torch.float32 if f32 else torch.bfloat16
    out = torch.full(y.shape, 7.0, dtype=dtype, device="cuda")
    kept = torch.full(z.shape, 7.0, dtype=torch.bfloat16, device="cuda") if pre else False
    got = ep.expert_product(s["x"], s["w"], s["offsets"], w_scale=s["w_scale"], bias=s["bias"], act=s["act"], residual=s["res"],
                            keep_pre=kept, out=out)
    at = s["range"]
    ref.within(out[at], y[at], (dy + (0 if f32 else ref.BF16) * (y.abs() + dy))[at], "y")
    assert (out[:at.start] == 7.0).all() and (out[at.stop:] == 7.0).all()   # rows of no expert
    if pre:
        ref.within(kept[at], z[at], (dz + ref.BF16 * (z.abs() + dz))[at], "pre")
        assert (kept[:at.start] == 7.0).all() and (kept[at.stop:] == 7.0).all()
    return got


COUNTS = [[1], [16], [0, 5, 0], [129], [17, 0, 1, 64], [128, 127, 300], [256, 257, 255], [1024, 0, 3]]


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("counts", COUNTS, ids=str)
def test_row_counts(counts, bits8):
    for K, N, act in ((208, 136, "silu"), (128, 264, "swiglu"), (1040, 520, "none")):
        say(f"expert_product rows={counts} K={K} N={N} {act} 8-bit={bits8}")
        check(make(counts, K, N, act, K + N, bits8=bits8))


@pytest.mark.parametrize("K", [8, 16, 56, 64, 72, 120, 128, 136, 192, 264, 512, 1448, 4104])
@pytest.mark.parametrize("rows", [1, 9, 40, 300])
def test_inner_lengths(rows, K):
    say(f"expert_product rows={rows} K={K}")
    check(make([rows], K, 72, "none", K))
    if K % 16 == 0:
        check(make([rows], K, 72, "none", K, bits8=True))


@pytest.mark.parametrize("N", [8, 16, 24, 40, 64, 120, 136, 256, 264, 1032])
@pytest.mark.parametrize("rows", [2, 33, 260])
def test_output_lengths(rows, N):
    say(f"expert_product rows={rows} N={N}")
    for act in ("none", "swiglu"):
        check(make([rows, rows // 2], 200, N, act, N))
        check(make([rows, rows // 2], 208, N, act, N, bits8=True))


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [3, 70, 500])
def test_epilogues(rows, act, bits8):
    say(f"expert_product {act} rows={rows} 8-bit={bits8}")
    for bias in (False, True):
        for residual in (False, True):
            for f32 in (False, True):
                check(make([rows, 7], 144, 88, act, rows, bits8=bits8, bias=bias, residual=residual), f32, pre=bias != residual)


@pytest.mark.parametrize("rows,K,N", [(1, 7168, 256), (256, 7168, 256), (4, 2048, 4096), (32, 4096, 1024), (100, 8192, 64)])
def test_few_rows_and_long_sums(rows, K, N):
    """The dense products of a decode step, where the contraction is split over workgroups."""
    say(f"expert_product dense rows={rows} K={K} N={N}")
    s = make([rows], K, N, "none", rows + K)
    check(s, f32=True, pre=False)
    one = ep.expert_product(s["x"], s["w"], None, out_dtype=torch.float32).out
    assert torch.equal(one, ep.expert_product(s["x"], s["w"], s["offsets"], out_dtype=torch.float32).out)
    check(make([rows], K, N, "swiglu", rows + K, bias=True, residual=True))


# Enough columns that every tile size has a tile for each compute unit: which size runs goes by
# the mean rows per expert, and between the two largest by how they fill the chip.
MANY = [[3, 0, 9], [20, 40], [37, 70, 60, 0], [100, 90, 140], [300, 190], [700, 513], [193, 1, 600], [1024], [2049]]


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("counts", MANY, ids=str)
def test_many_columns(counts, bits8):
    for K, N, act in ((144, 16392, "none"), (528, 8200, "swiglu")):
        say(f"expert_product many columns rows={counts} K={K} N={N} {act} 8-bit={bits8}")
        check(make(counts, K, N, act, K, bits8=bits8, bias=True, residual=act == "none"), f32=K == 144)


@pytest.mark.parametrize("act", ACTS)
def test_large_tiles_epilogues(act):
    for counts in ([300, 190], [90, 100, 81], [45, 60, 50]):
        say(f"expert_product many columns rows={counts} {act}")
        for bias, residual in ((False, True), (True, False)):
            check(make(counts, 72, 16392 if act != "swiglu" else 8200, act, 7, first=3, past=5, bias=bias, residual=residual))


def test_rows_of_no_expert_stay():
    for rows in ([0, 0], [5, 0], [200, 90]):
        say(f"expert_product inside a larger buffer: {rows}")
        check(make(rows, 136, 72, "gelu", 1, first=11, past=300))


def test_many_experts():
    g = torch.Generator().manual_seed(1)
    for E, most in ((200, 5), (70, 60), (2048, 2)):
        counts = torch.randint(0, most, (E,), generator=g).tolist()
        say(f"expert_product E={E}")
        check(make(counts, 72, 40, "swiglu", E), pre=False)


def test_no_rows():
    s = make([0, 0], 64, 32, "silu", 1)
    assert ep.expert_product(s["x"], s["w"], s["offsets"], act="silu").out.shape == (0, 32)


def test_offsets_out_of_range_stay_in_bounds():
    """Offsets below 0, past the rows, or falling: what they name within [0, rows) is computed."""
    say("expert_product: offsets out of range")
    s = make([40, 60, 50], 64, 32, "none", 1)
    s["offsets"] = torch.tensor([-5, 40, 100, 100000], dtype=torch.int32, device="cuda")
    want = ep.expert_product(s["x"], s["w"], torch.tensor([0, 40, 100, 150], dtype=torch.int32, device="cuda")).out
    assert torch.equal(ep.expert_product(s["x"], s["w"], s["offsets"]).out, want)
    falling = torch.tensor([100, 50, 150, 20], dtype=torch.int32, device="cuda")
    got = ep.expert_product(s["x"], s["w"], falling, out=torch.zeros_like(want)).out
    ref.within(got[50:150], s["xd"][50:150] @ s["wd"][1].t(), 1.0, "the rows of the one expert that has some")
    assert not got[:50].any()


def test_nan_and_infinity_stay_in_their_rows_and_columns():
    say("expert_product: NaN and infinities")
    for rows in ([20, 9], [300, 200]):
        s = make(rows, 264, 136, "silu", 5)
        clean = ep.expert_product(s["x"], s["w"], s["offsets"], act="silu").out
        s["x"][3, 100] = float("nan")
        s["x"][rows[0] + 2] = float("inf")
        got = ep.expert_product(s["x"], s["w"], s["offsets"], act="silu").out
        keep = [r for r in range(sum(rows)) if r not in (3, rows[0] + 2)]
        assert torch.equal(got[keep], clean[keep]) and got[3].isnan().all()
        s["x"][3], s["x"][rows[0] + 2] = 0, 0
        s["w"][0, 7] = float("nan")
        clean = ep.expert_product(s["x"], torch.nan_to_num(s["w"]), s["offsets"], act="silu").out
        got = ep.expert_product(s["x"], s["w"], s["offsets"], act="silu").out
        assert got[:rows[0], 7].isnan().all()
        got[:rows[0], 7] = clean[:rows[0], 7]
        assert torch.equal(got, clean)


def test_padding_bytes_of_8bit_rows_do_not_matter():
    """K = 16 less than a step: the scale and what stands behind it are not multiplied."""
    say("expert_product: bytes behind 8-bit rows")
    s = make([37], 112, 40, "none", 3, bits8=True)
    want = ep.expert_product(s["x"], s["w"], s["offsets"], w_scale=s["w_scale"]).out
    s["x"][:, 116:] = 0x7f      # e4m3 NaN
    assert torch.equal(ep.expert_product(s["x"], s["w"], s["offsets"], w_scale=s["w_scale"]).out, want)


def test_rows_past_4_gib():
    say("expert_product past 4 GiB")
    K, N = 2048, 64
    rows = (1 << 32) // (K * 2) + 5000
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    g = ref.gen(2)
    w = ref.normal((2, N, K), g)
    x[-300:] = ref.normal((300, K), g)
    offsets = torch.tensor([0, rows - 200, rows], dtype=torch.int32, device="cuda")
    got = ep.expert_product(x, w, offsets).out
    z = torch.cat([x[-300:-200].double() @ w[0].double().t(), x[-200:].double() @ w[1].double().t()])
    size = torch.cat([x[-300:-200].double().abs() @ w[0].double().abs().t(), x[-200:].double().abs() @ w[1].double().abs().t()])
    bound = size * (K + 8) * ref.U23
    ref.within(got[-300:], z, bound + ref.BF16 * (z.abs() + bound), "y")
    d_y = torch.zeros((rows, N), dtype=torch.bfloat16, device="cuda")
    d_y[-300:] = ref.normal((300, N), g)
    grad = ep.expert_product_grad(x, w, d_y, offsets)
    d = d_y[-300:].double()
    dx = torch.cat([d[:100] @ w[0].double(), d[100:] @ w[1].double()])
    size = torch.cat([d[:100].abs() @ w[0].double().abs(), d[100:].abs() @ w[1].double().abs()])
    bound = size * (N + 8) * ref.U23
    ref.within(grad.dx[-300:], dx, bound + ref.BF16 * (dx.abs() + bound), "dx")
    dw = torch.stack([d[:100].t() @ x[-300:-200].double(), d[100:].t() @ x[-200:].double()])
    size = torch.stack([d[:100].abs().t() @ x[-300:-200].double().abs(), d[100:].abs().t() @ x[-200:].double().abs()])
    bound = size * 308 * ref.U23   # zeros add nothing
    ref.within(grad.dw, dw, bound + ref.BF16 * (dw.abs() + bound), "dw")


def test_side_stream_and_graph():
    say("expert_product on a stream of its own and in a graph")
    s = make([60, 0, 300], 512, 256, "swiglu", 4)
    want = ep.expert_product(s["x"], s["w"], s["offsets"], act="swiglu").out
    few = make([8], 4096, 256, "none", 4)
    want_few = ep.expert_product(few["x"], few["w"], out_dtype=torch.float32).out
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        got = ep.expert_product(s["x"], s["w"], s["offsets"], act="swiglu", stream=side).out
        got_few = ep.expert_product(few["x"], few["w"], out_dtype=torch.float32, stream=side).out
        torch.empty_like(want).fill_(7.0)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(got_few, want_few)
    out, out_few = torch.empty_like(want), torch.empty_like(want_few)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ep.expert_product(s["x"], s["w"], s["offsets"], act="swiglu", out=out)
        ep.expert_product(few["x"], few["w"], out=out_few)
    for i in range(4):
        s["x"].mul_(-1.0)
        few["x"].mul_(-1.0)
        want = ep.expert_product(s["x"], s["w"], s["offsets"], act="swiglu").out
        want_few = ep.expert_product(few["x"], few["w"], out_dtype=torch.float32).out
        out.zero_(), out_few.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(out_few, want_few), i


# ------------------------------------------------------------------------------ gradient

def check_grad(counts, K, N, act, seed, bias=True, first=0, past=0):
    s = make(counts, K, N, act, seed, first, past)
    g = ref.gen(seed + 1)
    rows, wide = s["x"].shape[0], s["w"].shape[1]
    d_y = ref.normal((rows, N), g)
    pre = None if act == "none" else ref.normal((rows, wide), g)
    dz = d_y.double() if act == "none" else ref.act_grad(pre.double(), d_y.double(), act)
    # what activation_grad may be off: 2^-17 of the slope's terms, each at most |z| + 1.2 in size
    off = torch.zeros_like(dz)
    if act != "none":
        zd = pre.double()
        if act == "swiglu":
            gate, up = zd.chunk(2, 1)
            off = torch.cat([d_y.double().abs() * up.abs() * (gate.abs() + 1.2), d_y.double().abs() * gate.abs()], 1) * 2.0 ** -17
        else:
            off = d_y.double().abs() * (zd.abs() + 1.2) * 2.0 ** -17
    into = torch.full((rows, K), 7.0, dtype=torch.bfloat16, device="cuda")
    got = ep.expert_product_grad(s["x"], s["w"], d_y, s["offsets"], pre=pre, act=act, with_bias=bias, dx=into)
    term = dz.abs() * (0 if act == "none" else ref.BF16) + off
    ends = s["offsets"].tolist()
    assert (into[:ends[0]] == 7.0).all() and (into[ends[-1]:] == 7.0).all()
    for e in range(len(counts)):
        at = slice(ends[e], ends[e + 1])
        x, w, z = s["xd"][at], s["wd"][e], dz[at]
        dx = z @ w
        bound = term[at] @ w.abs() + (z.abs() + term[at]) @ w.abs() * (wide + 8) * ref.U23
        ref.within(got.dx[at], dx, bound + ref.BF16 * (dx.abs() + bound), f"dx {e}")
        n = max(1, counts[e])
        dw = z.t() @ x
        bound = term[at].t() @ x.abs() + (z.abs() + term[at]).t() @ x.abs() * (n + 8) * ref.U23
        ref.within(got.dw[e], dw, bound + ref.BF16 * (dw.abs() + bound), f"dw {e}")
        if bias:
            ref.within(got.dbias[e], z.sum(0), off[at].sum(0) + z.abs().sum(0) * (n + 8) * ref.U24, f"dbias {e}")
    assert bias or got.dbias is None
    return s, d_y, pre, got


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("counts", [[1], [0, 5, 0], [63, 64, 65, 0], [130, 1, 17], [300, 257]], ids=str)
def test_gradient(counts, act):
    for K, N in ((72, 40), (264, 136), (520, 264)):
        say(f"expert_product_grad rows={counts} K={K} N={N} {act}")
        check_grad(counts, K, N, act, K)


@pytest.mark.parametrize("K,N", [(8, 8), (16, 1032), (1032, 16), (1448, 72), (520, 520), (2056, 640)])
def test_gradient_lengths(K, N):
    for counts in ([40, 3], [500, 400]):
        say(f"expert_product_grad rows={counts} K={K} N={N}")
        check_grad(counts, K, N, "none", N, bias=False)
        check_grad(counts, K, N, "swiglu", N)


@pytest.mark.parametrize("counts", [[300, 190], [700, 513], [193, 1, 600], [1024], [2049], [0, 321, 0, 400]], ids=str)
def test_gradient_many_columns(counts):
    """dx over long rows and dw over many tiles: both large tiles."""
    for K, N in ((16392, 72), (4104, 1032)):
        say(f"expert_product_grad many columns rows={counts} K={K} N={N}")
        check_grad(counts, K, N, "none", K, bias=False)


@pytest.mark.parametrize("counts", [[5000], [3000, 0, 100], [1, 2500], [700] * 5], ids=str)
def test_gradient_of_many_rows(counts):
    """dw of few tiles, whose rows are split into parts, and the same bits at every call."""
    for K, N, act in ((72, 40, "none"), (520, 264, "gelu"), (136, 72, "swiglu")):
        say(f"expert_product_grad rows={counts} K={K} N={N} {act}")
        s, d_y, pre, got = check_grad(counts, K, N, act, K)
        again = ep.expert_product_grad(s["x"], s["w"], d_y, s["offsets"], pre=pre, act=act, with_bias=True)
        assert torch.equal(again.dw, got.dw) and torch.equal(again.dx, got.dx) and torch.equal(again.dbias, got.dbias)


def test_gradient_parts_and_empty():
    say("expert_product_grad: parts, rows of no expert, no rows")
    s, d_y, pre, whole = check_grad([90, 0, 200], 264, 136, "gelu", 3, first=5, past=70)
    for dx, dw, bias in ((True, False, False), (False, True, False), (False, False, True)):
        into = torch.full_like(whole.dx, 7.0) if dx else False
        got = ep.expert_product_grad(s["x"], s["w"], d_y, s["offsets"], pre=pre, act="gelu", with_bias=bias, dx=into, dw=dw)
        assert (got.dx is not None, got.dw is not None, got.dbias is not None) == (dx, dw, bias)
        for name in ("dx", "dw", "dbias"):
            assert getattr(got, name) is None or torch.equal(getattr(got, name), getattr(whole, name))
    empty = ep.expert_product_grad(s["x"][:0], s["w"], d_y[:0], torch.zeros(4, dtype=torch.int32, device="cuda"), pre=pre[:0],
                                   act="gelu", with_bias=True)
    assert empty.dx.shape == (0, 264) and not empty.dw.any() and not empty.dbias.any()


def test_gradient_against_differences():
    """Central differences of sum(d_y * act(x W^T + b)) in 64 bits at the forward's own pre."""
    say("expert_product_grad against differences")
    for act in ACTS:
        s = make([30, 21], 72, 40, act, 9, bias=True)
        g = ref.gen(4)
        d_y = ref.normal((51, 40), g)
        fwd = ep.expert_product(s["x"], s["w"], s["offsets"], bias=s["bias"], act=act, keep_pre=True)
        got = ep.expert_product_grad(s["x"], s["w"], d_y, s["offsets"], pre=fwd.pre, act=act, with_bias=True)

        def loss(x, w, b):
            z = torch.cat([x[:30] @ w[0].t() + b[0], x[30:] @ w[1].t() + b[1]])
            return (d_y.double() * ref.act(z, act)).sum()

        at = (s["xd"], s["wd"], s["bias"].double())
        for i, grad in enumerate((got.dx, got.dw, got.dbias)):
            v = torch.randn(at[i].shape, device="cuda", dtype=torch.float64, generator=g)
            h = 1e-5
            up, down = [list(at), list(at)]
            up[i], down[i] = at[i] + h * v, at[i] - h * v
            along = (loss(*up) - loss(*down)) / (2 * h)
            # pre is bf16: the slope is taken up to 2^-8 |z| beside z, and dz and the result are rounded
            assert abs((grad.double() * v).sum() - along) <= 0.02 * float((grad.double() * v).abs().sum()), (act, i)


def test_binding_refusals():
    """Wrong devices, types, layouts and shapes raise before anything is enqueued."""
    say("expert_product: refusals of the binding")
    s = make([3, 2], 64, 32, "none", 1)
    x, w, off = s["x"], s["w"], s["offsets"]
    for bad in (x.cpu(), x.float(), x.t(), x[:, :48], x[0]):
        with pytest.raises(ValueError):
            ep.expert_product(bad, w, off)
    for bad in (w.float(), w.transpose(1, 2), w[0], w.cpu()):
        with pytest.raises(ValueError):
            ep.expert_product(x, bad, off)
    for bad in (None, off[:2], off.long(), off.cpu()):
        with pytest.raises(ValueError):
            ep.expert_product(x, w, bad)
    for more in (dict(act="tanh"), dict(bias=w[0]), dict(residual=x), dict(out=x), dict(out_dtype=torch.float16),
                 dict(w_scale=torch.ones((2, 31), device="cuda")), dict(keep_pre=x)):
        with pytest.raises(ValueError):
            ep.expert_product(x, w, off, **more)
    with pytest.raises(ep.EPError):
        ep.expert_product(x, w, off, w_scale=torch.ones((2, 32), device="cuda"))   # scales go with 8-bit rows
    with pytest.raises(ValueError):
        ep.expert_product(ep.rows8_empty(5, 64), w.to(torch.float8_e4m3fn), off)
    d_y = torch.zeros((5, 32), dtype=torch.bfloat16, device="cuda")
    for bad in (None, d_y[:4], d_y.float()):
        with pytest.raises(ValueError):
            ep.expert_product_grad(x, w, bad, off)
    with pytest.raises(ValueError):
        ep.expert_product_grad(x, w, d_y, off, act="silu")


def test_gelu_of_negative_values_keeps_its_digits():
    """z Phi(z) over the range of its tail, through an identity: the exponent -z^2 / 2 and its
    exponential are off by 1.25 z^2 2^-24, the polynomial and its arithmetic by 24 2^-24; below 2^-120
    the exponential may come out as zero."""
    say("expert_product: gelu's tail")
    g = ref.gen(12)
    K = 64
    x = (torch.rand((400, K), device="cuda", generator=g) * 26 - 13).bfloat16()
    eye = torch.eye(K, device="cuda", dtype=torch.bfloat16)[None].contiguous()
    z = x.double()
    y = z * torch.exp(torch.special.log_ndtr(z))
    off = y.abs() * (1.25 * z.square() + 32) * ref.U24 + 2.0 ** -120
    wide = ep.expert_product(x, eye, act="gelu", out_dtype=torch.float32).out
    ref.within(wide, y, off, "fp32")
    ref.within(ep.expert_product(x, eye, act="gelu").out, y, (y.abs() + off) * ref.BF16 + off, "bf16")
    # the slope Phi(z) + z phi(z), through d_y of ones; its terms cancel near -0.75
    cdf, density = torch.exp(torch.special.log_ndtr(z)), z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    grad = ep.expert_product_grad(x, eye, torch.ones_like(x), pre=x, act="gelu", dw=False)
    size = (cdf + density.abs()) * (1.25 * z.square() + 32) * ref.U24 + 2.0 ** -118
    want = cdf + density
    # dz is rounded to bf16, which the product with the identity keeps
    ref.within(grad.dx, want, (want.abs() + size) * ref.BF16 + size, "slope")


def autograd_dz(pre, d_y, act):
    """The pre-activations' gradient by 64-bit autograd of the activation: no slope written by hand."""
    z = pre.double().detach().requires_grad_()
    if act == "gelu":
        y = z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    else:
        y = ref.act(z, act)
    (y * d_y.double()).sum().backward()
    return z.grad


def slope_error(pre, d_y, act):
    """What dz may be off before its rounding: 2^-17 of the slope's terms, each at most |z| + 1.2 in size."""
    z, d = pre.double().abs(), d_y.double().abs()
    if act != "swiglu":
        return d * (z + 1.2) * 2.0 ** -17
    gate, up = z.chunk(2, 1)
    return torch.cat([d * up * (gate + 1.2), d * gate], 1) * 2.0 ** -17


@pytest.mark.parametrize("act", ["relu", "silu", "gelu", "swiglu"])
def test_slopes_against_autograd(act):
    """dz itself, element by element (through an identity), and every element of dx, dw and dbias,
    against 64-bit autograd of the activation at the kept values."""
    say(f"expert_product_grad: slope of {act} against autograd")
    counts, K, N = [30, 21], 72, 40
    s, d_y, pre, got = check_grad(counts, K, N, act, 13)
    dz, off = autograd_dz(pre, d_y, act), slope_error(pre, d_y, act)
    wide = dz.shape[1]
    eye = torch.eye(wide, device="cuda", dtype=torch.bfloat16)[None].contiguous()
    alone = ep.expert_product_grad(torch.zeros((51, wide), device="cuda", dtype=torch.bfloat16), eye, d_y, pre=pre, act=act,
                                   dw=False).dx
    ref.within(alone, dz, (dz.abs() + off) * ref.BF16 + off, "dz")
    term = dz.abs() * ref.BF16 + off
    for e, at in enumerate((slice(0, 30), slice(30, 51))):
        w, x, n, most = s["wd"][e], s["xd"][at], counts[e], dz[at].abs() + term[at]
        want = dz[at] @ w
        bound = term[at] @ w.abs() + most @ w.abs() * (wide + 8) * ref.U23
        ref.within(got.dx[at], want, bound + ref.BF16 * (want.abs() + bound), "dx")
        want = dz[at].t() @ x
        bound = term[at].t() @ x.abs() + most.t() @ x.abs() * (n + 8) * ref.U23
        ref.within(got.dw[e], want, bound + ref.BF16 * (want.abs() + bound), "dw")
        ref.within(got.dbias[e], dz[at].sum(0), off[at].sum(0) + most.sum(0) * (n + 8) * ref.U24, "dbias")


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences_along_itself(act):
    """As test_gradient_against_differences, along the gradient's own signs, where every element adds
    to the difference.  The roundings of pre, dz and the result, at most 2^-8 of a value each and of
    random sign, over 80 elements and more: 3 * 2^-8 / sqrt(80) = 0.13%, three times that.  A slope
    without one of its terms is 0.9% off and more (silu 1.8, gelu 4.5, relu 39)."""
    say(f"expert_product_grad against differences along itself: {act}")
    for seed in (21, 22):
        s = make([30, 21], 72, 40, act, seed, bias=True)
        d_y = ref.normal((51, 40), ref.gen(seed + 10))
        fwd = ep.expert_product(s["x"], s["w"], s["offsets"], bias=s["bias"], act=act, keep_pre=True)
        got = ep.expert_product_grad(s["x"], s["w"], d_y, s["offsets"], pre=fwd.pre, act=act, with_bias=True)

        def loss(x, w, b):
            z = torch.cat([x[:30] @ w[0].t() + b[0], x[30:] @ w[1].t() + b[1]])
            return (d_y.double() * ref.act(z, act)).sum()

        at = (s["xd"], s["wd"], s["bias"].double())
        for i, grad in enumerate((got.dx, got.dw, got.dbias)):
            v, h = grad.double().sign(), 1e-6
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * v, at[i] - h * v
            along = (loss(*up) - loss(*down)) / (2 * h)
            whole = float(grad.double().abs().sum())
            assert abs(whole - float(along)) <= 0.004 * whole, (act, i)


# ------------------------------------------------------------------- long sums of 8-bit rows

# sums of 4000 terms and more are cut into more than four parts where rows are few
@pytest.mark.parametrize("K", [512, 528, 1040, 2048, 4096, 7168])
@pytest.mark.parametrize("counts", [[1], [8], [5, 0, 30], [70, 200], [300]], ids=str)
def test_long_sums_of_8bit_rows(counts, K):
    """fp32 results are sums of exact products: at 7168 terms of random signs, 16 to an addition, each
    addition truncated to 2^-23 of the sum so far, their 2-norm is off by at most 2^-23 sqrt(448) / 2 =
    1.3e-6 of the result's, so 2e-6 with the scales; twice that for a gate times an up.  bf16
    results go through the 8-bit instruction, off by less than 2^-15 in the 2-norm, before their own
    rounding of at most 2^-9."""
    for N, act in ((72, "none"), (40, "swiglu")):
        say(f"expert_product 8-bit rows={counts} K={K} N={N} {act}")
        s = make(counts, K, N, act, K + N, bits8=True)
        z, _ = ref.product_z(s["xd"], s["wd"], s["offsets"])
        y = ref.act(z, act)
        check(s, f32=True, pre=False)
        check(s)
        more = dict(w_scale=s["w_scale"], act=act)
        wide = ep.expert_product(s["x"], s["w"], s["offsets"], out_dtype=torch.float32, **more).out.double()
        assert float((wide - y).norm() / y.norm()) <= (2e-6 if act == "none" else 4e-6)
        pre = ep.expert_product(s["x"], s["w"], s["offsets"], keep_pre=True, **more).pre.double()
        assert float((pre - z).norm() / z.norm()) <= 2.0 ** -9 + 2.0 ** -15


@pytest.mark.parametrize("rows,K,N", [(1, 7168, 256), (256, 7168, 256), (4, 2048, 4096), (100, 8192, 64)])
def test_few_rows_keep_fp32_sums(rows, K, N):
    """As test_few_rows_and_long_sums, in the 2-norm: sums cut into parts stay in fp32 to the end."""
    say(f"expert_product dense rows={rows} K={K} N={N} in the 2-norm")
    s = make([rows], K, N, "none", rows + K)
    got = ep.expert_product(s["x"], s["w"], s["offsets"], out_dtype=torch.float32).out.double()
    want = s["xd"] @ s["wd"][0].t()
    assert float((got - want).norm() / want.norm()) <= 2e-6
