"""The layer operators write what is theirs and nothing beside it, on a stream of the caller's."""
import ctypes

import pytest
import torch

import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say
from paper_2609_40093_amd import _lib

pytestmark = pytest.mark.gpu

GUARD = 4096  # bytes before and behind an output


class Guarded:
    """Tensors cut out of buffers whose other bytes have to stay."""

    def __init__(self):
        self.held = []

    def __call__(self, shape, dtype=torch.bfloat16):
        n = torch.Size(shape).numel() * torch.empty((), dtype=dtype).element_size()
        whole = torch.full((GUARD + n + GUARD,), 0x5A, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()  # whatever stream writes it next
        self.held.append((whole, n))
        return whole[GUARD:GUARD + n].view(dtype).view(shape)

    def check(self):
        torch.cuda.synchronize()
        for i, (whole, n) in enumerate(self.held):
            assert bool((whole[:GUARD] == 0x5A).all()) and bool((whole[GUARD + n:] == 0x5A).all()), i


def run(streamed, call):
    """call(stream) on the current stream, or on another one behind the inputs' work."""
    if not streamed:
        return call(None)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = call(s)
    torch.cuda.current_stream().wait_stream(s)
    return got


@pytest.mark.parametrize("streamed", [False, True])
@pytest.mark.parametrize("T,H", [(1, 16), (3, 528), (37, 2896), (130, 7168), (5, 20000)])
def test_norm(T, H, streamed):
    say(f"norm {T} {H}")
    g, at = ref.gen(T + H), Guarded()
    x, r, w, d = ref.normal((T, H), g), ref.normal((T, H), g), ref.normal(H, g), ref.normal((T, H), g)
    got = run(streamed, lambda s: ep.rmsnorm(x, w, residual=r, total=at((T, H)), out=at((T, H)),
                                             rows8=at((T, H + 16), torch.uint8), stream=s))
    dx, dw = run(streamed, lambda s: ep.rmsnorm_grad(got.total, w, d, d_total=r, dx=at((T, H)), d_weight=at((H,), torch.float32),
                                                     stream=s))
    at.check()
    want = ep.rmsnorm(x, w, residual=r, rows8=True)
    want_dx, want_dw = ep.rmsnorm_grad(want.total, w, d, d_total=r)
    for a, b in ((got.total, want.total), (got.out, want.out), (got.rows8, want.rows8), (dx, want_dx), (dw, want_dw)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("streamed", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (3, 7, 7), (33, 65, 3), (70, 130, 8), (5, 257, 4), (9, 511, 6), (20, 513, 2),
                                   (7, 1027, 66), (4, 2047, 5)])
def test_route(T, E, k, dtype, streamed):
    say(f"route {T} {E} {k} {dtype}")
    g, at = ref.gen(T * E + k), Guarded()
    z = torch.randn((T, E), device="cuda", generator=g).to(dtype)
    dg, dl = torch.randn((T, k), device="cuda", generator=g), torch.ones(1, device="cuda")
    f32, i32 = torch.float32, torch.int32
    got = run(streamed, lambda s: ep.route(z, k, balance=0.5, stream=s, out=ep.Routing(
        at((T, k), i32), at((T, k), f32), at((E,), i32), at((E,), f32), at((1,), f32), None, True, 0.0)))
    dz = run(streamed, lambda s: ep.route_grad(z, got, dg, dl, out=at((T, E), dtype), stream=s))
    at.check()
    want = ep.route(z, k, balance=0.5)
    for name in ("topk_idx", "topk_w", "expert_counts", "prob_sums", "loss"):
        assert torch.equal(getattr(got, name), getattr(want, name)), name
    assert torch.equal(dz, ep.route_grad(z, want, dg, dl))


@pytest.mark.parametrize("streamed", [False, True])
@pytest.mark.parametrize("T,k,H", [(1, 1, 8), (5, 3, 520), (33, 8, 2888), (4, 2, 7168)])
def test_combine_grad(T, k, H, streamed):
    say(f"combine_grad {T} {k} {H}")
    g, at = ref.gen(T + k + H), Guarded()
    d, y = ref.normal((T, H), g), ref.normal((T * k, H), g)
    pos = torch.randperm(T * k, device="cuda", generator=g).int()
    w = torch.rand((T, k), device="cuda", generator=g)
    dy, dw = run(streamed, lambda s: ep.combine_grad(d, y, pos, w, dy=at((T * k, H)), d_topk_w=at((T, k), torch.float32),
                                                     stream=s))
    at.check()
    want = ep.combine_grad(d, y, pos, w)
    assert torch.equal(dy, want[0]) and torch.equal(dw, want[1])


@pytest.mark.parametrize("streamed", [False, True])
@pytest.mark.parametrize("counts,K,N", [([1], 8, 8), ([3, 0, 5], 72, 40), ([70, 130], 520, 264), ([300], 1448, 520),
                                        ([700, 1, 90], 264, 2888), ([40] * 9, 512, 776), ([9000], 136, 4104)])
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_product(counts, K, N, act, streamed):
    say(f"product {counts[:3]} {K} {N} {act}")
    E, rows, wide = len(counts), sum(counts), 2 * N if act == "swiglu" else N
    g, at = ref.gen(rows + K + N), Guarded()
    x, w, b = ref.normal((rows, K), g), ref.normal((E, wide, K), g), ref.normal((E, wide), g)
    r, d = ref.normal((rows, N), g), ref.normal((rows, N), g)
    off = torch.tensor([0] + counts, device="cuda").cumsum(0).int()
    got = run(streamed, lambda s: ep.expert_product(x, w, off, bias=b, act=act, residual=r, keep_pre=at((rows, wide)),
                                                    out=at((rows, N)), stream=s))
    wide_out = run(streamed, lambda s: ep.expert_product(x, w, off, act=act, out=at((rows, N), torch.float32), stream=s))
    grad = run(streamed, lambda s: ep.expert_product_grad(x, w, d, off, pre=got.pre, act=act, dx=at((rows, K)),
                                                          dw=at((E, wide, K)), dbias=at((E, wide), torch.float32), stream=s))
    at.check()
    want = ep.expert_product(x, w, off, bias=b, act=act, residual=r, keep_pre=True)
    assert torch.equal(got.out, want.out) and torch.equal(got.pre, want.pre)
    assert torch.equal(wide_out.out, ep.expert_product(x, w, off, act=act, out_dtype=torch.float32).out)
    want = ep.expert_product_grad(x, w, d, off, pre=want.pre, act=act, with_bias=True)
    for name in ("dx", "dw", "dbias"):
        assert torch.equal(getattr(grad, name), getattr(want, name)), name


@pytest.mark.parametrize("streamed", [False, True])
@pytest.mark.parametrize("counts,K,N", [([5], 16, 16), ([70, 0, 131], 528, 272), ([900], 1456, 520)])
def test_product_of_8bit_rows(counts, K, N, streamed):
    say(f"product 8 bit {counts} {K} {N}")
    E, rows = len(counts), sum(counts)
    g, at = ref.gen(rows + K), Guarded()
    x = ep.rmsnorm(ref.normal((rows, K), g), out=False, rows8=True).rows8
    w = ref.normal((E, N, K), g).to(torch.float8_e4m3fn)
    scale = torch.rand((E, N), device="cuda", generator=g)
    off = torch.tensor([0] + counts, device="cuda").cumsum(0).int()
    for dtype in (torch.bfloat16, torch.float32):
        got = run(streamed, lambda s: ep.expert_product(x, w, off, w_scale=scale, out=at((rows, N), dtype), stream=s))
        at.check()
        assert torch.equal(got.out, ep.expert_product(x, w, off, w_scale=scale, out_dtype=dtype).out)


@pytest.mark.parametrize("offsets", [[0, 300, 0, 300], [300, 0, 300, 0], [-5, 1000, -7, 2000], [0, 0, 0, 0]])
@pytest.mark.parametrize("act", ["none", "silu", "swiglu"])
def test_decreasing_offsets_stay_in_bounds(offsets, act):
    """What such offsets give is not defined; nothing beside the outputs is touched."""
    say(f"decreasing offsets {offsets} {act}")
    rows, E, K, N = 300, 3, 136, 72
    wide = 2 * N if act == "swiglu" else N
    g, at = ref.gen(5), Guarded()
    x, w, d = ref.normal((rows, K), g), ref.normal((E, wide, K), g), ref.normal((rows, N), g)
    pre = ref.normal((rows, wide), g)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    ep.expert_product(x, w, off, act=act, keep_pre=at((rows, wide)), out=at((rows, N)))
    ep.expert_product_grad(x, w, d, off, pre=pre, act=act, dx=at((rows, K)), dw=at((E, wide, K)),
                           dbias=at((E, wide), torch.float32))
    at.check()


@pytest.mark.parametrize("counts,K,N", [([70, 130], 520, 264), ([3000, 0, 100], 136, 72), ([5], 16, 16)])
@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
def test_product_gradient_within_the_workspace_of_its_results(counts, K, N, act):
    """Every choice of results, in a workspace of just the bytes that the query names for it."""
    say(f"product gradient in its own workspace {counts} {K} {N} {act}")
    lib, code = _lib.load(), _lib.EP_ACTIVATIONS[act]
    E, rows, wide = len(counts), sum(counts), 2 * N if act == "swiglu" else N
    g = ref.gen(rows + K)
    x, w, d = ref.normal((rows, K), g), ref.normal((E, wide, K), g), ref.normal((rows, N), g)
    pre = None if act == "none" else ref.normal((rows, wide), g)
    off = torch.tensor([0] + counts, device="cuda").cumsum(0).int()
    want = ep.expert_product_grad(x, w, d, off, pre=pre, act=act, with_bias=True)
    need = {}
    for dx, dw, db in ((1, 1, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)):
        at, n = Guarded(), ctypes.c_size_t()
        flags = db * _lib.EP_GRAD_DBIAS | (not dx) * _lib.EP_GRAD_WITHOUT_DX | (not dw) * _lib.EP_GRAD_WITHOUT_DW
        assert lib.ep_expert_product_grad_workspace_bytes(rows, E, K, N, code, flags, ctypes.byref(n)) == _lib.EP_OK
        need[dx, dw, db] = n.value
        outs = [at((rows, K)) if dx else None, at((E, wide, K)) if dw else None, at((E, wide), torch.float32) if db else None]
        work = at((n.value,), torch.uint8)
        ptr = [t.data_ptr() if t is not None else None for t in (x, off, w, pre, d, *outs, work)]
        assert lib.ep_expert_product_grad(ptr[0], rows, ptr[1], E, ptr[2], K, N, code, ptr[3], ptr[4], ptr[5], ptr[6], ptr[7],
                                          ptr[8], n.value, torch.cuda.current_stream().cuda_stream) == _lib.EP_OK
        at.check()
        for got, name in zip(outs, ("dx", "dw", "dbias")):
            assert got is None or torch.equal(got, getattr(want, name)), (dx, dw, db, name)
    assert need[1, 0, 0] == (0 if act == "none" else -(-rows * wide * 2 // 256) * 256)     # dz and nothing else
    assert need[0, 0, 1] == need[1, 0, 1] - need[1, 0, 0]                                   # no dz
