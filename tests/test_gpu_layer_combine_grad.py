"""The combine's gradient against a plain implementation in 64 bits.

dy is one fp32 product rounded to bf16: within 2^-24 and half a bf16 step of the product.
d_topk_w sums H products in fp32, at most H / 64 + 6 roundings deep per term."""
import pytest
import torch

import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say

pytestmark = pytest.mark.gpu


def check(T, k, H, rows, pos, seed):
    g = ref.gen(seed)
    d, y = ref.normal((T, H), g), ref.normal((rows, H), g)
    w = torch.randn((T, k), device="cuda", generator=g)
    out = torch.full((rows, H), 7.0, dtype=torch.bfloat16, device="cuda")
    dy, dw = ep.combine_grad(d, y, pos.reshape(-1), w, dy=out)
    assert dy is out
    has = (pos >= 0) & (pos < rows)
    at = pos.long()
    want = torch.full((rows, H), 7.0, dtype=torch.float64, device="cuda")  # rows that no slot names keep what they hold
    want[at[has]] = (w.double()[:, :, None] * d.double()[:, None, :])[has]
    named = torch.zeros(rows, dtype=torch.bool, device="cuda")
    named[at[has]] = True
    ref.within(dy, want, want.abs() * (ref.BF16 + 2.0 ** -20), "dy")
    assert (out[~named] == 7.0).all()
    terms = y.double()[torch.where(has, at, 0)] * d.double()[:, None, :] * has[:, :, None]
    ref.within(dw, terms.sum(2), terms.abs().sum(2) * (H / 64 + 8) * ref.U24, "d_topk_w")
    assert not dw[~has].any()
    for a, b in ((True, False), (False, True)):
        one = ep.combine_grad(d, y, pos.reshape(-1), w, dy=out.clone().fill_(7.0) if a else False, d_topk_w=b)
        assert (one[0] is None) == (not a) and (one[1] is None) == (not b)
        assert torch.equal(one[0], dy) if a else torch.equal(one[1], dw)


@pytest.mark.parametrize("H", [8, 64, 512, 520, 2048, 2056, 2888, 7168])
@pytest.mark.parametrize("k", [1, 2, 3, 6, 8, 9])
def test_shapes(k, H):
    say(f"combine_grad k={k} H={H}")
    for T in (1, 67):
        g = ref.gen(T * k * H)
        check(T, k, H, T * k, torch.randperm(T * k, device="cuda", generator=g).int().view(T, k), T)


@pytest.mark.parametrize("k", [1, 5, 8])
def test_slots_without_rows(k):
    say(f"combine_grad with missing slots k={k}")
    T, H = 301, 264
    g = ref.gen(k)
    rows = T * k + 9
    pos = torch.randperm(rows, device="cuda", generator=g)[:T * k].int().view(T, k)
    drop = torch.rand((T, k), device="cuda", generator=g)
    pos[drop < 0.3] = -1
    pos[drop > 0.9] = rows + 3
    pos[5] = 2 ** 31 - 1
    check(T, k, H, rows, pos, k)


def test_no_tokens_and_no_rows():
    e = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    dy, dw = ep.combine_grad(e, e, torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty((0, 2), device="cuda"))
    assert dy.shape == (0, 64) and dw.shape == (0, 2)
    d = torch.ones((3, 64), dtype=torch.bfloat16, device="cuda")
    dy, dw = ep.combine_grad(d, e, torch.zeros(6, dtype=torch.int32, device="cuda"), torch.ones((3, 2), device="cuda"))
    assert dy.shape == (0, 64) and not dw.any()


def test_it_is_the_gradient_of_combine_rows():
    """<d_out, combine_rows(y, w)> changes along (u, v) as <dy, u> + <dw, v>: the combine is linear
    in each, so a difference of any step is exact but for the fp32 output's rounding."""
    say("combine_grad against combine_rows")
    T, k, H = 40, 4, 256
    g = ref.gen(1)
    pos = torch.randperm(T * k, device="cuda", generator=g).int()
    y, d, w = ref.normal((T * k, H), g), ref.normal((T, H), g), torch.randn((T, k), device="cuda", generator=g)
    u = ref.normal((T * k, H), g)
    dy, dw = ep.combine_grad(d, y, pos, w)

    def out(a, b):
        return ep.combine_rows(a, pos, b, torch.empty((T, H), device="cuda")).double()

    along_y = (d.double() * out(u, w)).sum()
    assert abs((dy.double() * u.double()).sum() - along_y) <= (dy.double() * u.double()).abs().sum() * 2.0 ** -7
    v = torch.randn((T, k), device="cuda", generator=g)
    along_w = (d.double() * out(y, v)).sum()
    size = (d.double().abs() * out(y.abs(), v.abs())).sum()
    assert abs((dw.double() * v.double()).sum() - along_w) <= size * 2.0 ** -18


def test_rows_past_4_gib():
    """Rows whose byte offsets pass 32 bits."""
    say("combine_grad past 4 GiB")
    T, k, H = 3, 2, 4096
    rows = (1 << 32) // (H * 2) + 70000
    y = torch.empty((rows, H), dtype=torch.bfloat16, device="cuda")
    dy = torch.empty_like(y)
    pos = torch.tensor([rows - 1, 5, (1 << 31) // (H * 2) + 1, (1 << 32) // (H * 2) + 1, 0, rows - 2], dtype=torch.int32, device="cuda")
    g = ref.gen(3)
    y[pos.long()] = ref.normal((6, H), g)
    d, w = ref.normal((T, H), g), torch.randn((T, k), device="cuda", generator=g)
    _, dw = ep.combine_grad(d, y, pos, w, dy=dy)
    want = w.double().view(6, 1) * d.double().repeat_interleave(2, 0)
    ref.within(dy[pos.long()], want, want.abs() * (ref.BF16 + 2.0 ** -20), "dy")
    terms = y[pos.long()].double() * d.double().repeat_interleave(2, 0)
    ref.within(dw.view(-1), terms.sum(1), terms.abs().sum(1) * (H / 64 + 8) * ref.U24, "d_topk_w")


def test_new_dy_of_a_buffer_with_more_rows_than_slots():
    """Rows behind the last slot's are zeros in a new dy, whatever its memory held."""
    say("combine_grad: a new dy with rows that no slot names")
    T, k, H, more = 50, 3, 264, 37
    g = ref.gen(4)
    d, y, w = ref.normal((T, H), g), ref.normal((T * k + more, H), g), torch.rand((T, k), device="cuda", generator=g)
    pos = torch.randperm(T * k + more, device="cuda", generator=g)[:T * k].int()
    want, _ = ep.combine_grad(d, y, pos, w, dy=torch.zeros_like(y))
    for stream in (None, torch.cuda.Stream()):
        for _ in range(3):
            held = torch.full_like(y, float("nan"))
            torch.cuda.synchronize()
            del held                                # a new tensor of this size is likely to get its memory
            dy, _ = ep.combine_grad(d, y, pos, w, stream=stream)
            torch.cuda.synchronize()
            assert torch.equal(dy, want)
