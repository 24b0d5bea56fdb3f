"""The example layer (examples/moe_layer.py) as a whole: its training step against torch
autograd in 64 bits with the same experts chosen, and its serving step against its training
forward.

Bounds, in the 2-norm: a bf16 rounding is off by at most 2^-8 of a value.  A result passes at
most ten of them from the inputs on (norm, pre-activation, activation, expert's row, output;
gradient of the row, of the activation, of the rows added up, of the logits, of the stream):
10 * 2^-8.  An 8-bit rounding is off by at most 2^-4 of a value, of the rows and of the weights:
2 * 2^-4 beside them."""
import os
import subprocess
import sys

import pytest
import torch

import layer_ref as ref
from gpu_cases import say

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
import moe_layer  # noqa: E402

pytestmark = pytest.mark.gpu


def near(got, want, bound, what):
    off = float((got.double() - want).norm() / want.norm())
    assert off <= bound, f"{what}: {off:.4g} of its norm off"


@pytest.mark.parametrize("T,H,F,E,k", [(37, 64, 40, 8, 2), (300, 256, 136, 16, 4), (1000, 520, 264, 24, 3)])
def test_training_step(T, H, F, E, k):
    say(f"example layer T={T} H={H} F={F} E={E} k={k}")
    g = ref.gen(T)
    p = moe_layer.init(H, F, E, seed=T)
    p.bias.copy_(ref.normal((E, H), g, 0.1))
    p.norm.copy_(ref.normal(H, g, 0.1) + 1)
    x, r = ref.normal((T, H), g), ref.normal((T, H), g)
    mask = torch.arange(T, device="cuda") % 7 != 3
    d_out, d_total = ref.normal((T, H), g), ref.normal((T, H), g)
    layer = moe_layer.Layer(p, k, balance=0.5)
    out, total, loss = layer.forward(x, r, mask)
    got = layer.backward(d_out, d_total, torch.full((1,), 3.0, device="cuda"))

    leaf = {n: getattr(p, n).double().requires_grad_() for n in ("norm", "router", "up", "down", "bias")}
    s = (x.double() + r.double()).requires_grad_()
    n = s / (s.square().mean(1, keepdim=True) + 1e-6).sqrt() * leaf["norm"]
    z = n @ leaf["router"][0].t()
    idx = layer.routing.topk_idx.long()
    gates = torch.softmax(z.gather(1, idx), 1) * mask[:, None]
    want = torch.zeros((T, H), dtype=torch.float64, device="cuda")
    for e in range(E):
        t, j = torch.nonzero((idx == e), as_tuple=True)
        h = ref.act(n[t] @ leaf["up"][e].t(), "swiglu") @ leaf["down"][e].t() + leaf["bias"][e]
        want = want.index_add(0, t, gates[t, j][:, None] * h)
    live = int(mask.sum())
    counts = torch.bincount(idx[mask].reshape(-1), minlength=E).double()
    want_loss = 0.5 * E * (counts / (live * k) * torch.softmax(z, 1)[mask].sum(0) / live).sum()
    ((d_out.double() * want).sum() + (d_total.double() * s).sum() + 3.0 * want_loss).backward()
    bound = 10 * 2.0 ** -8
    near(out, want.detach(), bound, "out")
    near(total, s.detach(), bound, "total")
    assert abs(float(loss) - float(want_loss.detach())) <= bound * float(want_loss.detach())
    for name in leaf:
        near(getattr(got, name), leaf[name].grad, bound, name)
    near(got.x, s.grad, bound, "x")


def test_serving_step():
    say("example layer: serving from 8-bit rows")
    T, H, F, E, k = 200, 512, 128, 16, 4
    g = ref.gen(1)
    p = moe_layer.init(H, F, E)
    x, r = ref.normal((T, H), g), ref.normal((T, H), g)
    out, total, _ = moe_layer.Layer(p, k).forward(x, r)
    served, total8 = moe_layer.serve(moe_layer.to_8bit(p), x, r, k)
    assert torch.equal(total, total8)
    near(served, out.double(), 2 * 2.0 ** -4 + 10 * 2.0 ** -8, "served")
    one, _ = moe_layer.serve(moe_layer.to_8bit(p), x[:1].contiguous(), r[:1].contiguous(), k)   # a single token
    assert one.shape == (1, H) and torch.isfinite(one).all()


def test_the_command_runs_and_learns():
    say("example layer: the command")
    got = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "moe_layer.py"), "--tokens", "256", "--hidden", "256",
                          "--ffn", "128", "--experts", "8", "--steps", "6"], capture_output=True, text=True, timeout=110)
    assert got.returncode == 0, got.stderr[-2000:]
    errors = [float(line.split("per token ")[1].split(",")[0]) for line in got.stdout.splitlines() if line.startswith("step")]
    assert len(errors) == 6 and errors[-1] < errors[0]
    assert "served from 8-bit rows" in got.stdout
