"""A MoE layer on one GPU out of this package's operators: a training step (forward, backward,
update) and a serving step from 8-bit rows.

    python examples/moe_layer.py [--tokens 512] [--hidden 1024] [--experts 16] [--topk 2] [--steps 8] [--rate 0.1]

The layer is  out = sum over the chosen experts of gate * down(silu(gate_proj n) * up_proj n),
n = rmsnorm(x + residual).  One rank owns every expert here, so ep.pack groups the rows; across
ranks ep.dispatch and ep.combine move the same rows between the two products.
"""
from __future__ import annotations

import argparse
import os
import sys
from dataclasses import dataclass
from typing import Optional

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_40093_amd as ep  # noqa: E402


@dataclass
class Params:
    norm: torch.Tensor    # bf16 [H]
    router: torch.Tensor  # bf16 [1, E, H]
    up: torch.Tensor      # bf16 [E, 2F, H]: gates, then ups
    down: torch.Tensor    # bf16 [E, H, F]
    bias: torch.Tensor    # bf16 [E, H], of the down product


@dataclass
class Grads:
    norm: torch.Tensor
    router: torch.Tensor
    up: torch.Tensor
    down: torch.Tensor
    bias: torch.Tensor
    x: torch.Tensor       # of x and of the residual


def init(hidden: int, ffn: int, experts: int, seed: int = 0) -> Params:
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale):
        return (torch.randn(shape, device="cuda", generator=g) * scale).to(torch.bfloat16)

    return Params(torch.ones(hidden, device="cuda", dtype=torch.bfloat16), normal(1, experts, hidden, scale=hidden ** -0.5),
                  normal(experts, 2 * ffn, hidden, scale=hidden ** -0.5), normal(experts, hidden, ffn, scale=ffn ** -0.5),
                  torch.zeros(experts, hidden, device="cuda", dtype=torch.bfloat16))


class Layer:
    """One forward pass and what its backward reads."""

    def __init__(self, p: Params, topk: int, balance: float = 0.01):
        self.p, self.k, self.balance = p, topk, balance

    def forward(self, x, residual=None, mask: Optional[torch.Tensor] = None):
        """(out, total, balance loss): the layer's output, the residual stream, fp32 [1]."""
        p, (T, H) = self.p, x.shape
        E = p.up.shape[0]
        self.n = ep.rmsnorm(x, p.norm, residual=residual, total=True)
        self.logits = ep.expert_product(self.n.out, p.router, out_dtype=torch.float32).out
        self.routing = ep.route(self.logits, self.k, mask=mask, balance=self.balance)
        self.lay = ep.dispatch_layout(self.routing.topk_idx, E, 1)
        self.rows = ep.pack(self.n.out, self.lay.slot_pos, x.new_empty((T * self.k, H)), topk=self.k)
        offsets = self.lay.expert_offsets
        self.up = ep.expert_product(self.rows, p.up, offsets, act="swiglu", keep_pre=True)
        self.down = ep.expert_product(self.up.out, p.down, offsets, bias=p.bias).out
        out = ep.combine_rows(self.down, self.lay.slot_pos, self.routing.topk_w, torch.empty_like(x))
        return out, self.n.total, self.routing.loss

    def backward(self, d_out, d_total=None, d_loss: Optional[torch.Tensor] = None) -> Grads:
        p, slot_pos, offsets = self.p, self.lay.slot_pos, self.lay.expert_offsets
        d_down, d_gates = ep.combine_grad(d_out, self.down, slot_pos, self.routing.topk_w)
        down = ep.expert_product_grad(self.up.out, p.down, d_down, offsets, with_bias=True)
        up = ep.expert_product_grad(self.rows, p.up, down.dx, offsets, pre=self.up.pre, act="swiglu")
        # the gradient of the grouping: every token's rows added up, with gates of one
        d_n = ep.combine_rows(up.dx, slot_pos, torch.ones_like(d_gates), torch.empty_like(d_out))
        d_logits = ep.route_grad(self.logits, self.routing, d_gates, d_loss)
        router = ep.expert_product_grad(self.n.out, p.router, d_logits.to(torch.bfloat16))
        d_x, d_norm = ep.rmsnorm_grad(self.n.total, p.norm, d_n.add_(router.dx), d_total=d_total)
        return Grads(d_norm, router.dw, up.dw, down.dw, down.dbias, d_x)


@dataclass
class Params8:
    """The same layer for serving: the up product's weights in 8 bits, with a scale per row."""
    p: Params
    up: torch.Tensor
    up_scale: torch.Tensor


def to_8bit(p: Params) -> Params8:
    scale = p.up.abs().amax(2).float().clamp_min(2.0 ** -100) / 448
    return Params8(p, (p.up.float() / scale[:, :, None]).to(torch.float8_e4m3fn), scale)


def serve(q: Params8, x, residual, topk: int):
    """(out, total): the norm writes bf16 rows for the router and 8-bit rows, which carry their
    scales with them, for the experts; grouping moves the 8-bit rows as it moves any."""
    p, (T, H) = q.p, x.shape
    n = ep.rmsnorm(x, p.norm, residual=residual, rows8=True, total=True)
    logits = ep.expert_product(n.out, p.router, out_dtype=torch.float32).out
    routing = ep.route(logits, topk, counts=False)
    lay = ep.dispatch_layout(routing.topk_idx, p.up.shape[0], 1, with_row_src=False)
    rows = ep.rows8_empty(T * topk, H)
    ep.pack(n.rows8.view(torch.int16), lay.slot_pos, rows.view(torch.int16), topk=topk)
    up = ep.expert_product(rows, q.up, lay.expert_offsets, w_scale=q.up_scale, act="swiglu").out
    down = ep.expert_product(up, p.down, lay.expert_offsets, bias=p.bias).out
    out = ep.combine_rows(down, lay.slot_pos, routing.topk_w, torch.empty_like(x))
    return out, n.total


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("tokens", 512), ("hidden", 1024), ("ffn", 512), ("experts", 16), ("topk", 2), ("steps", 8)):
        ap.add_argument(f"--{name}", type=int, default=value)
    ap.add_argument("--rate", type=float, default=0.1)
    a = ap.parse_args()
    torch.manual_seed(0)
    p = init(a.hidden, a.ffn, a.experts)
    x = torch.randn(a.tokens, a.hidden, device="cuda").to(torch.bfloat16)
    want = torch.randn(a.tokens, a.hidden, device="cuda") * 0.1
    one = torch.ones(1, device="cuda")
    for step in range(a.steps):
        layer = Layer(p, a.topk)
        out, _, balance = layer.forward(x)
        off = out.float() - want
        g = layer.backward((off / a.tokens).to(torch.bfloat16), d_loss=one)
        for w, d in ((p.norm, g.norm), (p.router, g.router), (p.up, g.up), (p.down, g.down), (p.bias, g.bias)):
            w.sub_(d.to(w.dtype), alpha=a.rate)
        print(f"step {step}: squared error per token {float(off.square().sum()) / a.tokens:.4f}, "
              f"balance loss {float(balance):.4f}", flush=True)
    out, _, _ = Layer(p, a.topk).forward(x)
    served, _ = serve(to_8bit(p), x, None, a.topk)
    print(f"served from 8-bit rows: {float((served.float() - out.float()).norm() / out.float().norm()):.4f} "
          "of the output's norm away from bf16")


if __name__ == "__main__":
    main()
