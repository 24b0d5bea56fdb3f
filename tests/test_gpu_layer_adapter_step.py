"""The adapters and dropout together, as a fine-tuning step uses them: a normalised feed-forward block, trained through
adapters beside its fixed weights, against torch autograd in 64 bits with the generator's masks.

Bounds, in the 2-norm: a bf16 rounding is off by at most 2^-8 of a value, and a result passes at most twelve of them from
the inputs on (total, norm, what the activation reads, activation, base, sum; gradient of the sum, of the activation,
of what it reads, of the norm, of the rows through the adapters, of the stream): 12 * 2^-8."""
import pytest
import torch

import adapter_ref as ar
import dropout_ref as dr
import layer_ref as ref
import paper_2609_40093_amd as ep
from gpu_cases import say

pytestmark = pytest.mark.gpu
BOUND = 12 * 2.0 ** -8
P = 0.1


def near(got, want, what):
    off = float((got.double() - want).norm() / want.norm())
    assert off <= BOUND, f"{what}: {off:.4g} of its norm off"


class Block:
    """y = total + dropout(down(up(norm(total)))), total = stream + dropout(x).  up: gated, adapters in the projection's own
    pass; down: dropout before the adapters alone, which then join the base product."""

    def __init__(self, T, H, F, A, R, seed):
        g = ref.gen(seed)
        self.up, self.down = ref.normal((2 * F, H), g, H ** -0.5), ref.normal((H, F), g, F ** -0.5)
        self.norm = ref.normal(H, g, 0.1) + 1
        self.a = [ref.normal((A, R, H), g, H ** -0.5), ref.normal((A, R, F), g, F ** -0.5)]
        self.b = [ref.normal((A, 2 * F, R), g, R ** -0.5), ref.normal((A, H, R), g, R ** -0.5)]
        self.scale = torch.rand(A, device="cuda", generator=g) + 0.5
        self.all = torch.tensor([0, T], dtype=torch.int32, device="cuda")

    def forward(self, x, stream, ids, rng):
        self.x, self.rng, self.by = x, rng, ep.adapter_rows(ids, len(self.scale))
        self.n = ep.dropout_rmsnorm(x, P, rng, self.norm, site=0, residual=stream)
        self.u = ep.adapter_product(self.n.out, self.a[0], self.b[0], self.by, w=self.up, scale=self.scale, act="swiglu",
                                    keep_pre=True, keep_low=True)
        base = ep.expert_product(self.u.out, self.down[None], self.all)
        self.h = ep.dropout(self.u.out, P, rng, site=1)
        self.d = ep.adapter_product(self.h, self.a[1], self.b[1], self.by, scale=self.scale, residual=base.out, keep_low=True)
        return ep.dropout(self.d.out, P, rng, site=2, residual=self.n.total)

    def backward(self, dy):
        dd = ep.dropout(dy, P, self.rng, site=2)
        g1 = ep.adapter_product_grad(self.h, self.a[1], self.b[1], self.d.low, dd, self.by, scale=self.scale)
        base = ep.expert_product_grad(self.u.out, self.down[None], dd, self.all, dw=False)
        du = ep.dropout(g1.dx, P, self.rng, site=1, residual=base.dx)
        g0 = ep.adapter_product_grad(self.n.out, self.a[0], self.b[0], self.u.low, du, self.by, w=self.up, scale=self.scale,
                                     pre=self.u.pre, act="swiglu")
        dx, ds, dn = ep.dropout_rmsnorm_grad(self.n.total, self.norm, g0.dx, P, self.rng, site=0, d_total=dy)
        return {"x": dx, "stream": ds, "norm": dn, "a0": g0.da, "b0": g0.db, "a1": g1.da, "b1": g1.db}

    def exact(self, x, stream, ids, rng, dy):
        """The result and the gradients in 64 bits."""
        leaf = {"x": x, "stream": stream, "norm": self.norm, "a0": self.a[0], "b0": self.b[0], "a1": self.a[1], "b1": self.b[1]}
        leaf = {k: v.double().requires_grad_() for k, v in leaf.items()}
        A = len(self.scale)
        by = torch.cat([self.scale.double(), self.scale.new_zeros(1).double()])[ids.long()][:, None]  # ids of -1: the last

        def adapters(rows, a, b):
            low = rows.new_zeros((rows.shape[0], a.shape[1]))
            out = rows.new_zeros((rows.shape[0], b.shape[1]))
            for e in range(A):
                at = torch.nonzero(ids == e)[:, 0]
                low = low.index_add(0, at, rows[at] @ a[e].t())
                out = out.index_add(0, at, (low[at] * by[at]) @ b[e].t())
            return out

        total = leaf["stream"] + leaf["x"] * dr.factor(x.shape, P, rng, 0)
        n = total / (total.square().mean(1, keepdim=True) + 1e-6).sqrt() * leaf["norm"]
        u = ref.act(n @ self.up.double().t() + adapters(n, leaf["a0"], leaf["b0"]), "swiglu")
        d = u @ self.down.double().t() + adapters(u * dr.factor(u.shape, P, rng, 1), leaf["a1"], leaf["b1"])
        y = total + d * dr.factor(d.shape, P, rng, 2)
        y.backward(dy.double())
        return y.detach(), {k: v.grad for k, v in leaf.items()}


def rng_of(step):
    return torch.tensor([77, step], dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("T,H,F,A,R", [(9, 64, 40, 2, 8), (300, 264, 136, 5, 16), (1500, 520, 776, 24, 40), (5000, 520, 264, 1, 64)])
def test_training_step(T, H, F, A, R):
    say(f"adapters and dropout, a step T={T} H={H} F={F} A={A} R={R}")
    g = ref.gen(T)
    x, stream, dy = ref.normal((T, H), g), ref.normal((T, H), g), ref.normal((T, H), g)
    ids, block = ar.random_ids(T, A, T).int(), Block(T, H, F, A, R, T)
    y = block.forward(x, stream, ids, rng_of(3))
    got = block.backward(dy)
    want_y, want = block.exact(x, stream, ids, rng_of(3), dy)
    near(y, want_y, "y")
    for name in want:
        near(got[name], want[name], name)


def test_two_captured_steps():
    """Two graphs of one memory pool, each of a whole step, replayed in turn with eager steps between."""
    say("adapters and dropout, two captured steps")
    T, H, F, A, R = 200, 264, 136, 5, 16
    g = ref.gen(1)
    x, stream, dy = ref.normal((T, H), g), ref.normal((T, H), g), ref.normal((T, H), g)
    ids, rng = ar.random_ids(T, A, 1).int(), rng_of(0)
    blocks = [Block(T, H, F, A, R, seed) for seed in (1, 2)]

    def step(block):
        return {"y": block.forward(x, stream, ids, rng), **block.backward(dy)}

    for block in blocks:
        step(block)
    torch.cuda.synchronize()
    graphs, held = [], []
    for block in blocks:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=graphs[0].pool() if graphs else None):
            held.append(step(block))
        graphs.append(graph)
    for turn in range(3):
        rng.copy_(rng_of(turn))
        ids.copy_(ar.random_ids(T, A, turn + 5))
        x.copy_(ref.normal((T, H), ref.gen(turn + 9)))
        for graph, block, out in zip(graphs, blocks, held):
            graph.replay()
            torch.cuda.synchronize()
            got = {k: v.clone() for k, v in out.items()}
            want = step(block)
            for k in want:
                assert torch.equal(got[k], want[k]), (turn, k)
