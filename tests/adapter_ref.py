"""Inputs, plain results in 64 bits and bounds of the adapters' tests (test_gpu_layer_adapter*.py).

Bounds: products of bf16 values are exact in fp32; a sum of n terms in any order, each addition rounded
or truncated, is within (n + 8) 2^-23 of the sum of magnitudes (8 more for the scale, the bias, the
residual and the join of partial sums).  The low that a call keeps is rounded to bf16 (2^-8 of it); the low
and the v that are multiplied are the sum of two such values (2^-16).  An activation stretches an error by at most 1.2
(layer_ref.act_error); the gradient's dz is rounded to bf16 and its slope is within 2^-17."""
import torch

import layer_ref as ref
import paper_2609_40093_amd as ep

TWO = ref.BF16 ** 2    # what the sum of two bf16 values leaves of a number


def make(ids, A, R, K, N, seed, act="none", base=True, bias=False, residual=False, scaled=True):
    """ids: each row's adapter, -1 for none; a list or a tensor."""
    g = ref.gen(seed)
    ids = torch.as_tensor(ids, dtype=torch.int32, device="cuda")
    rows, wide = ids.shape[0], 2 * N if act == "swiglu" else N
    return {"ids": ids, "A": A, "R": R, "K": K, "N": N, "act": act, "x": ref.normal((rows, K), g),
            "a": ref.normal((A, R, K), g, K ** -0.5), "b": ref.normal((A, wide, R), g, R ** -0.5),
            "w": ref.normal((wide, K), g, K ** -0.5) if base else None,
            "scale": torch.rand(A, device="cuda", generator=g) + 0.5 if scaled else None,
            "bias": ref.normal(wide, g) if bias else None, "res": ref.normal((rows, N), g) if residual else None}


def sorted_ids(ids, A):
    """The adapters in the order of ep_adapter_rows, A for none; the order; the offsets."""
    ids = torch.where((ids < 0) | (ids >= A), A, ids).long()
    order = torch.sort(ids, stable=True)[1]
    counts = torch.bincount(ids, minlength=A + 1)[:A]
    return ids[order], order, torch.cat([counts.new_zeros(1), counts.cumsum(0)])


def rows_of(s, packed=False):
    """AdapterRows of the ids; `packed` wants ids in the adapters' order already."""
    of, order, offsets = sorted_ids(s["ids"], s["A"])
    if packed:
        assert torch.equal(order, torch.arange(len(order), device="cuda"))
    return ep.AdapterRows(None if packed else order.int(), offsets.int())


def scales(s, of):
    one = torch.ones(s["A"], dtype=torch.float64, device="cuda") if s["scale"] is None else s["scale"].double()
    return torch.cat([one, one.new_zeros(1)])[of][:, None]


def by_adapter(rows, of, weights):
    """rows[i] @ weights[of[i]] (zeros without an adapter), and the sums of the terms' magnitudes."""
    out = rows.new_zeros((rows.shape[0], weights.shape[2]))
    size = torch.zeros_like(out)
    for e in range(weights.shape[0]):
        at = of == e
        out[at] = rows[at] @ weights[e]
        size[at] = rows[at].abs() @ weights[e].abs()
    return out, size


def check(s, packed=False, keep=True, **more):
    """One forward call against 64 bits."""
    of, order, _ = sorted_ids(s["ids"], s["A"])
    rows, N, K, R = s["ids"].shape[0], s["N"], s["K"], s["R"]
    wide = s["b"].shape[1]
    out = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
    pre = torch.full((rows, wide), 7.0, dtype=torch.bfloat16, device="cuda") if keep else False
    low = torch.full((rows, R), 7.0, dtype=torch.bfloat16, device="cuda")
    got = ep.adapter_product(s["x"], s["a"], s["b"], rows_of(s, packed), w=s["w"], scale=s["scale"], bias=s["bias"],
                             act=s["act"], residual=s["res"], keep_pre=pre, keep_low=low, out=out, **more)
    x = s["x"].double()
    want, size = by_adapter(x[order], of, s["a"].double().transpose(1, 2))
    by = scales(s, of)
    off = size * by * (K + 8) * ref.U23
    ref.within(low, want * by, off + ref.BF16 * (want.abs() * by + off), "low")
    b = s["b"].double().transpose(1, 2)
    part, size = by_adapter(want * by, of, b)
    part_off, _ = by_adapter(off + TWO * (want.abs() * by + off), of, b.abs())
    z, all_sizes, z_off = torch.zeros_like(part), torch.zeros_like(part), torch.zeros_like(part)
    z[order], all_sizes[order], z_off[order] = part, size, part_off
    if s["w"] is not None:
        z += x @ s["w"].double().t()
        all_sizes += x.abs() @ s["w"].double().abs().t()
    if s["bias"] is not None:
        z += s["bias"].double()
        all_sizes += s["bias"].double().abs()
    off = z_off + (all_sizes + z_off) * (K + 2 * R + 8) * ref.U23
    if keep:
        ref.within(pre, z, off + ref.BF16 * (z.abs() + off), "pre")
    y, dy = ref.act(z, s["act"]), ref.act_error(z, off, s["act"])
    if s["res"] is not None:
        y = y + s["res"].double()
        dy = dy + (y.abs() + s["res"].double().abs()) * ref.U23
    ref.within(out, y, dy + ref.BF16 * (y.abs() + dy), "y")
    return got


def check_grad(s, packed=False, seed=5, **more):
    """One backward call against 64 bits."""
    of, order, _ = sorted_ids(s["ids"], s["A"])
    rows, N, K, R, A = s["ids"].shape[0], s["N"], s["K"], s["R"], s["A"]
    wide = s["b"].shape[1]
    g = ref.gen(seed)
    d_y, low = ref.normal((rows, N), g), ref.normal((rows, R), g)
    pre = None if s["act"] == "none" else ref.normal((rows, wide), g)
    got = ep.adapter_product_grad(s["x"], s["a"], s["b"], low, d_y, rows_of(s, packed), w=s["w"], scale=s["scale"], pre=pre,
                                  act=s["act"], **more)
    d = d_y.double()
    dz, off = d, torch.zeros_like(d)  # and what dz may be off
    if pre is not None:
        zd = pre.double()
        dz = ref.act_grad(zd, d, s["act"])
        if s["act"] == "swiglu":
            gate, up = zd.chunk(2, 1)
            off = torch.cat([d.abs() * up.abs() * (gate.abs() + 1.2), d.abs() * gate.abs()], 1) * 2.0 ** -17
        else:
            off = d.abs() * (zd.abs() + 1.2) * 2.0 ** -17
        off = off + ref.BF16 * (dz.abs() + off)
    dz, off, x, by = dz[order], off[order], s["x"].double()[order], scales(s, of)
    b, a = s["b"].double(), s["a"].double()
    v, size = by_adapter(dz, of, b)
    v_off = by * (by_adapter(off, of, b.abs())[0] + size * (wide + 8) * ref.U23)
    v = v * by
    v_off = v_off + TWO * (v.abs() + v_off)
    if got.dx is not None:
        dx, size = by_adapter(v, of, a)
        dx_off = by_adapter(v_off, of, a.abs())[0]
        terms = 2 * R
        if s["w"] is not None:
            w = s["w"].double()
            dx, size, dx_off, terms = dx + dz @ w, size + dz.abs() @ w.abs(), dx_off + off @ w.abs(), terms + wide
        dx_off = dx_off + (size + dx_off) * (terms + 8) * ref.U23
        ref.within(got.dx[order], dx, dx_off + ref.BF16 * (dx.abs() + dx_off), "dx")
    for e in range(A):
        at = of == e
        n = int(at.sum())
        if got.da is not None:
            want = v[at].t() @ x[at]
            o = v_off[at].t() @ x[at].abs() + (v[at].abs() + v_off[at]).t() @ x[at].abs() * (2 * n + 8) * ref.U23
            ref.within(got.da[e], want, o + ref.BF16 * (want.abs() + o), f"da {e}")
        if got.db is not None:
            u = low.double()[at]
            want = dz[at].t() @ u
            o = off[at].t() @ u.abs() + (dz[at].abs() + off[at]).t() @ u.abs() * (n + 8) * ref.U23
            ref.within(got.db[e], want, o + ref.BF16 * (want.abs() + o), f"db {e}")
    return got


def random_ids(rows, A, seed, none=0.2):
    g = ref.gen(seed)
    ids = torch.randint(0, A, (rows,), device="cuda", generator=g)
    return torch.where(torch.rand(rows, device="cuda", generator=g) < none, -1, ids)


def packed_ids(counts, none=0):
    return [e for e, n in enumerate(counts) for _ in range(n)] + [-1] * none
