"""The cleartext norm with gate and residual and its gradients against the definition in 64 bits; the block it stands in."""
import pytest
import torch

import paper_2608_17442_b200 as fesc
from clear_ref import TYPES, norm, off, scan, wide

pytestmark = pytest.mark.gpu
EPS = 1e-5
F32 = torch.float32


def inputs(rows, d, t, gate, residual, scale, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T = TYPES[t]
    n = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    return {"y": n(rows, d).to(T), "gamma": n(d), "gate": (2 * n(rows, d)).to(T) if gate else None, "residual": n(rows, d).to(T) if residual else None,
            "scale": n(d) if scale else None, "dn": n(rows, d).to(T), "dh": n(rows, d).to(T) if residual else None}


def forward(s, groups=1):
    n = torch.full(s["y"].shape, 7.0, device="cuda", dtype=s["y"].dtype)
    h = torch.full_like(n, 7.0)
    fesc.clear_norm(s["y"], s["gamma"], n, EPS, gate=s["gate"], residual=s["residual"], scale=s["scale"], h=h, groups=groups)
    return n, h


def backward(s, groups=1):
    like = lambda t: None if t is None else torch.full(t.shape, 7.0, device="cuda", dtype=t.dtype)  # noqa: E731
    o = {"y": like(s["y"]), "gamma": like(s["gamma"]), "gate": like(s["gate"]), "residual": like(s["residual"]), "scale": like(s["scale"])}
    fesc.clear_norm_backward(s["y"], s["gamma"], s["dn"], o["y"], o["gamma"], EPS, gate=s["gate"], dgate=o["gate"], residual=s["residual"],
                             dresidual=o["residual"], scale=s["scale"], dscale=o["scale"], dh=s["dh"], groups=groups)
    return {k: v for k, v in o.items() if v is not None}


def reference(s, groups):
    names = [k for k in ("y", "gamma", "gate", "residual", "scale") if s[k] is not None]
    leaves = {k: wide(s[k]).requires_grad_() for k in names}
    n, h = norm(leaves["y"], leaves["gamma"], EPS, leaves.get("gate"), leaves.get("residual"), leaves.get("scale"), groups)
    total = (n * wide(s["dn"])).sum() + ((h * wide(s["dh"])).sum() if s["dh"] is not None else 0)
    return n.detach(), h.detach(), dict(zip(names, torch.autograd.grad(total, [leaves[k] for k in names])))


CASES = [(1, 1, 1, "fp32", 1, 1, 1), (8, 1536, 1, "bf16", 1, 0, 0), (37, 768, 1, "bf16", 0, 1, 1), (5, 770, 2, "fp32", 1, 1, 1), (3, 2048, 1, "fp16", 1, 1, 0),
         (7, 2050, 1, "bf16", 1, 0, 0), (4, 8192, 1, "fp32", 1, 1, 1), (4, 16384, 2, "bf16", 0, 0, 0), (33, 40, 5, "fp16", 1, 1, 1), (2, 1025, 1, "fp32", 0, 1, 0),
         (1300, 24, 1, "bf16", 1, 1, 1), (3000, 256, 2, "fp32", 1, 0, 0), (9, 513, 1, "bf16", 1, 1, 1), (64, 4096, 1, "bf16", 1, 1, 1)]


@pytest.mark.parametrize("rows, d, groups, t, gate, residual, scale", CASES)
def test_norm_and_gradients_against_the_definition(rows, d, groups, t, gate, residual, scale):
    s = inputs(rows, d, t, gate, residual, scale, rows + d)
    check(s, groups, *forward(s, groups), backward(s, groups))


def check(s, groups, n, h, o):
    (rows, d), T = s["y"].shape, s["y"].dtype
    gate, residual, scale = (s[k] is not None for k in ("gate", "residual", "scale"))
    wn, wh, grads = reference(s, groups)
    # magnitudes of what is summed; a sum of a row is a tree over its threads behind at most 16 terms of a thread: below 32 roundings of 2^-24, the
    # functions 2 units each
    u = 2.0 ** -18
    y, r = wide(s["y"]).abs(), wide(s["residual"]).abs() if residual else 0
    v = y if not gate else y * (wide(s["gate"]).abs() / (1 + torch.exp(-wide(s["gate"]))))
    c = wide(s["scale"]).abs() if scale else 1
    hm = c * v + r
    rho = 1 / torch.sqrt(wh.reshape(rows, groups, -1).square().mean(2, keepdim=True) + EPS)
    spread = lambda m: m.expand(rows, groups, d // groups).reshape(rows, d)  # noqa: E731
    assert off(h, wh, u * hm, T) <= 0
    gamma = wide(s["gamma"]).abs()
    # relative error of the mean square: twice that of h, of which a sum of two terms may keep little
    part = spread(rho ** 2 * (hm * wh.abs()).reshape(rows, groups, -1).mean(2, keepdim=True))
    assert off(n, wn, u * gamma * spread(rho) * (hm + wh.abs() * (1 + part)), T) <= 0
    w = gamma * wide(s["dn"]).abs()
    inner = spread(rho ** 3 * (w * hm).reshape(rows, groups, -1).mean(2, keepdim=True))
    dt = (spread(rho) * w + hm * inner) * (2 + part) + (wide(s["dh"]).abs() if residual else 0)
    if residual:
        assert off(o["residual"], grads["residual"], u * dt, T) <= 0
    dv = c * dt
    slope = 1
    if gate:
        z = wide(s["gate"])
        sig = 1 / (1 + torch.exp(-z))
        slope = z.abs() * sig
        assert off(o["gate"], grads["gate"], u * dv * y * sig * (1 + z.abs() * (1 - sig)), T) <= 0
    assert off(o["y"], grads["y"], u * dv * slope, T) <= 0
    # sums over rows: a thread's own rows one after the other, at most rows / 592 rounded up, then in 64 bits
    k = u + 2.0 ** -23 * (rows / 592 + 10)
    assert off(o["gamma"], grads["gamma"], (k * wide(s["dn"]).abs() * hm * spread(rho) * (2 + part)).sum(0), F32) <= 0
    if scale:
        assert off(o["scale"], grads["scale"], (k * dt * v).sum(0), F32) <= 0


def test_views_unaligned_rows_and_shared_rows():
    s = inputs(50, 96, "bf16", 1, 1, 1, 3)
    n, h = forward(s, 2)
    o = backward(s, 2)
    check(s, 2, n, h, o)
    for extra, shifts in ((16, (0, 8, 16)), (17, (0, 1, 8))):        # rows that allow 16-byte accesses, and rows that do not
        first = None
        for shift in shifts:
            pad = {k: v for k, v in s.items()}
            for k in ("y", "gate", "residual", "dn", "dh"):
                room = torch.zeros((50, 96 + extra), dtype=torch.bfloat16, device="cuda")[:, shift:shift + 96]
                room.copy_(s[k])
                pad[k] = room
            n2, h2 = forward(pad, 2)
            o2 = backward(pad, 2)
            check(s, 2, n2, h2, o2)
            first = first or ((n, h, o) if extra == 16 else (n2, h2, o2))      # a row is added up in one order per kind of access
            assert torch.equal(first[0], n2) and torch.equal(first[1], h2) and all(torch.equal(first[2][k], o2[k]) for k in o)
    one = dict(s, residual=s["residual"][:1].expand(50, 96))
    n2, _ = forward(one)
    n3, _ = forward(dict(s, residual=one["residual"].contiguous()))
    assert torch.equal(n2, n3)


def test_rows_of_zeros_and_extreme_gates():
    s = inputs(4, 100, "fp32", 1, 1, 1, 4)
    s["y"][0], s["residual"][0] = 0, 0
    s["gate"][1], s["gate"][2] = -1e4, 1e4
    n, h = forward(s)
    assert (n[0] == 0).all() and torch.equal(h[1], s["residual"][1]) and torch.isfinite(n).all()
    o = backward(s)
    assert all(torch.isfinite(v).all() for v in o.values()) and (o["y"][1] == 0).all()
    _, _, want = reference(s, 1)
    assert off(o["residual"][0], want["residual"][0], 2.0 ** -18 * want["residual"][0].abs() + 1e-3, F32) <= 0


@pytest.mark.parametrize("rows, d, groups, t, gate", [(5, 770, 2, "fp32", 1), (40, 1536, 1, "bf16", 1), (7, 2050, 1, "fp16", 0), (3, 8192, 1, "bf16", 1)])
def test_the_gradient_of_h_without_a_residual(rows, d, groups, t, gate):
    s = inputs(rows, d, t, gate, 0, 0, d)
    s["dh"] = inputs(rows, d, t, 0, 1, 0, d + 1)["dh"]
    n, h = forward(s, groups)
    o = backward(s, groups)
    wn, wh, grads = reference(s, groups)
    # as in check(), with the magnitude of dh
    u = 2.0 ** -18
    sig = 1 / (1 + torch.exp(-wide(s["gate"]))) if gate else 1
    slope = wide(s["gate"]).abs() * sig if gate else 1
    hm = wide(s["y"]).abs() * slope
    spread = lambda m: m.expand(rows, groups, d // groups).reshape(rows, d)  # noqa: E731
    rho = 1 / torch.sqrt(wh.reshape(rows, groups, -1).square().mean(2, keepdim=True) + EPS)
    w = wide(s["gamma"]).abs() * wide(s["dn"]).abs()
    part = spread(rho ** 2 * (hm * hm).reshape(rows, groups, -1).mean(2, keepdim=True))
    dt = (spread(rho) * w + hm * spread(rho ** 3 * (w * hm).reshape(rows, groups, -1).mean(2, keepdim=True))) * (2 + part) + wide(s["dh"]).abs()
    T = s["y"].dtype
    assert off(o["y"], grads["y"], u * dt * slope, T) <= 0
    if gate:
        assert off(o["gate"], grads["gate"], u * dt * wide(s["y"]).abs() * sig * (1 + wide(s["gate"]).abs() * (1 - sig)), T) <= 0
    assert off(o["gamma"], grads["gamma"], (2 * u * wide(s["dn"]).abs() * hm * spread(rho) * (2 + part)).sum(0), F32) <= 0


def test_a_row_of_zeros_with_a_tiny_eps():
    y, dn = torch.randn((3, 64), device="cuda"), torch.randn((3, 64), device="cuda")
    y[1] = 0
    gamma, dy, dgamma = torch.ones(64, device="cuda"), torch.full((3, 64), 7.0, device="cuda"), torch.empty(64, device="cuda")
    fesc.clear_norm_backward(y, gamma, dn, dy, dgamma, 1e-30)        # 1 / sqrt(eps) = 1e15, its cube is beyond float32
    assert torch.isfinite(dy).all() and torch.isfinite(dgamma).all()
    want = dn[1].double() / torch.tensor(1e-30, dtype=torch.float32).double().sqrt().item()
    assert off(dy[1], want, 2.0 ** -20 * want.abs(), F32) <= 0


def test_streams_graphs_and_the_same_bits_again():
    s = inputs(3000, 768, "bf16", 1, 1, 1, 5)
    n, h = forward(s)
    o = backward(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        n2, h2 = forward(s)
        o2 = backward(s)
    torch.cuda.synchronize()
    assert torch.equal(n, n2) and torch.equal(h, h2) and all(torch.equal(o[k], o2[k]) for k in o)
    if fesc.debug_bounds():      # registers every tensor with the device, which cannot be captured
        return
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        n3, h3 = forward(s)
        o3 = backward(s)
    for _ in range(2):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(n, n3) and torch.equal(h, h3) and all(torch.equal(o[k], o3[k]) for k in o)


def test_no_rows():
    s = inputs(1, 64, "bf16", 1, 1, 1, 6)
    none = {k: (v[:0] if k not in ("gamma", "scale") else v) for k, v in s.items()}
    forward(none)
    o = backward(none)
    assert (o["gamma"] == 0).all() and (o["scale"] == 0).all()


def test_a_block_forward_and_backward():
    """Scan, gated norm, residual norm, as a block runs them (the projections between them are the caller's), against the same chain in 64 bits from the
    library's own rounded intermediates, and the gradients chained through all three."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    b, L, H, P, N = 2, 130, 3, 32, 16
    d = H * P
    n = lambda *sh: torch.randn(sh, generator=gen, device="cuda")  # noqa: E731
    z_x_bc = n(b, L, 2 * d + 2 * N)                      # one projection's output: gate, x, B, C side by side
    z, x = z_x_bc[..., :d], z_x_bc[..., d:2 * d].unflatten(-1, (H, P))
    B, C = z_x_bc[..., 2 * d:2 * d + N].unsqueeze(2), z_x_bc[..., 2 * d + N:].unsqueeze(2)
    g, skip, g1, g2, scale, r = -n(b, L, H).abs(), n(H), n(d), n(d), n(d), n(b, L, d)
    y = torch.empty((b, L, H, P), device="cuda")
    fesc.clear_scan(x, g, B, C, y, skip=skip)
    flat = lambda t: t.reshape(b * L, -1)  # noqa: E731
    rows_z = z_x_bc.view(b * L, -1)[:, :d]
    m1, out, h = (torch.empty((b * L, d), device="cuda") for _ in range(3))
    fesc.clear_norm(flat(y), g1, m1, EPS, gate=rows_z)
    fesc.clear_norm(m1, g2, out, EPS, residual=flat(r), scale=scale, h=h)
    dout, dh = n(b * L, d), n(b * L, d)
    dm1, dr, dy, dz = (torch.empty((b * L, d), device="cuda") for _ in range(4))
    dg1, dg2, ds, dskip = torch.empty(d, device="cuda"), torch.empty(d, device="cuda"), torch.empty(d, device="cuda"), torch.empty(H, device="cuda")
    fesc.clear_norm_backward(m1, g2, dout, dm1, dg2, EPS, residual=flat(r), dresidual=dr, scale=scale, dscale=ds, dh=dh)
    fesc.clear_norm_backward(flat(y), g1, dm1, dy, dg1, EPS, gate=rows_z, dgate=dz)
    dx, dg, dB, dC = torch.empty((b, L, H, P), device="cuda"), torch.empty_like(g), torch.empty((b, L, 1, N), device="cuda"), torch.empty((b, L, 1, N), device="cuda")
    fesc.clear_scan_backward(x, g, B, C, dy.view(b, L, H, P), dx, dg, dB, dC, skip=skip, dskip=dskip)
    leaf = {k: v.detach().double().requires_grad_() for k, v in dict(x=x, g=g, B=B, C=C, skip=skip, z=z, g1=g1, g2=g2, scale=scale, r=r).items()}
    yw, _ = scan(leaf["x"], leaf["g"], leaf["B"], leaf["C"], leaf["skip"])
    mw, _ = norm(flat(yw), leaf["g1"], EPS, gate=flat(leaf["z"]))
    ow, hw = norm(mw, leaf["g2"], EPS, residual=flat(leaf["r"]), scale=leaf["scale"])
    total = (ow * dout.double()).sum() + (hw * dh.double()).sum()
    want = dict(zip(leaf, torch.autograd.grad(total, list(leaf.values()))))
    got = dict(x=dx, g=dg, B=dB, C=dC, skip=dskip, z=dz.view(b, L, d), g1=dg1, g2=dg2, scale=ds, r=dr.view(b, L, d))
    # each of the three steps is off by a few 2^-18 of its magnitudes at most (tests of the steps); a chain of six, with norms that pass
    # errors on as they are on the whole: 2^-14 of the whole
    for a, w in ((out, ow.detach()), (h, hw.detach()), *((got[k], want[k]) for k in leaf)):
        assert float((a.double() - w).norm()) <= 2.0 ** -14 * float(w.norm())
