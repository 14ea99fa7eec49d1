"""Plain definitions in 64 bits of the cleartext operators, and bounds on how far a result may be from them."""
import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def scan(x, g, B, C, skip=None, h0=None, lengths=None):
    """(y, h_out) token by token; differentiable.  Tokens behind a sequence's end give zeros."""
    b, L, H, P = x.shape
    G, N = B.shape[2:]
    of = torch.arange(H, device=x.device) // (H // G)
    h = h0 if h0 is not None else torch.zeros((b, H, P, N), dtype=x.dtype, device=x.device)
    ys = []
    a = torch.exp(g)
    for t in range(L):
        new = a[:, t, :, None, None] * h + x[:, t, :, :, None] * B[:, t][:, of, None, :]
        y = torch.einsum("bhpn,bhn->bhp", new, C[:, t][:, of])
        if skip is not None:
            y = y + skip[:, None] * x[:, t]
        if lengths is not None:
            live = t < lengths
            new = torch.where(live[:, None, None, None], new, h)
            y = torch.where(live[:, None, None], y, torch.zeros_like(y))
        h = new
        ys.append(y)
    return (torch.stack(ys, 1) if ys else x.clone()), h


def norm(y, gamma, eps, gate=None, residual=None, scale=None, groups=1):
    v = y if gate is None else y * gate / (1 + torch.exp(-gate))
    h = v if residual is None else residual + (v if scale is None else scale * v)
    p = h.reshape(h.shape[0], groups, -1)
    return (p / torch.sqrt((p * p).mean(2, keepdim=True) + eps)).reshape(h.shape) * gamma, h


def wide(t):
    return None if t is None else t.double()


def make(case, seed=0):
    """Inputs of a scan case (b, L, H, P, N, G, type, start, lengths)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    b, L, H, P, N, G = (case[k] for k in ("b", "L", "H", "P", "N", "G"))
    T = TYPES[case["type"]]

    def normal(*s, dtype=T):
        return torch.randn(s, generator=gen, device="cuda").to(dtype)

    f = torch.float32
    s = {"x": normal(b, L, H, P), "B": normal(b, L, G, N), "C": normal(b, L, G, N), "skip": normal(H, dtype=f),
         "g": -torch.exp(torch.rand((b, L, H), generator=gen, device="cuda") * 7 - 6), "dy": normal(b, L, H, P),
         "h0": normal(b, H, P, N, dtype=f) if case.get("start") else None, "dh_out": normal(b, H, P, N, dtype=f) if case.get("start") else None}
    s["lengths"] = torch.tensor(case["lengths"], dtype=torch.int32, device="cuda") if case.get("lengths") else None
    return s


INPUTS = ("x", "g", "B", "C", "skip", "h0")


def gradients(s):
    """Gradients of the plain recurrence by automatic differentiation in 64 bits, keyed as the library's outputs."""
    leaves = {k: wide(s[k]).requires_grad_() for k in INPUTS if s[k] is not None}
    g = {k: leaves.get(k) for k in INPUTS}
    if g["h0"] is None:
        b, _, H, P = s["x"].shape
        g["h0"] = leaves["h0"] = torch.zeros((b, H, P, s["B"].shape[3]), dtype=torch.float64, device="cuda", requires_grad=True)
    y, h = scan(*(g[k] for k in ("x", "g", "B", "C")), g["skip"], g["h0"], s["lengths"])
    total = (y * wide(s["dy"])).sum()
    if s["dh_out"] is not None:
        total = total + (h * wide(s["dh_out"])).sum()
    names = list(leaves)
    got = dict(zip(names, torch.autograd.grad(total, [leaves[k] for k in names], allow_unused=True)))
    return {k: torch.zeros_like(leaves[k]) if v is None else v for k, v in got.items()}


def magnitudes(s):
    """The inputs with their magnitudes in place of their values: sums of them bound what rounding can do (decays are positive as they are)."""
    return {k: (v if v is None or k in ("g", "lengths") else v.abs()) for k, v in s.items()}


def share(case):
    """Rounding of a result before its own, as a share of the sum of the magnitudes behind it.  Numbers cut into two bfloat16 numbers are off by
    2^-18 (each leaves at most 2^-9 of what is cut), the products of their second parts, which are left out, are below 2^-18 twice: at most
    2^-16 over scores and states.  Sums and decays: fewer than 32 + 16 for each chunk of 64 tokens operations in float32, 2^-22 each (the
    tensor cores may cut instead of rounding).  Of float32 inputs and of states three parts are kept: 2^-26 and less, in the second term."""
    chunks = (case["L"] + 63) // 64
    return 2.0 ** -22 * (32 + 16 * chunks), 2.0 ** -16


def off(got, want, bound, T):
    """Largest excess of |got - want| over half a unit in the last place of `want` plus `bound` (numbers above 0 are failures); the smallest
    numbers of a type are a distance apart."""
    d = (got.double() - want).abs() - torch.finfo(T).eps / 2 * (want.abs() + bound) - bound - torch.finfo(T).tiny * torch.finfo(T).eps
    assert torch.isfinite(got).all() and torch.isfinite(want).all()
    return float(d.max()) if d.numel() else -1.0
