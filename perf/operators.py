"""The cleartext operators of a Mamba-2 block: plain forms, cases and what each cannot do without.

A case is one call: `op` (scan, scan_backward, step, norm, norm_backward), a type and sizes.  With `own` false `run` computes
the operator with elementary torch operations in 32 bits (sums of log decays in 64), with `own` true it calls the library.
Outputs are buffers that the state holds; rows of a padded batch behind a sequence's end stay zero in them.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
CHUNK = 64      # tokens per quadratic piece of the plain scan


def listed():
    block = {"H": 24, "P": 64, "N": 128, "G": 1}        # the deployed layer: 24 heads of 64 channels, d_s = 128
    return [
        # one new token of one document: latency
        {"name": "step_one", "op": "step", "type": "bf16", "b": 1, **block},
        # one new token of many documents: the states are larger than L2
        {"name": "step_many", "op": "step", "type": "bf16", "b": 192, **block},
        # one document of the benchmark's length, as served or checked against decrypted results
        {"name": "scan_document", "op": "scan", "type": "bf16", "b": 1, "L": 2048, **block, "start": False, "ragged": False},
        # a prefill or a training batch: the largest
        {"name": "scan_batch", "op": "scan", "type": "bf16", "b": 16, "L": 4096, **block, "start": False, "ragged": False},
        # a padded batch that continues from earlier states, odd sizes, two groups, full precision
        {"name": "scan_ragged", "op": "scan", "type": "fp32", "b": 5, "L": 777, "H": 6, "P": 40, "N": 24, "G": 2, "start": True,
         "ragged": True},
        # a training step on one document
        {"name": "scan_backward_document", "op": "scan_backward", "type": "bf16", "b": 1, "L": 2048, **block, "start": False,
         "ragged": False},
        # a training step on a batch
        {"name": "scan_backward_batch", "op": "scan_backward", "type": "bf16", "b": 8, "L": 2048, **block, "start": False,
         "ragged": False},
        # truncated back-propagation through a padded batch, odd sizes, full precision
        {"name": "scan_backward_ragged", "op": "scan_backward", "type": "fp32", "b": 3, "L": 331, "H": 4, "P": 72, "N": 56, "G": 1,
         "start": True, "ragged": True},
        # the gated norm of a few new tokens: latency
        {"name": "norm_tokens", "op": "norm", "type": "bf16", "rows": 8, "d": 1536, "groups": 1, "gate": True, "residual": False},
        # residual, layer scale and the next block's norm over a batch
        {"name": "norm_batch", "op": "norm", "type": "bf16", "rows": 32768, "d": 768, "groups": 1, "gate": False, "residual": True},
        # the gated norm's backward pass over a training batch
        {"name": "norm_backward_batch", "op": "norm_backward", "type": "bf16", "rows": 16384, "d": 1536, "groups": 1, "gate": True,
         "residual": False},
        # everything at once, odd width, full precision
        {"name": "norm_backward_odd", "op": "norm_backward", "type": "fp32", "rows": 999, "d": 770, "groups": 2, "gate": True,
         "residual": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["scan", "scan_backward", "step", "norm", "norm_backward"])
    t = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("norm", "norm_backward"):
        groups = rng.choice([1, 1, 2, 3])
        d = groups * _log(rng, 40 // groups, 4000 // groups)
        rows = _log(rng, 1, min(32768, 24000000 // d))
        gate, residual = rng.choice([(True, False), (False, True), (True, True), (False, False)])
        return {"op": op, "type": t, "rows": rows, "d": d, "groups": groups, "gate": gate, "residual": residual}
    G = rng.choice([1, 1, 2])
    H = G * rng.randint(1, 12)
    P, N = rng.choice([64, 64, rng.randint(1, 128)]), rng.choice([128, 64, rng.randint(1, 128)])
    if op == "step":
        b = _log(rng, 1, 192)
        return {"op": op, "type": t, "b": b, "H": H, "P": P, "N": N, "G": G}
    b = _log(rng, 1, 16)
    L = _log(rng, 1, (8192 if op == "scan" else 4096) // b)
    return {"op": op, "type": t, "b": b, "L": L, "H": H, "P": P, "N": N, "G": G, "start": rng.random() < 0.5, "ragged": rng.random() < 0.5}


def _lengths(case, seed):
    """Lengths of a padded batch: one sequence is full, one empty, one a single token, the others anything."""
    b, L = case["b"], case["L"]
    if not case["ragged"]:
        return None
    few = [L, 0, 1]
    return [few[i] if i < 3 else (2654435761 * (i + 1) + seed * 40503) % (L + 1) for i in range(b)]


def _inputs(case, seed):
    """The call's inputs, from the seed alone, on the GPU."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T = TYPES[case["type"]]

    def normal(*shape, scale=1.0, dtype=T):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)

    def uniform(*shape, lo=0.0, hi=1.0):
        return torch.rand(shape, generator=gen, device="cuda") * (hi - lo) + lo

    op, f = case["op"], torch.float32
    if op in ("norm", "norm_backward"):
        rows, d = case["rows"], case["d"]
        s = {"y": normal(rows, d), "gamma": uniform(d, lo=0.5, hi=1.5)}
        if case["gate"]:      # a column range of the input projection's output, which is wider
            s["gate"] = normal(rows, 2 * d)[:, :d]
        if case["residual"]:
            s["residual"], s["scale"] = normal(rows, d), uniform(d, lo=0.1, hi=1.0)
        if op == "norm_backward":
            s["dn"] = normal(rows, d)
            if case["residual"]:
                s["dh"] = normal(rows, d)
        return s
    b, L, H, P, N, G = case["b"], case.get("L", 1), case["H"], case["P"], case["N"], case["G"]
    width = H * P + 2 * G * N      # x, B and C lie side by side, as the convolution leaves them
    xbc = normal(b, L, width)
    s = {"x": xbc[..., :H * P].unflatten(-1, (H, P)), "B": xbc[..., H * P:H * P + G * N].unflatten(-1, (G, N)),
         "C": xbc[..., H * P + G * N:].unflatten(-1, (G, N)), "skip": uniform(H, lo=0.5, hi=1.5)}
    # decays exp(-dt A): from ones that forget in a few tokens to ones that remember thousands
    s["g"] = -torch.exp(uniform(b, L, H, lo=math.log(1e-3), hi=0.0)) * uniform(H, lo=0.05, hi=2.0)
    if op == "step":
        s = {k: v[:, 0] if k not in ("skip",) else v for k, v in s.items()}
        s["state"] = normal(b, H, P, N, dtype=f)
        return s
    if case["start"]:
        s["h0"] = normal(b, H, P, N, dtype=f)
    lengths = _lengths(case, seed)
    if lengths is not None:
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if op == "scan_backward":
        s["dy"] = normal(b, L, H, P)
        s["dh_out"] = normal(b, H, P, N, dtype=f, scale=0.1)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op, T = case["op"], TYPES[case["type"]]
    f = {"device": "cuda", "dtype": torch.float32}
    s["case"] = case
    if op in ("norm", "norm_backward"):
        rows, d = case["rows"], case["d"]
        new = lambda: torch.zeros((rows, d), device="cuda", dtype=T)  # noqa: E731
        if op == "norm":
            s["out"] = {"n": new()}
            if case["residual"]:
                s["out"]["h"] = new()
        else:
            s["out"] = {"dy": new(), "dgamma": torch.zeros(d, **f)}
            if case["gate"]:
                s["out"]["dgate"] = new()
            if case["residual"]:
                s["out"]["dresidual"], s["out"]["dscale"] = new(), torch.zeros(d, **f)
        return s
    b, L, H, P, N, G = case["b"], case.get("L", 1), case["H"], case["P"], case["N"], case["G"]
    if op == "step":
        s["out"] = {"y": torch.zeros((b, H, P), device="cuda", dtype=T), "state": torch.zeros((b, H, P, N), **f)}
    elif op == "scan":
        s["out"] = {"y": torch.zeros((b, L, H, P), device="cuda", dtype=T), "h_out": torch.zeros((b, H, P, N), **f)}
    else:
        s["out"] = {"dx": torch.zeros((b, L, H, P), device="cuda", dtype=T), "dg": torch.zeros((b, L, H), **f),
                    "dB": torch.zeros((b, L, G, N), device="cuda", dtype=T), "dC": torch.zeros((b, L, G, N), device="cuda", dtype=T),
                    "dskip": torch.zeros(H, **f), "dh0": torch.zeros((b, H, P, N), **f)}
    return s


def run(state):
    case, op = state["case"], state["case"]["op"]
    if own:
        import paper_2608_17442_b200 as fesc

        s, o = state, state["out"]
        if op == "step":
            fesc.clear_scan_step(s["x"], s["g"], s["B"], s["C"], s["state"], o["y"], skip=s["skip"], state_out=o["state"])
        elif op == "scan":
            fesc.clear_scan(s["x"], s["g"], s["B"], s["C"], o["y"], skip=s["skip"], h0=s.get("h0"), h_out=o["h_out"],
                            lengths=s.get("lengths"))
        elif op == "scan_backward":
            fesc.clear_scan_backward(s["x"], s["g"], s["B"], s["C"], s["dy"], o["dx"], o["dg"], o["dB"], o["dC"], skip=s["skip"],
                                     dskip=o["dskip"], h0=s.get("h0"), dh_out=s["dh_out"], dh0=o["dh0"], lengths=s.get("lengths"))
        elif op == "norm":
            fesc.clear_norm(s["y"], s["gamma"], o["n"], 1e-5, gate=s.get("gate"), residual=s.get("residual"), scale=s.get("scale"),
                            h=o.get("h"), groups=case["groups"])
        else:
            fesc.clear_norm_backward(s["y"], s["gamma"], s["dn"], o["dy"], o["dgamma"], 1e-5, gate=s.get("gate"), dgate=o.get("dgate"),
                                     residual=s.get("residual"), dresidual=o.get("dresidual"), scale=s.get("scale"),
                                     dscale=o.get("dscale"), dh=s.get("dh"), groups=case["groups"])
        return o
    return {"step": _step, "scan": _scan, "scan_backward": _scan_backward, "norm": _norm, "norm_backward": _norm_backward}[op](state)


# ---- plain forms ------------------------------------------------------------------------------------------------------------


def _step(s):
    x, B, C = s["x"].float(), _heads(s["B"].float(), s), _heads(s["C"].float(), s)
    h = torch.exp(s["g"])[..., None, None] * s["state"] + x[..., None] * B[:, :, None, :]
    y = (h * C[:, :, None, :]).sum(-1) + s["skip"][:, None] * x
    return {"y": y.to(s["x"].dtype), "state": h}


def _heads(t, s):
    """[..., G, N] -> [..., H, N]"""
    return t.repeat_interleave(s["case"]["H"] // s["case"]["G"], dim=-2)


def _sweep(q, k, v, g, h):
    """out_t = sum_{s<=t} exp(g_{s+1} + .. + g_t) (q_t . k_s) v_s + exp(g_0 + .. + g_t) q_t h, and the state behind the last token.
    q, k [b,L,H,K], v [b,L,H,V], g [b,L,H] in 64 bits, h [b,H,K,V]; L a multiple of CHUNK."""
    b, L, H, K = q.shape
    c = L // CHUNK
    q, k, v = (t.view(b, c, CHUNK, H, -1).transpose(2, 3) for t in (q, k, v))                  # [b,c,H,Q,*]
    cum = g.view(b, c, CHUNK, H).transpose(2, 3).cumsum(-1)                                     # [b,c,H,Q]
    total = cum[..., -1]
    low = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=q.device).tril()
    decay = torch.exp((cum[..., :, None] - cum[..., None, :]).masked_fill(~low, -math.inf)).float()
    out = ((q @ k.transpose(-1, -2)) * decay) @ v
    local = (k * torch.exp(total[..., None] - cum).float()[..., None]).transpose(-1, -2) @ v    # [b,c,H,K,V]
    # states before every chunk: the start and the chunks before it, each decayed by the chunks between
    along = torch.cat([torch.zeros_like(total[:, :1]), total.cumsum(1)], 1)                     # [b,c+1,H]
    lower = torch.ones(c + 1, c + 1, dtype=torch.bool, device=q.device).tril()
    over = torch.exp((along[:, :, None] - along[:, None, :]).masked_fill(~lower[..., None], -math.inf)).float()
    pieces = torch.cat([h[:, None], local], 1)                                                  # piece i enters before chunk i
    states = (over.permute(0, 3, 1, 2) @ pieces.transpose(1, 2).flatten(3)).unflatten(-1, local.shape[-2:]).transpose(1, 2)
    out = out + torch.exp(cum).float()[..., None] * (q @ states[:, :-1])
    return out.transpose(2, 3).reshape(b, L, H, -1), states[:, -1]


def _padded(s):
    """x, g, B, C (per head) and dy in 32 bits (g in 64) with zeros behind the sequences' ends, and the count of tokens."""
    L = s["x"].shape[1]
    pad = -L % CHUNK
    keep = None
    if "lengths" in s:
        keep = torch.arange(L, device="cuda")[None, :, None, None] < s["lengths"][:, None, None, None]

    def full(t, wide=False):
        t = t.double() if wide else t.float()
        if keep is not None:
            t = torch.where(keep if t.dim() == 4 else keep[..., 0], t, torch.zeros_like(t))
        return torch.nn.functional.pad(t, (0, 0) * (t.dim() - 2) + (0, pad))

    g = full(s["g"], True).clamp(min=-1000.0)
    got = [full(s["x"]), g, _heads(full(s["B"]), s), _heads(full(s["C"]), s)]
    return got + [full(s["dy"])] if "dy" in s else got


def _start(s):
    c = s["case"]
    return s["h0"] if "h0" in s else torch.zeros((c["b"], c["H"], c["P"], c["N"]), device="cuda")


def _scan(s):
    x, g, B, C = _padded(s)
    L = s["x"].shape[1]
    y, h = _sweep(C, B, x, g, _start(s).transpose(-1, -2))
    y = (y + s["skip"][:, None] * x)[:, :L]
    return {"y": y.to(s["x"].dtype), "h_out": h.transpose(-1, -2).contiguous()}


def _scan_backward(s):
    T, L, G = s["x"].dtype, s["x"].shape[1], s["case"]["G"]
    x, g, B, C, dy = _padded(s)
    dC, h_last = _sweep(dy, x, B, g, _start(s))
    # backwards in time: the decay between two tokens belongs to the later one
    g_back = torch.cat([torch.zeros_like(g[:, :1]), g.flip(1)[:, :-1]], 1)
    xr, Br, Cr, dyr = (t.flip(1) for t in (x, B, C, dy))
    dx, _ = _sweep(Br, Cr, dyr, g_back, s["dh_out"].transpose(-1, -2))
    dB, dh = _sweep(xr, dyr, Cr, g_back, s["dh_out"])
    dx, dB = dx.flip(1) + s["skip"][:, None] * dy, dB.flip(1)
    row, col = (C * dC).sum(-1, dtype=torch.float64), (B * dB).sum(-1, dtype=torch.float64)
    end = (h_last.double() * s["dh_out"].double()).sum((-1, -2))
    dg = (row - col).flip(1).cumsum(1).flip(1) + end[:, None]
    if "lengths" in s:
        keep = torch.arange(dg.shape[1], device="cuda")[None, :, None] < s["lengths"][:, None, None]
        dg = torch.where(keep, dg, torch.zeros_like(dg))
    groups = lambda t: t[:, :L].unflatten(2, (G, -1)).sum(3).to(T)  # noqa: E731
    return {"dx": dx[:, :L].to(T), "dg": dg[:, :L].float(), "dB": groups(dB), "dC": groups(dC),
            "dskip": (dy * x).sum((0, 1, 3), dtype=torch.float64).float(), "dh0": torch.exp(g[:, 0]).float()[..., None, None] * dh}


def _norm_parts(s):
    y, groups = s["y"].float(), s["case"]["groups"]
    v = y * (s["gate"].float() * torch.sigmoid(s["gate"].float())) if "gate" in s else y
    h = s["residual"].float() + s["scale"] * v if "residual" in s else v
    rho = torch.rsqrt(h.unflatten(-1, (groups, -1)).square().mean(-1, keepdim=True) + 1e-5).expand(-1, -1, y.shape[-1] // groups)
    return y, v, h, rho.flatten(1)


def _norm(s):
    T = s["y"].dtype
    _, _, h, rho = _norm_parts(s)
    out = {"n": (s["gamma"] * h * rho).to(T)}
    if "residual" in s:
        out["h"] = h.to(T)
    return out


def _norm_backward(s):
    T, groups = s["y"].dtype, s["case"]["groups"]
    y, v, h, rho = _norm_parts(s)
    w = s["gamma"] * s["dn"].float()
    mean = (w * h).unflatten(-1, (groups, -1)).mean(-1, keepdim=True).expand(-1, -1, y.shape[-1] // groups).flatten(1)
    d = rho * w - h * rho * rho * rho * mean
    out = {"dgamma": (s["dn"].float() * h * rho).sum(0, dtype=torch.float64).float()}
    if "residual" in s:
        d = d + s["dh"].float()
        out["dresidual"], out["dscale"] = d.to(T), (d * v).sum(0, dtype=torch.float64).float()
        d = s["scale"] * d
    if "gate" in s:
        z = s["gate"].float()
        sig = torch.sigmoid(z)
        out["dgate"] = (d * y * sig * (1 + z * (1 - sig))).to(T)
        d = d * z * sig
    out["dy"] = d.to(T)
    return {k: out[k] for k in ("dy", "dgamma", "dgate", "dresidual", "dscale") if k in out}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------


def work(case):
    e = 4 if case["type"] == "fp32" else 2
    op = case["op"]
    if op in ("norm", "norm_backward"):
        n = case["rows"] * case["d"]
        tensors = (1 if op == "norm" else 3) + (1 if op == "norm" else 0)                      # y, n or y, dn, dy
        tensors += case["gate"] * (1 if op == "norm" else 2) + case["residual"] * (2 if op == "norm" else 3)
        return {"bytes": n * e * tensors + 4 * case["d"] * (1 + (op != "norm")) * (1 + case["residual"]),
                "flops": n * (12 if op == "norm" else 30)}
    b, H, P, N, G = (case[k] for k in ("b", "H", "P", "N", "G"))
    states = b * H * P * N * 4
    if op == "step":
        return {"bytes": 2 * states + b * (e * (2 * H * P + 2 * G * N) + 4 * H), "flops": 5 * b * H * P * N}
    tokens = b * case["L"]
    if case["ragged"]:
        tokens = sum(_lengths(case, 0))
    if op == "scan":
        return {"bytes": tokens * (e * (2 * H * P + 2 * G * N) + 4 * H) + states * (1 + case["start"]), "flops": 5 * tokens * H * P * N}
    return {"bytes": tokens * (e * (3 * H * P + 4 * G * N) + 8 * H) + states * (2 + case["start"]), "flops": 15 * tokens * H * P * N}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------


def exact(case, seed):
    s = _inputs(case, seed)
    d = {k: (v.double() if v.is_floating_point() else v) for k, v in s.items()}
    op = case["op"]
    if op in ("norm", "norm_backward"):
        return _exact_norm(case, d)
    H, G = case["H"], case["G"]
    of = torch.arange(H, device="cuda") // (H // G)             # the group of a head
    a = torch.exp(d["g"])
    if op == "step":
        h = a[:, :, None, None] * d["state"] + d["x"][:, :, :, None] * d["B"][:, of, None, :]
        return {"y": torch.einsum("bhpn,bhn->bhp", h, d["C"][:, of]) + d["skip"][None, :, None] * d["x"], "state": h}
    b, L, P, N = case["b"], case["L"], case["P"], case["N"]
    length = d["lengths"] if "lengths" in d else torch.full((b,), L, device="cuda")
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    h = d["h0"] if "h0" in d else torch.zeros((b, H, P, N), dtype=torch.float64, device="cuda")

    def after(h, t):
        new = a[:, t, :, None, None] * h + d["x"][:, t, :, :, None] * d["B"][:, t][:, of, None, :]
        return torch.where((t < length)[:, None, None, None], new, h)

    if op == "scan":
        y = torch.zeros((b, L, H, P), dtype=torch.float64, device="cuda")
        for t in range(L):
            h = after(h, t)
            got = torch.einsum("bhpn,bhn->bhp", h, d["C"][:, t][:, of]) + d["skip"][None, :, None] * d["x"][:, t]
            y[:, t] = torch.where((t < length)[:, None, None], got, zero)
        return {"y": y, "h_out": h}
    # states are kept every so many tokens and computed again between
    every, kept = 64, []
    for t in range(L):
        if t % every == 0:
            kept.append(h)
        h = after(h, t)
    out = {k: torch.zeros_like(d[n]) for k, n in (("dx", "x"), ("dg", "g"), ("dB", "B"), ("dC", "C"))}
    dskip, dh = torch.zeros(H, dtype=torch.float64, device="cuda"), d["dh_out"]
    for first in reversed(range(0, L, every)):
        before = [kept[first // every]]
        for t in range(first, min(first + every, L)):
            before.append(after(before[-1], t))
        for t in reversed(range(first, min(first + every, L))):
            live = t < length
            dy, x = d["dy"][:, t], d["x"][:, t]
            total = dh + dy[..., None] * d["C"][:, t][:, of, None, :]
            by_group = lambda v: v.unflatten(1, (G, -1)).sum(2)  # noqa: E731
            row = {"dx": torch.einsum("bhpn,bhn->bhp", total, d["B"][:, t][:, of]) + d["skip"][None, :, None] * dy,
                   "dB": by_group(torch.einsum("bhpn,bhp->bhn", total, x)),
                   "dC": by_group(torch.einsum("bhpn,bhp->bhn", before[t - first + 1], dy)),
                   "dg": a[:, t] * torch.einsum("bhpn,bhpn->bh", before[t - first], total)}
            for k, v in row.items():
                out[k][:, t] = torch.where(live.view(-1, *[1] * (v.dim() - 1)), v, zero)
            dskip = dskip + torch.where(live[:, None], (dy * x).sum(-1), zero).sum(0)
            dh = torch.where(live[:, None, None, None], a[:, t, :, None, None] * total, dh)
    return {**out, "dskip": dskip, "dh0": dh}


def _exact_norm(case, d):
    groups = case["groups"]
    leaves = {k: d[k].clone().requires_grad_() for k in ("y", "gamma", "gate", "residual", "scale") if k in d}
    with torch.enable_grad():
        h = leaves["y"]
        if "gate" in d:
            h = h * leaves["gate"] / (1 + torch.exp(-leaves["gate"]))
        if "residual" in d:
            h = leaves["residual"] + leaves["scale"] * h
        per = h.reshape(case["rows"], groups, -1)
        n = (per / (per.pow(2).mean(2, keepdim=True) + 1e-5).sqrt()).reshape(h.shape) * leaves["gamma"]
        if case["op"] == "norm":
            return {"n": n.detach(), "h": h.detach()} if "residual" in d else {"n": n.detach()}
        total = (n * d["dn"]).sum() + ((h * d["dh"]).sum() if "dh" in d else 0)
        grads = dict(zip(leaves, torch.autograd.grad(total, list(leaves.values()))))
    return {"d" + k: grads[k] for k in ("y", "gamma", "gate", "residual", "scale") if k in grads}
