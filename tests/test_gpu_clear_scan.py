"""The cleartext gated linear recurrence, its gradients and its single token against the definition in 64 bits."""
import pytest
import torch

import paper_2608_17442_b200 as fesc
from clear_ref import TYPES, gradients, magnitudes, make, off, scan, share, wide

pytestmark = pytest.mark.gpu


def case(b, L, H, P, N, G=1, type="bf16", start=False, lengths=None):
    return dict(b=b, L=L, H=H, P=P, N=N, G=G, type=type, start=start, lengths=lengths)


CASES = [
    case(1, 1, 1, 1, 1), case(1, 1, 2, 64, 128, type="fp32", start=True), case(2, 63, 2, 64, 128), case(1, 64, 3, 64, 64, 3), case(2, 65, 2, 64, 128, start=True),
    case(1, 130, 4, 40, 24, 2, "fp32", True), case(2, 200, 2, 72, 56, 1, "fp32"), case(2, 129, 2, 72, 65, 2, "fp16", True),
    case(1, 128, 1, 128, 128, 1, "fp16"), case(3, 70, 2, 5, 3, 1, "bf16", True), case(1, 100, 2, 33, 127, 1, "bf16"), case(1, 192, 6, 64, 128, 2, "bf16", True),
    case(5, 150, 2, 64, 128, 1, "bf16", True, [150, 0, 1, 64, 97]), case(4, 90, 4, 40, 24, 2, "fp32", True, [0, 90, 65, 1]),
    case(3, 77, 2, 64, 64, 1, "fp16", False, [77, 0, 500]), case(1, 1500, 2, 64, 128, 1, "bf16", True), case(2, 700, 1, 70, 40, 1, "fp32", True, [700, 333]),
    case(1, 40, 2, 200, 16, 1, "bf16"), case(1, 128, 1, 64, 128, 1, "bf16", True), case(3, 400, 50, 64, 128, 2, "bf16", True), case(1, 1000, 4, 72, 96, 2, "bf16", True),
    case(5, 300, 30, 40, 72, 1, "bf16", True, [300, 129, 128, 1, 0]), case(1, 257, 2, 200, 128, 1, "bf16"), case(2, 640, 2, 8, 80, 1, "bf16", True, [600, 7]),
    case(1, 900, 150, 16, 128, 1, "bf16", True), case(40, 130, 4, 64, 72, 4, "bf16"),
]
IDS = ["-".join(str(v) for v in c.values()).replace(" ", "") for c in CASES]


def forward(s, y=None, **kw):
    b, L, H, P = s["x"].shape
    y = torch.full_like(s["x"], 7.0) if y is None else y
    h = torch.full((b, H, P, s["B"].shape[3]), 7.0, device="cuda")
    fesc.clear_scan(s["x"], s["g"], s["B"], s["C"], y, skip=s["skip"], h0=s["h0"], h_out=h, lengths=s["lengths"], **kw)
    return y, h


def backward(s, **kw):
    x, B, g = s["x"], s["B"], s["g"]
    b, L, H, P = x.shape
    o = {"x": torch.full(x.shape, 7.0, device="cuda", dtype=x.dtype), "g": torch.full(g.shape, 7.0, device="cuda"), "B": torch.full(B.shape, 7.0, device="cuda", dtype=x.dtype),
         "C": torch.full(B.shape, 7.0, device="cuda", dtype=x.dtype), "skip": torch.full((H,), 7.0, device="cuda"), "h0": torch.full((b, H, P, B.shape[3]), 7.0, device="cuda")}
    fesc.clear_scan_backward(x, g, B, s["C"], s["dy"], o["x"], o["g"], o["B"], o["C"], skip=s["skip"], dskip=o["skip"] if s["skip"] is not None else None, h0=s["h0"],
                             dh_out=s["dh_out"], dh0=o["h0"], lengths=s["lengths"], **kw)
    return o


def dead(s, L):
    """[b, L]: tokens behind a sequence's end"""
    if s["lengths"] is None:
        return None
    return torch.arange(L, device="cuda")[None] >= s["lengths"].clamp(0, L)[:, None]


def check_forward(s, c, y, h):
    fesc.clear_sync()
    T = s["x"].dtype
    want, hw = scan(*(wide(s[k]) for k in ("x", "g", "B", "C", "skip", "h0")), s["lengths"])
    m = magnitudes(s)
    ym, hm = scan(*(wide(m[k]) for k in ("x", "g", "B", "C", "skip", "h0")), s["lengths"])
    sums, cut = share(c)
    gone = dead(s, c["L"])
    if gone is not None:
        assert (y[gone] == 7.0).all()
        y = y.masked_fill(gone[..., None, None], 0.0)
    assert off(y, want, (sums + (cut if T != torch.float32 else 0)) * ym, T) <= 0
    assert off(h, hw, sums * hm, torch.float32) <= 0


def check_backward(s, c, o):
    fesc.clear_sync()
    T = s["x"].dtype
    want, m = gradients(s), gradients(magnitudes(s))
    sums, cut = share(c)
    gone = dead(s, c["L"])
    if gone is not None:
        for k in ("x", "g", "B", "C"):
            assert (o[k][gone] == 7.0).all(), k
            o[k] = o[k].masked_fill(gone.view(*gone.shape, *[1] * (o[k].dim() - 2)), 0.0)
    assert off(o["x"], want["x"], (sums + (cut if T != torch.float32 else 0)) * m["x"], T) <= 0
    for k in ("B", "C"):
        assert off(o[k], want[k], sums * m[k], T) <= 0, k
    assert off(o["skip"], want["skip"], sums * m["skip"], torch.float32) <= 0 if s["skip"] is not None else True
    assert off(o["h0"], want["h0"], sums * m["h0"], torch.float32) <= 0
    # the log decays' gradient is summed back from a segment's end, at most the sequence's: rows and columns of all heads and tokens
    # behind, and what is there
    rows = (wide(s["C"]).abs() * m["C"]).sum((-1, -2)) + (wide(s["B"]).abs() * m["B"]).sum((-1, -2))
    ends = m["g"].amax(1, keepdim=True) + ((m["h0"] * wide(s["h0"]).abs()).sum((-1, -2))[:, None] if s["h0"] is not None else 0)
    behind = rows.flip(1).cumsum(1).flip(1)[..., None] + ends
    assert off(o["g"], want["g"], sums * behind, torch.float32) <= 0
    # and as close as float32 sums are, over all
    d = (o["g"].double() - want["g"]).norm()
    assert d <= 2.0 ** -17 * want["g"].norm() + 2.0 ** -20 * m["g"].norm(), float(d / want["g"].norm())


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_scan_against_the_definition(c):
    s = make(c, 1)
    check_forward(s, c, *forward(s))


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_gradients_against_differentiation_of_the_definition(c):
    s = make(c, 2)
    check_backward(s, c, backward(s))


def test_options_may_be_left_out():
    c = case(2, 70, 2, 24, 16, 1, "fp32")
    s = make(c, 3)
    s["skip"] = None
    y = torch.empty_like(s["x"])
    fesc.clear_scan(s["x"], s["g"], s["B"], s["C"], y)
    want, _ = scan(*(wide(s[k]) for k in ("x", "g", "B", "C")))
    m = magnitudes(s)
    assert off(y, want, share(c)[0] * scan(*(wide(m[k]) for k in ("x", "g", "B", "C")))[0], torch.float32) <= 0
    check_backward(s, c, backward(s))


@pytest.mark.parametrize("kind", ["drop", "strong", "none", "mixed"])
@pytest.mark.parametrize("t", ["bf16", "fp32"])
def test_decays_of_zero_of_one_and_strong_ones(kind, t):
    c = case(2, 150, 2, 40, 72, 1, t, True)
    s = make(c, 4)
    if kind == "drop":
        s["g"][:, 10::37] = -float("inf")
    elif kind == "strong":
        s["g"].mul_(200.0)
    elif kind == "none":
        s["g"].zero_()
    else:
        s["g"][:, ::3] = -250.0
        s["g"][:, 1::3] = -0.0
    check_forward(s, c, *forward(s))
    if kind == "drop":      # differentiation of exp(-inf) * h is fine in 64 bits: 0
        assert (backward(s)["g"][:, 10::37] == 0).all()
    check_backward(s, c, backward(s))


def test_what_lies_behind_a_sequence_is_not_read():
    c = case(3, 140, 2, 64, 128, 1, "bf16", True, [140, 70, 0])
    s = make(c, 5)
    y, h = forward(s)
    o = backward(s)
    gone = dead(s, 140)
    for k in ("x", "B", "C", "dy", "g"):
        s[k][gone] = float("nan")
    y2, h2 = forward(s)
    o2 = backward(s)
    assert torch.equal(y, y2) and torch.equal(h, h2) and all(torch.equal(o[k], o2[k]) for k in o)


def test_negative_and_excessive_lengths_are_taken_into_range():
    c = case(3, 66, 2, 16, 16, 1, "fp32", True, [-5, 66, 1 << 30])
    s = make(c, 6)
    y, h = forward(s)
    s["lengths"] = torch.tensor([0, 66, 66], dtype=torch.int32, device="cuda")
    y2, h2 = forward(s)
    assert torch.equal(y, y2) and torch.equal(h, h2)


@pytest.mark.parametrize("t", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kind", ["columns", "odd", "shifted", "time_major", "shared"])
def test_strides_and_alignment(kind, t):
    c = case(2, 131, 2, 40, 24, 2, t, True)
    s = make(c, 7)
    T, (b, L, H, P, N, G) = TYPES[t], (2, 131, 2, 40, 24, 2)
    r = dict(s)

    def into(base, view):
        view.copy_(base)
        return view

    y = None
    if kind in ("columns", "odd", "shifted"):        # shifted: strides that allow 16-byte accesses, addresses that do not
        extra = {"columns": 8, "odd": 3, "shifted": 1}[kind]
        wide_ = torch.zeros((b, L, H * P + 2 * G * N + {"columns": 16, "odd": 6, "shifted": 8}[kind]), dtype=T, device="cuda")
        cols = wide_[..., extra:]
        r["x"] = into(s["x"], cols[..., :H * P].unflatten(-1, (H, P)))
        r["B"] = into(s["B"], cols[..., H * P:H * P + G * N].unflatten(-1, (G, N)))
        r["C"] = into(s["C"], cols[..., H * P + G * N:H * P + 2 * G * N].unflatten(-1, (G, N)))
        y = torch.zeros((b, L, H, P + extra), dtype=T, device="cuda")[..., extra:]
    elif kind == "time_major":
        for k in ("x", "B", "C", "dy", "g"):
            r[k] = into(s[k], torch.empty_like(s[k].transpose(0, 1).contiguous()).transpose(0, 1))
        r["g"] = into(s["g"], torch.empty((H, L, b), device="cuda").permute(2, 1, 0))
        y = torch.empty((L, b, H, P), dtype=T, device="cuda").transpose(0, 1)
    else:                                # one row of B for all tokens and groups: a stride of zero
        r["B"] = s["B"][:1, :1, :1].expand(b, L, G, N)
    # alignment decides which kernels run: what they give is held to the definition, and to itself
    got, o = forward(r, y), backward(r)
    check_forward(r, c, *got)
    check_backward(r, c, dict(o))
    again = forward(r)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1]) and all(torch.equal(v, backward(r)[k]) for k, v in o.items())


def test_offsets_beyond_32_bits():
    c = case(2, 70, 2, 64, 128, 1, "bf16", True)
    s = make(c, 8)
    want, wo = forward(s), backward(s)
    far = (1 << 32) + 8 * 5
    big = torch.empty(far + 70 * 2 * 64, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided(s["x"].shape, (far, 128, 64, 1))
    x.copy_(s["x"])
    got = forward(dict(s, x=x))
    assert torch.equal(got[0], want[0])
    o = backward(dict(s, x=x))
    assert all(torch.equal(o[k], wo[k]) for k in o)
    y = big.as_strided(s["x"].shape, (far, 128, 64, 1))
    forward(s, y)
    assert torch.equal(y, want[0])


def test_the_same_bits_again_on_another_stream_and_in_two_graphs():
    c = case(1, 900, 2, 64, 128, 1, "bf16", True)
    s, s2 = make(c, 9), make(c, 10)
    want, want2, wo, wo2 = forward(s), forward(s2), backward(s), backward(s2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a, ao = forward(s), backward(s)
    b, bo = forward(s2), backward(s2)                # at the same time
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for got, w in ((a, want), (b, want2)):
        assert torch.equal(got[0], w[0]) and torch.equal(got[1], w[1])
    assert all(torch.equal(ao[k], wo[k]) and torch.equal(bo[k], wo2[k]) for k in wo)
    if fesc.debug_bounds():                          # registers every tensor with the device, which cannot be captured
        return
    held, graphs, outs = {k: v.clone() if v is not None else None for k, v in s.items()}, [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append((forward(held), backward(held)))
        graphs.append(g)
    for src, w, o in ((s, want, wo), (s2, want2, wo2)):
        for k, v in src.items():
            if v is not None:
                held[k].copy_(v)
        for g, (f, back) in zip(graphs, outs):
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(f[0], w[0]) and torch.equal(f[1], w[1]) and all(torch.equal(back[k], o[k]) for k in o)


def test_gradients_against_differences_of_the_forward_kernel():
    """<gradient, d> = (f(+e d) - f(-e d)) / 2e + O(e^2), f = <y, dy> + <h_out, dh_out> in 64 bits from float32 results: with e = 2^-7 the
    results' own rounding (2^-20 of a sum of magnitudes, over 2e) and the third order (e^2 of it) stay below 2^-10 of the magnitudes."""
    c = case(2, 100, 2, 24, 16, 1, "fp32", True)
    s = make(c, 11)
    o = backward(s)
    gen = torch.Generator(device="cuda").manual_seed(12)
    e = 2.0 ** -7

    def f(t):
        y, h = forward(t)
        return float((y.double() * t["dy"].double()).sum() + (h.double() * t["dh_out"].double()).sum())

    y, h = forward(s)
    size = float((y.double() * s["dy"].double()).norm() + (h.double() * s["dh_out"].double()).norm())
    for k in ("x", "g", "B", "C", "skip", "h0"):
        d = torch.randn(s[k].shape, generator=gen, device="cuda")
        if k == "g":
            d = d * s["g"].abs()
        got = (f(dict(s, **{k: s[k] + e * d})) - f(dict(s, **{k: s[k] - e * d}))) / (2 * e)
        want = float((o[k].double() * d.double()).sum())
        assert abs(got - want) <= 2.0 ** -10 * (size + abs(want) + float((o[k].double() * d.double()).norm())), k


@pytest.mark.parametrize("b, H, P, N, G, t", [(1, 24, 64, 128, 1, "bf16"), (3, 4, 40, 24, 2, "fp32"), (2, 2, 7, 1, 1, "fp16"), (40, 24, 64, 128, 1, "bf16"),
                                              (2, 3, 65, 127, 1, "fp32"), (200, 6, 72, 56, 3, "fp16")])
def test_one_token(b, H, P, N, G, t):
    c = case(b, 1, H, P, N, G, t, True)
    s = make(c, 13)
    y, h = torch.empty_like(s["x"][:, 0]), torch.empty_like(s["h0"])
    before = s["h0"].clone()
    args = (s["x"][:, 0], s["g"][:, 0], s["B"][:, 0], s["C"][:, 0], s["h0"])
    fesc.clear_scan_step(*args, y, skip=s["skip"], state_out=h)
    assert torch.equal(s["h0"], before)
    want, hw = scan(*(wide(s[k]) for k in ("x", "g", "B", "C", "skip", "h0")))
    m = magnitudes(s)
    ym, hm = scan(*(wide(m[k]) for k in ("x", "g", "B", "C", "skip", "h0")))
    # a row of at most 128 products, a product and a sum for the state, the decay: fewer than 16 roundings on any way (sums over a lane's
    # four columns and then in a tree), 2^-24 each, the decay 2 units
    assert off(y[:, None], want, 2.0 ** -20 * ym, s["x"].dtype) <= 0 and off(h, hw, 2.0 ** -21 * hm, torch.float32) <= 0
    y2 = torch.empty_like(y)
    fesc.clear_scan_step(*args, y2, skip=s["skip"])        # in place
    assert torch.equal(y, y2) and torch.equal(s["h0"], h)


def test_a_document_then_tokens_equals_one_scan_and_matches_the_recurrence_of_the_encrypted_path():
    """x, a, B, C of the encrypted scan's synthetic inputs: prefill of 90 tokens, ten steps, against the sequential loop the encrypted results
    are held to."""
    import numpy as np

    from oracle.scan import float_recurrence

    rng = np.random.default_rng(3)
    L, H, P, N = 100, 2, 4, 8
    x, a = rng.normal(size=(L, H, P)), rng.uniform(0.9, 1, size=(L, H))
    B, C = rng.normal(size=(2, L, 1, N)) / N ** 0.5
    want = torch.tensor(float_recurrence(x, a, B, C), device="cuda")
    f = {"dtype": torch.float32, "device": "cuda"}
    x, g, B, C = (torch.tensor(v, **f)[None] for v in (x, np.log(a), B, C))
    y, h = torch.empty_like(x), torch.empty((1, H, P, N), **f)
    fesc.clear_scan(x[:, :90], g[:, :90], B[:, :90], C[:, :90], y[:, :90], h_out=h)
    for t in range(90, L):
        fesc.clear_scan_step(x[:, t], g[:, t], B[:, t], C[:, t], h, y[:, t])
    m = torch.tensor(float_recurrence(*(v[0].abs().double().cpu().numpy() for v in (x, g.exp(), B, C))), device="cuda")
    # inputs are rounded to float32 (2^-24 each, log decays 2^-24 of their size a token): below 2^-20 over a hundred tokens
    assert off(y[0], want, (2.0 ** -20 + share({"L": L})[0]) * m, torch.float32) <= 0


def test_empty_calls():
    c = case(2, 1, 2, 8, 8, 1, "bf16", True)
    s = make(c, 14)
    none = {k: (v[:, :0] if k in ("x", "g", "B", "C", "dy") else v) for k, v in s.items()}
    _, h = forward(none)
    assert torch.equal(h, s["h0"])
    o = backward(none)
    assert torch.equal(o["h0"], s["dh_out"]) and (o["skip"] == 0).all()
    nobody = {k: (v[:0] if v is not None and k != "skip" else v) for k, v in s.items()}
    forward(nobody)
    assert (backward(nobody)["skip"] == 0).all()
    fesc.clear_scan_step(*(nobody[k][:, 0] for k in ("x", "g", "B", "C")), nobody["h0"], nobody["x"][:, 0].clone())


def test_a_wait_that_runs_out_is_reported_and_nothing_else_is_lost():
    c = case(1, 300, 2, 64, 128, 1, "bf16", True)
    s = make(c, 15)
    fesc.clear_sync()
    fesc.clear_selftest_wait_limit()
    with pytest.raises(fesc.FescError) as e:
        fesc.clear_sync()
    assert e.value.code == fesc.ETIMEOUT
    check_forward(s, c, *forward(s))       # and a later call is sound again


@pytest.mark.parametrize("t", ["bf16", "fp32"])
def test_many_calls_with_different_inputs_in_turn(t):
    """Three sets of inputs in turn, many times: the waits inside the kernels hold at every interleaving, and each set gives its own bits."""
    sets = [make(case(1, 600 + 17 * k, 4, 64, 128, 1, t, True), 20 + k) for k in range(3)]
    want = [(forward(s), backward(s)) for s in sets]
    for k in range(60):
        s, (f, b) = sets[k % 3], want[k % 3]
        got, o = forward(s), backward(s)
        if k >= 57:
            assert torch.equal(got[0], f[0]) and torch.equal(got[1], f[1]) and all(torch.equal(o[n], b[n]) for n in o)
    fesc.clear_sync()


def test_step_reads_no_length():
    d = fesc.ClearScanDesc(1, 0xffffffff, 1, 8, 1, 8, 2)
    d.x[:], d.y[:], d.g[:], d.B[:], d.C[:] = (0, 0, 0), (0, 0, 0), (0, 0, 0), (0, 0, 0), (0, 0, 0)
    z = {k: torch.ones(n, device="cuda") for k, n in (("x", 8), ("g", 1), ("B", 8), ("C", 8), ("h", 64), ("y", 8))}
    p = {k: v.data_ptr() for k, v in z.items()}
    for v in z.values() if fesc.debug_bounds() else ():       # the binding does it elsewhere
        fesc.lib().fesc_debug_bounds_register(v.data_ptr(), v.numel() * 4)
    assert fesc.lib().fesc_clear_scan_step(d, p["x"], p["g"], p["B"], p["C"], None, p["h"], p["h"], p["y"], fesc._stream()) == fesc.OK
    torch.cuda.synchronize()
    assert torch.allclose(z["h"], torch.full_like(z["h"], 2.718281828 + 1), rtol=1e-6)
