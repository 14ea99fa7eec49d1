"""The cleartext operators at the edges of what they promise: addresses, dropped states, buffers of autograd, waits that run out."""
import pytest
import torch

import paper_2608_17442_b200 as fesc
from clear_ref import make
from test_gpu_clear_scan import backward, case, check_backward, check_forward, forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("c", [case(2, 131, 2, 40, 24, 2, "bf16", True), case(3, 300, 3, 72, 128, 1, "bf16", True, [300, 129, 1]), case(1, 70, 3, 64, 64, 1, "bf16"),
                               case(2, 200, 1, 33, 127, 1, "bf16", True), case(2, 90, 3, 40, 72, 1, "fp16", True), case(1, 131, 2, 64, 128, 1, "fp32", True)],
                         ids=lambda c: "-".join(str(v) for v in c.values()).replace(" ", ""))
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_log_decays_at_any_address(c, shift):
    """g and its gradient as a column range of a wider float32 buffer, on 4 or 8 bytes, where the other operands lie on 16."""
    s = make(c, 30)
    b, L, H = s["g"].shape
    room = torch.full((b, L, H + 3 + shift), float("nan"), device="cuda")
    g = room[..., shift:shift + H]
    g.copy_(s["g"])
    assert g.data_ptr() % 16 == 4 * shift
    s["g"] = g
    check_forward(s, c, *forward(s))
    o = backward(s)
    room_out = torch.full((b, L, H + 3 + shift), 7.0, device="cuda")
    dg = room_out[..., shift:shift + H]
    rest = {k: torch.empty_like(o[k]) for k in ("x", "B", "C")}
    fesc.clear_scan_backward(s["x"], g, s["B"], s["C"], s["dy"], rest["x"], dg, rest["B"], rest["C"], skip=s["skip"], h0=s["h0"], dh_out=s["dh_out"], lengths=s["lengths"])
    assert torch.equal(dg, o["g"]) and (room_out[..., :shift] == 7.0).all() and (room_out[..., shift + H:] == 7.0).all()
    check_backward(s, c, o)


def test_a_wait_that_runs_out_at_a_kernels_end_is_reported_too():
    fesc.clear_sync()
    fesc.clear_selftest_wait_limit()
    with pytest.raises(fesc.FescError, match="still under way") as e:
        fesc.clear_sync()
    assert e.value.code == fesc.ETIMEOUT
    fesc.clear_sync()


@pytest.mark.parametrize("t", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("L, drop, P, N", [(1, 0, 64, 128), (40, 17, 40, 24), (300, 150, 64, 128), (1500, 700, 40, 72), (1500, 1024, 64, 128)])
def test_a_dropped_state_leaves_nothing_behind_also_an_infinite_one(L, drop, P, N, t):
    """A log decay of -inf between infinities and finite tokens: what lies on the far side is what it is without them, bit for bit."""
    s = make(case(2, L, 2, P, N, 1, t, True), 31)
    s["g"][:, drop] = -float("inf")
    y, h = forward(s)
    o = backward(s)
    # states before the drop: outputs and gradients from the drop on
    lost = dict(s, h0=s["h0"].clone())
    lost["h0"][:, 0], lost["h0"][0, 1] = float("inf"), float("nan")
    y2, h2 = forward(lost)
    o2 = backward(lost)
    assert torch.isfinite(h).all() and torch.equal(h, h2) and torch.equal(y[:, drop:], y2[:, drop:])
    for k in ("g", "C"):
        assert torch.equal(o[k][:, drop:], o2[k][:, drop:]), k
    for k in ("x", "B", "skip", "h0"):
        assert torch.equal(o[k], o2[k]), k
    # gradients of the state behind the drop: gradients before it
    lost = dict(s, dh_out=s["dh_out"].clone())
    lost["dh_out"][:, 1], lost["dh_out"][1, 0] = -float("inf"), float("nan")
    o2 = backward(lost)
    for k in ("x", "B", "g"):
        assert torch.equal(o[k][:, :drop], o2[k][:, :drop]), k
    for k in ("C", "skip", "h0"):
        assert torch.equal(o[k], o2[k]), k
    assert (o2["g"][:, drop] == 0).all()


def test_one_token_and_a_scan_of_one_token_drop_alike():
    s = make(case(3, 1, 2, 40, 24, 1, "fp32", True), 32)
    s["g"][0], s["g"][1] = -float("inf"), -150.0          # both are decays of zero in float32
    s["h0"][:2] = float("inf")
    y, h = forward(s)
    y1, h1 = torch.empty_like(s["x"][:, 0]), torch.empty_like(h)
    fesc.clear_scan_step(s["x"][:, 0], s["g"][:, 0], s["B"][:, 0], s["C"][:, 0], s["h0"], y1, skip=s["skip"], state_out=h1)
    assert all(torch.isfinite(v).all() for v in (y, h, y1, h1))
    assert (h[:2] - h1[:2]).abs().max() <= 2.0 ** -20 * h1[:2].abs().max()      # one product each


def test_what_a_call_writes_counts_as_changed_in_place():
    s = make(case(1, 70, 2, 40, 24, 1, "bf16", True), 33)
    f = {"device": "cuda", "dtype": torch.float32}

    def written(call, *outputs):
        before = [t._version for t in outputs]
        call()
        assert all(t._version > v for t, v in zip(outputs, before))

    y, h = torch.empty_like(s["x"]), torch.empty_like(s["h0"])
    written(lambda: fesc.clear_scan(s["x"], s["g"], s["B"], s["C"], y, h_out=h), y, h)
    o = [torch.empty_like(s[k]) for k in ("x", "g", "B", "C", "skip", "h0")]
    written(lambda: fesc.clear_scan_backward(s["x"], s["g"], s["B"], s["C"], s["dy"], *o[:4], skip=s["skip"], dskip=o[4], h0=s["h0"], dh0=o[5]), *o)
    token = [s[k][:, 0] for k in ("x", "g", "B", "C")]
    written(lambda: fesc.clear_scan_step(*token, h, y[:, 0]), h, y)            # in place; a view counts for its base
    other = torch.empty_like(h)
    left = h._version
    written(lambda: fesc.clear_scan_step(*token, h, y[:, 0], state_out=other), other, y)
    assert h._version == left and s["x"]._version == 0
    rows, gamma = torch.randn((6, 48), **f), torch.randn(48, **f)
    n, hh = torch.empty_like(rows), torch.empty_like(rows)
    written(lambda: fesc.clear_norm(rows, gamma, n, 1e-5, h=hh), n, hh)
    d = [torch.empty_like(t) for t in (rows, gamma, rows, rows, gamma)]
    written(lambda: fesc.clear_norm_backward(rows, gamma, n, d[0], d[1], 1e-5, gate=hh, dgate=d[2], residual=rows, dresidual=d[3], scale=gamma, dscale=d[4]), *d)
    # autograd notices: the values that this product's gradient needs are gone
    w = torch.ones((6, 48), **f, requires_grad=True)
    total = (w * n).sum()
    fesc.clear_norm(rows, gamma, n, 1e-5)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        total.backward()
    with torch.inference_mode():
        fesc.clear_norm(rows, gamma, torch.empty_like(rows), 1e-5)


def test_a_workspace_that_does_not_fit_is_torchs_own_error():
    """64 x 2^20 tokens of four heads, all of them the same one in memory: the partial sums alone would take 256 GB."""
    x, g, B = (torch.zeros((1, 1, 1, *n), device="cuda").expand(64, 1 << 20, h, *n) for n, h in (((64,), 4), ((), 4), ((128,), 1)))
    with pytest.raises(torch.cuda.OutOfMemoryError):
        fesc.clear_scan_backward(x, g, B, B, x, x, g, B, B)
    with pytest.raises(fesc.FescError, match="overlap"):          # with a workspace the call is refused: outputs of one token's memory
        fesc.clear_scan_backward(x, g, B, B, x, x, g, B, B, work=torch.empty(256, dtype=torch.uint8, device="cuda"))


def test_the_gate_of_float32_rows_is_as_exact_as_float32():
    """h = y z / (1 + exp(-z)) over the gate's range: the exponential and the reciprocal are off by one unit (2^-23) at most, the sum and the two products
    by half a unit each: 3.5 x 2^-23 < 2^-21.  Backwards sigma (1 + z (1 - sigma)) as well, with 1 - sigma and the sum around it off by units of terms that do not exceed 1 + |z|."""
    gen = torch.Generator(device="cuda").manual_seed(34)
    d = 4096
    z = (torch.rand((2, d), generator=gen, device="cuda") * 100 - 80)
    y, dh = (torch.randn((2, d), generator=gen, device="cuda") for _ in range(2))
    gamma, n, h = torch.ones(d, device="cuda"), torch.empty_like(y), torch.empty_like(y)
    fesc.clear_norm(y, gamma, n, 1e-5, gate=z, h=h)
    sig = 1 / (1 + torch.exp(-z.double()))
    want = y.double() * z.double() * sig
    assert ((h.double() - want).abs() <= 2.0 ** -21 * want.abs() + 2.0 ** -149).all()
    # dn of zero: dy = dh silu(z), dz = dh y sigma (1 + z (1 - sigma))
    dy, dgamma, dz = torch.empty_like(y), torch.empty_like(gamma), torch.empty_like(y)
    fesc.clear_norm_backward(y, gamma, torch.zeros_like(y), dy, dgamma, 1e-5, gate=z, dgate=dz, dh=dh)
    want = dh.double() * z.double() * sig
    assert ((dy.double() - want).abs() <= 2.0 ** -21 * want.abs() + 2.0 ** -149).all()
    want = dh.double() * y.double() * sig * (1 + z.double() * (1 - sig))
    size = (dh.double() * y.double()).abs() * sig * (1 + z.double().abs())
    assert ((dz.double() - want).abs() <= 2.0 ** -21 * size + 2.0 ** -149).all()
