"""Refusals of the cleartext operators and sizes of their workspaces: checked on the host before anything is launched, so no GPU is needed (the
addresses are never followed)."""
import ctypes

import pytest

import paper_2608_17442_b200 as fesc

A = [4096 * (i + 1) for i in range(20)]         # distinct aligned addresses


def scan_desc(batch=2, L=100, H=4, P=64, G=2, N=128, type=0, **strides):
    d = fesc.ClearScanDesc(batch, L, H, P, G, N, type)
    full = {"x": (L * H * P, H * P, P), "g": (L * H, H, 1), "B": (L * G * N, G * N, N)}
    for k in ("x", "y", "g", "B", "C", "dx", "dg", "dB", "dC"):
        getattr(d, k)[:] = strides.get(k, full[{"y": "x", "dx": "x", "dg": "g", "C": "B", "dB": "B", "dC": "B"}.get(k, k)])
    return d


def refused(rc, text):
    assert rc == fesc.EINVAL
    assert text in fesc.lib().fesc_clear_last_error().decode(), fesc.lib().fesc_clear_last_error()


BIG = 1 << 40


def scan(d, x=A[0], g=A[1], B=A[2], C=A[3], y=A[4], h0=None, h_out=None, work=A[5], nbytes=BIG):
    return fesc.lib().fesc_clear_scan(d, x, g, B, C, None, h0, None, y, h_out, work, nbytes, None)


def scan_backward(d, dx=A[5], dg=A[6], dB=A[7], dC=A[8], dskip=None, dh0=None, work=A[9], nbytes=BIG):
    return fesc.lib().fesc_clear_scan_backward(d, A[0], A[1], A[2], A[3], None, None, None, A[4], None, dx, dg, dB, dC, dskip, dh0, work, nbytes, None)


@pytest.mark.parametrize("change, text", [
    (dict(type=3), "type"), (dict(H=0), "empty"), (dict(P=0), "empty"), (dict(N=0), "empty"), (dict(G=0), "empty"), (dict(G=3), "divide"), (dict(N=129), "128"),
    (dict(P=4097), "4096"), (dict(L=1 << 30), "2^30"), (dict(batch=65536), "too many"), (dict(batch=60000, L=1 << 29), "too many"),
    (dict(x=(-1, 256, 64)), "negative"), (dict(B=(0, -8, 0)), "negative"), (dict(y=(0, 256, 64)), "overlap"), (dict(y=(25600, 256, 63)), "overlap"),
    (dict(y=(25600, 255, 64)), "overlap"), (dict(x=(1 << 41, 256, 64)), "2^40")])
def test_scan_refuses_descriptors(change, text):
    refused(scan(scan_desc(**change)), text)
    if "y" not in change:        # y holds the strides of dy there, which may overlap
        refused(scan_backward(scan_desc(**change)), text)


def test_scan_refuses_buffers():
    d = scan_desc()
    for k in ("x", "g", "B", "C", "y"):
        refused(scan(d, **{k: None}), "have to be given")
    refused(scan(d, y=A[0]), "output is an input")
    refused(scan(d, h0=A[6], h_out=A[6]), "output is an input")
    need = fesc.lib().fesc_clear_scan_work(scan_desc(L=4096))
    assert need > 0
    for work, n in ((None, BIG), (A[5] + 8, BIG), (A[5], need - 1)):
        refused(scan(scan_desc(L=4096), work=work, nbytes=n), "workspace")
    for k in ("dx", "dg", "dB", "dC"):
        refused(scan_backward(d, **{k: None}), "have to be given")
        refused(scan_backward(d, **{k: A[0]}), "output is an input")
    refused(scan_backward(d, dh0=A[5]), "two outputs")
    for k, v in (("dx", (0, 256, 64)), ("dg", (400, 4, 0)), ("dB", (25600, 256, 100)), ("dC", (25600, 0, 128))):
        refused(scan_backward(scan_desc(**{k: v})), "overlap")
    need = fesc.lib().fesc_clear_scan_backward_work(d)
    refused(scan_backward(d, nbytes=need - 1), "workspace")
    f = fesc.lib().fesc_clear_scan_step
    refused(f(d, A[0], A[1], A[2], A[3], None, None, A[5], A[6], None), "have to be given")
    refused(f(d, A[0], A[1], A[2], A[3], None, A[4], A[5], A[0], None), "y is an input")
    refused(f(scan_desc(y=(255, 0, 64)), A[0], A[1], A[2], A[3], None, A[4], A[5], A[6], None), "overlap")
    assert fesc.lib().fesc_clear_scan(None, *[None] * 10, 0, None) == fesc.EINVAL


def test_scan_refuses_log_decays_as_an_output():
    d = scan_desc(type=2)
    refused(scan(d, y=A[1]), "output is an input")
    refused(scan_backward(d, dg=A[1]), "output is an input")
    refused(fesc.lib().fesc_clear_scan_step(d, A[0], A[1], A[2], A[3], None, A[4], A[5], A[1], None), "y is an input")


def test_calls_without_work_succeed_without_a_gpu():
    assert scan(scan_desc(batch=0)) == fesc.OK
    assert fesc.lib().fesc_clear_scan_step(scan_desc(batch=0), *[None] * 9) == fesc.OK
    assert norm(norm_desc(rows=0)) == fesc.OK


def norm_desc(rows=10, d=96, groups=2, type=0, eps=1e-5, **strides):
    n = fesc.ClearNormDesc(rows, d, groups, type, eps)
    for k in ("y", "gate", "residual", "n", "h", "dn", "dh", "dy", "dgate", "dresidual"):
        setattr(n, k + "_stride", strides.get(k, d))
    return n


def norm(d, y=A[0], gamma=A[1], gate=None, residual=None, scale=None, n=A[2], h=None):
    return fesc.lib().fesc_clear_norm(d, y, gamma, gate, residual, scale, n, h, None)


def norm_backward(d, gate=None, residual=None, scale=None, dh=None, dy=A[4], dgamma=A[5], dgate=None, dresidual=None, dscale=None, work=A[9], nbytes=BIG):
    return fesc.lib().fesc_clear_norm_backward(d, A[0], A[1], gate, residual, scale, A[2], dh, dy, dgamma, dgate, dresidual, dscale, work, nbytes, None)


@pytest.mark.parametrize("change, text", [
    (dict(type=7), "type"), (dict(groups=0), "divide"), (dict(groups=5), "divide"), (dict(d=0), "divide"), (dict(d=8193, groups=1), "8192"), (dict(eps=0.0), "eps"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(rows=1 << 31), "rows"), (dict(y=-1), "stride")])
def test_norm_refuses_descriptors(change, text):
    refused(norm(norm_desc(**change)), text)
    refused(norm_backward(norm_desc(**change)), text)


def test_norm_refuses_buffers():
    d = norm_desc()
    refused(norm(d, n=None), "have to be given")
    refused(norm(d, scale=A[3]), "belongs to a residual")
    refused(norm(d, n=A[0]), "output is an input")
    refused(norm(d, residual=A[3], h=A[3]), "output is an input")
    refused(norm(d, h=A[2]), "another output")
    refused(norm(norm_desc(n=95)), "overlap")
    refused(norm_backward(norm_desc(dy=10)), "overlap")
    refused(norm_backward(d, gate=A[3]), "together")
    refused(norm_backward(d, residual=A[3], dresidual=A[6], dscale=A[7]), "together")
    refused(norm_backward(d, dy=A[0]), "output is an input")
    refused(norm_backward(d, dgamma=A[4]), "two outputs")
    refused(norm_backward(d, work=None), "workspace")
    refused(norm_backward(d, nbytes=fesc.lib().fesc_clear_norm_backward_work(d) - 1), "workspace")


def test_workspaces_are_as_large_as_documented_sizes_need_and_not_with_bad_descriptors():
    L = fesc.lib()
    assert L.fesc_clear_scan_work(scan_desc(N=200)) == 0 and L.fesc_clear_norm_backward_work(norm_desc(eps=0.0)) == 0
    assert L.fesc_clear_scan_work(None) == 0 and L.fesc_clear_scan_backward_work(None) == 0
    assert L.fesc_clear_scan_work(scan_desc(batch=1000, L=64)) == 0                      # enough heads: no segments
    # beyond 32 bits
    assert L.fesc_clear_scan_backward_work(scan_desc(batch=64, L=1 << 20)) >= 64 * (1 << 20) * 4 * 128 * 4 * 2 > 1 << 32


def test_the_binding_refuses_tensors():
    import torch

    x = torch.zeros((1, 2, 1, 4), dtype=torch.bfloat16)
    with pytest.raises(fesc.FescError, match="CUDA device"):
        fesc.clear_scan(x, x, x, x, x)
    with pytest.raises(fesc.FescError, match="CUDA device"):
        fesc.clear_norm(x, x, x, 1e-5)
    assert ctypes.sizeof(fesc.ClearScanDesc) == 32 + 9 * 24 and ctypes.sizeof(fesc.ClearNormDesc) == 24 + 80
