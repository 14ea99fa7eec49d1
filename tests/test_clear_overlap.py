"""Calls of the cleartext operators in which one address is given twice: refused on the host for every pair of an output and an input or another output
(the addresses are never followed, no GPU is needed)."""
import itertools

import pytest

import paper_2608_17442_b200 as fesc
from test_clear_args import A, BIG, norm_desc, refused, scan_desc

L = fesc.lib()
# name: (entry point, descriptor, arguments in order, outputs, arguments behind them, pairs that may be one buffer)
CALLS = {
    "clear_scan": (L.fesc_clear_scan, scan_desc(), ["x", "g", "B", "C", "skip", "h0", "lengths", "y", "h_out"], ["y", "h_out"], [A[15], BIG, None], []),
    "clear_scan_backward": (L.fesc_clear_scan_backward, scan_desc(),
                            ["x", "g", "B", "C", "skip", "h0", "lengths", "dy", "dh_out", "dx", "dg", "dB", "dC", "dskip", "dh0"],
                            ["dx", "dg", "dB", "dC", "dskip", "dh0"], [A[15], BIG, None], []),
    "clear_scan_step": (L.fesc_clear_scan_step, scan_desc(), ["x", "g", "B", "C", "skip", "state", "state_out", "y"], ["state_out", "y"], [None], [("state", "state_out")]),
    "clear_norm": (L.fesc_clear_norm, norm_desc(), ["y", "gamma", "gate", "residual", "scale", "n", "h"], ["n", "h"], [None], []),
    "clear_norm_backward": (L.fesc_clear_norm_backward, norm_desc(),
                            ["y", "gamma", "gate", "residual", "scale", "dn", "dh", "dy", "dgamma", "dgate", "dresidual", "dscale"],
                            ["dy", "dgamma", "dgate", "dresidual", "dscale"], [A[15], BIG, None], []),
}
PAIRS = [(k, a, b) for k, (_, _, names, outs, _, fine) in CALLS.items() for a, b in itertools.combinations(names, 2) if (a in outs or b in outs) and (a, b) not in fine]


@pytest.mark.parametrize("call, a, b", PAIRS)
def test_an_address_given_twice_is_refused(call, a, b):
    f, d, names, _, rest, _ = CALLS[call]
    at = dict(zip(names, A))
    at[b] = at[a]
    refused(f(d, *at.values(), *rest), "an input" if call != "clear_scan_step" else "clear_scan_step: y is an input")
