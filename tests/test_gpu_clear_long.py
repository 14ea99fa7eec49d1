"""The cleartext operators where a CTA has many chunks or rows in a row, and where float32 needs every bit of its operands."""
import pytest
import torch

import paper_2608_17442_b200 as fesc
from clear_ref import make
from test_gpu_clear_norm import backward as norm_backward, check, forward as norm_forward, inputs
from test_gpu_clear_scan import backward, case, check_backward, check_forward, forward

pytestmark = pytest.mark.gpu

# 160 sequences and heads fill the SMs: nothing is cut into segments, and a CTA goes through 9 to 16 chunks of 128 tokens, or twice as many of 64
LONG = [case(4, 2048, 40, 8, 8, 1, "bf16", True), case(4, 1100, 40, 8, 72, 2, "bf16", True, [1100, 1024, 1, 900]), case(4, 1100, 40, 8, 7, 1, "bf16", True),
        case(4, 1100, 40, 8, 16, 4, "fp16", True, [1099, 0, 1100, 640]), case(4, 1100, 40, 8, 16, 1, "fp32", True)]
IDS = ["-".join(str(v) for v in c.values()).replace(" ", "") for c in LONG]


def segments_are_whole(c):
    d = fesc.ClearScanDesc(c["b"], c["L"], c["H"], c["P"], c["G"], 8 * ((c["N"] + 7) // 8), {"bf16": 0, "fp16": 1, "fp32": 2}[c["type"]])
    return fesc.lib().fesc_clear_scan_work(d) == 0


@pytest.mark.parametrize("c", LONG, ids=IDS)
def test_many_chunks_in_a_row_against_the_definition(c):
    assert segments_are_whole(c)
    s = make(c, 40)
    check_forward(s, c, *forward(s))
    check_backward(s, c, backward(s))


@pytest.mark.parametrize("t", ["bf16", "fp16", "fp32"])
def test_calls_of_many_chunks_in_turn_give_their_own_bits_every_time(t):
    """Long, padded and (bfloat16) copied operands in turn, launched back to back; every call's outputs are compared, on the device."""
    sets = [make(case(4, 2048 - 130 * k, 40, 64, n, 1, t, True, lengths), 41 + k) for k, (n, lengths) in enumerate(((128, None), (64, [1918, 5, 1024, 1500]), (37, None)))]
    want = [(forward(s), backward(s)) for s in sets]
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    for k in range(45):
        s, (f, b) = sets[k % 3], want[k % 3]
        got, o = forward(s), backward(s)
        for x, y in ((got[0], f[0]), (got[1], f[1]), *((o[n], b[n]) for n in o)):
            bad += (x != y).any()
    fesc.clear_sync()
    assert int(bad) == 0


@pytest.mark.parametrize("rows, d, groups, t, gate, residual, scale", [(4000, 768, 1, "bf16", 0, 1, 1), (3000, 1536, 1, "bf16", 1, 0, 0), (12000, 24, 1, "bf16", 1, 1, 1),
                                                                       (5000, 770, 2, "fp32", 1, 1, 1), (1000, 4096, 1, "fp16", 1, 1, 1), (700, 8192, 1, "fp32", 1, 0, 0),
                                                                       (9000, 100, 4, "fp16", 0, 0, 0), (2500, 2048, 1, "fp32", 1, 0, 0)])
def test_norm_of_many_rows_a_team_against_the_definition(rows, d, groups, t, gate, residual, scale):
    """More rows than the teams that are resident: a team takes two rows and more, each fetched while the one before is computed."""
    s = inputs(rows, d, t, gate, residual, scale, rows)
    check(s, groups, *norm_forward(s, groups), norm_backward(s, groups))


def test_float32_operands_keep_all_their_bits():
    """One token, channel and column, so that results are products of two or three numbers; all of them are the number that loses most when it is cut into
    two bfloat16 numbers: 2^-17 of itself, each time in the same direction.  Rounding as it is: a product of numbers cut into three is six products,
    the scores join three sums and are cut again: at most 16 operations, 2^-22 each (the tensor cores may cut instead of rounding)."""
    bound = 16 * 2.0 ** -22
    all_ = 1 + torch.arange(1 << 23, device="cuda") * 2.0 ** -23
    rest = all_ - all_.bfloat16().float()
    rest = rest - rest.bfloat16().float()
    v = float(all_[rest.argmax()])
    assert 2 * float(rest.max()) / v > 3 * bound          # two factors cut into two would show
    one = {"device": "cuda", "dtype": torch.float32}
    x, B, C, dy = (torch.full((1, 1, 1, 1), v, **one) for _ in range(4))
    g, h0, zero = torch.zeros((1, 1, 1), **one), torch.full((1, 1, 1, 1), v, **one), torch.zeros((1, 1, 1, 1), **one)
    y, h = torch.empty_like(x), torch.empty_like(h0)

    def near(got, want):
        assert abs(float(got) - want) <= bound * abs(want), (float(got), want)

    fesc.clear_scan(x, g, B, C, y, h_out=h)
    near(y, v ** 3), near(h, v ** 2)
    fesc.clear_scan(zero, g, B, C, y, h0=h0, h_out=h)
    near(y, v ** 2), near(h, v)
    for xi, start in ((x, None), (zero, h0)):
        o = [torch.empty_like(t) for t in (x, g, B, C, h0)]
        fesc.clear_scan_backward(xi, g, B, C, dy, *o[:4], h0=start, dh0=o[4])
        near(o[0], v ** 3), near(o[4], v ** 2)
        near(o[3], v ** 3 if start is None else v ** 2), near(o[2], v ** 3 if start is None else 0.0)
        if start is not None:
            near(o[1], v ** 3)


@pytest.mark.parametrize("t, shift", [("bf16", 0), ("bf16", 1), ("fp16", 0), ("fp32", 0)])
@pytest.mark.parametrize("slow", [0.0, 1e-4])
def test_a_state_that_forgets_little_does_not_lose_to_one_side(t, shift, slow):
    """Positive terms of 4096 tokens.  What 16 tokens add is six products one after the other, each cut by 2^-22 at most: 2^-19.4 in all, to one side.  Adding it to the
    state, and the state's decay, round to either side: 64 chunks with at most four sums and two products, 2^-24 each, are below 2^-19.7 in the mean square, and
    below 2^-17.7 by four of those, with much less in the mean of 2^16 elements.  bfloat16 operands off 16 bytes take the other sweep."""
    b, L, H, P, N = 4, 4096, 40, 16, 24
    gen = torch.Generator(device="cuda").manual_seed(50)
    T = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[t]

    def positive(*shape):
        room = torch.zeros(shape[:-1] + (shape[-1] + 8,), dtype=T, device="cuda")[..., shift:shift + shape[-1]]
        return room.copy_(torch.rand(shape, generator=gen, device="cuda"))

    x, B, C = positive(b, L, H, P), positive(b, L, 1, N), positive(b, L, 1, N)
    g = -slow * torch.rand((b, L, H), generator=gen, device="cuda")
    y, h = torch.empty((b, L, H, P), dtype=T, device="cuda"), torch.empty((b, H, P, N), device="cuda")
    fesc.clear_scan(x, g, B, C, y, h_out=h)
    fesc.clear_sync()
    behind = torch.exp(g.double().flip(1).cumsum(1).flip(1) - g.double())            # decay from a token to the end
    want = torch.einsum("blhp,bln,blh->bhpn", x.double(), B[:, :, 0].double(), behind)
    off = (h.double() - want) / want
    assert abs(float(off.mean())) <= 2.0 ** -19 and float(off.abs().max()) <= 2.0 ** -17, (float(off.mean()), float(off.abs().max()))
