"""grim_glr_sequence, its backward pass and grim_glr_step against the recurrence written out in 64 bits, token by token.

Bounds, carried along with the reference: a gate sigmoid(z) in fp32 is off by (8 + 3 |z|) x 2^-24 of itself (two roundings of
the exponent, which scale with z, and an exponential, an addition, a reciprocal and a product of one unit each), and a state
that takes part in n steps by the sum of what the steps add, scaled by the gates in between -- whether the steps are taken one
after another or composed first.  Every product and sum adds a unit of its own size; 4 per formula cover them."""
import random

import pytest
import torch

import paper_2108_11033_amd as g
from lm_helpers import DTYPES, EPS32, close, out_rows, randn, rows, untouched

TINIEST = 2.0 ** -120          # exponents are cut off at 2^126


def _gate(z):
    s, k = torch.sigmoid(z), torch.sigmoid(-z)
    return s, k, (8 + 3 * z.abs().clamp(max=300)) * EPS32


def reference(gates, bias, h0, starts, dy=None, dh_last=None):
    """(results, slacks): y, h_last and, with dy, dz, dbias, dh0."""
    H = gates.shape[1] // 3
    z = gates.double() + bias.double()
    f, k, df = _gate(z[:, :H])
    o, ko, do = _gate(z[:, 2 * H:])
    c = z[:, H:2 * H]
    N, q = z.shape[0], len(starts) - 1
    h, before, size, err, err_before, size_before = (torch.zeros_like(c) for _ in range(6))
    h_last, h_last_err = h0.double().clone(), torch.zeros_like(h0.double())
    for s in range(q):
        state, big, e = h0[s].double(), h0[s].double().abs(), torch.zeros_like(h0[s].double())
        for t in range(starts[s], starts[s + 1]):
            before[t], size_before[t], err_before[t] = state, big, e
            state = f[t] * state + k[t] * c[t]
            e = f[t] * e + (df[t] + 4 * EPS32) * (f[t] * big + k[t] * c[t].abs())
            big = f[t] * big + k[t] * c[t].abs()
            h[t], size[t], err[t] = state, big, e
        h_last[s], h_last_err[s] = state, e
    out, slack = [o * h, h_last], [o * err + (do + 2 * EPS32) * o * size + TINIEST, h_last_err + TINIEST]
    if dy is None:
        return out, slack
    d = dy.double()
    G, Gs, Ge = torch.zeros_like(c), torch.zeros_like(c), torch.zeros_like(c)
    dh0, dh0_err = dh_last.double().clone(), torch.zeros_like(dh_last.double())
    for s in range(q):
        R, Rs, Re = dh_last[s].double(), dh_last[s].double().abs(), torch.zeros_like(dh_last[s].double())
        for t in range(starts[s + 1] - 1, starts[s] - 1, -1):
            own = d[t] * o[t]
            G[t], Gs[t] = own + R, own.abs() + Rs
            Ge[t] = Re + (do[t] + 4 * EPS32) * own.abs() + 2 * EPS32 * Rs
            R, Rs = f[t] * G[t], f[t] * Gs[t]
            Re = f[t] * Ge[t] + (df[t] + 2 * EPS32) * Rs
        dh0[s], dh0_err[s] = R, Re
    du, dc, dv = G * f * k * (before - c), G * k, d * h * o * ko
    dist = size_before + c.abs()
    eu = f * k * (Ge * dist + Gs * err_before + (3 * df + 6 * EPS32) * Gs * dist)
    ec = k * (Ge + (2 * df + 2 * EPS32) * Gs)
    ev = d.abs() * o * ko * (err + (3 * do + 6 * EPS32) * size)
    dz, ez = torch.cat([du, dc, dv], 1), torch.cat([eu, ec, ev], 1) + TINIEST
    # rows of a chunk, its waves and the sets: fewer additions than rows / 8 + 200 on the way of one term
    return out + [dz, dz.sum(0), dh0], slack + [ez, ez.sum(0) + (N / 8 + 200) * EPS32 * dz.abs().sum(0), dh0_err + TINIEST]


def _uniform(n, q):
    return [n * i // q for i in range(q + 1)]


def _cuts(seed, n, q):
    r = random.Random(seed)
    return [0] + sorted(r.randint(0, n) for _ in range(q - 1)) + [n]


CASES = [
    (1, 1, [0, 1]), (7, 3, [0, 7]), (5, 2, [0, 0, 0, 2, 5, 5]), (64, 33, [0, 1, 2, 33, 64]), (128, 64, _uniform(128, 2)),
    (129, 65, [0, 129]), (200, 261, [0, 0, 8, 8, 9, 16, 199, 200, 200, 200]), (600, 70, list(range(601))), (512, 96, _uniform(512, 8)),
    (300, 40, _cuts(1, 300, 900)), (1100, 1000, _cuts(2, 1100, 70)), (1500, 1024, [0, 1500]), (2500, 515, _cuts(3, 2500, 9)),
]


def _operands(dtype, N, H, q, pad, offset, seed):
    gates, _ = rows(randn(seed, N, 3 * H) * 1.3, dtype, pad, offset)
    bias = 0.3 * randn(seed + 1, 3 * H)
    bias[:H] += 2.0
    dy, _ = rows(randn(seed + 2, N, H), dtype, pad + 1, offset)
    return gates, bias, 0.5 * randn(seed + 3, q, H), dy, randn(seed + 4, q, H)


def _scratch(n):
    return torch.empty(max(1, n), dtype=torch.uint8, device="cuda")


def _train(dtype, gates, bias, h0, seq, q, N, H, dy, dh_last, pad=0, offset=0, ws=None, states=None):
    y, ybuf = out_rows(N, H, dtype, pad, offset)
    dg, dgbuf = out_rows(N, 3 * H, dtype, pad + 2, offset)
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")
    h_last, dbias, dh0 = nan(q, H), nan(3 * H), nan(q, H)
    ws = _scratch(g.glr_workspace(N, H)).fill_(255) if ws is None else ws
    states = _scratch(g.glr_states(N, H)).fill_(255) if states is None else states
    stream = torch.cuda.current_stream()
    g.glr_sequence(gates, dtype, gates.stride(0), bias, h0, seq, q, N, H, y, H + pad, h_last, states, ws, stream)
    g.glr_sequence_backward(gates, dtype, gates.stride(0), bias, h0, seq, q, N, H, states, dy, dy.stride(0), dh_last, dg,
                            3 * H + pad + 2, dbias, dh0, ws, stream)
    assert untouched(y, ybuf) and untouched(dg, dgbuf)
    return [y, h_last, dg, dbias, dh0]


NAMES = ["y", "h_last", "dgates", "dbias", "dh0"]


def _check(got, want, slack, dtype):
    for name, a, b, e in zip(NAMES, got, want, slack):
        close(a, b, e, dtype if name in ("y", "dgates") else "f32", name)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,H,starts", CASES, ids=[f"{n}x{h}s{len(s) - 1}" for n, h, s in CASES])
def test_forward_and_backward(dtype, N, H, starts):
    q = len(starts) - 1
    pad, offset = (0, 0) if N % 2 else (3, 1)
    gates, bias, h0, dy, dh_last = _operands(dtype, N, H, q, pad, offset, 50)
    seq = torch.tensor(starts, dtype=torch.int32, device="cuda")
    got = _train(dtype, gates, bias, h0, seq, q, N, H, dy, dh_last, pad, offset)
    _check(got, *reference(gates, bias, h0, starts, dy, dh_last), dtype)
    again = _train(dtype, gates, bias, h0, seq, q, N, H, dy, dh_last, pad, offset)
    assert all(torch.equal(a, b) for a, b in zip(got, again)), "a second call gave other bits"


# Several units of a lane (from 2 M units), operands of more than 128 MiB, rows of whole cache lines and others.
WIDE = [("bf16", 2100, 1024, 0), ("f16", 2310, 1001, 3), ("f32", 5000, 1000, 1), ("bf16", 20000, 512, 0), ("f16", 17000, 1000, 0), ("bf16", 27400, 1000, 0), ("f16", 26700, 1024, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,N,H,pad", WIDE)
def test_wide_and_large(dtype, N, H, pad):
    starts = _cuts(H, N, 7)
    gates, bias, h0, dy, dh_last = _operands(dtype, N, H, 7, pad, pad, 80)
    seq = torch.tensor(starts, dtype=torch.int32, device="cuda")
    got = _train(dtype, gates, bias, h0, seq, 7, N, H, dy, dh_last, pad, pad)
    _check(got, *reference(gates, bias, h0, starts, dy, dh_last), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("N", [0, 1, 100, 700])
def test_left_out_operands(N):
    """No bias, no states before, no starts, no gradient behind, no states kept, no extra results."""
    H, dtype = 130, "f16"
    gates, _, _, dy, _ = _operands(dtype, N, H, 1, 0, 0, 60)
    zero, none = torch.zeros(3 * H, device="cuda"), torch.zeros(1, H, device="cuda")
    want, slack = reference(gates, zero, none, [0, N], dy, none)
    ws = _scratch(g.glr_workspace(N, H))
    y, dg = out_rows(N, H, dtype)[0], out_rows(N, 3 * H, dtype)[0]
    g.glr_sequence(gates, dtype, 3 * H, None, None, None, 1, N, H, y, H, None, None, ws)
    close(y, want[0], slack[0], dtype, "y")
    states, h_last = _scratch(g.glr_states(N, H)), torch.empty(1, H, device="cuda")
    g.glr_sequence(gates, dtype, 3 * H, None, None, None, 1, N, H, y, H, h_last, states, ws)
    close(h_last, want[1], slack[1], "f32", "h_last")
    g.glr_sequence_backward(gates, dtype, 3 * H, None, None, None, 1, N, H, states, dy, dy.stride(0), None, dg, 3 * H, None, None,
                            ws)
    close(dg, want[2], slack[2], dtype, "dgates")


@pytest.mark.gpu
def test_no_tokens_at_all():
    H, q = 70, 5
    h0, dh_last, seq = randn(1, q, H), randn(2, q, H), torch.zeros(q + 1, dtype=torch.int32, device="cuda")
    empty = torch.empty(0, 3 * H, dtype=torch.float16, device="cuda")
    _, h_last, _, dbias, dh0 = _train("f16", empty, None, h0, seq, q, 0, H, empty[:, :H], dh_last)
    assert torch.equal(h_last, h0) and torch.equal(dh0, dh_last) and not dbias.any()


@pytest.mark.gpu
@pytest.mark.parametrize("N", [120, 900])
def test_gates_that_are_shut_or_open(N):
    H, q = 64, 3
    starts = [0, N // 3, N // 2, N]
    gates, bias, h0, dy, dh_last = _operands("f32", N, H, q, 0, 0, 70)
    gates[:, 0], gates[:, 1], gates[:, 2] = 300.0, -300.0, 60.0
    gates[:, 3], gates[:, 4] = float("inf"), -float("inf")
    gates[:, 2 * H], gates[:, 2 * H + 1] = 300.0, -300.0
    gates[:, 2 * H + 2], gates[:, 2 * H + 3] = float("inf"), -float("inf")
    seq = torch.tensor(starts, dtype=torch.int32, device="cuda")
    got = _train("f32", gates, bias, h0, seq, q, N, H, dy, dh_last)
    want, slack = reference(gates, bias, h0, starts, dy, dh_last)
    _check(got, want, slack, "f32")
    assert all(torch.isfinite(t).all() for t in got)


@pytest.mark.gpu
@pytest.mark.parametrize("N", [100, 3000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_sequence(N, bad):
    H, q, dtype = 96, 4, "bf16"
    starts = [0, N // 4, N // 2, N // 2 + 3, N]
    seq = torch.tensor(starts, dtype=torch.int32, device="cuda")
    gates, bias, h0, dy, dh_last = _operands(dtype, N, H, q, 0, 0, 80)
    clean = _train(dtype, gates, bias, h0, seq, q, N, H, dy, dh_last)
    gates, dy, h0 = gates.clone(), dy.clone(), h0.clone()
    gates[starts[1] + 5, H:2 * H] = bad                       # a candidate of sequence 1, a gradient of sequence 1, a state of 2
    dy[starts[2] - 7] = bad
    h0[2] = bad
    y, h_last, dg, dbias, dh0 = _train(dtype, gates, bias, h0, seq, q, N, H, dy, dh_last)
    for s in (0, 3):
        r = slice(starts[s], starts[s + 1])
        assert torch.equal(y[r], clean[0][r]) and torch.equal(dg[r], clean[2][r])
        assert torch.equal(h_last[s], clean[1][s]) and torch.equal(dh0[s], clean[4][s])
    head = slice(starts[1], starts[1] + 5)
    assert torch.equal(y[head], clean[0][head])
    # behind it, the state of sequence 1 is lost for good, however far its gates have decayed
    assert not torch.isfinite(y[starts[1] + 5:starts[2]].float()).any() and not torch.isfinite(h_last[1:3]).any()
    assert not torch.isfinite(dh0[1]).any()


@pytest.mark.gpu
def test_backward_against_differences():
    """A smooth function of all operands along one direction: h^2 / 6 of a third derivative of the size of the gradient times
    |v|^2 per entry (h = 1/64) and rounding of 1e-6 / h leave less than 5e-3 of the gradient's size."""
    N, H, q, h = 150, 20, 3, 1 / 64
    starts = [0, 40, 41, 150]
    seq = torch.tensor(starts, dtype=torch.int32, device="cuda")
    gates, bias, h0, dy, dh_last = _operands("f32", N, H, q, 0, 0, 90)
    v = [randn(95, N, 3 * H), randn(96, 3 * H), randn(97, q, H)]

    def value(t):
        y, last = torch.empty(N, H, device="cuda"), torch.empty(q, H, device="cuda")
        g.glr_sequence((gates + t * v[0]).contiguous(), "f32", 3 * H, bias + t * v[1], h0 + t * v[2], seq, q, N, H, y, H, last, None,
                       _scratch(g.glr_workspace(N, H)))
        return float((y.double() * dy).sum() + (last.double() * dh_last).sum())

    _, _, dg, dbias, dh0 = _train("f32", gates, bias, h0, seq, q, N, H, dy, dh_last)
    along = sum(float((a.double() * b).sum()) for a, b in zip((dg, dbias, dh0), v))
    size = sum(float((a.double() ** 2).sum()) for a in (dg, dbias, dh0)) ** 0.5 * sum(float((b.double() ** 2).sum()) for b in v) ** 0.5
    assert abs((value(h) - value(-h)) / (2 * h) - along) <= 5e-3 * size


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    N, H, ld, dtype = 70000, 32, 32771, "f16"
    values = randn(1, N, 3 * H)
    wide = torch.empty(N * ld, dtype=torch.float16, device="cuda").as_strided((N, 3 * H), (ld, 1))
    wide.copy_(values)
    tight, dy, dh_last = values.half(), randn(2, N, H).half(), randn(3, 1, H)
    a = _train(dtype, tight, None, None, None, 1, N, H, dy, dh_last)
    states, ws = _scratch(g.glr_states(N, H)), _scratch(g.glr_workspace(N, H))
    y, h_last, dbias = torch.empty(N, H, dtype=torch.float16, device="cuda"), torch.empty(1, H, device="cuda"), torch.empty(3 * H, device="cuda")
    g.glr_sequence(wide, dtype, ld, None, None, None, 1, N, H, y, H, h_last, states, ws)
    assert torch.equal(y, a[0]) and torch.equal(h_last, a[1])
    del y
    out = torch.empty(N * ld, dtype=torch.float16, device="cuda").as_strided((N, 3 * H), (ld, 1))
    g.glr_sequence_backward(wide, dtype, ld, None, None, None, 1, N, H, states, dy, H, dh_last, out, ld, dbias, None, ws)
    assert torch.equal(out.contiguous(), a[2]) and torch.equal(dbias, a[3])


@pytest.mark.gpu
def test_replays_of_a_captured_graph():
    N, H, q, dtype = 900, 192, 3, "bf16"
    starts = [0, 500, 501, 900]
    seq = torch.tensor(starts, dtype=torch.int32, device="cuda")
    gates, bias, h0, dy, dh_last = _operands(dtype, N, H, q, 0, 0, 100)
    ws, states = _scratch(g.glr_workspace(N, H)), _scratch(g.glr_states(N, H))
    y, dg = out_rows(N, H, dtype)[0], out_rows(N, 3 * H, dtype)[0]
    h_last, dbias, dh0 = torch.empty(q, H, device="cuda"), torch.empty(3 * H, device="cuda"), torch.empty(q, H, device="cuda")

    def both():
        st = torch.cuda.current_stream()
        g.glr_sequence(gates, dtype, 3 * H, bias, h0, seq, q, N, H, y, H, h_last, states, ws, st)
        g.glr_sequence_backward(gates, dtype, 3 * H, bias, h0, seq, q, N, H, states, dy, dy.stride(0), dh_last, dg, 3 * H, dbias, dh0,
                                ws, st)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for turn in range(3):
        gates.copy_(rows(randn(200 + turn, N, 3 * H), dtype)[0])
        for t in (y, dg, h_last, dbias, dh0):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, h_last, dg, dbias, dh0)]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, h_last, dg, dbias, dh0))), turn


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,batch,pad", [(1, 1, 0), (1024, 1, 0), (100, 7, 3), (1024, 32, 0), (33, 300, 1)])
def test_step(dtype, H, batch, pad):
    ld = batch + pad
    gates, bias, h = randn(1, 3 * H, ld) * 2, randn(2, 3 * H), randn(3, H, ld)
    h_new, y = torch.full((H, ld), float("nan"), device="cuda"), torch.full((H, ld), float("nan"), device="cuda").to(out_rows(1, 1, dtype)[0].dtype)
    g.glr_step(gates, ld, bias, h, ld, h_new, ld, y, dtype, ld, H, batch, torch.cuda.current_stream())
    assert not pad or (torch.isnan(h_new[:, batch:]).all() and torch.isnan(y[:, batch:]).all())
    # a caller is a sequence of one token whose state before is the column of h
    want, slack = reference(gates[:, :batch].t().contiguous(), bias, h[:, :batch].t().contiguous(), list(range(batch + 1)))
    close(h_new[:, :batch].t(), want[1], slack[1] + 2 * EPS32 * (want[1].abs() + 8), "f32", "h")
    close(y[:, :batch].t(), want[0], slack[0] + 2 * EPS32 * (want[0].abs() + 8), dtype, "y")
    mine = h.clone()
    g.glr_step(gates, ld, bias, mine, ld, mine, ld, None, dtype, 0, H, batch)
    assert torch.equal(mine[:, :batch], h_new[:, :batch])


@pytest.mark.gpu
def test_steps_agree_with_the_sequence():
    T, H = 40, 64
    gates, bias = randn(1, T, 3 * H), randn(2, 3 * H)
    y, h_last, h = torch.empty(T, H, device="cuda"), torch.empty(1, H, device="cuda"), torch.zeros(H, 1, device="cuda")
    g.glr_sequence(gates, "f32", 3 * H, bias, None, None, 1, T, H, y, H, h_last, None, _scratch(g.glr_workspace(T, H)))
    one = torch.empty(H, 1, device="cuda")
    for t in range(T):
        g.glr_step(gates[t].contiguous(), 1, bias, h, 1, h, 1, one, "f32", 1, H, 1)
        assert float((one[:, 0] - y[t]).abs().max()) <= 64 * EPS32 * float(y.abs().max())
    assert float((h[:, 0] - h_last[0]).abs().max()) <= 64 * EPS32 * float(h_last.abs().max())


def test_refusals():
    def name(fn, *args, **kw):
        with pytest.raises(g.GrimError) as e:
            fn(*args, **kw)
        return e.value.name

    N, H = 100, 64
    ws = torch.empty(g.glr_workspace(N, H), dtype=torch.uint8)
    fwd = lambda gates=256, dt="f16", ldg=3 * H, seq=512, nseq=2, N=N, H=H, y=768, ldy=H, ws=ws: g.glr_sequence(
        gates, dt, ldg, None, None, seq, nseq, N, H, y, ldy, None, None, ws)
    bwd = lambda states=1024, dy=1280, lddy=H, dg=1536, lddg=3 * H, ws=ws: g.glr_sequence_backward(
        256, "f16", 3 * H, None, None, 512, 2, N, H, states, dy, lddy, None, dg, lddg, None, None, ws)
    for kw in [dict(gates=None), dict(y=None), dict(ws=None)]:
        assert name(fwd, **kw) == "GRIM_ERR_NULL", kw
    for kw in [dict(ldg=3 * H - 1), dict(ldy=H - 1), dict(nseq=0), dict(seq=None), dict(N=-1), dict(N=2 ** 30 + 1), dict(H=0), dict(ws=ws[:-4]),
               dict(ldg=2 ** 60)]:
        assert name(fwd, **kw) == "GRIM_ERR_SHAPE", kw
    for kw in [dict(states=None), dict(dy=None), dict(dg=None), dict(ws=None)]:
        assert name(bwd, **kw) == "GRIM_ERR_NULL", kw
    for kw in [dict(lddy=H - 1), dict(lddg=3 * H - 1), dict(ws=ws[:-4])]:
        assert name(bwd, **kw) == "GRIM_ERR_SHAPE", kw
    step = lambda gates=256, ldg=4, h=512, ldh=4, new=768, y=1024, ldy=4, H=H, b=4: g.glr_step(gates, ldg, None, h, ldh, new, 4, y, "f16", ldy, H, b)
    for kw in [dict(gates=None), dict(h=None), dict(new=None)]:
        assert name(step, **kw) == "GRIM_ERR_NULL", kw
    for kw in [dict(ldg=3), dict(ldh=3), dict(ldy=3), dict(H=0), dict(b=-1), dict(H=2 ** 40)]:
        assert name(step, **kw) == "GRIM_ERR_SHAPE", kw
    from paper_2108_11033_amd import lm
    assert lm._lib().grim_glr_sequence(256, 9, 3 * H, None, None, None, 1, N, H, 512, H, None, None, 768, 1 << 30, None) == 4


def test_states_in_place_are_refused():
    """Workgroups finish at different times: a sequence's last state would take the place of one that another workgroup has yet to read."""
    N, H, q = 100, 64, 3
    ws = torch.empty(g.glr_workspace(N, H), dtype=torch.uint8)
    size = 4 * q * H
    at = 1 << 20

    def name(fn, *args):
        with pytest.raises(g.GrimError) as e:
            fn(*args)
        return e.value.name

    fwd = lambda h0, h_last: g.glr_sequence(256, "f16", 3 * H, None, h0, 512, q, N, H, 768, H, h_last, None, ws)
    bwd = lambda dh_last, dh0: g.glr_sequence_backward(256, "f16", 3 * H, None, None, 512, q, N, H, 1024, 1280, H, dh_last, 1536, 3 * H, None, dh0, ws)
    for fn in (fwd, bwd):
        for a, b in [(at, at), (at, at + 4), (at + 4, at), (at, at + size - 4), (at + size - 4, at)]:
            assert name(fn, a, b) == "GRIM_ERR_UNSUPPORTED", (a, b)


@pytest.mark.gpu
def test_states_side_by_side():
    """The states before and after in halves of one buffer, in either order: neighbours, not in place."""
    N, H, q, dtype = 900, 64, 3, "f16"
    starts = [0, 300, 301, 900]
    seq = torch.tensor(starts, dtype=torch.int32, device="cuda")
    gates, bias, h0, dy, dh_last = _operands(dtype, N, H, q, 0, 0, 120)
    want = _train(dtype, gates, bias, h0, seq, q, N, H, dy, dh_last)
    for first in (0, 1):
        a, b = torch.zeros(2 * q, H, device="cuda"), torch.zeros(2 * q, H, device="cuda")
        before, after, d_after, d_before = a[first * q:][:q], a[(1 - first) * q:][:q], b[first * q:][:q], b[(1 - first) * q:][:q]
        before.copy_(h0), d_after.copy_(dh_last)
        ws, states = _scratch(g.glr_workspace(N, H)), _scratch(g.glr_states(N, H))
        y, dg = out_rows(N, H, dtype)[0], out_rows(N, 3 * H, dtype)[0]
        g.glr_sequence(gates, dtype, 3 * H, bias, before, seq, q, N, H, y, H, after, states, ws)
        g.glr_sequence_backward(gates, dtype, 3 * H, bias, before, seq, q, N, H, states, dy, dy.stride(0), d_after, dg, 3 * H, None, d_before, ws)
        assert torch.equal(after, want[1]) and torch.equal(d_before, want[4]) and torch.equal(before, h0) and torch.equal(d_after, dh_last)
