"""grim_policy_loss against the formulas in 64 bits.

Bounds: with d = (z - max) / tau in base 2, q is off by (4 |d| + 4 mean |d| + 264) x 2^-24 of itself (an exponential by 4 |d| + 2, a sum of them by the mean of that
and 256 additions at most) and lp by e = (4 |d at the word| + 4 mean |d| + 264 + 4 |lp|) x 2^-24; the ratio by that, by the rounding of lp - old and 4 x 2^-24
of itself, and likewise the exponential of the KL term."""
import math

import pytest
import torch

import paper_2108_11033_amd as g
from lm_helpers import DTYPES, EPS32, close, out_rows, randn, rows, untouched

LOW, HIGH = 0.2, 0.3


def reference(z, ids, tau, old, ref, A, w, kl):
    """loss, lp, dz and their slacks (rows whose word is none: zeros)."""
    V = z.shape[1]
    none = (ids < 0) | (ids >= V)
    at = ids.long().clamp(0, V - 1)[:, None]
    z, A, w = z.double() / tau, A.double(), w.double()
    d = z - z.amax(1, keepdim=True)
    q = torch.exp(d)
    total = q.sum(1, keepdim=True)
    q, lq = q / total, d - torch.log(total)
    lp = lq.gather(1, at)[:, 0]
    old = lp if old is None else old.double()
    r, D = torch.exp(lp - old), (torch.zeros_like(lp) if ref is None else ref.double() - lp)
    kl = 0.0 if ref is None else kl
    plain, cut = r * A, r.clamp(1 - LOW, 1 + HIGH) * A
    active = plain <= cut
    term = kl * (torch.expm1(D) - D) if kl else torch.zeros_like(lp)
    loss = w * (term - torch.minimum(plain, cut))
    s = torch.where(active, -plain, torch.zeros_like(plain)) - (kl * torch.expm1(D) if kl else 0.0)
    hot = torch.zeros_like(z).scatter_(1, at, 1.0)
    dz = (w * s / tau)[:, None] * (hot - q)
    d2 = (d.abs() / math.log(2)).clamp(max=1e4)
    mean = (q * torch.where(q > 0, d2, torch.zeros_like(d2))).sum(1)
    e = (4 * d2.gather(1, at)[:, 0] + 4 * mean + 264 + 4 * lp.abs()) * EPS32
    er = e + EPS32 * (4 + (lp - old).abs())
    ed = e + EPS32 * (4 + D.abs())
    sl = w.abs() * (er * torch.minimum(plain.abs(), cut.abs()) + (kl * (ed * (torch.expm1(D).abs() + 1) + 4 * EPS32 * (torch.expm1(D).abs() + D.abs())) if kl else 0) + 8 * EPS32 * loss.abs())
    ss = torch.where(active, er * plain.abs(), torch.zeros_like(er)) + (kl * ed * torch.exp(D) * 2 if kl else 0.0) + 8 * EPS32 * s.abs()
    rq = (4 * d2 + 4 * mean[:, None] + 270) * EPS32
    sdz = (w.abs() / tau)[:, None] * (s.abs()[:, None] * (q * rq + 4 * EPS32 * hot) + ss[:, None] * (hot - q).abs())
    for t in (loss, lp, dz, sl, e, sdz):
        t[none] = 0
    for t in (loss, dz, sl, sdz):
        t[w == 0] = 0
    return loss, lp, dz, sl, e, sdz + 2.0 ** -125


def operands(dtype, N, V, tau, pad, offset, seed):
    z, _ = rows(randn(seed, N, V) * 2.5, dtype, pad, offset)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    ids = torch.randint(0, V, (N,), device="cuda", generator=gen).to(torch.int32)
    lp = torch.log_softmax(z.double() / tau, 1).gather(1, ids.long()[:, None])[:, 0]
    ratio = 0.25 * randn(seed + 2, N)                       # (none near a border, where a rounding decides which side is taken)
    for edge in (math.log1p(HIGH), math.log1p(-LOW)):
        ratio = torch.where((ratio - edge).abs() < 2e-3, torch.full_like(ratio, edge + 4e-3), ratio)
    old = (lp - ratio).float()
    return z, ids, old, old + 0.2 * randn(seed + 3, N), randn(seed + 4, N), torch.rand(N, device="cuda", generator=gen)


def call(z, dtype, ldz, ids, N, V, dz=None, lddz=0, stream=None, loss=True, logp=True, **kw):
    ws = torch.empty(g.policy_loss_workspace(N, V), dtype=torch.uint8, device="cuda").fill_(255)
    out = [torch.full((N,), float("nan"), device="cuda") if want else None for want in (loss, logp)]
    g.policy_loss(z, dtype, ldz, ids, N, V, *out, dz, lddz, ws, clip_low=LOW, clip_high=HIGH, stream=stream, **kw)
    return out


SHAPES = [(1, 1), (3, 2), (5, 7), (200, 8), (4, 33), (300, 1000), (2, 1023), (130, 2049), (129, 4100), (2, 5003), (140, 8197), (150, 20001), (130, 40003),
          (128, 70001), (129, 131072), (161, 131070), (160, 32769), (3, 131075), (2, 300001), (1, 16384), (24, 30000)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V", SHAPES)
def test_loss_and_gradient(dtype, N, V):
    tau, kl, pad, offset = [1.0, 2.0, 0.5][V % 3], [0.05, 0.0][N % 2], [0, 3][V % 2], [0, 1][N % 2]
    z, ids, old, ref, A, w = operands(dtype, N, V, tau, pad, offset, N + V)
    if N > 3:
        w[N // 2], ids[0], ids[3] = 0, -1, V
    dz, buf = out_rows(N, V, dtype, pad + 1, offset)
    more = dict(old_logp=old, ref_logp=ref, advantage=A, weight=w, temperature=tau, kl=kl)
    loss, logp = call(z, dtype, V + pad, ids, N, V, dz, V + pad + 1, torch.cuda.current_stream(), **more)
    assert untouched(dz, buf)
    wl, wp, wdz, sl, sp, sdz = reference(z, ids, tau, old, ref, A, w, kl)
    close(loss, wl, sl, "f32", "loss")
    close(logp, wp, sp, "f32", "logp")
    close(dz, wdz, sdz, dtype, "dz")
    assert torch.equal(call(z, dtype, V + pad, ids, N, V, logp=False, **more)[0], loss)
    assert torch.equal(call(z, dtype, V + pad, ids, N, V, loss=False, temperature=tau)[1], logp)
    first = dz.clone()
    mine, mbuf = rows(z.float(), dtype, pad, offset)                         # in place, and without loss and logarithm
    call(mine, dtype, V + pad, ids, N, V, mine, V + pad, loss=False, logp=False, **more)
    assert torch.equal(mine, first) and untouched(mine, mbuf)


# logits and gradients of more than 128 MiB, written past the caches
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,N,V", [("bf16", 9001, 4100), ("f16", 1100, 32771), ("f32", 600, 30000)])
def test_operands_beyond_the_caches(dtype, N, V):
    test_loss_and_gradient(dtype, N, V)


@pytest.mark.gpu
def test_without_old_and_weights():
    N, V, dtype = 50, 700, "f32"
    z, ids, _, ref, A, _ = operands(dtype, N, V, 1.0, 0, 0, 3)
    dz = torch.empty(N, V, device="cuda")
    loss, logp = call(z, dtype, V, ids, N, V, dz, V, advantage=A, ref_logp=ref, kl=0.1)
    wl, wp, wdz, sl, sp, sdz = reference(z, ids, 1.0, None, ref, A, torch.ones(N, device="cuda"), 0.1)
    close(loss, wl, sl, "f32", "loss")
    close(logp, wp, sp, "f32", "logp")
    close(dz, wdz, sdz, "f32", "dz")


@pytest.mark.gpu
def test_gradient_against_differences():
    N, V = 12, 40
    z, ids, old, ref, A, w = operands("f32", N, V, 1.0, 0, 0, 9)
    dz = torch.empty(N, V, device="cuda")
    call(z, "f32", V, ids, N, V, dz, V, old_logp=old, ref_logp=ref, advantage=A, weight=w, kl=0.1)
    step = 1e-4
    for j in range(V):
        up, down = z.double().clone(), z.double().clone()
        up[:, j] += step
        down[:, j] -= step
        diff = (reference(up, ids, 1.0, old, ref, A, w, 0.1)[0] - reference(down, ids, 1.0, old, ref, A, w, 0.1)[0]) / (2 * step)
        # (third derivatives below 10 in these units: step^2 / 6 of them, and 2^-24 x 300 of the gradient)
        assert float((dz[:, j].double() - diff).abs().max()) <= 2e-5 * float(A.abs().max() + 1), j


@pytest.mark.gpu
@pytest.mark.parametrize("N,V", [(6, 50000), (200, 5000)])
def test_masked_words_and_rows_without_an_answer(N, V):
    z, ids, old, ref, A, w = operands("f32", N, V, 1.0, 0, 0, 5)
    w[:] = 1
    ids[:2] = V - 1
    z[0, V // 3:V - 1] = -math.inf
    z[1, : V - 1] = torch.finfo(torch.float32).min
    z[2] = torch.finfo(torch.float32).min
    z[3], z[4, 7], z[5, V - 1] = -math.inf, math.nan, math.inf
    dz = torch.empty(N, V, device="cuda")
    lp = torch.log_softmax(z.double(), 1).gather(1, ids.long()[:, None])[:, 0]
    old = torch.where(torch.isfinite(lp), lp - 0.01, old.double()).float()
    loss, logp = call(z, "f32", V, ids, N, V, dz, V, old_logp=old, ref_logp=old, advantage=A, weight=w, kl=0.1)
    keep = [0, 1, 2] + list(range(6, N))
    wl, wp, wdz, sl, sp, sdz = (t[keep] for t in reference(z, ids, 1.0, old, old, A, w, 0.1))
    close(loss[keep], wl, sl, "f32", "loss")
    close(logp[keep], wp, sp, "f32", "logp")
    close(dz[keep], wdz, sdz, "f32", "dz")
    assert torch.isnan(loss[3:6]).all() and torch.isnan(dz[3:6]).all() and torch.isnan(logp[3:6]).all()
    w[3:6] = 0                                                               # rows of weight 0 count for nothing, whatever they hold
    loss, _ = call(z, "f32", V, ids, N, V, dz, V, old_logp=old, ref_logp=old, advantage=A, weight=w, kl=0.1)
    assert not loss[3:6].any() and not dz[3:6].any()
    ids[3:6], w[3:6] = -1, 1
    loss, logp = call(z, "f32", V, ids, N, V, dz, V, old_logp=old, ref_logp=old, advantage=A, weight=w, kl=0.1)
    assert not loss[3:6].any() and not dz[3:6].any() and not logp[3:6].any()


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    N, V = 20, 131075
    z, ids, old, ref, A, w = operands("f16", N, V, 1.0, 0, 0, 7)
    more = dict(old_logp=old, ref_logp=ref, advantage=A, weight=w, kl=0.1, clip_low=LOW, clip_high=HIGH)
    ws = torch.empty(g.policy_loss_workspace(N, V), dtype=torch.uint8, device="cuda")
    loss, logp, dz = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(z)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        g.policy_loss(z, "f16", V, ids, N, V, loss, logp, dz, V, ws, stream=stream, **more)
    stream.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        g.policy_loss(z, "f16", V, ids, N, V, loss, logp, dz, V, ws, stream=stream, **more)
    for seed in range(3):
        z.copy_(randn(seed, N, V))
        graph.replay()
        torch.cuda.synchronize()
        got = loss.clone(), logp.clone(), dz.clone()
        g.policy_loss(z, "f16", V, ids, N, V, loss, logp, dz, V, ws, stream=torch.cuda.current_stream(), **more)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (loss, logp, dz)))


A_, B_, C_, D_, E_, WS = (1 << 20 << i for i in range(6))


def _name(*args, **kw):
    with pytest.raises(g.GrimError) as e:
        g.policy_loss(*args, **kw)
    return e.value.name


def test_refusals():
    room = (WS, 1 << 40)
    good = dict(advantage=C_)
    assert _name(A_, "f16", 63, B_, 4, 64, D_, None, None, 0, room, **good) == "GRIM_ERR_SHAPE"
    assert _name(A_, "f16", 64, B_, 4, 64, D_, None, E_, 63, room, **good) == "GRIM_ERR_SHAPE"
    assert _name(A_, "f16", 64, B_, 4, 64, D_, None, A_, 65, room, **good) == "GRIM_ERR_SHAPE"
    assert _name(A_, "f16", 64, B_, -1, 64, D_, None, E_, 64, room, **good) == "GRIM_ERR_SHAPE"
    assert _name(A_, "f16", 64, B_, 4, 0, D_, None, E_, 64, room, **good) == "GRIM_ERR_SHAPE"
    assert _name(A_, "f16", 1 << 17, B_, 4, 1 << 17, D_, None, E_, 1 << 17, (WS, 16), **good) == "GRIM_ERR_SHAPE"
    for bad in (dict(temperature=0.0), dict(temperature=math.nan), dict(temperature=1e31), dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-1.0),
                dict(clip_high=math.inf), dict(kl=-0.1), dict(kl=math.nan)):
        assert _name(A_, "f16", 64, B_, 4, 64, D_, None, E_, 64, room, **good, **bad) == "GRIM_ERR_SHAPE", bad
    assert _name(None, "f16", 64, B_, 4, 64, D_, None, E_, 64, room, **good) == "GRIM_ERR_NULL"
    assert _name(A_, "f16", 64, None, 4, 64, D_, None, E_, 64, room, **good) == "GRIM_ERR_NULL"
    assert _name(A_, "f16", 64, B_, 4, 64, D_, None, E_, 64, room) == "GRIM_ERR_NULL"
    assert _name(A_, "f16", 64, B_, 4, 64, None, None, None, 0, room, **good) == "GRIM_ERR_NULL"
    assert _name(A_, "f16", 64, B_, 4, 64, D_, None, E_, 64, None, **good) == "GRIM_ERR_NULL"
    g.policy_loss(None, "f16", 64, None, 0, 64, None, None, None, 0, None)
    assert g.policy_loss_workspace(-1, 5) == 0 and g.policy_loss_workspace(4, 0) == 0
