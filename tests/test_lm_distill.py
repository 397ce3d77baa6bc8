"""grim_distill_topk against the formulas in 64 bits.

Bounds: an exponential of d = (z - max) / tau in base 2 is off by (4 |d| + 2) x 2^-24 of itself; a sum of them over a row, by the
mean of that over the terms and 256 x 2^-24 for the additions (128 elements a thread, the waves, the slices) -- so q by (4 |d| + 4 mean |d| +
264) x 2^-24, p by (4 |d| + 64) x 2^-24, and a log of either by the same in absolute terms plus 4 x 2^-24 of its size."""
import math

import pytest
import torch

import paper_2108_11033_amd as g
from lm_helpers import DTYPES, EPS32, close, out_rows, randn, rows, untouched


def reference(z, top, ids, tau, weight):
    """loss, dz and their slacks."""
    N, V = z.shape
    z, top, w = z.double() / tau, top.double() / tau, weight.double()
    there = (ids >= 0) & (ids < V)
    t = torch.where(there, top, torch.full_like(top, -math.inf))
    some = (t > -math.inf).any(1) & (w != 0)
    t = t - torch.where(torch.isnan(t).any(1), torch.full((N,), math.nan, device="cuda").double(), t.amax(1))[:, None]
    x = torch.where(there & (top > -math.inf), torch.exp(t), torch.zeros_like(t))
    total = x.sum(1, keepdim=True)
    p, logp = x / total, t - torch.log(total)
    d = z - z.amax(1, keepdim=True)
    q = torch.exp(d)
    sq = q.sum(1, keepdim=True)
    q, logq = q / sq, d - torch.log(sq)
    at = ids.long().clamp(0, V - 1)
    used = there & (p > 0) | torch.isnan(p)
    terms = torch.where(used, p * (logp - logq.gather(1, at)), torch.zeros_like(p))
    ps = torch.zeros_like(z).scatter_add_(1, at, torch.where(there, p, torch.zeros_like(p)))
    loss, dz = w * tau ** 2 * terms.sum(1), w[:, None] * tau * (q - ps)
    d2, t2 = (d.abs() / math.log(2)).clamp(max=1e4), (t.abs() / math.log(2)).clamp(max=1e4)
    mean = (q * torch.where(q > 0, d2, torch.zeros_like(d2))).sum(1, keepdim=True)
    rq, rp = (4 * d2 + 4 * mean + 264) * EPS32, (4 * t2 + 64) * EPS32
    pe = torch.zeros_like(z).scatter_add_(1, at, torch.where(there & (p > 0), p * rp, torch.zeros_like(p)))
    slack_dz = w.abs()[:, None] * tau * (torch.where(q > 0, q * rq, q) + pe + 2.0 ** -125)
    each = p * (rp * (logp - logq.gather(1, at)).abs() + rp + rq.gather(1, at) + 4 * EPS32 * (logp.abs() + logq.gather(1, at).abs()))
    slack_loss = w.abs() * tau ** 2 * torch.where(used, each + 32 * EPS32 * terms.abs(), torch.zeros_like(each)).sum(1)
    zero = ~some
    loss[zero], dz[zero], slack_loss[zero], slack_dz[zero] = 0, 0, 0, 0
    return loss, dz, torch.nan_to_num(slack_loss, nan=0, posinf=0), torch.nan_to_num(slack_dz, nan=0, posinf=0)


def _operands(dtype, N, V, k, pad, offset, seed):
    z, _ = rows(randn(seed, N, V) * 2.5, dtype, pad, offset)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    ids = torch.randint(-1, V + 1, (N, k), device="cuda", generator=gen).to(torch.int32)     # duplicates, and some out of range
    return z, 2 * randn(seed + 2, N, k) + 4, ids, torch.rand(N, device="cuda", generator=gen)


def _run(z, dtype, V, top, ids, tau, weight, N, k, ldz, dz=None, lddz=0, stream=None):
    ws = torch.empty(g.distill_topk_workspace(N, V), dtype=torch.uint8, device="cuda").fill_(255)
    loss = torch.full((N,), float("nan"), device="cuda")
    g.distill_topk(z, dtype, ldz, top, ids, k, top.stride(0) if N else k, tau, weight, N, V, loss, dz, lddz, ws, stream)
    return loss


SHAPES = [(1, 1, 1), (3, 2, 3), (5, 7, 4), (200, 8, 2), (4, 33, 33), (300, 1000, 10), (2, 1023, 64), (130, 2049, 65), (129, 4100, 7),
          (2, 5003, 100), (140, 8197, 256), (150, 20001, 128), (130, 40003, 16), (128, 70001, 32), (129, 131072, 64), (3, 131075, 200),
          (2, 300001, 1024), (1, 16384, 1), (24, 30000, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V,k", SHAPES)
def test_loss_and_gradient(dtype, N, V, k):
    tau = [1.0, 2.0, 0.5][V % 3]
    pad, offset = (0, 0) if k % 2 else (3, 1)
    z, top, ids, weight = _operands(dtype, N, V, k, pad, offset, V + k)
    weight[N // 2] = 0 if N > 2 else 1
    if N > 3:
        ids[3] = -1                                                          # a row that lists nothing
    dz, buf = out_rows(N, V, dtype, pad + 1, offset)
    loss = _run(z, dtype, V, top, ids, tau, weight, N, k, V + pad, dz, V + pad + 1, torch.cuda.current_stream())
    assert untouched(dz, buf)
    want, wdz, sl, sdz = reference(z, top, ids, tau, weight)
    close(loss, want, sl, "f32", "loss")
    close(dz, wdz, sdz, dtype, "dz")
    alone = _run(z, dtype, V, top, ids, tau, weight, N, k, V + pad)
    assert torch.equal(alone, loss)
    first = dz.clone()
    mine, mbuf = rows(z.float(), dtype, pad, offset)                         # in place
    again = _run(mine, dtype, V, top, ids, tau, weight, N, k, V + pad, mine, V + pad)
    assert torch.equal(mine, first) and torch.equal(again, loss) and untouched(mine, mbuf)


# logits and gradients of more than 128 MiB, written past the caches up to 128 listed words
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,N,V,k", [("bf16", 9001, 4100, 64), ("f16", 1100, 32771, 129), ("f32", 600, 30000, 32)])
def test_operands_beyond_the_caches(dtype, N, V, k):
    test_loss_and_gradient(dtype, N, V, k)


@pytest.mark.gpu
@pytest.mark.parametrize("N,V", [(4, 50000), (200, 5000)])
def test_masked_words(N, V):
    """-infinity and the type's lowest value as masks, most of a row masked, listed words among the masked, listed logits of -infinity."""
    k, dtype, tau = 12, "f32", 0.5
    z, top, ids, _ = _operands(dtype, N, V, k, 0, 0, 5)
    ids = (ids % V).contiguous()
    weight = torch.ones(N, device="cuda")
    low = torch.finfo(torch.float32).min
    z[0, V // 3:] = -math.inf
    z[1, : V - 2] = low
    z[1, V - 2:] = 3.0
    ids[1, :] = V - 1
    z[2] = low                                                              # all alike: the uniform distribution
    z[3, ids[3, 0].long()] = -math.inf                                      # a word with probability that cannot come
    top[0, 4:] = -math.inf
    ids[0, :] = torch.arange(k, device="cuda", dtype=torch.int32)
    dz = torch.empty(N, V, device="cuda")
    loss = _run(z, dtype, V, top, ids, tau, weight, N, k, V, dz, V)
    want, wdz, sl, sdz = reference(z, top, ids, tau, weight)
    close(loss, want, sl, dtype, "loss")
    close(dz, wdz, sdz, dtype, "dz")
    assert float(loss[3]) == math.inf and torch.isfinite(dz).all()


@pytest.mark.gpu
@pytest.mark.parametrize("N,V", [(6, 50000), (200, 5000)])
def test_rows_that_have_no_answer(N, V):
    k, dtype = 5, "f16"
    z, top, ids, _ = _operands(dtype, N, V, k, 0, 0, 6)
    ids = (ids % V).contiguous()
    weight = torch.ones(N, device="cuda")
    z[0], z[1, 7], z[2, V - 1] = -math.inf, math.nan, math.inf
    top[3, 2] = math.nan
    top[4], z[5] = -math.inf, math.nan
    weight[5] = 0
    dz = torch.full((N, V), 7.0, dtype=torch.float16, device="cuda")
    loss = _run(z, dtype, V, top, ids, 1.0, weight, N, k, V, dz, V)
    assert torch.isnan(loss[:4]).all() and torch.isnan(dz[:4]).all()
    assert not loss[4:6].any() and not dz[4:6].any()
    if N > 6:
        assert torch.isfinite(loss[6:]).all() and torch.isfinite(dz[6:]).all()


@pytest.mark.gpu
def test_gradient_against_differences():
    """h = 1/64 along a direction: h^2 / 6 of a third derivative below 2 |v|^3 p, and the loss's rounding (2e-6) over h."""
    N, V, k, tau, h = 7, 60, 6, 2.0, 1 / 64
    z, top, ids, weight = _operands("f32", N, V, k, 0, 0, 7)
    v = randn(8, N, V)
    dz = torch.empty(N, V, device="cuda")
    _run(z, "f32", V, top, ids, tau, weight, N, k, V, dz, V)
    value = lambda t: float(_run((z + t * v).contiguous(), "f32", V, top, ids, tau, weight, N, k, V).double().sum())
    along = float((dz.double() * v).sum())
    assert abs((value(h) - value(-h)) / (2 * h) - along) <= 2e-3 * float(dz.double().norm() * v.double().norm())


@pytest.mark.gpu
def test_no_weights_strided_lists_no_rows():
    N, V, k = 9, 700, 5
    z, top, ids, _ = _operands("bf16", N, V, k, 0, 0, 9)
    wide_t, wide_i = torch.zeros(N, k + 3, device="cuda"), torch.zeros(N, k + 3, dtype=torch.int32, device="cuda")
    wide_t[:, :k], wide_i[:, :k] = top, ids
    want = _run(z, "bf16", V, top, ids, 1.0, torch.ones(N, device="cuda"), N, k, V)
    got = _run(z, "bf16", V, wide_t, wide_i, 1.0, None, N, k, V)
    assert torch.equal(got, want)
    assert _run(z[:0], "bf16", V, top[:0], ids[:0], 1.0, None, 0, k, V).numel() == 0


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    N, V, k, ld = 5, 40000, 9, 2 ** 29 + 5
    values, top, ids, weight = _operands("f16", N, V, k, 0, 0, 11)
    wide = torch.empty(N * ld, dtype=torch.float16, device="cuda").as_strided((N, V), (ld, 1))
    wide.copy_(values)
    dz = torch.empty(N, V, dtype=torch.float16, device="cuda")
    want = _run(values, "f16", V, top, ids, 2.0, weight, N, k, V, dz, V)
    got = _run(wide, "f16", V, top, ids, 2.0, weight, N, k, ld, wide, ld)
    assert torch.equal(got, want) and torch.equal(wide.contiguous(), dz)


def test_refusals():
    def name(**kw):
        a = dict(z=256, dt="f16", ldz=100, top=512, ids=768, k=4, ldt=4, tau=1.0, N=6, V=100, loss=1024, dz=1280, lddz=100, ws=None)
        a["ws"] = torch.empty(g.distill_topk_workspace(6, 100), dtype=torch.uint8)
        a.update(kw)
        with pytest.raises(g.GrimError) as e:
            g.distill_topk(a["z"], a["dt"], a["ldz"], a["top"], a["ids"], a["k"], a["ldt"], a["tau"], None, a["N"], a["V"], a["loss"],
                           a["dz"], a["lddz"], a["ws"])
        return e.value.name

    for kw in [dict(z=None), dict(top=None), dict(ids=None), dict(loss=None), dict(ws=None)]:
        assert name(**kw) == "GRIM_ERR_NULL", kw
    for kw in [dict(ldz=99), dict(lddz=99), dict(k=0), dict(ldt=3), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")), dict(tau=float("inf")),
               dict(N=-1), dict(V=0), dict(V=2 ** 31, ldz=2 ** 31, lddz=2 ** 31), dict(ldz=2 ** 60),
               dict(ws=torch.empty(g.distill_topk_workspace(6, 100) - 1, dtype=torch.uint8))]:
        assert name(**kw) == "GRIM_ERR_SHAPE", kw
    assert name(k=1025, ldt=1025) == "GRIM_ERR_UNSUPPORTED"


# temperatures at the ends of their range and between, with weights that keep the results within fp32
@pytest.mark.gpu
@pytest.mark.parametrize("N,V", [(5, 50000), (200, 3000)])
@pytest.mark.parametrize("tau,scale", [(1e-30, 1.0), (1e-30, 1e30), (1e-23, 1.0), (1e-12, 1.0), (1e-3, 1.0), (1e6, 1.0), (1e18, 1.0), (1e19, 0.01), (1e24, 1e-24),
                                       (1e30, 1e-30), (1e30, 1e-38)])
def test_temperatures(N, V, tau, scale):
    k = 7
    z, top, ids, weight = _operands("f32", N, V, k, 0, 0, 13)
    weight = (0.5 + weight) * scale
    z[0, ids[0].long().clamp(0, V - 1)] = -1e4
    dz = torch.empty(N, V, device="cuda")
    loss = _run(z, "f32", V, top, ids, tau, weight, N, k, V, dz, V)
    want, wdz, sl, sdz = reference(z, top, ids, tau, weight)
    close(loss, want, sl, "f32", "loss")
    close(dz, wdz, sdz, "f32", "dz")


@pytest.mark.gpu
@pytest.mark.parametrize("tau", [0.25, 1.0])
@pytest.mark.parametrize("N,V", [(3, 50000), (200, 3000)])
def test_listed_words_of_the_lowest_value(N, V, tau):
    """The teacher's best word is masked by the type's lowest value: the loss is as large as that, and no infinity."""
    k = 3
    z, top, ids, _ = _operands("f32", N, V, k, 0, 0, 14)
    ids = torch.arange(k, device="cuda", dtype=torch.int32).repeat(N, 1)
    top[:, 0] = top.amax(1) + 1
    weight = torch.full((N,), 0.25, device="cuda")
    z[0, 0] = torch.finfo(torch.float32).min
    loss = _run(z, "f32", V, top, ids, tau, weight, N, k, V)
    want, _, sl, _ = reference(z, top, ids, tau, weight)
    close(loss, want, sl, "f32", "loss")
    assert torch.isfinite(loss).all() and float(loss[0]) > 1e30


# More rows than compute units of 1793 to 2688 pieces of 16 bytes: rows of eight waves with six pieces a thread.
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,N,V,k", [("bf16", 300, 18001, 64), ("f16", 301, 21503, 100), ("f32", 300, 9001, 65), ("f32", 257, 10752, 16), ("bf16", 270, 14337, 7)])
def test_many_rows_of_a_middling_vocabulary(dtype, N, V, k):
    test_loss_and_gradient(dtype, N, V, k)
