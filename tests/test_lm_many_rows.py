"""More rows than one launch may have threads for (2^32 - 1: 2^24 - 1 workgroups of 256).  Rows on both sides of where launches meet are
held against a small call on the same rows, bit by bit; sums over all rows against 64 bits."""
import pytest
import torch

import paper_2108_11033_amd as g
from lm_helpers import EPS32, TORCH, close

MOST_THREADS = 2 ** 32 - 1


def _pick(n, meet):
    """Rows at the start, at the end, and around row `meet`."""
    return torch.cat([torch.arange(0, 20), torch.arange(meet - 20, meet + 20), torch.arange(n - 20, n)]).clamp(0, n - 1).cuda()


def _normal(n, c, dtype, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.empty(n, c, dtype=TORCH[dtype], device="cuda").normal_(generator=gen)


# (the last: teams of sixteen lanes, sixteen rows a workgroup)
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,C,per_group", [("bf16", 4, 1), ("f32", 1, 1), ("bf16", 8, 16)])
def test_layer_norm(dtype, C, per_group):
    meet = MOST_THREADS // 256 * per_group
    N = meet + 37
    x = _normal(N, C, dtype, 1)
    gamma, beta = torch.linspace(0.5, 2, C, device="cuda"), torch.linspace(-1, 1, C, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    g.layer_norm(x, dtype, C, gamma, beta, 1e-5, N, C, y, C, mean, rstd)
    at = _pick(N, meet)
    n, few = len(at), x[at].contiguous()
    sy, sm, sr = torch.empty_like(few), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    g.layer_norm(few, dtype, C, gamma, beta, 1e-5, n, C, sy, C, sm, sr)
    assert torch.equal(y[at], sy) and torch.equal(mean[at], sm) and torch.equal(rstd[at], sr)


@pytest.mark.gpu
@pytest.mark.parametrize("sums", [False, True])
def test_layer_norm_backward(sums):
    C, dtype, meet = 4, "bf16", MOST_THREADS // 256
    N = meet + 37
    x, dy = _normal(N, C, dtype, 1), _normal(N, C, dtype, 2)
    mean, rstd = 0.1 * _normal(N, 1, "f32", 3)[:, 0], 1 + 0.1 * _normal(N, 1, "f32", 4)[:, 0]
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = torch.empty(g.layer_norm_workspace(N, C), dtype=torch.uint8, device="cuda")
    g.layer_norm_backward(dy, C, x, C, dtype, None, mean, rstd, N, C, dx, C, dgamma if sums else None, dbeta if sums else None, ws if sums else None)
    at = _pick(N, meet)
    n, few = len(at), torch.empty(len(at), C, dtype=TORCH[dtype], device="cuda")
    g.layer_norm_backward(dy[at].contiguous(), C, x[at].contiguous(), C, dtype, None, mean[at].contiguous(), rstd[at].contiguous(), n, C, few, C,
                          None, None, None)
    assert torch.equal(dx[at], few)
    if sums:                                            # N / 1024 rows a thread, then 1024 sums
        d, xh = dy.double(), (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        size = (x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None]
        steps = (N / 1024 + 200) * EPS32
        close(dgamma, (d * xh).sum(0), steps * (d.abs() * size).sum(0), "f32", "dgamma")
        close(dbeta, d.sum(0), steps * d.abs().sum(0), "f32", "dbeta")


# rows of their own workgroup (128 threads), and slices (320 threads)
@pytest.mark.gpu
@pytest.mark.parametrize("V,threads", [(8, 128), (3, 320)])
def test_distillation(V, threads):
    dtype, k, meet = "bf16", 2, MOST_THREADS // threads
    N = meet + 37
    z, top = _normal(N, V, dtype, 1), _normal(N, k, "f32", 2)
    ids = torch.randint(-1, V, (N, k), device="cuda", generator=torch.Generator("cuda").manual_seed(3), dtype=torch.int32)
    weight = _normal(N, 1, "f32", 4)[:, 0].abs()

    def run(z, top, ids, weight, dz):
        n = z.shape[0]
        loss = torch.full((n,), float("nan"), device="cuda")
        ws = torch.empty(g.distill_topk_workspace(n, V), dtype=torch.uint8, device="cuda")
        g.distill_topk(z, dtype, V, top, ids, k, k, 2.0, weight, n, V, loss, dz, V, ws)
        return loss

    dz = torch.empty_like(z)
    loss = run(z, top, ids, weight, dz)
    # (a call of few rows of 8 words runs on the same kernel)
    at = _pick(N, meet)
    few = torch.empty(len(at), V, dtype=TORCH[dtype], device="cuda")
    want = run(z[at].contiguous(), top[at].contiguous(), ids[at].contiguous(), weight[at].contiguous(), few)
    assert torch.equal(loss[at], want) and torch.equal(dz[at], few)
    assert torch.isfinite(loss).all()


@pytest.mark.gpu
@pytest.mark.parametrize("columns,V", [(False, 2), (True, 1)])
def test_logit_rules(columns, V):
    dtype, meet = "f16", MOST_THREADS // 512 * (8 if columns else 1)
    batch, L, nb = meet + 37, 2, 1
    z = _normal(*((V, batch) if columns else (batch, V)), dtype, 1)
    gen = torch.Generator("cuda").manual_seed(2)
    whole = lambda lo, hi, *s: torch.randint(lo, hi, s, device="cuda", generator=gen, dtype=torch.int32)
    real = lambda *s: torch.rand(s, device="cuda", generator=gen)
    r = dict(history=whole(0, V + 1, batch, L), history_len=whole(0, L + 1, batch), repetition=1 + real(batch), frequency=real(batch), presence=real(batch),
             bias_ids=whole(0, V + 1, batch, nb), bias_values=real(batch, nb), allowed=whole(0, 4, batch, 1))
    sizes = dict(ld_history=L, max_history=L, nbias=nb, ld_bias=nb, ld_allowed=1)
    out = torch.empty_like(z)
    g.logit_rules(z, dtype, z.stride(0), V, batch, out, out.stride(0), columns=columns, **r, **sizes)
    at = _pick(batch, meet)
    n = len(at)
    few = z[:, at].contiguous() if columns else z[at].contiguous()
    want = torch.empty_like(few)
    g.logit_rules(few, dtype, few.stride(0), V, n, want, want.stride(0), columns=columns, **{k: v[at].contiguous() for k, v in r.items()}, **sizes)
    got = out[:, at] if columns else out[at]
    assert torch.equal(got, want) and not torch.isnan(want).any()


def test_sizes_beyond_the_limits_are_refused():
    """Found on the host, before anything is enqueued; no GPU is needed to see them."""
    def name(fn, *args, **kw):
        with pytest.raises(g.GrimError) as e:
            fn(*args, **kw)
        return e.value.name

    ws = torch.empty(1 << 20, dtype=torch.uint8)
    assert name(g.layer_norm, 256, "f32", 1, None, None, 1e-5, 2 ** 31, 1, 512, 1) == "GRIM_ERR_SHAPE"
    assert name(g.layer_norm_backward, 256, 1, 512, 1, "f32", None, 768, 768, 2 ** 31, 1, 1024, 1, None, None, None) == "GRIM_ERR_SHAPE"
    C = 16776961
    assert name(g.layer_norm_backward, 256, C, 512, C, "f32", None, 768, 768, 1, C, 1024, C, None, None, None) == "GRIM_ERR_SHAPE"
    assert name(g.distill_topk, 256, "f32", 1, 512, 768, 1, 1, 1.0, None, 2 ** 31, 1, 1024, None, 0, ws) == "GRIM_ERR_SHAPE"
    assert name(g.glr_step, 256, 2 ** 16, None, 512, 2 ** 16, 768, 2 ** 16, None, "f32", 0, 2 ** 16, 2 ** 16) == "GRIM_ERR_SHAPE"
