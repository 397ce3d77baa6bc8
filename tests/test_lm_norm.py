"""grim_layer_norm and its backward pass against the formulas in 64 bits.

Bounds: a row's sums run over at most 64 terms per thread and 10 levels of reduction, so a mean is off by at most 80 x 2^-24
of the mean of |terms|; results add a dozen roundings.  96 x 2^-24 of the terms' sizes covers both.  Column sums over N rows
take N / 64 + 100 additions at most on the way of one term."""
import pytest
import torch

import paper_2108_11033_amd as g
from lm_helpers import DTYPES, EPS32, close, out_rows, randn, rows, untouched

SHAPES = [(1, 1), (1, 7), (3, 8), (5, 33), (2, 997), (300, 1024), (9, 2048), (3, 2049), (4, 5000), (2, 8192), (3, 10000),
          (2, 32768), (2, 40000), (1000, 72), (70000, 64)]


def _stats(x, eps):
    m = x.mean(1, keepdim=True)
    return m, (((x - m) ** 2).mean(1, keepdim=True) + eps).rsqrt()


def _operands(dtype, N, C, pad, offset, seed):
    x, _ = rows(randn(seed, N, C) * 1.5 + 0.5, dtype, pad, offset)
    return x, 1 + 0.3 * randn(seed + 1, C), 0.3 * randn(seed + 2, C)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C", SHAPES)
def test_forward(dtype, N, C):
    for pad, offset, params in [(0, 0, True), (3, 1, True), (8, 0, False)]:
        x, gamma, beta = _operands(dtype, N, C, pad, offset, 10)
        y, buf = out_rows(N, C, dtype, pad + 2, offset)
        mean, rstd = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        gb = (gamma, beta) if params else (None, None)
        g.layer_norm(x, dtype, C + pad, *gb, 1e-5, N, C, y, C + pad + 2, mean, rstd, torch.cuda.current_stream())
        assert untouched(y, buf)
        x64 = x.double()
        m, s = _stats(x64, 1e-5)
        g64, b64 = (gamma.double(), beta.double()) if params else (torch.ones_like(gamma.double()), torch.zeros_like(beta.double()))
        size = s * (x64.abs() + x64.abs().mean(1, keepdim=True))
        # the variance's own relative error reaches s through half its value; rows of one element have s = eps^-1/2
        close(y, (x64 - m) * s * g64 + b64, 96 * EPS32 * (size * g64.abs() + b64.abs()), dtype, f"y {N}x{C}")
        close(mean, m[:, 0], 96 * EPS32 * x64.abs().mean(1), "f32", "mean")
        close(rstd, s[:, 0], 96 * EPS32 * s[:, 0] * (1 + (s[:, 0] * x64.abs().mean(1)) ** 2 * EPS32 * 96), "f32", "rstd")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C", SHAPES)
def test_backward(dtype, N, C):
    for pad, offset, params in [(0, 0, True), (5, 3, False)]:
        x, gamma, _ = _operands(dtype, N, C, pad, offset, 20)
        dy, _ = rows(randn(23, N, C), dtype, pad + 1, offset)
        m, s = _stats(x.double(), 1e-5)
        mean, rstd = m[:, 0].float(), s[:, 0].float()
        m, s = mean.double()[:, None], rstd.double()[:, None]
        dx, buf = out_rows(N, C, dtype, pad, offset)
        dgamma, dbeta = torch.full((C,), float("nan"), device="cuda"), torch.full((C,), float("nan"), device="cuda")
        ws = torch.empty(g.layer_norm_workspace(N, C), dtype=torch.uint8, device="cuda")
        call = lambda: g.layer_norm_backward(dy, C + pad + 1, x, C + pad, dtype, gamma if params else None, mean, rstd, N, C, dx,
                                             C + pad, dgamma, dbeta, ws, torch.cuda.current_stream())
        call()
        assert untouched(dx, buf)
        x64, d64 = x.double(), dy.double()
        g64 = gamma.double() if params else torch.ones_like(gamma.double())
        xh, d = (x64 - m) * s, d64 * g64
        size = s * (x64.abs() + m.abs())                                    # of xh before its difference cancels
        want = s * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))
        slack = s * (d.abs() + d.abs().mean(1, keepdim=True) + 2 * size * (d.abs() * size).mean(1, keepdim=True))
        close(dx, want, 96 * EPS32 * slack, dtype, f"dx {N}x{C}")
        steps = (N / 64 + 100) * EPS32
        close(dgamma, (d64 * xh).sum(0), steps * (d64.abs() * size).sum(0), "f32", "dgamma")
        close(dbeta, d64.sum(0), steps * d64.abs().sum(0), "f32", "dbeta")
        first = [t.clone() for t in (dx, dgamma, dbeta)]
        call()
        assert all(torch.equal(a, b) for a, b in zip(first, (dx, dgamma, dbeta))), "a second call gave other bits"


# operands of more than 128 MiB, which are written past the caches: rows in registers and rows that are walked
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,N,C", [("f16", 35001, 1001), ("bf16", 36000, 1024), ("f32", 4200, 4100), ("bf16", 900, 40001)])
def test_operands_beyond_the_caches(dtype, N, C):
    test_forward(dtype, N, C)
    test_backward(dtype, N, C)


@pytest.mark.gpu
def test_backward_against_differences():
    """sum(dy y) along a direction, both ways, of the fp32 kernel itself: the difference quotient at h = 1/64 is off by
    h^2 / 6 of a third derivative of size about 6 |v|^3 of the normed row (below 1e-3 of the gradient's size here) and by
    the outputs' rounding, 1e-7 x sqrt(N C) / h."""
    N, C, h = 6, 200, 1 / 64
    x, gamma, beta = randn(1, N, C) * 2, 1 + 0.3 * randn(2, C), 0.2 * randn(3, C)
    dy, v, vg, vb = randn(4, N, C), randn(5, N, C), randn(6, C), randn(7, C)

    def value(t):
        y = torch.empty(N, C, device="cuda")
        g.layer_norm(x + t * v, "f32", C, gamma + t * vg, beta + t * vb, 1e-5, N, C, y, C)
        return float((y.double() * dy.double()).sum())

    y, mean, rstd = torch.empty(N, C, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    g.layer_norm(x, "f32", C, gamma, beta, 1e-5, N, C, y, C, mean, rstd)
    dx, dgamma, dbeta = torch.empty(N, C, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = torch.empty(g.layer_norm_workspace(N, C), dtype=torch.uint8, device="cuda")
    g.layer_norm_backward(dy, C, x, C, "f32", gamma, mean, rstd, N, C, dx, C, dgamma, dbeta, ws)
    along = float((dx.double() * v).sum() + (dgamma.double() * vg).sum() + (dbeta.double() * vb).sum())
    size = float((dx.double() ** 2).sum().sqrt() * (v.double() ** 2).sum().sqrt())
    assert abs((value(h) - value(-h)) / (2 * h) - along) <= 2e-3 * size


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", [5, 1000, 6000, 70000])
def test_in_place_and_partial_outputs(dtype, C):
    N = 40
    x, gamma, beta = _operands(dtype, N, C, 3, 1, 30)
    y, _ = out_rows(N, C, dtype)
    g.layer_norm(x, dtype, C + 3, gamma, beta, 1e-5, N, C, y, C)
    mine = rows(x.float(), dtype, 3, 1)[0]
    g.layer_norm(mine, dtype, C + 3, gamma, beta, 1e-5, N, C, mine, C + 3)
    assert torch.equal(mine, y)
    m, s = _stats(x.double(), 1e-5)
    dy = rows(randn(31, N, C), dtype)[0]
    ws = torch.empty(g.layer_norm_workspace(N, C), dtype=torch.uint8, device="cuda")
    args = (x, C + 3, dtype, gamma, m[:, 0].float(), s[:, 0].float(), N, C)
    dx, dgamma, dbeta = out_rows(N, C, dtype)[0], torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    g.layer_norm_backward(dy, C, *args, dx, C, dgamma, dbeta, ws)
    only = torch.empty(C, device="cuda")
    g.layer_norm_backward(dy, C, *args, None, 0, None, only, ws)
    assert torch.equal(only, dbeta)
    g.layer_norm_backward(dy, C, *args, None, 0, only, None, ws)
    assert torch.equal(only, dgamma)
    mine = dy.clone()
    g.layer_norm_backward(mine, C, *args, mine, C, None, None, None)         # dx over dy, no column sums, no workspace
    assert torch.equal(mine, dx)
    again = [torch.empty(C, device="cuda") for _ in range(2)]
    g.layer_norm_backward(dy, C, *args, dy, C, *again, ws)                   # dx over dy, which the column sums read too
    assert torch.equal(dy, dx) and torch.equal(again[0], dgamma) and torch.equal(again[1], dbeta)


@pytest.mark.gpu
def test_no_rows():
    dgamma, dbeta = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    ws = torch.empty(g.layer_norm_workspace(0, 64), dtype=torch.uint8, device="cuda")
    g.layer_norm(None, "f16", 64, None, None, 1e-5, 0, 64, None, 64)
    g.layer_norm_backward(None, 64, None, 64, "f16", None, None, None, 0, 64, None, 0, dgamma, dbeta, ws)
    assert not dgamma.any() and not dbeta.any()


@pytest.mark.gpu
def test_odd_rows_stay_their_own():
    """A row of NaN, one with an infinity, one of equal values: the others are as without them, equal values give beta."""
    N, C = 8, 256
    x, gamma, beta = randn(1, N, C), 1 + 0.3 * randn(2, C), 0.2 * randn(3, C)
    y0, y = torch.empty(N, C, device="cuda"), torch.empty(N, C, device="cuda")
    g.layer_norm(x, "f32", C, gamma, beta, 1e-5, N, C, y0, C)
    x[1], x[3, 7], x[5] = float("nan"), float("inf"), 3.25
    g.layer_norm(x, "f32", C, gamma, beta, 1e-5, N, C, y, C)
    assert torch.isnan(y[1]).all() and torch.isnan(y[3]).any() and torch.equal(y[5], beta)
    keep = [0, 2, 4, 6, 7]
    assert torch.equal(y[keep], y0[keep])


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    N, C, ld = 6, 520, 2 ** 29 + 3
    x = torch.empty(N * ld, dtype=torch.float16, device="cuda").as_strided((N, C), (ld, 1))
    x.copy_(randn(1, N, C))
    small, want = x.contiguous(), torch.empty(N, C, dtype=torch.float16, device="cuda")
    g.layer_norm(small, "f16", C, None, None, 1e-5, N, C, want, C)
    g.layer_norm(x, "f16", ld, None, None, 1e-5, N, C, x, ld)
    assert torch.equal(x.contiguous(), want)


@pytest.mark.gpu
def test_runs_on_the_stream_it_is_given():
    N, C = 4096, 2048
    side = torch.cuda.Stream()
    x, y = randn(1, N, C).half(), torch.empty(N, C, dtype=torch.float16, device="cuda")
    want = torch.empty_like(y)
    g.layer_norm(x, "f16", C, None, None, 1e-5, N, C, want, C)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        late = torch.zeros_like(x)
        for _ in range(50):
            late.add_(1)
        late.copy_(x)
        g.layer_norm(late, "f16", C, None, None, 1e-5, N, C, y, C, stream=side)
    side.synchronize()
    assert torch.equal(y, want)


def test_refusals():
    """Argument errors are found on the host: no GPU is needed to see them."""
    def status(fn, *args):
        with pytest.raises(g.GrimError) as e:
            fn(*args)
        return e.value.name

    fwd = lambda x=256, dt="f16", ldx=64, eps=1e-5, N=4, C=64, y=512, ldy=64: g.layer_norm(x, dt, ldx, None, None, eps, N, C, y, ldy)
    assert status(fwd, None) == "GRIM_ERR_NULL"
    assert status(lambda: fwd(y=None)) == "GRIM_ERR_NULL"
    for bad in [dict(ldx=63), dict(ldy=63), dict(N=-1), dict(C=0), dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(ldx=2 ** 62)]:
        assert status(lambda: fwd(**bad)) == "GRIM_ERR_SHAPE", bad
    from paper_2108_11033_amd import lm
    assert lm._lib().grim_layer_norm(256, 7, 64, None, None, 1e-5, 4, 64, 512, 64, None, None, None) == 4      # GRIM_ERR_DTYPE
    ws = torch.empty(g.layer_norm_workspace(4, 64) - 4, dtype=torch.uint8)
    bwd = lambda dy=256, x=512, mean=768, ws=ws, dgamma=1024, lddx=64: g.layer_norm_backward(dy, 64, x, 64, "f16", None, mean, 768, 4,
                                                                                         64, 1280, lddx, dgamma, None, ws)
    assert status(bwd) == "GRIM_ERR_SHAPE"                                                                # workspace too small
    assert status(lambda: bwd(ws=None)) == "GRIM_ERR_NULL"
    assert status(lambda: bwd(dy=None)) == "GRIM_ERR_NULL"
    assert status(lambda: bwd(mean=None)) == "GRIM_ERR_NULL"
    assert status(lambda: bwd(lddx=8)) == "GRIM_ERR_SHAPE"
