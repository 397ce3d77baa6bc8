"""grim_gdr_step against the formulas in 64 bits.

Bounds: a sum over dk rows has chains of at most 8 products in a thread, two and four joins: off by 16 x 2^-24 of the terms' sizes; a decay by (2 + |g|) x 2^-24
of itself, a length by 12 x 2^-24.  These are counted through u, the new states and y, with 40 x 2^-24 of each product's size for all of them."""
import math

import pytest
import torch

import paper_2108_11033_amd as g
from lm_helpers import DTYPES, EPS32, close, out_rows, randn, rows, untouched


def reference(q, k, v, decay, beta, s, heads, key_heads, dk, dv, scale, eps, batch):
    """y (heads dv x batch), the new states, and their slacks."""
    d = lambda t: t.double().t()
    q, k = (d(t).reshape(batch, key_heads, dk).repeat_interleave(heads // key_heads, 1) for t in (q, k))
    if eps > 0:
        q, k = (t / torch.sqrt((t * t).sum(2, keepdim=True) + eps) for t in (q, k))
    q = q * scale
    v, a, b = d(v).reshape(batch, heads, dv), torch.exp(d(decay))[..., None, None], d(beta)[..., None]
    D = a * s.double()
    ea = 40 + d(decay).abs().clamp(max=1e4)[..., None, None]
    u = b * (v - (k[..., None] * D).sum(2))
    eu = b.abs() * EPS32 * (4 * v.abs() + (k[..., None] * D * ea).abs().sum(2)) + 4 * EPS32 * u.abs()
    S = D + k[..., None] * u[:, :, None]
    eS = EPS32 * (ea * D.abs() + 40 * (k[..., None] * u[:, :, None]).abs()) + k.abs()[..., None] * eu[:, :, None]
    y = (q[..., None] * S).sum(2)
    ey = (q[..., None].abs() * (EPS32 * (ea * D.abs() + 40 * (k[..., None] * u[:, :, None]).abs()) + k.abs()[..., None] * eu[:, :, None])).sum(2)
    flat = lambda t: t.reshape(batch, heads * dv).t()
    return flat(y), S, flat(ey), eS


def operands(heads, key_heads, dk, dv, batch, seed, pad=0):
    wide = lambda i, n: rows(randn(seed + i, n, batch), "f32", pad)[0]
    gates = -torch.nn.functional.softplus(randn(seed + 4, heads, batch) * 2 - 2)
    return (wide(1, key_heads * dk), wide(2, key_heads * dk), wide(3, heads * dv), rows(gates, "f32", pad)[0],
            rows(torch.sigmoid(randn(seed + 5, heads, batch)), "f32", pad)[0], 0.3 * randn(seed + 6, batch, heads, dk, dv))


SHAPES = [(1, 1, 1, 1, 1), (2, 1, 3, 5, 3), (16, 16, 64, 64, 1), (4, 2, 40, 72, 5), (8, 2, 128, 128, 7), (3, 3, 65, 33, 2), (1, 1, 128, 1, 64), (6, 1, 16, 127, 4), (16, 4, 100, 66, 33)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,key_heads,dk,dv,batch", SHAPES)
@pytest.mark.parametrize("eps", [1e-6, 0.0])
def test_step(dtype, heads, key_heads, dk, dv, batch, eps):
    pad = batch % 3
    q, k, v, decay, beta, s = operands(heads, key_heads, dk, dv, batch, heads + dk, pad)
    if eps == 0:
        q, k = q * dk ** -0.5, k * dk ** -0.5
    decay[0, 0] = -math.inf                                                  # a state that is forgotten
    new = torch.full_like(s, float("nan"))
    y, buf = out_rows(heads * dv, batch, dtype, pad + 1)
    args = (decay.stride(0), heads, key_heads, dk, dv, 0.7, eps, batch)
    call = lambda s, s_new, y, ldy: g.gdr_step(q, k, v, q.stride(0), k.stride(0), v.stride(0), decay, beta, args[0], s, s_new, y, dtype, ldy, *args[1:],
                                               torch.cuda.current_stream())
    call(s, new, y, batch + pad + 1)
    assert untouched(y, buf)
    wy, ws, ey, es = reference(q, k, v, decay, beta, s, heads, key_heads, dk, dv, 0.7, eps, batch)
    close(y, wy, ey, dtype, "y")
    close(new, ws, es, "f32", "states")
    mine = s.clone()
    call(mine, mine, None, 0)                                                # in place, states alone
    assert torch.equal(mine, new)


@pytest.mark.gpu
def test_more_callers_than_a_launch_takes():
    """heads x blocks x 256 threads x callers at 2^32 and beyond."""
    heads, batch = 4096, 4100
    q, k, v = (randn(i, n, batch) for i, n in ((1, 1), (2, 1), (3, heads)))
    decay, beta = torch.zeros(heads, batch, device="cuda"), torch.ones(heads, batch, device="cuda")
    s = torch.zeros(batch, heads, 1, 1, device="cuda")
    g.gdr_step(q, k, v, batch, batch, batch, decay, beta, batch, s, s, None, "f32", 0, heads, 1, 1, 1, 1.0, 0.0, batch)
    # (one product of two fp32 numbers: half a unit)
    assert bool(((s[:, :, 0, 0] - (k[0][:, None] * v.t())).abs() <= 2 * EPS32 * s[:, :, 0, 0].abs()).all())


@pytest.mark.gpu
def test_infinities_stay_with_their_caller_and_head():
    q, k, v, decay, beta, s = operands(4, 2, 16, 8, 3, 1)
    want = torch.empty_like(s)
    y = torch.empty(32, 3, device="cuda")
    call = lambda: g.gdr_step(q, k, v, 3, 3, 3, decay, beta, 3, s, want, y, "f32", 3, 4, 2, 16, 8, 1.0, 1e-6, 3)
    call()
    clean, cy = want.clone(), y.clone()
    s[1, 2, 3, 4] = math.nan
    v[3 * 8 + 1, 0] = math.inf
    call()
    same = torch.ones(3, 4, dtype=torch.bool, device="cuda")
    same[1, 2] = same[0, 3] = False
    assert torch.equal(want[same], clean[same]) and not torch.isfinite(want[1, 2]).all() and not torch.isfinite(want[0, 3]).all()
    assert torch.equal(y.view(4, 8, 3).permute(2, 0, 1)[same], cy.view(4, 8, 3).permute(2, 0, 1)[same])


A_, B_, C_, D_, E_, F_, G_, H_ = (1 << 30 << i for i in range(8))


def test_refusals():
    def name(q=A_, ldq=4, ldk=4, ldv=4, ldg=4, s=D_, new=E_, y=F_, ldy=4, heads=4, key_heads=2, dk=16, dv=8, scale=1.0, eps=0.0, batch=4, decay=G_):
        with pytest.raises(g.GrimError) as e:
            g.gdr_step(q, B_, C_, ldq, ldk, ldv, decay, H_, ldg, s, new, y, "f16", ldy, heads, key_heads, dk, dv, scale, eps, batch)
        return e.value.name
    for bad in (dict(ldq=3), dict(ldk=3), dict(ldv=3), dict(ldg=3), dict(ldy=3), dict(heads=0), dict(heads=5), dict(heads=4097, key_heads=1), dict(key_heads=0), dict(dk=0), dict(dv=-1),
                dict(scale=math.inf), dict(scale=math.nan), dict(eps=-1.0), dict(scale=1e-31), dict(scale=-1e31),
                dict(eps=1e-17), dict(eps=1e31), dict(eps=math.nan), dict(eps=math.inf), dict(batch=-1)):
        assert name(**bad) == "GRIM_ERR_SHAPE", bad
    assert name(dk=129) == "GRIM_ERR_UNSUPPORTED" and name(dv=200) == "GRIM_ERR_UNSUPPORTED" and name(new=D_ + 4) == "GRIM_ERR_UNSUPPORTED"
    for bad in (dict(q=None), dict(s=None), dict(new=None), dict(decay=None)):
        assert name(**bad) == "GRIM_ERR_NULL", bad
    g.gdr_step(None, None, None, 0, 0, 0, None, None, 0, None, None, None, "f32", 0, 1, 1, 1, 1, 1.0, 0.0, 0)
