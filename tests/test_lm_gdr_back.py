"""grim_gdr_sequence_backward against PyTorch's gradients of the formulas in 64 bits, token by token (gdr_reference.py has the bounds), and against differences."""
import math

import pytest
import torch

import paper_2108_11033_amd as g
from gdr_reference import run as reference
from lm_helpers import DTYPES, close, out_rows, randn, rows, untouched
from test_lm_gdr import SHAPES, Call

NAMES = ["dq", "dk", "dv", "ddecay", "dbeta", "ds0"]


class Back(Call):
    def __init__(self, *args, last=True, **kw):
        super().__init__(*args, **kw)
        seed = 100 + self.dk
        self.dy = rows(randn(seed, self.N, self.heads * self.dv), self.dtype, self.pad + 2, self.offset)[0]
        self.ds_last = 0.3 * randn(seed + 1, self.nseq, self.heads, self.dk, self.dv) if last else None

    def buffers(self, ds0=True):
        N, keys, values = self.N, self.key_heads * self.dk, self.heads * self.dv
        self.out = {"dq": out_rows(N, keys, self.dtype, self.pad, self.offset), "dk": out_rows(N, keys, self.dtype, self.pad + 1),
                    "dv": out_rows(N, values, self.dtype, self.pad + 3), "ddecay": out_rows(N, self.heads, "f32", self.pad),
                    "dbeta": out_rows(N, self.heads, "f32", self.pad)}
        self.out["ds0"] = (torch.full((self.nseq, self.heads, self.dk, self.dv), float("nan"), device="cuda"),) * 2 if ds0 else (None, None)
        self.states = torch.empty(max(1, g.gdr_states(N, self.nseq, self.heads, self.dk, self.dv)), dtype=torch.uint8, device="cuda").fill_(255)

    def call(self, stream=None):
        keys, values, o = self.key_heads * self.dk + self.pad, self.heads * self.dv + self.pad, self.out
        g.gdr_sequence_backward(*self.head(), self.states, self.dy, values + 2, self.ds_last, o["dq"][0], keys, o["dk"][0], keys + 1, o["dv"][0], values + 3, o["ddecay"][0],
                                o["dbeta"][0], self.heads + self.pad, o["ds0"][0], self.ws, stream)

    def backward(self, ds0=True, stream=None):
        self.buffers(ds0)
        self.forward(self.states, stream)
        self.ws.fill_(255)                                                   # (nothing of the forward call's is left in it)
        self.call(stream)
        for name in NAMES[:5]:
            assert untouched(*self.out[name]), name
        return {name: self.out[name][0] for name in NAMES}

    def check(self):
        got, want = self.backward(ds0=self.dk != 65), self.want(dy=self.dy, ds_last=self.ds_last)
        for name in NAMES:
            if got[name] is not None:
                close(got[name], *want[name], self.dtype if name in ("dq", "dk", "dv") else "f32", name)
        return got


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("starts,heads,key_heads,dk,dv", SHAPES)
@pytest.mark.parametrize("eps", [1e-6, 0.0])
def test_backward(dtype, starts, heads, key_heads, dk, dv, eps):
    c = Back(dtype, starts, heads, key_heads, dk, dv, seed=dk + dv, pad=dv % 3, offset=dk % 2, eps=eps, s0=dk != 16, last=dk != 40)
    once = {n: t.clone() for n, t in c.check().items() if t is not None}
    again = c.backward()
    assert all(torch.equal(again[n], once[n]) for n in once)


# in runs, as of test_lm_gdr.py
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("starts,heads,key_heads,dk,dv", [([0, 1025], 2, 1, 64, 64), ([0, 1800], 1, 1, 128, 128), ([0, 512, 1536, 2049, 2100], 2, 2, 24, 100), ([0, 100, 2100], 1, 1, 128, 40)])
def test_runs(dtype, starts, heads, key_heads, dk, dv):
    Back(dtype, starts, heads, key_heads, dk, dv, seed=dk + dv, pad=dv % 3).check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_gates_at_their_ends(dtype):
    c = Back(dtype, [0, 90, 200], 3, 3, 32, 16, seed=7)
    c.decay[10], c.decay[70], c.decay[71] = -math.inf, -1e30, -20000.0
    c.decay[100:140] = 0.0
    c.decay[150, 1] = -90.0
    c.beta[40:50], c.beta[110:140] = 0.0, 1.0
    got = c.check()
    assert not got["ddecay"][[10, 70, 71]].any()


@pytest.mark.gpu
def test_scale_of_zero():
    """No output reaches the queries, and theirs is no division by the scale."""
    c = Back("f32", [0, 70], 2, 1, 16, 8, seed=5, scale=0.0)
    assert not c.check()["dq"].any()


@pytest.mark.gpu
def test_infinities_stay_in_their_sequence_and_key_head():
    starts = [0, 70, 75, 160]
    c = Back("f32", starts, 4, 2, 16, 24, seed=3)
    whole = {n: t.clone() for n, t in c.backward().items()}
    c.v[100, 1 * 24 + 3] = math.nan                                          # sequence 2, head 1
    c.s0[1, 2, 0, 0] = math.inf                                              # sequence 1, head 2
    c.dy[3, 0] = math.inf                                                    # sequence 0, head 0
    hurt = c.backward()
    heads = torch.ones(160, 4, dtype=torch.bool, device="cuda")
    heads[0:70, 0] = heads[70:75, 2] = heads[75:160, 1] = False
    keys = heads.view(160, 2, 2).all(2)
    for name, clean, n in [("dq", keys, 2), ("dk", keys, 2), ("dv", heads, 4), ("ddecay", heads, 4), ("dbeta", heads, 4)]:
        split = lambda t: t.reshape(160, n, -1)[clean]
        assert torch.equal(split(hurt[name]), split(whole[name])), name
    assert not torch.isfinite(hurt["dq"]).all()


@pytest.mark.gpu
def test_no_tokens():
    c = Back("bf16", [0, 0, 0], 2, 1, 16, 16)
    assert torch.equal(c.backward()["ds0"], c.ds_last)
    c.ds_last = None
    assert not c.backward()["ds0"].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_behind_the_last_sequence(dtype):
    """Rows that no sequence has are neither read nor written."""
    c = Back(dtype, [0, 40, 90], 2, 1, 16, 24, seed=13)
    whole = {n: t.clone() for n, t in c.backward().items()}
    y = c.forward()[0].clone()
    c.seq = torch.tensor([0, 40, 70], dtype=torch.int32, device="cuda")
    for t in (c.q, c.k, c.v, c.decay, c.beta, c.dy):
        t[70:] = math.nan
    cut, _ = c.forward()
    assert torch.equal(cut[:40], y[:40]) and torch.isfinite(cut[:70]).all() and torch.isnan(cut[70:]).all()
    got = c.backward()
    for n in NAMES[:5]:
        assert torch.isfinite(got[n][:70]).all() and torch.isnan(got[n][70:]).all() and torch.equal(got[n][:40], whole[n][:40]), n


@pytest.mark.gpu
def test_rows_far_apart():
    """Offsets beyond 32 bits: 600 rows of 4 M elements, the operands beside each other in them."""
    c = Back("bf16", [0, 100, 600], 2, 1, 16, 24, seed=21)
    near, ld = c.backward(), 4_000_000
    y, s_last = c.forward()
    far_in, far_out = (torch.empty(600 * ld, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def place(buf, at, t):
        view = buf.as_strided((600, t.shape[1]), (ld, 1), ld - 256 + at)
        view.copy_(t)
        return view
    q, k, v, dy = (place(far_in, 64 * i, t) for i, t in enumerate((c.q, c.k, c.v, c.dy)))
    Y, dq, dk, dv = (place(far_out, 64 * i, torch.full_like(t, math.nan)) for i, t in enumerate((c.v, c.q, c.k, c.v)))
    rest = c.head()
    again = torch.empty_like(s_last)
    g.gdr_sequence(q, k, v, "bf16", ld, ld, ld, *rest[7:], Y, ld, again, c.states, c.ws)
    gates = [torch.empty(600, 2, device="cuda") for _ in range(2)]
    ds0 = torch.empty_like(s_last)
    g.gdr_sequence_backward(q, k, v, "bf16", ld, ld, ld, *rest[7:], c.states, dy, ld, c.ds_last, dq, ld, dk, ld, dv, ld, *gates, 2, ds0, c.ws)
    for a, b in ((Y, y), (again, s_last), (dq, near["dq"]), (dk, near["dk"]), (dv, near["dv"]), (gates[0], near["ddecay"]), (gates[1], near["dbeta"]), (ds0, near["ds0"])):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_differences():
    """Along a direction, the gradients add up to the difference of the 64-bit formula's results; what the difference of step h is off by is at most what steps h and 2 h differ
    by, and the sums' own errors are their slacks and half a step of their type along the direction."""
    c = Back("f32", [0, 37, 80], 2, 1, 12, 20, seed=9)
    got, want = c.backward(), c.want(dy=c.dy, ds_last=c.ds_last)
    names = {"dq": "q", "dk": "k", "dv": "v", "ddecay": "decay", "dbeta": "beta", "ds0": "s0"}
    kept = {x: getattr(c, x).double().clone() for x in names.values()}
    for n, x in names.items():
        way = randn(len(x) + 40, *kept[x].shape).double()
        value = lambda step: reference(*[kept[i] + (step * way if i == x else 0) for i in ("q", "k", "v", "decay", "beta", "s0")], c.starts, c.heads, c.key_heads, c.dk, c.dv, c.scale,
                                       c.eps)
        def slope(h):
            a, b = value(h), value(-h)
            return float((((a["y"][0] - b["y"][0]) * c.dy.double()).sum() + ((a["s_last"][0] - b["s_last"][0]) * c.ds_last.double()).sum()) / (2 * h))
        h = 2.0 ** -14
        one, two = slope(h), slope(2 * h)
        allowed = float((way.abs() * (want[n][1] + 2.0 ** -24 * want[n][0].abs())).sum()) + abs(one - two) + 1e-9
        assert abs(float((got[n].double() * way).sum()) - one) <= allowed, n


A_, B_, C_, D_, E_, F_, G_, H_, I_ = (1 << 32 << i for i in range(9))


def test_refusals():
    def name(q=A_, dtype="f16", ldq=32, ldk=32, ldv=32, decay=D_, ldg=4, seq=G_, nseq=2, N=100, heads=4, key_heads=2, dk=16, dv=8, scale=1.0, eps=0.0, states=H_, dy=I_, lddy=32,
             ds_last=F_, dq=A_ * 3, lddq=32, dkey=A_ * 5, lddk=32, dvalue=A_ * 7, lddv=32, ddecay=A_ * 9, dbeta=A_ * 11, lddg=4, ds0=F_ * 3, ws=E_ * 64, room=1 << 40):
        with pytest.raises(g.GrimError) as e:
            g.gdr_sequence_backward(q, B_, C_, dtype, ldq, ldk, ldv, decay, E_, ldg, None, seq, nseq, N, heads, key_heads, dk, dv, scale, eps, states, dy, lddy, ds_last, dq, lddq,
                                    dkey, lddk, dvalue, lddv, ddecay, dbeta, lddg, ds0, (ws, room))
        return e.value.name
    for bad in (dict(ldq=31), dict(ldk=31), dict(ldv=31), dict(ldg=3), dict(lddy=31), dict(lddq=31), dict(lddk=31), dict(lddv=31), dict(lddg=3), dict(N=-1), dict(N=(1 << 30) + 1),
                dict(nseq=0), dict(seq=None), dict(heads=3), dict(key_heads=0), dict(dk=0), dict(dv=0), dict(scale=math.nan), dict(eps=-1.0), dict(scale=1e-31), dict(scale=-1e31),
                dict(eps=1e-17), dict(eps=1e31),
                dict(room=g.gdr_workspace(100, 2, 4, 2, 16, 8) - 1)):
        assert name(**bad) == "GRIM_ERR_SHAPE", bad
    assert name(dk=129, ldq=300, ldk=300, lddq=300, lddk=300) == "GRIM_ERR_UNSUPPORTED" and name(N=1 << 24) == "GRIM_ERR_UNSUPPORTED" and name(nseq=1 << 20) == "GRIM_ERR_UNSUPPORTED"
    assert g.gdr_states(1 << 24, 2, 4, 16, 8) == g.gdr_workspace(1 << 24, 2, 4, 2, 16, 8) == 0
    assert name(ds0=F_) == "GRIM_ERR_UNSUPPORTED" and name(ds0=F_ + 4) == "GRIM_ERR_UNSUPPORTED"
    for bad in (dict(q=None), dict(decay=None), dict(states=None), dict(dy=None), dict(dq=None), dict(dkey=None), dict(dvalue=None), dict(ddecay=None), dict(dbeta=None), dict(ws=None)):
        assert name(**bad) == "GRIM_ERR_NULL", bad
