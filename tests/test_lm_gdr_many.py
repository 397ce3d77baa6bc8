"""The gated delta rule with more heads and sequences than compute units (walks of four waves, no waves that help, their maps of runs) and with more sequences than one look of a wave
finds a place among, against the formulas token by token in 64 bits (gdr_reference.py has the bounds)."""
import pytest
import torch

from lm_helpers import DTYPES, close, untouched
from test_lm_gdr import Call
from test_lm_gdr_back import NAMES, Back


def starts_of(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths) + 1)]


# 100 sequences: most of a token or a few, some empty, some of more than a chunk of either size; two empty ones first and one last
SHORT = starts_of([0, 0, 33, 1, 2, 0, 64, 65] + [(i * i) % 5 for i in range(88)] + [70, 1, 31, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dk,dv", [(64, 64), (40, 33)])
def test_many_short_sequences(dtype, dk, dv):
    c = Back(dtype, SHORT, 8, 4, dk, dv, seed=dk + dv, pad=dv % 2, offset=dv % 2)
    once = {n: t.clone() for n, t in c.check().items()}
    y, s_last = c.forward()
    want = c.want()
    assert untouched(y, c.ybuf)
    close(s_last, *want["s_last"], "f32", "s_last")
    close(y, *want["y"], dtype, "y")
    again = c.backward()
    assert all(torch.equal(again[n], once[n]) for n in NAMES)


# in runs of two to five chunks, 288 and more of them over all heads
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("starts,dk,dv", [([0, 1025], 64, 64), ([0, 700, 700, 1090], 40, 33)])
def test_runs_of_many_heads(dtype, starts, dk, dv):
    c = Back(dtype, starts, 32, 8, dk, dv, seed=dk + dv, pad=dv % 2)
    c.check()
    y, s_last = c.forward()
    want = c.want()
    assert untouched(y, c.ybuf)
    close(s_last, *want["s_last"], "f32", "s_last")
    close(y, *want["y"], dtype, "y")


@pytest.mark.gpu
@pytest.mark.parametrize("nseq", [64, 65, 4096, 4097, 5000])
def test_places_among_many_sequences(nseq):
    """One look finds a place among 64 sequences, two among 4096: a hundred tokens among empty sequences, one long sequence among them."""
    lengths = [0] * nseq
    for i in range(60):
        lengths[(i * 997) % nseq] += 1
    lengths[nseq // 2] += 40
    starts = starts_of(lengths)
    c = Call("f32", starts, 2, 1, 8, 16, seed=nseq)
    y, s_last = c.forward()
    want = c.want()
    close(s_last, *want["s_last"], "f32", "s_last")
    close(y, *want["y"], "f32", "y")
    empty = torch.tensor([n == 0 for n in lengths], device="cuda")
    assert torch.equal(s_last[empty], c.s0[empty])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("before,behind,starts,heads,dk,dv", [(333, 500, [0, 900, 2100], 1, 128, 128), (1200, 3, [0, 500, 1300], 4, 40, 33), (70, 65, [0, 1, 1, 30], 2, 64, 64)])
def test_rows_of_no_sequence_around_runs(dtype, before, behind, starts, heads, dk, dv):
    """Sequences that start after the first row and end before the last: what is around them is neither read nor written, however they are cut."""
    c = Back(dtype, starts, heads, 1, dk, dv, seed=dk)
    want, inside = c.want(dy=c.dy, ds_last=c.ds_last), slice(before, before + starts[-1])
    p = Back(dtype, [0] * (len(starts) - 1) + [before + starts[-1] + behind], heads, 1, dk, dv, seed=dk)
    p.seq = torch.tensor(starts, dtype=torch.int32, device="cuda") + before
    for name in ("q", "k", "v", "decay", "beta", "dy"):
        getattr(p, name).fill_(float("nan"))
        getattr(p, name)[inside] = getattr(c, name)
    p.s0, p.ds_last = c.s0, c.ds_last
    y, s_last = p.forward()
    got = dict(p.backward(), y=y)
    close(s_last, *want["s_last"], "f32", "s_last")
    close(got.pop("ds0"), *want["ds0"], "f32", "ds0")
    for name, t in got.items():
        close(t[inside], *want[name], "f32" if name in ("ddecay", "dbeta") else dtype, name)
        assert torch.isnan(t[:before]).all() and torch.isnan(t[before + starts[-1]:]).all(), name
