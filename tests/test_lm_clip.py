"""grim_grad_norm and grim_grad_clip against the formulas in 64 bits: the norm is rounded once from fp64 (of fp16, sums of eight squares in fp32 before:
8 x 2^-24 of a sum, half of that of its root), an output by its factor's rounding and its own."""
import math

import pytest
import torch

import paper_2108_11033_amd as g
from lm_helpers import DTYPES, EPS32, TORCH, UNIT, close, randn

SIZES = [0, 1, 7, 8, 9, 255, 8191, 8192, 8193, 20000, 100003]


def tensors(dtype, sizes, seed, scale=0.01, offset=0):
    return [(randn(seed + i, n + offset)[offset:] * (scale * (1 + i % 3))).to(TORCH[dtype]) if n else torch.empty(0, dtype=TORCH[dtype], device="cuda")
            for i, n in enumerate(sizes)]


def clipped(lst, max_norm, unscale, stream=None):
    norm = torch.full((1,), float("nan"), device="cuda")
    ws = torch.empty(max(1, lst.workspace), dtype=torch.uint8, device="cuda").fill_(255)
    g.grad_clip(lst, max_norm, unscale, norm, ws, stream)
    alone = torch.full((1,), float("nan"), device="cuda")
    return norm, alone, ws


def check(grads, outs, before, norm, max_norm, unscale):
    want = abs(unscale) * math.sqrt(sum(float((t.double() ** 2).sum()) for t in before))
    assert abs(float(norm) - want) <= want * 6 * EPS32, (float(norm), want)
    factor = unscale * (min(1.0, max_norm / want) if want > 0 else 1.0)
    for a, b in zip(outs, before):
        dtype = {v: k for k, v in TORCH.items()}[a.dtype]
        close(a, b.double() * factor, (b.double() * factor).abs() * 10 * EPS32, dtype, f"{tuple(b.shape)}")


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["same", "f32", "place"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("max_norm,unscale", [(0.5, 1.0), (1e9, 1.0), (0.5, 1 / 1024), (0.25, -4.0), (0.0, 1.0), (math.inf, 0.5)])
def test_clip(dtype, out, max_norm, unscale):
    grads = tensors(dtype, SIZES, 1, offset=1)
    before = [t.clone() for t in grads]
    if out == "place":
        outs = grads
    else:
        flat = torch.full((sum(SIZES) + 9,), float("nan"), dtype=TORCH[dtype if out == "same" else "f32"], device="cuda")
        outs, at = [], 3
        for n in SIZES:
            outs.append(flat[at:at + n])
            at += n
    lst = g.GradList(grads, None if out == "place" else outs)
    norm, alone, ws = clipped(lst, max_norm, unscale, torch.cuda.current_stream())
    check(grads, outs, before, norm, max_norm, unscale)
    if out != "place":
        assert torch.isnan(flat[:3]).all() and torch.isnan(flat[at:]).all() and all(torch.equal(a, b) for a, b in zip(grads, before))
        g.grad_norm(lst, unscale, alone, ws, torch.cuda.current_stream())
        assert torch.equal(alone, norm)


@pytest.mark.gpu
@pytest.mark.parametrize("count", [1, 100, 101, 250, 2048])
def test_many_tensors(count):
    grads = [t for d in DTYPES for t in tensors(d, [(i * 37) % 300 for i in range(count // 3 + 1)], 5)][:count]
    outs = [torch.empty_like(t, dtype=torch.float32) for t in grads]
    norm, _, _ = clipped(g.GradList(grads, outs), 0.1, 1.0)
    check(grads, outs, grads, norm, 0.1, 1.0)


@pytest.mark.gpu
def test_more_runs_than_workgroups_and_beyond_the_caches():
    grads = [randn(1, 30_000_001) * 0.01, (randn(2, 20_000_003) * 0.01).bfloat16(), (randn(3, 5) * 0.01).half()]
    outs = [torch.empty_like(t) for t in grads]
    norm, _, _ = clipped(g.GradList(grads, outs), 1.0, 1.0)
    check(grads, outs, grads, norm, 1.0, 1.0)
    before = [t.clone() for t in grads]
    norm2, _, _ = clipped(g.GradList(grads), 1.0, 1.0)
    assert torch.equal(norm, norm2) and all(torch.equal(a, b) for a, b in zip(grads, outs))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,size", [("f32", 1e30), ("f32", 1e-30), ("bf16", 1e30), ("bf16", 1e-30)])
def test_squares_that_fp32_does_not_hold(dtype, size):
    grads = [(randn(4, 1000) * size).to(TORCH[dtype])]
    outs = [torch.empty_like(grads[0])]
    norm, _, _ = clipped(g.GradList(grads, outs), size, 1.0)
    check(grads, outs, grads, norm, size, 1.0)


@pytest.mark.gpu
def test_norms_that_are_none():
    for bad in (math.inf, math.nan):
        grads = tensors("f32", [100, 9000], 6)
        grads[1][8500] = bad
        outs = [torch.empty_like(t) for t in grads]
        norm, _, _ = clipped(g.GradList(grads, outs), 0.01, 0.5)
        assert not math.isfinite(float(norm))
        assert torch.equal(outs[0], grads[0] * 0.5) and torch.equal(outs[1].nan_to_num(nan=7, posinf=8), (grads[1] * 0.5).nan_to_num(nan=7, posinf=8))
    zeros = [torch.zeros(50, device="cuda")]
    norm, _, _ = clipped(g.GradList(zeros), 1.0, 1.0)
    assert float(norm) == 0 and not zeros[0].any()
    norm, _, _ = clipped(g.GradList([]), 1.0, 1.0)
    assert float(norm) == 0
    norm, _, _ = clipped(g.GradList([torch.empty(0, device="cuda")]), 1.0, 1.0)
    assert float(norm) == 0


@pytest.mark.gpu
def test_captured():
    grads = tensors("bf16", SIZES, 8)
    outs = [torch.empty_like(t, dtype=torch.float32) for t in grads]
    lst, norm = g.GradList(grads, outs), torch.empty(1, device="cuda")
    ws = torch.empty(lst.workspace, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.grad_clip(lst, 0.3, 1.0, norm, ws, torch.cuda.current_stream())
    del lst                                                                  # the graph has copies of the list
    for seed in range(3):
        for t, new in zip(grads, tensors("bf16", SIZES, 20 * seed)):
            t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        check(grads, outs, grads, norm, 0.3, 1.0)


class Fake:
    """What the list asks of a tensor."""

    def __init__(self, at, n, dtype="torch.float32", whole=True):
        self.at, self.n, self.dtype, self.whole, self.shape = at, n, dtype, whole, (n,)

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def is_contiguous(self):
        return self.whole


def test_refusals():
    name = lambda *a: pytest.raises(g.GrimError, g.GradList, *a).value.name
    A, B = 1 << 20, 1 << 21
    assert name([Fake(A, 10), Fake(A, 10)]) == "GRIM_ERR_SHAPE"                                   # the same tensor twice, in place
    assert name([Fake(A, 10), Fake(A + 36, 10)]) == "GRIM_ERR_SHAPE"
    assert name([Fake(A, 10), Fake(A + 40, 10)], [Fake(B, 10), Fake(B + 39, 10)]) == "GRIM_ERR_SHAPE"
    assert name([Fake(A, 10), Fake(A + 40, 10)], [Fake(A + 40, 10), Fake(A, 10)]) == "GRIM_ERR_SHAPE"
    assert name([Fake(A, 10, "torch.bfloat16")], [Fake(A, 10)]) == "GRIM_ERR_SHAPE"
    assert name([Fake(A, 10)], [Fake(A + 4, 10)]) == "GRIM_ERR_SHAPE"
    assert name([Fake(0, 10)]) == "GRIM_ERR_NULL"
    g.GradList([Fake(A, 10), Fake(A, 10)], [Fake(B, 10), Fake(B + 40, 10)])                       # read twice
    g.GradList([Fake(A, 10), Fake(A + 40, 10), Fake(0, 0)])
    for args in (([Fake(A, 10)], []), ([Fake(A, 10)], [Fake(B, 9)]), ([Fake(A, 10, whole=False)],), ([Fake(A, 10, "torch.float64")],)):
        with pytest.raises(ValueError):
            g.GradList(*args)
    lst = g.GradList([Fake(A, 10)])
    assert lst.workspace == 8
    bad = lambda *a: pytest.raises(g.GrimError, *a).value.name
    room = (B, 8)
    for max_norm, unscale in ((-1.0, 1.0), (math.nan, 1.0), (1.0, math.inf), (1.0, math.nan)):
        assert bad(g.grad_clip, lst, max_norm, unscale, A, room) == "GRIM_ERR_SHAPE"
    assert bad(g.grad_clip, lst, 1.0, 1.0, A, (B, 7)) == "GRIM_ERR_SHAPE"
    assert bad(g.grad_clip, lst, 1.0, 1.0, None, room) == "GRIM_ERR_NULL"
    assert bad(g.grad_norm, lst, 1.0, A, None) == "GRIM_ERR_NULL"
    none = g.GradList([Fake(A, 10)], [Fake(0, 10)])                                              # a list for norms alone
    assert bad(g.grad_clip, none, 1.0, 1.0, A, room) == "GRIM_ERR_NULL"
