"""Shared plumbing of the language-model operators' tests: strided operands with guarded surroundings, and error bounds in the
form unit roundoff of the result's type x |result| + (a count of fp32 roundings) x 2^-24 x (the sum of the terms' sizes)."""
import torch

DTYPES = ["f32", "f16", "bf16"]
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}       # half a unit in the last place, relative
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}    # half the smallest number, absolute
EPS32 = 2.0 ** -24


def rows(values, dtype, pad=0, offset=0):
    """The values as rows of width + pad elements, `offset` elements into a buffer of NaN: (view, whole buffer)."""
    n, c = values.shape
    buf = torch.full((n * (c + pad) + offset + 8,), float("nan"), dtype=TORCH[dtype], device="cuda")
    view = buf[offset:offset + n * (c + pad)].view(n, c + pad)[:, :c]
    view.copy_(values)
    return view, buf


def out_rows(n, c, dtype, pad=0, offset=0):
    return rows(torch.full((n, c), float("nan"), device="cuda"), dtype, pad, offset)


def untouched(view, buf):
    """Nothing around the rows was written."""
    if view.numel() == 0:
        return bool(torch.isnan(buf).all())
    probe = buf.clone()
    probe.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(float("nan"))
    return bool(torch.isnan(probe).all())


def randn(seed, *shape):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(shape, dtype=torch.float32, device="cuda", generator=gen)


def close(got, want, slack, dtype, what):
    """|got - want| <= unit x |want| + slack (64-bit tensors of what arithmetic in fp32 may be off by), element by element;
    infinities and NaN in the same places."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    inf = odd & ~torch.isnan(want)
    assert bool((got[inf] == want[inf]).all()), f"{what}: infinities differ"
    bound = UNIT[dtype] * want.abs() * (1 + 2.0 ** -7) + slack + TINY[dtype]
    over = (got - want).abs()[~odd] - bound.expand_as(want)[~odd]
    if over.numel():
        worst = float(over.max())
        assert worst <= 0, f"{what}: {worst:.3e} above its bound (largest value {float(want[~odd].abs().max()):.3e})"
