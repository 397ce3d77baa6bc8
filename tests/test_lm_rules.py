"""grim_apply_logit_rules against the rules written out in 64 bits.

Bounds: a division or product, three additions and the bias's sum of n values, each 2^-24 of what it adds up."""
import math

import pytest
import torch

import paper_2108_11033_amd as g
from lm_helpers import DTYPES, EPS32, TORCH, close, randn


def reference(z, r, batch, V):
    """z: batch x V in 64 bits; (result, slack)."""
    out, slack = z.clone(), torch.zeros_like(z)
    for b in range(batch):
        row = z[b].clone()
        size = row.abs()
        if r.get("history") is not None:
            n = r["max_history"] if r.get("history_len") is None else min(max(int(r["history_len"][b]), 0), r["max_history"])
            h = r["history"][b, :n].long()
            count = torch.bincount(h[(h >= 0) & (h < V)], minlength=V).double()
            pick = lambda key, none: r[key][b].double() if r.get(key) is not None else torch.tensor(none, device="cuda").double()
            rep, fr, pr = pick("repetition", 1.0), pick("frequency", 0.0), pick("presence", 0.0)
            seen = count > 0
            row = torch.where(seen, torch.where(row > 0, row / rep, row * rep) - fr * count - pr, row)
            size = torch.where(seen, size * torch.maximum(rep, 1 / rep) + (fr * count).abs() + pr.abs(), size)
        if r.get("nbias"):
            for i in range(r["nbias"]):
                v = int(r["bias_ids"][b, i])
                if 0 <= v < V:
                    row[v] += r["bias_values"][b, i].double()
                    size[v] += r["bias_values"][b, i].double().abs()
        if r.get("allowed") is not None:
            v = torch.arange(V, device="cuda")
            row[((r["allowed"][b].long()[v // 32] >> (v % 32)) & 1) == 0] = -math.inf
        out[b], slack[b] = row, (6 + r.get("nbias", 0)) * EPS32 * size
    return out, torch.nan_to_num(slack, nan=0, posinf=0)


def _rules(V, batch, L, nb, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rand = lambda *s: torch.rand(s, device="cuda", generator=gen)
    history = torch.randint(-2, V + 3, (batch, L + 2), device="cuda", generator=gen).to(torch.int32)
    history[:, : L // 2] %= max(1, V // 50)                                                     # words that come often
    lens = torch.randint(-1, L + 3, (batch,), device="cuda", generator=gen).to(torch.int32)       # some to be clamped
    lens[0] = L
    ids = torch.randint(-1, min(V, 3 * nb) + 1, (batch, nb + 1), device="cuda", generator=gen).to(torch.int32)   # words listed twice
    words = torch.randint(-2 ** 31, 2 ** 31, (batch, (V + 31) // 32 + 1), device="cuda", generator=gen).to(torch.int32)
    return dict(history=history, ld_history=L + 2, max_history=L, history_len=lens, repetition=0.7 + rand(batch), frequency=rand(batch) - 0.3,
                presence=rand(batch), bias_ids=ids, bias_values=2 * randn(seed + 1, batch, nb + 1), nbias=nb, ld_bias=nb + 1, allowed=words,
                ld_allowed=(V + 31) // 32 + 1)


def _logits(dtype, V, batch, columns, pad, seed):
    """The logits as the call takes them (a view of a guarded buffer), and a batch x V view of the same."""
    r, c = (V, batch) if columns else (batch, V)
    buf = torch.full((r, c + pad), float("nan"), dtype=TORCH[dtype], device="cuda")
    buf[:, :c] = 3 * randn(seed, r, c)
    return buf, buf[:, :c].t() if columns else buf[:, :c]


SHAPES = [(1, 1, 1, 1), (7, 3, 5, 2), (31, 1, 64, 0), (1000, 2, 300, 7), (2048, 1, 4, 1), (2049, 5, 1000, 40), (4099, 9, 17, 3), (32771, 1, 200, 16),
          (50003, 33, 5000, 128), (6000, 300, 40, 5), (700, 4, 20000, 1024)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("columns", [False, True])
@pytest.mark.parametrize("V,batch,L,nb", SHAPES)
def test_all_rules(dtype, columns, V, batch, L, nb):
    r = _rules(V, batch, L, nb, V + batch)
    buf, view = _logits(dtype, V, batch, columns, 3, V)
    view[0, 0], view[batch - 1, V - 1] = -math.inf, torch.finfo(TORCH[dtype]).min
    out, oview = _logits(dtype, V, batch, columns, 5, 1)
    out.fill_(float("nan"))
    g.logit_rules(buf, dtype, buf.stride(0), V, batch, out, out.stride(0), columns=columns, stream=torch.cuda.current_stream(), **r)
    want, slack = reference(view.double(), r, batch, V)
    close(oview, want, slack, dtype, "logits")
    width = batch if columns else V
    assert torch.isnan(out[:, width:]).all()
    g.logit_rules(buf, dtype, buf.stride(0), V, batch, buf, buf.stride(0), columns=columns, **r)      # in place
    assert torch.equal(view, oview)


@pytest.mark.gpu
@pytest.mark.parametrize("columns", [False, True])
@pytest.mark.parametrize("keep", [(), ("history",), ("history", "repetition"), ("history", "frequency"), ("history", "presence", "history_len"),
                                  ("bias_ids", "bias_values", "nbias"), ("allowed",)])
def test_each_rule_alone(columns, keep):
    V, batch, L, nb = 5000, 3, 100, 9
    full = _rules(V, batch, L, nb, 3)
    r = {k: v for k, v in full.items() if k in keep or k.startswith("ld_") or (k == "max_history" and "history" in keep)}
    buf, view = _logits("f32", V, batch, columns, 0, 4)
    out, oview = _logits("f32", V, batch, columns, 0, 5)
    g.logit_rules(buf, "f32", buf.stride(0), V, batch, out, out.stride(0), columns=columns, **r)
    want, slack = reference(view.double(), r, batch, V)
    close(oview, want, slack, "f32", str(keep))


@pytest.mark.gpu
def test_grammar_that_allows_nothing_and_nan():
    V, batch = 3000, 2
    z = randn(1, batch, V)
    z[0, 5], z[1, 6] = float("nan"), float("nan")
    allowed = torch.zeros(batch, (V + 31) // 32, dtype=torch.int32, device="cuda")
    allowed[1] = -1
    out = torch.empty_like(z)
    g.logit_rules(z, "f32", V, V, batch, out, V, allowed=allowed, ld_allowed=allowed.stride(0))
    assert (out[0] == -math.inf).all()                        # a word that may not come is not NaN either
    assert torch.isnan(out[1, 6]) and torch.equal(torch.nan_to_num(out[1]), torch.nan_to_num(z[1]))


@pytest.mark.gpu
@pytest.mark.parametrize("columns", [False, True])
def test_longest_lists_of_one_word(columns):
    """A word's count and its entry of the bias list at their most, together: a history of 2^20 times one word, that word first and last of 1024."""
    V, batch, L, nb = 1500, 2, 2 ** 20, 1024
    ids = torch.arange(100, 100 + nb, device="cuda", dtype=torch.int32).repeat(batch, 1)
    ids[:, 0] = ids[:, nb - 1] = 7
    r = dict(history=torch.full((batch, L), 7, device="cuda", dtype=torch.int32), ld_history=L, max_history=L, frequency=torch.full((batch,), 0.25, device="cuda"),
             bias_ids=ids, bias_values=randn(3, batch, nb), nbias=nb, ld_bias=nb)
    buf, view = _logits("f32", V, batch, columns, 0, 4)
    out, oview = _logits("f32", V, batch, columns, 0, 1)
    g.logit_rules(buf, "f32", buf.stride(0), V, batch, out, out.stride(0), columns=columns, **r)
    want, slack = reference(view.double(), r, batch, V)
    close(oview, want, slack, "f32", "logits")


@pytest.mark.gpu
def test_same_bits_again_and_no_callers():
    V, batch = 40000, 17
    r = _rules(V, batch, 3000, 200, 8)
    z, a, b = randn(2, batch, V).half(), torch.empty(batch, V, dtype=torch.float16, device="cuda"), torch.empty(batch, V, dtype=torch.float16, device="cuda")
    g.logit_rules(z, "f16", V, V, batch, a, V, **r)
    g.logit_rules(z, "f16", V, V, batch, b, V, **r)
    assert torch.equal(a, b)
    g.logit_rules(None, "f16", V, V, 0, None, V)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    V, batch, ld = 3000, 5, 2 ** 29 + 1
    r = _rules(V, batch, 50, 4, 9)
    values, want = randn(3, batch, V).half(), torch.empty(batch, V, dtype=torch.float16, device="cuda")
    wide = torch.empty(batch * ld, dtype=torch.float16, device="cuda").as_strided((batch, V), (ld, 1))
    wide.copy_(values)
    g.logit_rules(values, "f16", V, V, batch, want, V, **r)
    g.logit_rules(wide, "f16", ld, V, batch, wide, ld, **r)
    assert torch.equal(wide.contiguous(), want)


def test_refusals():
    def name(z=256, dt="f16", ldz=64, V=64, batch=2, out=512, ldo=64, **kw):
        with pytest.raises(g.GrimError) as e:
            g.logit_rules(z, dt, ldz, V, batch, out, ldo, **kw)
        return e.value.name

    assert name(z=None) == "GRIM_ERR_NULL" and name(out=None) == "GRIM_ERR_NULL"
    assert name(nbias=3, ld_bias=3) == "GRIM_ERR_NULL"
    for kw in [dict(ldz=63), dict(ldo=63), dict(V=0), dict(V=2 ** 31, ldz=2 ** 31, ldo=2 ** 31), dict(batch=-1), dict(columns=True, ldz=1),
               dict(history=768, ld_history=4, max_history=5), dict(history=768, max_history=-1),
               dict(nbias=-1), dict(nbias=4, ld_bias=3, bias_ids=768, bias_values=1024), dict(allowed=768, ld_allowed=1), dict(ldz=2 ** 60)]:
        assert name(**kw) == "GRIM_ERR_SHAPE", kw
    assert name(nbias=1025, ld_bias=1025, bias_ids=768, bias_values=1024) == "GRIM_ERR_UNSUPPORTED"
    assert name(history=768, max_history=2 ** 20 + 1, ld_history=2 ** 21) == "GRIM_ERR_UNSUPPORTED"
    from paper_2108_11033_amd import lm
    assert lm._lib().grim_apply_logit_rules(256, 0, 0, 64, 64, 2, None, 512, 64, None) == 1              # GRIM_ERR_NULL: no rules


# Columns of more than 2^22 logits run in tiles of 8192 places, with room for up to 128 biases a caller or for 1024; 2^22 itself is the first such call.
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,batch,L,nb", [(131075, 33, 700, 16), (131072, 64, 300, 129), (2 ** 17, 32, 5, 128), (14001, 301, 60, 40), (1400003, 3, 3000, 1024)])
def test_many_logits_in_columns(dtype, V, batch, L, nb):
    assert V * batch >= 1 << 22
    r = _rules(V, batch, L, nb, V + batch)
    buf, view = _logits(dtype, V, batch, True, 3, V)
    view[0, 0], view[batch - 1, V - 1] = -math.inf, torch.finfo(TORCH[dtype]).min
    out, oview = _logits(dtype, V, batch, True, 5, 1)
    out.fill_(float("nan"))
    call = lambda to: g.logit_rules(buf, dtype, buf.stride(0), V, batch, to, to.stride(0), columns=True, stream=torch.cuda.current_stream(), **r)
    call(out)
    # the same callers' rows a few at a time in 64 bits
    for b0 in range(0, batch, 16):
        n = min(16, batch - b0)
        some = {k: v[b0:b0 + n] if torch.is_tensor(v) else v for k, v in r.items()}
        want, slack = reference(view[b0:b0 + n].double(), some, n, V)
        close(oview[b0:b0 + n], want, slack, dtype, f"callers {b0}..")
    assert torch.isnan(out[:, batch:]).all()
    call(buf)                                                                                             # in place
    assert torch.equal(view, oview) and torch.isnan(buf[:, batch:]).all()
