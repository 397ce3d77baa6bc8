"""Calls in place need one leading dimension: rows that move would be written over rows that other workgroups have yet to read."""
import pytest

import paper_2108_11033_amd as g

A, B, C, D, E, WS = (1 << 20 << i for i in range(6))


class _Room:
    nbytes = 1 << 40

    @staticmethod
    def data_ptr():
        return WS


def _name(fn, *args, **kw):
    with pytest.raises(g.GrimError) as e:
        fn(*args, **kw)
    return e.value.name


def test_other_leading_dimensions_in_place_are_refused():
    for ld, out in [(64, 72), (72, 64)]:
        assert _name(g.layer_norm, A, "f16", ld, None, None, 1e-5, 4, 64, A, out) == "GRIM_ERR_SHAPE"
        assert _name(g.layer_norm_backward, A, ld, B, 64, "f16", None, C, D, 4, 64, A, out, None, None, None) == "GRIM_ERR_SHAPE"
        assert _name(g.distill_topk, A, "f16", ld, B, C, 2, 2, 1.0, None, 4, 64, D, A, out, _Room) == "GRIM_ERR_SHAPE"
        assert _name(g.logit_rules, A, "f16", ld, 64, 4, A, out, allowed=B, ld_allowed=2) == "GRIM_ERR_SHAPE"
        assert _name(g.logit_rules, A, "f16", ld, 64, 4, A, out, columns=True, allowed=B, ld_allowed=2) == "GRIM_ERR_SHAPE"
        assert _name(g.glr_step, A, 72, None, B, ld, B, out, D, "f16", 72, 64, 4) == "GRIM_ERR_SHAPE"


@pytest.mark.gpu
def test_one_row_in_place_has_no_leading_dimension():
    import torch
    V, H = 100, 1
    z, want = torch.randn(1, V, device="cuda"), torch.empty(1, V, device="cuda")
    allowed = torch.full((1, 4), 0x55555555, dtype=torch.int32, device="cuda")
    g.logit_rules(z, "f32", V, V, 1, want, V, allowed=allowed, ld_allowed=4)
    g.logit_rules(z, "f32", V, V, 1, z, V + 7, allowed=allowed, ld_allowed=4)
    assert torch.equal(z, want)
    x = torch.randn(1, V, device="cuda")
    g.layer_norm(x, "f32", V, None, None, 1e-5, 1, V, want, V)
    g.layer_norm(x, "f32", V, None, None, 1e-5, 1, V, x, V + 7)
    assert torch.equal(x, want)
    gates, h, new = torch.randn(3 * H, 5, device="cuda"), torch.randn(H, 5, device="cuda"), torch.empty(H, 5, device="cuda")
    g.glr_step(gates, 5, None, h, 5, new, 5, None, "f32", 0, H, 5)
    g.glr_step(gates, 5, None, h, 5, h, 9, None, "f32", 0, H, 5)
    assert torch.equal(h, new)
