"""The sizes of workspaces and states for any numbers: no GPU is needed to ask for them, and none makes the library end the program."""
import pytest

import paper_2108_11033_amd as g

EDGES = [-2 ** 63, -1, 0, 1, 7, 64, 2 ** 21, 2 ** 30, 2 ** 31 - 1, 2 ** 31, 2 ** 40, 2 ** 40 + 1, 2 ** 56, 2 ** 58, 2 ** 60, 2 ** 61, 2 ** 62, 2 ** 63 - 1]


@pytest.mark.parametrize("fn", [g.layer_norm_workspace, g.glr_workspace, g.glr_states, g.distill_topk_workspace])
def test_sizes_of_any_numbers(fn):
    for rows in EDGES:
        for width in EDGES:
            n = fn(rows, width)
            assert 0 <= n < 2 ** 62, (rows, width, n)
            if rows >= 2 ** 31 or width > 2 ** 40 or rows < 0 or width < 1:
                assert n == 0, (rows, width, n)                       # calls of such sizes are refused


class _Room:
    """A buffer as other libraries hand it over: an address and a size."""
    def __init__(self, nbytes):
        self.nbytes = nbytes

    @staticmethod
    def data_ptr():
        return 1 << 20


def test_workspaces_as_addresses():
    """A workspace may be an address with its size: too small ones are refused as they are of tensors, an address alone says what is missing."""
    N, H, V, k = 100, 64, 100, 4
    A = 1 << 22
    calls = [(g.layer_norm_workspace(N, H), lambda ws: g.layer_norm_backward(A, H, A + 4096, H, "f16", None, A, A, N, H, None, 0, A, None, ws)),
             (g.glr_workspace(N, H), lambda ws: g.glr_sequence(A, "f16", 3 * H, None, None, None, 1, N, H, A, H, None, None, ws)),
             (g.glr_workspace(N, H), lambda ws: g.glr_sequence_backward(A, "f16", 3 * H, None, None, None, 1, N, H, A, A, H, None, A, 3 * H, None, None, ws)),
             (g.distill_topk_workspace(N, V), lambda ws: g.distill_topk(A, "f16", V, A, A, k, k, 1.0, None, N, V, A, None, 0, ws))]
    for need, call in calls:
        for ws in (_Room(need - 1), ((1 << 20), need - 1), (_Room(0), need - 1)):
            with pytest.raises(g.GrimError) as e:
                call(ws)
            assert e.value.name == "GRIM_ERR_SHAPE"
        with pytest.raises(g.GrimError) as e:
            call((None, need))
        assert e.value.name == "GRIM_ERR_NULL"
        with pytest.raises(TypeError, match="size"):
            call(1 << 20)


@pytest.mark.gpu
def test_a_workspace_given_by_its_address():
    import torch
    N, C = 50, 200
    x, dy, mean, rstd = torch.randn(N, C, device="cuda"), torch.randn(N, C, device="cuda"), torch.zeros(N, device="cuda"), torch.ones(N, device="cuda")
    ws = torch.empty(g.layer_norm_workspace(N, C), dtype=torch.uint8, device="cuda")
    a, b = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    g.layer_norm_backward(dy, C, x, C, "f32", None, mean, rstd, N, C, None, 0, a, None, ws)
    g.layer_norm_backward(dy, C, x, C, "f32", None, mean, rstd, N, C, None, 0, b, None, (ws.data_ptr(), ws.nbytes))
    assert torch.equal(a, b)
