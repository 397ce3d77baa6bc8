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
