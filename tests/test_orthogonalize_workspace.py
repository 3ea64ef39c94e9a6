"""What sdl_orthogonalize_workspace_bytes asks for (CPU only)."""
import pytest

import paper_2501_18512_amd as sdl
from test_training_refusals import INVALID, call

BYTES = sdl.sdl_orthogonalize_workspace_bytes


@pytest.mark.parametrize("out", [0, 1])
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (6000, 10, 60), (65535, 16, 16), (65535, 8, 8), (65535, 24, 24), (4000, 64, 64), (30, 96, 48), (1, 100, 131), (300, 131, 100)])
def test_matrices_that_a_workgroup_works_on_need_what_x_takes_in_fp32(batch, rows, cols, out):
    """All of them, whatever the batch: 65535 of 16 x 16 are 67 MB."""
    assert BYTES(batch, rows, cols, out) == batch * rows * cols * 4


def test_less_is_refused():
    one = 2 * 30 * 40 * 4
    assert BYTES(2, 30, 40, 1) == one
    assert call("sdl_orthogonalize", workspace_bytes=one - 1) == INVALID and call("sdl_orthogonalize", workspace=None) == INVALID


def test_larger_matrices_still_get_their_images():
    """Three images of 4 bytes an element and X in fp32, and two of n by n; of one image a half of that and less."""
    for n, m in ((400, 801), (2048, 2048), (768, 8192)):
        assert BYTES(3, n, m, 0) >= 3 * (n * m * (4 + 4 + 4) + n * n * (4 + 4))
        assert BYTES(3, n, m, 1) >= 3 * (n * m * (2 + 2 + 2) + n * n * (2 + 2))
