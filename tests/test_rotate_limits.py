"""Sizes octo_op_rotate refuses because no launch takes them, without a GPU."""
import ctypes as C

import pytest

from paper_2502_01277_amd import binding
from test_tokens_host import _rotate_op


@pytest.mark.parametrize("dim,dtype,n,heads,x,pairs", [(256, 2, 2 ** 30, 1, 8192, (128, 0)), (256, 0, 2 ** 31 - 2 ** 17, 1, 8192, (64, 64)), (128, 1, 2 ** 20, 1024, 8194, (64, 0)),
                                                       (126, 2, 2 ** 27, 15, 8192, (63, 0))])
def test_more_blocks_than_a_launch_takes(dim, dtype, n, heads, x, pairs):
    op = _rotate_op()
    op.dim, op.dtype, op.n_tokens = dim, dtype, n
    op.sections[:2] = pairs
    p = op.part[0]
    p.heads, p.d_x, p.x_token, p.x_head, p.y_token, p.y_head = heads, x, dim * heads, dim, dim * heads, dim
    assert binding.lib().octo_op_rotate(C.byref(op), None) == binding.EINVAL
