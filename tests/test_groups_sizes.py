"""Sizes of workspaces, on the CPU: as the library states them, and as the binding asks for them."""
import ctypes as C

import pytest

import paper_2508_13478_b200 as dhq
from paper_2508_13478_b200 import groups


@pytest.mark.parametrize("t,n,k,group,kind", [((1 << 31) - 1, 16, 1 << 24, 32, 1), ((1 << 31) - 1, 1 << 24, 1 << 24, 128, 0), (1 << 30, 5, 1 << 20, 64, 2),
                                              (100000, 64, 8192, 32, 0), (9, 4, 100, 32, 1), (65, 16, 4097, 64, 2)])
@pytest.mark.parametrize("rotation", [dhq.DHQ_ROT_INPUT, dhq.DHQ_ROT_NONE])
def test_workspace_of_products_of_any_size(t, n, k, group, kind, rotation):
    # terms as fp16 numbers for whole blocks of 256 inputs and up to 64 columns, a factor and an offset (8 bytes) for each group of a column
    terms = 2 if kind == 0 or (kind == 2 and rotation == dhq.DHQ_ROT_INPUT) else 1
    width = next(w for w in (8, 16, 32, 64) if min(64, t * terms) <= w)
    tokens = min(width // terms, t)
    columns = -(-t // tokens) * width
    blocks = -(-k // 256)
    need = C.c_int64(-1)
    assert groups._functions()["dhq_w4_linear_workspace"](t, n, k, group, rotation, kind, C.byref(need)) == 0
    assert need.value == columns * blocks * 256 * 2 + columns * blocks * (256 // group) * 8
