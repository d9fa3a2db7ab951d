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


def test_weight_gradients_of_more_blocks_than_a_launch_has():
    need = C.c_int64(-1)
    ask = groups._functions()["dhq_checkpoint_weight_grad_workspace"]
    rows = (1 << 31) - 1
    for t, n, k, kind, out in ((rows, 1 << 20, 1 << 20, 2, 2), (rows, 1 << 14, 1 << 24, 2, 2), (rows, 1 << 24, 1 << 18, 1, 1)):
        assert ask(t, n, k, 64, dhq.DHQ_ROT_NONE, kind, 1 << 20, n, out, C.byref(need)) == 2, (t, n, k)
    # the most rows, for one tile: a part of it (128 x 128 sums) for every 16,384 of fp16
    assert ask(rows, 64, 64, 64, dhq.DHQ_ROT_NONE, 2, 1 << 20, 64, 2, C.byref(need)) == 0 and need.value == (1 << 17) * 128 * 128 * 4
    assert ask(8192, 8192, 8192, 128, dhq.DHQ_ROT_INPUT, 1, 1 << 20, 8192, 1, C.byref(need)) == 0


def test_the_binding_asks_the_library_for_every_size(monkeypatch):
    """No rule of the library's is repeated in Python: what dhq_w4_linear_workspace says is what the call gets."""
    torch = pytest.importorskip("torch")
    seen = []

    def need(name, t, n, k, group, rotation, kind):
        seen.append((name, t, k))
        return 0

    class Stop(Exception):
        pass

    def stop(*_):
        raise Stop

    monkeypatch.setattr(groups, "_need", need)
    if hasattr(groups, "_linear_need"):   # (answers of this test's own are not remembered)
        monkeypatch.setattr(groups, "_linear_need", lambda *sizes: need("dhq_w4_linear_workspace", *sizes))
    monkeypatch.setattr(groups, "_matrix", lambda t, what: (*t.shape, t.shape[1], 0, 1 << 20))
    monkeypatch.setattr(groups, "_result", lambda t, *_: (t.shape[1], 1 << 20))
    monkeypatch.setattr(groups, "_stream_of", lambda *_: None)
    monkeypatch.setattr(groups, "_store", stop)
    for t, k in ((1, 64), (2, 4000), (3, 64), (1, 9000)):
        with pytest.raises(Stop):
            groups.dhq_w4_linear(None, None, torch.zeros(t, k), torch.zeros(t, 24), group=32)
        assert seen[-1][1:] == (t, k)
