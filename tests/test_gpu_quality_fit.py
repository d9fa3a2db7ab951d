"""The fit of the quality harness runs the form of checkpoints that it is asked for."""
import numpy as np
import pytest

import dhq_inputs
from paper_2508_13478_b200 import binding, quality, training

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gabor_s0", [0.0, 3.0])
@pytest.mark.parametrize("rotation", [None, binding.DHQ_ROT_INPUT, binding.DHQ_ROT_NONE])
def test_rotation_of_the_checkpoints(monkeypatch, rotation, gabor_s0):
    seen = []
    for name in ("dhq_checkpoint_save", "dhq_checkpoint_weight_grad", "dhq_checkpoint_act_grad"):
        call = getattr(training, name)
        monkeypatch.setattr(training, name, lambda *a, call=call, **kw: (seen.append((kw["group"], kw["rotation"])), call(*a, **kw))[1])
    asked = {} if rotation is None else {"checkpoint_rotation": rotation}
    target = np.zeros((16 * 16, 3), dtype=np.float32)
    weights, biases, out = quality.fit_network((2, 64, 64, 3), 30.0, target, dhq_inputs.grid_coords(16, 16), 2, 1e-4, 7, gabor_s0, checkpoints=32, **asked)
    assert set(seen) == {(32, binding.DHQ_ROT_INPUT if rotation is None else rotation)}   # (rotated by default)
    assert all(np.isfinite(w).all() for w in weights + biases) and np.isfinite(out).all()
