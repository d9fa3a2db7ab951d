"""The group operators recorded into a CUDA graph by a process's very first calls of them."""
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

PROGRAM = """
import sys
import torch
import paper_2508_13478_b200 as dhq

kind, dtype = sys.argv[1], getattr(torch, sys.argv[2])
gen = torch.Generator(device="cuda").manual_seed(1)
t, n, k, g = 300, 264, 512, 64


def normal(*shape):
    return torch.randn(*shape, generator=gen, device="cuda").to(dtype)


x, dy = normal(t, k), normal(t, n)
codes, exponents = torch.empty(t, k, dtype=torch.int8, device="cuda"), torch.empty(t, k // g, dtype=torch.uint8, device="cuda")
w, packed, scales = normal(n, k), torch.empty(n, k // 2, dtype=torch.uint8, device="cuda"), torch.empty(n, k // g, dtype=torch.bfloat16, device="cuda")
form = dict(group=g, rotation=dhq.DHQ_ROT_INPUT)


def calls():
    outs = []
    if kind == "linear":
        dhq.dhq_w4_pack(w, packed, scales, **form)
        for rows in (1, 2, 9, 20, 40, 64):
            outs.append(torch.zeros(rows, n, dtype=dtype, device="cuda"))
            dhq.dhq_w4_linear(packed, scales, x[:rows], outs[-1], **form)
    else:
        outs += [torch.zeros_like(x), torch.zeros_like(x), torch.zeros(n, k, device="cuda"), torch.zeros(n, k, dtype=dtype, device="cuda")]
        dhq.dhq_checkpoint_save(x, codes, exponents, out=outs[0], activation=dhq.DHQ_ACT_GELU, **form)
        dhq.dhq_checkpoint_act_grad(codes, exponents, x, outs[1], activation=dhq.DHQ_ACT_GELU, **form)
        for dW in outs[2:]:
            dhq.dhq_checkpoint_weight_grad(codes, exponents, dy, dW, **form)
    return outs


torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = calls()
graph.replay()
kept = [o.clone() for o in got]
for a, b in zip(kept, calls()):
    assert torch.equal(a, b) and b.isfinite().all() and b.abs().max() > 0
print("as the eager calls")
"""


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("kind", ["linear", "checkpoint"])
def test_first_calls_of_a_process_in_a_graph(kind, dtype):
    ran = subprocess.run([sys.executable, "-c", PROGRAM, kind, dtype], capture_output=True, text=True, timeout=300)
    assert ran.returncode == 0 and "as the eager calls" in ran.stdout, ran.stderr[-2000:]
