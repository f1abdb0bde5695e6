"""Order of the experts' rows at the edges of its launches."""
import os
import subprocess
import sys

import pytest
import torch

from tests.conftest import ROOT
from tests.test_gpu_experts import gen, hif4, plan  # noqa: F401  (hif4: fixture)

pytestmark = pytest.mark.gpu

# Shared memory of 49088 to 49152 bytes, which with the kernel's own 68 bytes is more than a launch gets without asking
FIRST_CALLS = [(241, 8, 768), (300, 8, 767), (184, 8, 1024), (230, 8, 819)]


@pytest.mark.parametrize("T,k,E", FIRST_CALLS)
def test_plan_as_the_first_call_of_a_process(T, k, E):
    """No earlier call has asked for more shared memory on this device."""
    program = f"""
import torch
import paper_2602_11287_b200 as hif4
from tests.test_gpu_experts import gen, plan
ids = torch.randint(0, {E}, ({T}, {k}), generator=gen(1), device="cuda", dtype=torch.int32)
got, want = hif4.hif4_expert_plan(ids, {E}), plan(ids, {E})
assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
print("the plan is right")
"""
    done = subprocess.run([sys.executable, "-c", program], cwd=ROOT, env={**os.environ, "PYTHONPATH": ROOT}, capture_output=True, text=True, timeout=600)
    assert done.returncode == 0 and "the plan is right" in done.stdout, done.stderr[-2000:]


# fewer warps with assignments than the sums over the experts take; experts past one pass of these sums
@pytest.mark.parametrize("T,k,E", FIRST_CALLS + [(1, 1, 1000), (3, 8, 1024), (17, 8, 600), (20, 8, 513), (16, 8, 512), (256, 8, 511), (257, 8, 513), (2048, 1, 1023), (4097, 32, 1024)])
@pytest.mark.parametrize("drop", [0.0, 0.3, 1.0])
def test_plan(hif4, T, k, E, drop):  # noqa: F811
    g = gen(T + E)
    ids = torch.randint(0, E, (T, k), generator=g, device="cuda", dtype=torch.int32)
    ids[torch.rand(T, k, generator=g, device="cuda") < drop] = -1
    if drop == 0.3:
        ids[T // 2, 0], ids[T // 3, -1] = E, 2 ** 31 - 1
    off, row_of = hif4.hif4_expert_plan(ids, E)
    want = plan(ids, E)
    assert torch.equal(off, want[0]) and torch.equal(row_of, want[1])
