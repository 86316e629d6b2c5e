"""Draft verification at the ends of its parameters' ranges, vs the fp64 oracle."""
import numpy as np
import pytest

from paper_2607_20791_gb300 import binding
from test_gpu_verify import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("certain", [False, True])
def test_a_cutoff_past_fp32_keeps_everything(gpu_lib, certain):
    """T ln p_min below fp32's range is -inf: every row is decided, and the workspace serves the next call."""
    c = Case(24, 3, 600, "f32", seed=21, certain=certain, temps=(3.3e36, 1e37, 1e38, 3e38), min_ps=(0.01, 1e-30, 0.3), probe_every=100)
    c.active[:] = 1
    with np.errstate(over="ignore"):
        c.run().check()
    assert not bool(c.ws.any())
    after = Case(24, 3, 600, "f32", seed=22)
    after.run(workspace=c.ws).check()
    assert not bool(c.ws.any())
