"""The drafting example reports what its gate reports, all but the -1 behind a row's tokens."""
import pytest

from paper_2607_20791_gb300 import binding
from test_gpu_drafted_decode import _example

pytestmark = pytest.mark.gpu


def test_the_gates_status_is_reported(gpu_lib):
    d, _, _ = _example().run(draft=3, steps=2)
    assert int(d.gate_status.item()) in (0, binding.RGD_DEV_BAD_TOKEN)
    d.check()
    for bit in (binding.RGD_DEV_WAIT_TIMEOUT, binding.RGD_DEV_BAD_PARAM):
        d.gate_status.fill_(bit | binding.RGD_DEV_BAD_TOKEN)
        with pytest.raises(RuntimeError, match=str(bit)):
            d.check()
