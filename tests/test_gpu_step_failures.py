"""A failure of the device's is raised, and not taken for a refusal after which the call is made once more."""
import pytest
import torch

from paper_2605_04478_amd import ccld, step
from tests.test_step_calls import _arguments

DEV = "cuda:0"


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(_arguments("cpu")))
def test_a_failure_is_raised_by_the_first_call(name):
    """The runtime keeps a thread's last error, here that of asking for a device that there is not, for the launch that asks next."""
    L, args = ccld.lib(), _arguments(DEV)[name]
    several = lambda out: out if isinstance(out, tuple) else (out,)
    want = several(getattr(step, name)(*args))
    try:
        assert L.hipSetDevice(9999) != 0
        with pytest.raises(ccld.CcldError, match=f"ccld_{name}: E_HIP") as e:
            getattr(step, name)(*args)
    finally:
        L.hipGetLastError()
    assert e.value.name == "E_HIP" and e.value.status == -11
    assert all(torch.equal(a, b) for a, b in zip(several(getattr(step, name)(*args)), want))
