"""The generator's state on the device is not looked at without dropout, whatever the pointer is (no GPU: valid calls get as far as
asking for the device)."""
import pytest

from paper_2306_06098_b200 import binding as B
from test_rows_abi import CALLS, FAKE, desc, no_gpu


@no_gpu
@pytest.mark.parametrize("call", CALLS)
def test_a_pointer_that_is_not_looked_at(call):
    assert call(desc(p=0.0, rng=FAKE + 4)) == B.ECUDA


@no_gpu
@pytest.mark.parametrize("call", [c for c in CALLS if c.__name__ != "quantize"])
def test_one_that_is(call):
    more = {"h": FAKE} if call.__name__ == "forward" else {}
    assert call(desc(p=0.1, rng=FAKE), **more) == B.ECUDA
    assert call(desc(p=0.1, rng=FAKE + 4), **more) == B.EINVAL
