"""Settings of verify_attn_scored that the call's 32 bits cannot hold."""
import pytest

import paper_2508_21706_amd as pkg
from test_gpu_devices import inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("softcap", [1e-50, -1e-50, 1e-42, 1e39, float("nan")])
def test_caps_out_of_range_are_not_taken_for_off(softcap):
    x = inputs()
    with pytest.raises(pkg.SpecMoEError) as e:
        pkg.verify_attn_scored(x["q"], x["k"], x["v"], x["ctx"], x["chunk"], 0.125, softcap=softcap)
    assert e.value.status == -17
