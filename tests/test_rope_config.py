"""Configurations whose numbers leave the range of what is kept: refused, like those that are not finite."""
import pytest

import paper_2607_09153_gb300 as kp


@pytest.mark.parametrize("bad", [dict(magnitude=1e39), dict(magnitude=-1e39), dict(base=1e300, scaling="base", factor=1e10)])
def test_out_of_range(bad):
    with pytest.raises(kp.KvprmError) as e:
        kp.Rope(64, **bad)
    assert e.value.code == kp.KVPRM_EINVAL and "kvprm_rope_create" in str(e.value)


def test_in_range():
    for fine in (dict(magnitude=3e38), dict(magnitude=-0.5), dict(base=1e30, scaling="base", factor=1e10)):
        assert len(kp.Rope(64, **fine).turns()) == 32
