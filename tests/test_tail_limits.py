"""Limits of the trained tail's descriptors (no GPU needed)."""
import pytest

import paper_2210_08650_amd as H


@pytest.mark.parametrize("t", [3e-39, 1e-25, 2.0 ** -61, 2.0 ** 61, 1e25, 3e38, -1.0])
def test_temperatures_whose_square_or_reciprocal_is_lost_are_refused(t):
    d = H.Head(H.HAPI_F32, 4, 64, 10, top=2, temperature=t)
    with pytest.raises(H.HapiError) as e:
        H.hapi_head_workspace_bytes(d, True)
    assert e.value.code == H.HAPI_E_INVAL and "temperature" in str(e.value)


@pytest.mark.parametrize("t", [2.0 ** -60, 1e-3, 1.0, 1e3, 2.0 ** 60])
def test_temperatures_in_range(t):
    assert H.hapi_head_workspace_bytes(H.Head(H.HAPI_F32, 4, 64, 10, top=2, temperature=t), True) > 0
