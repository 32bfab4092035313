"""Numbers that the binding of sampling and routing hands to the library: none is cut to
the width of its field."""
import pytest
import torch

import paper_1805_02867_amd as osm


def test_a_top_k_of_any_size():
    """0, negative or at least V: all."""
    x = torch.zeros(2, 8)
    for k, want in ((5, 5), (0, 0), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1),
                    (2 ** 32 + 5, 2 ** 31 - 1), (-2 ** 31 - 1, -2 ** 31), (-2 ** 40 + 3, -2 ** 31)):
        pointer, number = osm._setting(k, torch.int32, x, 2, "top_k")
        assert pointer is None
        assert osm.SampleParams(None, None, None, None, 1.0, number, 1.0, 0.0).top_k_all == want


@pytest.mark.parametrize("place", range(4))
@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32 + 1, -2 ** 32 + 1])
def test_router_options_outside_of_their_type(place, value):
    args = [0, 1, 1, 1]
    args[place] = value
    with pytest.raises(ValueError):
        osm._route(*args, True, 1.0)


def test_scales_that_compare_equal_are_told_apart():
    def sign(scale):
        return str(osm._route(0, 1, 1, 1, True, scale)._obj.scale)
    assert [sign(0.0), sign(-0.0), sign(0.0)] == ["0.0", "-0.0", "0.0"]
