"""What the built kernels on packed batches take of a compute unit (registers a lane, scratch), which the waves they are launched for rest
on: a SIMD has 512 vector registers, in blocks of 8 a wave."""
import re

import pytest

from test_kernel_resources import kernels  # noqa: F401 (a fixture)


def named(kernels, pattern):
    found = {n: k for n, k in kernels.items() if re.search(pattern, n)}
    assert found, pattern
    return found


@pytest.mark.parametrize("pattern, waves", [
    (r"\d+k_packed_(scan|ends)I", 4),                            # the tile rule's most
    (r"\d+k_packed_bwd_endsI\w+Li\dELb1E", 3),                   # whole waves of states; the others two
    (r"\d+k_packed_bwd_endsI\w+Li\dELb0E", 2),
    (r"\d+k_packed_bwdI", 2),
    (r"\d+k_conv_packed_bwdI", 3),                               # runs are cut for three
    (r"\d+k_packed_stepI", 8),
])
def test_registers_leave_room_for_the_waves(kernels, pattern, waves):  # noqa: F811
    for name, k in named(kernels, pattern).items():
        assert k[".vgpr_count"] <= 512 // waves // 8 * 8, name


def test_scratch(kernels):  # noqa: F811
    """None, but for the gradients of more than 64 states: eight waves with all of a compute unit's LDS keep one register there."""
    for name, k in named(kernels, r"\d+k_(pack|packed|conv_packed)_?").items():
        most = 8 if re.search(r"k_packed_bwdI\w+Li8E", name) else 0
        assert k[".private_segment_fixed_size"] <= most and k[".vgpr_spill_count"] <= most // 8, name
        assert k[".group_segment_fixed_size"] <= 160 * 1024, name
