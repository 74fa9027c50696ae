"""What include/sketchssm_attention.h says a call takes, against what the library takes, on the CPU: no call here gets to a launch."""
import re

import pytest

from paper_2609_33051_amd import binding as B
from paper_2609_33051_amd import build
from test_attention_abi_cpu import M, lib, rot  # noqa: F401


@pytest.mark.parametrize("io", [B.BF16, B.F32])
def test_channels_of_rotary(lib, io):  # noqa: F811
    """The header names a multiple and a largest number of channels, for either type; those are taken and others are not."""
    text = open(build.INCLUDE + "/sketchssm_attention.h").read()
    step, most = map(int, re.search(r"sketchssm_rotary -- .*\(dim a multiple of (\d+), up to (\d+)\)", text).groups())
    call = lambda D: lib.sketchssm_rotary(io, 0, 3, D, rot(rotated=2), 6 * M, 4 * most, most, 7 * M, 4 * most, most, None)  # noqa: E731
    for D in range(1, most + 2 * step):
        assert (call(D) == 0) == (D % step == 0 and D <= most), D
