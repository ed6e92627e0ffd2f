"""Instructions that the library must not contain, as every rank of a program on several GPUs loads it."""
from __future__ import annotations

import os
import re

import pytest

from paper_2608_12574_gb300 import _build


@pytest.mark.parametrize("name", sorted(os.listdir(_build.CSRC)))
def test_no_multicast_loads(name):
    """Copies that write the shared memory of several CTAs at once: only for programs on one GPU, reading its own
    memory. (An MMA's arrival on both CTAs of a pair, tcgen05.commit, is none.)"""
    with open(os.path.join(_build.CSRC, name)) as f:
        text = re.sub(r'"\s*"', "", f.read())  # a string's parts
    assert not re.findall(r"cp\.async\.bulk[^;\"]*\.multicast", text)
