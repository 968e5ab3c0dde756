"""Sizes of checkpoints that no 64-bit product holds (no GPU needed)."""
import pytest

from paper_1901_09290_b200 import binding as B
from paper_1901_09290_b200 import build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def test_scale_bytes_do_not_wrap():
    for npix, C in ((1 << 62, 256), (1 << 60, 2048), ((1 << 63) - 1, 1), ((1 << 40) + 1, 8), (1 << 40, 2049), (10, (1 << 31) - 1)):
        assert B.pt_act_scale_bytes(npix, C) == 0, (npix, C)
    assert B.pt_act_scale_bytes(1 << 40, 2048) == 64 << 40 and B.pt_act_scale_bytes(3, 2048) == 192
