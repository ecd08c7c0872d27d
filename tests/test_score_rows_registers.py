"""Registers and scratch memory of the score rows' kernels, from the compiler's remarks (no device needed)."""
import re

import pytest


@pytest.fixture(scope="module")
def usage():
    from paper_2306_15685_amd import build
    return build.resource_usage()


def test_tiles_keep_two_waves_on_a_simd(usage):
    """At most 256 registers.  Tiles of 128 x 256 need all of them and may spill a few numbers that are used once a tile; no
    other tile spills."""
    tiles = {k: v for k, v in usage.items() if "tile_kernel" in k}
    assert len(tiles) == 2 * 3 * 2 * 4 + 3 * 2   # (16-bit types x output types x activation or not x four sizes; fp32: one size)
    for k, v in tiles.items():
        kind = re.search(r"Lb([01])ELi1ELi4ELi(\d)ELi(\d)E", k).groups()
        limit = 16 if kind[1:] == ("8", "4") else 0
        assert v["vgprs"] <= 256 and v["scratch"] <= limit, (k, v)
        if kind[1:] in (("2", "2"), ("4", "2")):
            assert v["vgprs"] <= 128, (k, v)   # (four waves)


def test_waves_that_share_k_and_label_sampling_spill_nothing(usage):
    narrow = {k: v for k, v in usage.items() if "narrow_kernel" in k}
    sample = {k: v for k, v in usage.items() if "sample_kernel" in k}
    assert len(narrow) == 8 and len(sample) == 12
    for k, v in {**narrow, **sample}.items():
        assert v["vgprs"] <= 128 and v["scratch"] == 0, (k, v)
    for k, v in sample.items():   # (a held row has 144 KB of the 160 beside this)
        assert v["lds"] <= (16 * 1024 if k.count("Lb1E") else 80 * 1024), (k, v)
