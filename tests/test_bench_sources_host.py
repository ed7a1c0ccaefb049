"""The traffic figures of bench.py are tied to the sources of the kernels they were measured on: every header of this library that
these sources include has to be among them."""
import os
import re

import pytest

import bench

CSRC = os.path.join(os.path.dirname(os.path.abspath(bench.__file__)), "paper_2603_04428_amd", "csrc")


@pytest.mark.parametrize("name", ["DECODE_FILES", "LATENT_FILES", "CODEC_FILES", "CHUNK_FILES"])
def test_every_included_header_is_hashed(name):
    files = getattr(bench, name)
    for f in files:
        with open(os.path.join(CSRC, f)) as src:
            included = re.findall(r'^#include "([^"/]+)"', src.read(), re.M)
        assert set(included) <= set(files), f
