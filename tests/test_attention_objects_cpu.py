"""Where the kernels of attention over the cache are compiled: once each, by the file of their type."""
import os
import re

import pytest

import __graft_entry__ as entry

KERNEL = re.compile(rb"_ZN3lba17cache_attn_kernelI(\w+?)EEvNS_15CacheAttnParamsE")


def kernels(source):
    path = os.path.join(entry.BUILD_DIR, source + ".o")
    if not os.path.exists(path):
        pytest.skip("no object of a build here")
    with open(path, "rb") as f:
        return set(KERNEL.findall(f.read()))


def test_kernels_are_compiled_once():
    bf16, f32 = kernels("lba_cache_attn_bf16"), kernels("lba_cache_attn_f32")
    assert len(bf16) == 16 and len(f32) == 8 and not bf16 & f32      # D, rows of a tile, pieces of the weights
    assert not kernels("lba_cache_attn")
