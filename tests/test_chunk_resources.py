"""The compiler gave the kernels of santa_rope_append, santa_attend_chunk and santa_decode_window
registers for everything: a spilled one is read back through the counter that the copies into LDS
are waited for with, and stalls them (measured: 562 against 837 us on an 8k prompt)."""

import os

import pytest

from tests.test_kernel_resources import READELF, scratch_bytes


@pytest.mark.skipif(not os.path.exists(READELF), reason="no llvm-readelf")
def test_no_scratch(tmp_path):
    scratch = scratch_bytes(tmp_path)
    for kernel in ("k_rope_append", "k_attend_few", "k_attend_many", "k_attend_merge"):
        found = {n: b for n, b in scratch.items() if f"{len(kernel)}{kernel}I" in n}
        assert found, kernel
        assert not any(found.values()), {n: b for n, b in found.items() if b}
