"""Chunk attention's requests into LDS, read in the assembly that its source compiles to (no GPU): they are written as inline assembly, in front of which the
compiler inserts no wait for what it has written."""
import os

import pytest
from test_device_code_cpu import CSRC, assembly, late_writers


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    code = assembly(os.path.join(CSRC, "kv8_chunk.hip"), tmp_path_factory.mktemp("asm") / "kv8_chunk.s")
    return {n: v for n, v in code.items() if "kv8_chunk_kernel" in n}


def test_requests_read_an_address_that_is_there(kernels):
    assert len(kernels) == 4
    for name, code in kernels.items():
        assert sum(s.startswith("global_load_lds") for s in code) >= 8, name
        assert not late_writers(code), name


def test_each_request_sets_its_place_in_lds(kernels):
    """m0 is written directly in front of a request, or of the two that read a page's halves 1 KiB apart."""
    for name, code in kernels.items():
        for i, s in enumerate(code):
            if s.startswith("global_load_lds"):
                j = i - 1
                while code[j].startswith(("s_nop", "global_load_lds")):
                    j -= 1
                assert code[j].startswith("s_mov_b32 m0,"), (name, code[j:i + 1])
