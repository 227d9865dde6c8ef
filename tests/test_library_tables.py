"""What the host refuses of the page tables' buffers, on the CPU: the library's
host code linked with stand-ins for the kernels (stub_launches.cpp)."""

import ctypes

import pytest

import paper_2512_20968_amd as ma
from paper_2512_20968_amd import _binding as b

from helpers import cache_host_library

REQUESTS, FREE, ROWS, MAX_PAGES = 3, 5, 7, 4
# Bytes of every buffer, in the order of the arguments.
INPUTS = dict(lens=4 * REQUESTS, new_lens=4 * REQUESTS, free_pages=4 * FREE,
              free_range=8)
OUTPUTS = dict(block_table=4 * REQUESTS * MAX_PAGES, lens_out=4 * REQUESTS,
               cu_new=4 * (REQUESTS + 1), slots=8 * ROWS, positions=4 * ROWS,
               free_range_out=8, refused=4)
SIZES = dict(INPUTS, **OUTPUTS)
APART = {name: 0x10000 * (i + 1) for i, name in enumerate(SIZES)}


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    lib = cache_host_library(tmp_path_factory.mktemp("tables"))
    if lib is None:
        pytest.skip("g++ not available")
    cache = ma.Cache.make(dict(num_pages=8, page_size=16, num_kv_heads=2,
                               head_dim=64, max_pages=MAX_PAGES))

    def tables(at, requests=REQUESTS, free=FREE, rows=ROWS):
        return lib.mesh_attn_cache_tables(
            ctypes.byref(cache), requests, at["lens"], at["new_lens"],
            at["free_pages"], free, at["free_range"], at["block_table"],
            at["lens_out"], at["cu_new"], rows, at["slots"], at["positions"],
            at["free_range_out"], at["refused"], None)

    return tables


@pytest.mark.parametrize("out", OUTPUTS)
def test_an_output_over_another_buffer_is_refused(call, out):
    """The outermost addresses that overlap are refused, the next ones are
    not."""
    assert call(APART) == b.MA_OK
    align = 8 if out == "slots" else 4
    for other in SIZES:
        if other == out:
            continue
        last = (SIZES[other] - 1) // align * align
        first = -((SIZES[out] - 1) // align * align)
        for at in (0, first, last):
            assert call(dict(APART, **{out: APART[other] + at})) \
                == b.MA_ERR_INVALID_ARG, (other, at)
        for at in (first - align, last + align):
            assert call(dict(APART, **{out: APART[other] + at})) \
                == b.MA_OK, (other, at)


def test_buffers_of_no_bytes_overlap_nothing(call):
    at = dict(APART, slots=APART["cu_new"], positions=APART["lens"])
    assert call(at) == b.MA_ERR_INVALID_ARG
    assert call(at, rows=0) == b.MA_OK
    at = dict(APART, lens=APART["refused"], new_lens=APART["refused"],
              lens_out=APART["refused"], block_table=APART["refused"],
              free_pages=APART["refused"])
    assert call(at) == b.MA_ERR_INVALID_ARG
    assert call(at, requests=0, free=0) == b.MA_OK


def test_inputs_may_overlap(call):
    assert call(dict(APART, lens=APART["new_lens"])) == b.MA_OK
