"""Which rows of A the adapters' kernels load (csrc/adapter_rows.h), tried on the
host for every rank: loads are unconditional, so a rank past an adapter's own has
to fall back to a row of the same adapter, also in blocks that begin past the
rank (ranks 33 to 48 and 65 to 112), where one of the last adapter's would
otherwise lie past the end of A."""
import ctypes as ct
import os
import subprocess

import pytest

import paper_2607_08643_amd as bsq

CSRC = os.path.join(os.path.dirname(bsq.__file__), "csrc")

SOURCE = """
#include "adapter_rows.h"
extern "C" int blocks(int rank) { return bsq::rank_blocks(rank); }
extern "C" long long row(long long ad, int rank, int r, int own) { return bsq::adapter_row(ad, rank, r, own); }
"""


@pytest.fixture(scope="module")
def rows(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows")
    src, so = d / "rows.cpp", d / "rows.so"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
    lib = ct.CDLL(str(so))
    lib.row.restype, lib.row.argtypes = ct.c_longlong, [ct.c_longlong, ct.c_int, ct.c_int, ct.c_int]
    return lib


@pytest.mark.parametrize("rank", range(1, 129))
def test_every_row_is_of_the_adapter(rank, rows):
    blocks = rows.blocks(rank)
    assert 16 * blocks >= rank
    for own in sorted({0, 1, rank // 2, rank - 1, rank}):
        for ad in (0, 1, 1023):
            for r in range(16 * blocks):
                got = rows.row(ad, rank, r, own)
                assert ad * rank <= got < (ad + 1) * rank, (own, ad, r)
                if r < own:
                    assert got == ad * rank + r


def test_rows_of_the_largest_pool_pass_32_bits(rows):
    assert rows.row(1 << 26, 128, 127, 128) == (1 << 33) + 127
