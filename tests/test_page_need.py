"""How many pages a row of a page table takes, from the library's own header compiled for the host: whatever lengths a caller's memory holds, the pages of the rows
that are added up in 32 bits stay within them."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2404_04541_amd", "csrc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("page_need")
    src = d / "need.cpp"
    src.write_text('#include "page_need.hpp"\n'
                   'extern "C" int need(long long len, long long pages) { return spg::page_need(len, pages); }\n'
                   'extern "C" long long most() { return spg::kMaxPages; }\n')
    so = d / "need.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", CSRC, "-o", str(so), str(src)], check=True)
    lib = C.CDLL(str(so))
    lib.need.argtypes, lib.need.restype, lib.most.restype = [C.c_longlong, C.c_longlong], C.c_int, C.c_longlong
    return lib


def test_pages_of_a_length(lib):
    for pages in (0, 1, 7, 1000, lib.most() - 1):
        for n in (0, 1, 63, 64, 65, 128, 64 * 7, 64 * 7 + 1, 64000, 64001, 2 ** 31 - 1):
            want = -(-n // 64)
            assert lib.need(n, pages) == (want if want <= pages else -1), (n, pages)


def test_a_wave_of_rows_adds_up_in_32_bits(lib):
    """64 rows of any length over any cache: no partial sum leaves 32 bits, also for lengths near 2^31, which alone would be 64 times 2^25 pages."""
    for pages in (1, 6, 1 << 20, lib.most() - 1):
        for n in (2 ** 31 - 1, 64 * pages, 64 * pages + 1, 64 * (pages - 1) + 1):
            need = max(lib.need(n, pages), 0)
            assert 64 * need < 2 ** 31, (n, pages)
