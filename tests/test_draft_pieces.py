"""How trees' attention cuts its work into pieces, from the library's own header compiled for the host: the launch and the memory that the host asks for are enough for whatever lengths there are, and no piece
is longer than twice the average of a workgroup's place."""
import ctypes as C
import math
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2404_04541_amd", "csrc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("pieces")
    src = d / "pieces.cpp"
    src.write_text('#include "draft_pieces.hpp"\n'
                   'extern "C" int per(float work, float units, int places, float off) { return spg::pages_of_piece(work, units, places, [=](float x) { return 1.0f / x * (1.0f + off); }); }\n'
                   'extern "C" long long pieces(long long work, long long units, int places) { return spg::most_pieces(work, units, places); }\n'
                   'extern "C" int chunk(long long work, int places) { return spg::chunk_pages(work, places); }\n'
                   'extern "C" long long chunk_cell(long long at, int chunk) { return spg::chunk_cell(at, chunk); }\n'
                   'extern "C" long long cells(long long work, int places) { return spg::most_cells(work, places); }\n')
    so = d / "pieces.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", CSRC, "-o", str(so), str(src)], check=True)
    lib = C.CDLL(str(so))
    lib.per.argtypes = [C.c_float, C.c_float, C.c_int, C.c_float]
    lib.pieces.argtypes, lib.pieces.restype = [C.c_longlong, C.c_longlong, C.c_int], C.c_longlong
    lib.cells.argtypes, lib.cells.restype = [C.c_longlong, C.c_int], C.c_longlong
    lib.chunk.argtypes, lib.chunk_cell.argtypes, lib.chunk_cell.restype = [C.c_longlong, C.c_int], [C.c_longlong, C.c_int], C.c_longlong
    return lib


def cut(lib, units, places, off=0.0):
    """(pages of a piece, all pieces, those of cut units) of (pages, how many) units."""
    work, count = sum(p * n for p, n in units), sum(n for p, n in units if p)
    per = lib.per(work, count, places, off)
    each = [(-(-p // per), n) for p, n in units]
    return per, sum(k * n for k, n in each), sum(k * n for k, n in each if k > 1), work, count


PLACES = (512, 768)


@pytest.mark.parametrize("places", PLACES)
def test_the_launch_and_the_cells_are_enough(lib, places):
    rng = random.Random(places)
    for _ in range(20000):
        heads = rng.choice([1, 2, 8, 16, 64])
        top = 2 ** rng.uniform(0, 12)
        units = [(int(2 ** rng.uniform(0, math.log2(top + 1))) * rng.choice([0, 1, 1, 1]), heads * rng.randint(1, 4)) for _ in range(rng.choice([1, 2, 5, rng.randint(1, 512)]))]
        if rng.random() < 0.5:
            units[0] = (rng.randint(1, 20000), heads)
        if rng.random() < 0.4 and len(units) > 1:       # as many units as a number of turns has places, and a few more or less
            units[1] = (rng.randint(1, 9), max(1, rng.randint(1, 4) * places - sum(n for p, n in units[:1] + units[2:] if p) + rng.randint(-3, 3)))
        # (the reciprocal of the card is off by less than 2^-22, sums in 24 digits by less than 2^-12)
        per, pieces, cells, work, count = cut(lib, units, places, rng.choice([0, 2.0 ** -22, -2.0 ** -22, 2.0 ** -12, -2.0 ** -12]))
        assert per >= 4 and pieces <= lib.pieces(work, count, places) and cells <= lib.cells(work, places), (units, per, pieces, cells)
        assert per <= max(math.ceil(2 * work / places * (1 + 2.0 ** -11)), 4), (units, per)


@pytest.mark.parametrize("places", PLACES)
def test_long_sequences_are_cut_whatever_the_number_of_the_others(lib, places):
    """A sequence of 60 000 tokens among short ones, 8 key heads: no piece takes more than a few times what all pieces take together, also where units are nearly as many as the turns have places."""
    for seqs in range(2, 513):
        per, pieces, _, work, count = cut(lib, [(938, 8), (8, 8 * (seqs - 1))], places)
        assert min(per, 938) <= max(2.01 * work / places + 1, 8), (seqs, per)


@pytest.mark.parametrize("places", PLACES)
def test_chunks_have_cells_of_their_own(lib, places):
    """Rows of a table one after another: the pieces of those that are cut have different cells, all within what the host asks for, and that is a few for each place of the card."""
    rng = random.Random(places + 1)
    for _ in range(300):
        heads, tiles = rng.choice([1, 8, 16]), rng.choice([1, 2, 8])
        rows = [rng.choice([0, 1, 2, 9, int(2 ** rng.uniform(0, 11))]) for _ in range(rng.randint(513, 900))]
        if rng.random() < 0.3:
            rows[rng.randrange(len(rows))] = rng.randint(1000, 40000)
        nnz = sum(rows)
        chunk = lib.chunk(nnz * heads * tiles, places)
        at, end = 0, 0
        for p in rows:
            pieces, cell = -(-p // chunk), lib.chunk_cell(at, chunk)
            if pieces > 1:
                assert cell >= end
                end = cell + pieces
            at += p
        assert end <= lib.chunk_cell(nnz, chunk) and lib.chunk_cell(nnz, chunk) * heads * tiles <= 4 * places


def test_chunks_of_very_large_tables(lib):
    """Pages of all rows, key heads and tiles go far beyond 32 bits; a chunk is never longer than a sequence can be."""
    for places in PLACES:
        for work in (1, 2 ** 20, 2 ** 35, 2 ** 35 + 1, 2 ** 41, 2 ** 42, 2 ** 57):
            chunk = lib.chunk(work, places)
            assert 8 <= chunk <= 2 ** 25 and chunk % 4 == 0 and (chunk == 2 ** 25 or chunk * 2 * places >= work), (work, places)
