"""How the attention's lines of work are cut into stretches and items (csrc/stretch.h), compiled for the host, against whole numbers
of any size."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_18573_amd", "csrc")

SOURCE = """
#include "stretch.h"
extern "C" int64_t begin_of(int w, int64_t steps, int parts) { return e3::begin_of(w, steps, parts); }
extern "C" int part_of(int64_t step, int64_t steps, int parts) { return e3::part_of(step, steps, parts); }
extern "C" void piece_at(int64_t offset, int64_t left, int item_steps, int* out)
{
    const e3::Piece p = e3::piece_at(offset, left, item_steps);
    out[0] = p.item; out[1] = p.from; out[2] = p.n;
}
"""


@pytest.fixture(scope="module")
def stretch(tmp_path_factory):
    d = tmp_path_factory.mktemp("stretch")
    src, lib = os.path.join(d, "stretch.cpp"), os.path.join(d, "stretch.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + CSRC, "-o", lib, src], check=True)
    L = C.CDLL(lib)
    L.begin_of.argtypes, L.begin_of.restype = [C.c_int, C.c_int64, C.c_int], C.c_int64
    L.part_of.argtypes, L.part_of.restype = [C.c_int64, C.c_int64, C.c_int], C.c_int
    L.piece_at.argtypes, L.piece_at.restype = [C.c_int64, C.c_int64, C.c_int, C.c_void_p], None
    return L


# items and steps of a unit: ordinary ones; one row of 65,536 queries x 128 heads on 2^21 tokens, and 4096 rows of 128 queries and eight
# key heads on a prefix of 2^20, whose steps pass 2^31; and the most that fits a line
UNITS = [(1, 5), (4, 12), (256, 40), (131_072, 16_388), (65_536, 32_772), (3584, 312_504), (1 << 25, 1 << 26)]


@pytest.mark.parametrize("items,steps", UNITS)
@pytest.mark.parametrize("parts", [1, 2, 511, 768, 3072])
def test_stretches_cover_the_line(stretch, items, steps, parts):
    total = items * steps
    parts = min(parts, total)
    edges = sorted({0, 1, 2, parts // 3, parts // 2, parts - 2, parts - 1, parts} & set(range(parts + 1)))
    for w in edges:
        assert stretch.begin_of(w, total, parts) == w * total // parts
    for w in edges[:-1]:
        begin, end = w * total // parts, (w + 1) * total // parts
        assert end > begin
        for step in {begin, (begin + end) // 2, end - 1}:
            assert stretch.part_of(step, total, parts) == w


@pytest.mark.parametrize("items,steps", UNITS)
def test_pieces_of_a_unit(stretch, items, steps):
    total, out = items * steps, (C.c_int * 3)()
    offsets = {0, steps - 1, steps, total // 2, 2 ** 31 - 1, 2 ** 31, 2 ** 31 + 1, 2 ** 32 - 1, 2 ** 32, total - steps - 1, total - steps, total - 1}
    for offset in offsets & set(o for o in offsets if 0 <= o < total):
        for left in {1, steps - 1 or 1, steps, total - offset, total}:
            stretch.piece_at(offset, left, steps, out)
            item, start = divmod(offset, steps)
            assert list(out) == [item, start, min(left, steps - start)]


@pytest.mark.parametrize("items,steps,parts", [(5, 7, 3), (40, 9, 11), (131_072, 16_388, 3), (65_536, 32_772, 2)])
def test_a_walk_meets_every_item_once(stretch, items, steps, parts):
    # as a worker goes along its stretch; of the long ones only the stretches' beginnings and the unit's end
    total, out = items * steps, (C.c_int * 3)()
    for w in range(parts):
        at, end = stretch.begin_of(w, total, parts), stretch.begin_of(w + 1, total, parts)
        for walk in ((at, end),) if items < 100 else ((at, at + 5 * steps), (end - 5 * steps, end)):
            at, stop = walk
            while at < stop:
                stretch.piece_at(at, stop - at, steps, out)
                item, start, n = list(out)
                assert 0 <= item < items and 0 <= start < steps and n > 0 and item * steps + start == at
                at += n
            assert at == stop
