"""Between which bounds a weight gradient looks for the length of its chunks: the search with the kernels' own bounds, run on the host, finds the chunk that whole
numbers say, so that no row is left out."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2305_09887_b200 import build

LEAST, MOST = 256, 2 ** 31 - 1
SOURCE = """
#include "grouped_linear.cuh"
template <int STEP>
int64_t fit_rows(int parts, const int32_t* rows, int64_t least, int64_t tiles, int32_t* bounds, int* tries) {
    int most = 1;
    int64_t all = 0;
    for (int g = 0; g < parts; ++g) {
        most = rows[g] > most ? rows[g] : most;
        all += grouped::steps_of<STEP>(rows[g]);
    }
    const grouped::ChunkBounds b = grouped::chunk_bounds<STEP>(all, grouped::steps_of<STEP>(most), least, tiles, parts);
    bounds[0] = b.least;
    bounds[1] = b.fits;
    *tries = 0;
    return (int64_t)STEP * grouped::fit_chunk(b.least, b.fits, tiles, [&](int steps) {
        int64_t count = 0;
        ++*tries;
        for (int g = 0; g < parts; ++g) count += (grouped::steps_of<STEP>(rows[g]) + steps - 1) / steps;
        return count;
    });
}
extern "C" int64_t fit(int parts, const int32_t* rows, int64_t least, int step, int64_t tiles, int32_t* bounds, int* tries) {
    return step == 32 ? fit_rows<32>(parts, rows, least, tiles, bounds, tries) : fit_rows<64>(parts, rows, least, tiles, bounds, tries);
}
"""


@pytest.fixture(scope="module")
def fit(tmp_path_factory):
    where = tmp_path_factory.mktemp("bounds")
    source, shared = os.path.join(where, "fit.cu"), os.path.join(where, "fit.so")
    with open(source, "w") as f:
        f.write(SOURCE)
    subprocess.run([build._nvcc()] + build.NVCC_FLAGS + ["-shared", source, "-o", shared], check=True)
    call = ctypes.CDLL(shared).fit
    call.restype = ctypes.c_int64
    call.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_int32), ctypes.c_int64, ctypes.c_int, ctypes.c_int64, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int)]

    def run(rows, step, tiles):
        bounds, tries = (ctypes.c_int32 * 2)(), ctypes.c_int()
        chunk = call(len(rows), (ctypes.c_int32 * len(rows))(*rows), LEAST, step, tiles, bounds, ctypes.byref(tries))
        return chunk, step * max(bounds), tries.value
    return run


def check(fit, rows, step, tiles):
    chunk, upper, tries = fit(rows, step, tiles)
    count = lambda c: sum(-(-r // c) for r in rows)  # noqa: E731
    assert count(upper) <= tiles, (upper, count(upper), tiles)  # the search trusts that its upper bound fits
    assert chunk % step == 0 and LEAST <= chunk <= upper
    assert count(chunk) <= tiles, (chunk, count(chunk), tiles)  # every row is in a chunk
    assert chunk == LEAST or count(chunk - step) > tiles, chunk  # and they are as short as can be
    assert tries <= 31


CASES = [[MOST], [MOST - 63], [2_140_000_000], [2 ** 30], [0, MOST - 700, 0, 700], [2 ** 30, 2 ** 30 - 1], [1] * 299 + [MOST - 299], [1] * 511 + [MOST - 511],
         [MOST // 512] * 512, [0], [0] * 512, [1], [256], [257], [1_000_000], [0, 5, 70_000, 0], [257] * 512, [64 * 7 + 1, 64 * 9, 31, 0, 33]]


@pytest.mark.parametrize("step", [32, 64])
@pytest.mark.parametrize("above", [0, 1, 2, 17, 295, 591])
@pytest.mark.parametrize("rows", CASES)
def test_tiles_from_as_many_as_parts_on(fit, rows, above, step):
    check(fit, rows, step, len(rows) + above)


@pytest.mark.parametrize("step", [32, 64])
@pytest.mark.parametrize("tiles", [1, 18, 148, 296, 592])
@pytest.mark.parametrize("rows", CASES)
def test_tiles_as_a_call_sets_them(fit, rows, tiles, step):
    check(fit, rows, step, min(max(len(rows), tiles), sum(rows) // LEAST + len(rows)))


def test_any_parts(fit):
    rng = random.Random(5)
    for _ in range(400):
        left, rows = rng.choice((MOST, 10 ** rng.randint(1, 9))), []
        for _ in range(rng.choice((1, 2, 7, 64, 512))):
            rows.append(rng.randint(0, left) if rng.random() < 0.5 else min(left, rng.randint(0, 1000)))
            left -= rows[-1]
        check(fit, rows, rng.choice((32, 64)), len(rows) + rng.choice((0, 1, 5, 37, 296, 592)))


@pytest.mark.parametrize("step", [32, 64])
def test_parts_that_overlap(fit, step):
    """Offsets that do not ascend: more rows in all than there are."""
    for rows in ([MOST, 0] * 256, [MOST] * 512, [2 ** 30] * 7):
        for above in (0, 1, 296):
            check(fit, rows, step, len(rows) + above)
