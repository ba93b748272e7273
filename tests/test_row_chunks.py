"""Into how long chunks of rows a weight gradient's parts are cut, up to the most rows that a call takes: the kernels' own function,
run on the host, against whole numbers of any size."""
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
int64_t fit_rows(int parts, const int32_t* rows, int64_t least, int64_t tiles) {
    int most = 1;
    for (int g = 0; g < parts; ++g) most = rows[g] > most ? rows[g] : most;
    return (int64_t)STEP * grouped::fit_chunk((int)least / STEP, grouped::steps_of<STEP>(most), tiles, [&](int steps) {
        int64_t count = 0;
        for (int g = 0; g < parts; ++g) count += (grouped::steps_of<STEP>(rows[g]) + steps - 1) / steps;
        return count;
    });
}
extern "C" int64_t fit(int parts, const int32_t* rows, int64_t least, int step, int64_t tiles) {
    return step == 32 ? fit_rows<32>(parts, rows, least, tiles) : fit_rows<64>(parts, rows, least, tiles);
}
"""


@pytest.fixture(scope="module")
def fit(tmp_path_factory):
    where = tmp_path_factory.mktemp("chunks")
    source, shared = os.path.join(where, "fit.cu"), os.path.join(where, "fit.so")
    with open(source, "w") as f:
        f.write(SOURCE)
    subprocess.run([build._nvcc()] + build.NVCC_FLAGS + ["-shared", source, "-o", shared], check=True)
    call = ctypes.CDLL(shared).fit
    call.restype = ctypes.c_int64
    call.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_int32), ctypes.c_int64, ctypes.c_int, ctypes.c_int64]
    return lambda rows, step, tiles: call(len(rows), (ctypes.c_int32 * len(rows))(*rows), LEAST, step, tiles)


def check(fit, rows, step, tiles):
    tiles = min(max(len(rows), tiles), sum(rows) // LEAST + len(rows))  # as a call sets it
    chunk = fit(rows, step, tiles)
    count = lambda c: sum(-(-r // c) for r in rows)  # noqa: E731
    assert chunk % step == 0 and chunk >= LEAST
    assert count(chunk) <= tiles, (chunk, count(chunk), tiles)  # every row is in a chunk
    assert chunk == LEAST or count(chunk - step) > tiles, chunk


@pytest.mark.parametrize("step", [32, 64])
@pytest.mark.parametrize("tiles", [1, 18, 296, 592])
@pytest.mark.parametrize("rows", [[MOST], [MOST - 63], [2_140_000_000], [2 ** 30], [0, MOST - 700, 0, 700], [2 ** 30, 2 ** 30 - 1], [1] * 299 + [MOST - 299],
                                  [1] * 511 + [MOST - 511], [MOST // 512] * 512, [0], [1], [256], [257], [1_000_000], [0, 5, 70_000, 0]])
def test_chunks_of_many_rows(fit, rows, step, tiles):
    check(fit, rows, step, tiles)


def test_chunks_of_any_parts(fit):
    rng = random.Random(3)
    for _ in range(300):
        left, rows = rng.choice((MOST, 10 ** rng.randint(1, 9))), []
        for _ in range(rng.choice((1, 2, 7, 64, 512))):
            rows.append(rng.randint(0, left) if rng.random() < 0.5 else min(left, rng.randint(0, 1000)))
            left -= rows[-1]
        check(fit, rows, rng.choice((32, 64)), rng.choice((1, 37, 296, 592)))
