"""The paged cache's host arithmetic at its limits (CPU only)."""
import ctypes as C
import os
import random
import subprocess
from decimal import Decimal, getcontext
from fractions import Fraction

import pytest

from paper_2509_20883_amd import recis as R


def _pi(bits):
    """pi 2^bits, by Machin's formula in whole numbers."""
    one = 1 << (bits + 16)

    def atan_inv(n):
        total, term, k, sign = 0, one // n, 1, 1
        while term:
            total += sign * (term // k)
            term //= n * n
            k, sign = k + 2, -sign
        return total

    return (4 * (4 * atan_inv(5) - atan_inv(239))) >> 16


BITS = 600
TWO_PI = Fraction(2 * _pi(BITS), 1 << BITS)


def _off(got, f):
    """How far a fraction of 2^64 is from the frequency's, in units of 2^-64 turns, around the turn."""
    want = f / TWO_PI
    d = Fraction(got, 1 << 64) - (want - want.__floor__())
    return abs(d - round(d)) * 2 ** 64


FREQS = [0.0, 1.0, -1.0, 6.25, 6.283185307179586, 100.0, -100.0, 1e5, -1e5, 12345.678, 1e9, 1e15, 2.0 ** 63, 1.7e30, -1.2345 * 2.0 ** 100,
         2.0 ** 127 * 1.999, 0.1, 1e-3, 2.0 ** -60, 1.7 * 2.0 ** -62, 2.0 ** -70, 5e-324]


def test_own_frequencies_are_exact():
    """A frequency is the double that it is, whatever its size: its fraction of a turn is off by the last rounding."""
    got = (C.c_uint64 * len(FREQS))()
    assert R.lib().rs_rotation_turns((C.c_double * len(FREQS))(*FREQS), 0.0, 2 * len(FREQS), got) == R.OK
    for f, g in zip(FREQS, got):
        assert _off(g, Fraction(f)) <= 0.5 + 2.0 ** -20, f


@pytest.mark.parametrize("f", [2.0 ** 128, -2.0 ** 128, 1e300, float("inf"), float("nan")])
def test_frequencies_that_are_refused(f):
    got = (C.c_uint64 * 2)()
    assert R.lib().rs_rotation_turns((C.c_double * 2)(1.0, f), 0.0, 4, got) == R.EINVAL


def test_a_base_whose_powers_are_refused():
    got = (C.c_uint64 * 64)()
    assert R.lib().rs_rotation_turns(None, 5e-324, 128, got) == R.EINVAL  # up to 2^1057


@pytest.mark.parametrize("base,rotary", [(10000.0, 128), (500000.0, 64), (1.0, 6), (1e300, 32), (0.5, 48)])
def test_frequencies_of_a_base(base, rotary):
    """base^(-2 i / rotary) in 64 bits: the power is off by less than its last, 2^-63 of itself, its exponent by 2^-64 of itself, which
    is ln f of the power; then the last rounding.  One unit is never passed from base 1 on."""
    getcontext().prec = 60
    got = (C.c_uint64 * (rotary // 2))()
    assert R.lib().rs_rotation_turns(None, base, rotary, got) == R.OK
    for i in range(rotary // 2):
        f = (Decimal(base).ln() * Decimal(-2 * i) / Decimal(rotary)).exp()
        bound = 0.5 + float(f) / 6.28 * (2 + abs(float(f.ln())))
        assert _off(got[i], Fraction(f)) <= bound and (base < 1 or bound < 1), i


SHIM = r"""
#include "select_tiles.h"
extern "C" {
int rows_log(int64_t seqs, int64_t rows, int64_t pad, int64_t window, int64_t most) { return rs::tile_rows_log(seqs, rows, pad, window, most); }
void tiles(int64_t seqs, int64_t rows, int64_t pad, int log, int64_t row0, int64_t n, int64_t* out) {
  const rs::TileRange r = rs::tiles_of_rows(seqs, rows, pad, log, row0, n);
  out[0] = r.first;
  out[1] = r.count;
}
}
"""


@pytest.fixture(scope="module")
def st(tmp_path_factory):
    d = tmp_path_factory.mktemp("select_tiles")
    (d / "shim.cpp").write_text(SHIM)
    so = str(d / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(R.PKG, "csrc"),
                    str(d / "shim.cpp"), "-o", so], check=True)
    L = C.CDLL(so)
    i64 = C.c_int64
    L.rows_log.argtypes = [i64] * 5
    L.tiles.argtypes = [i64, i64, i64, C.c_int, i64, i64, C.POINTER(i64)]
    return L


def _windows(st, seqs, rows, pad, log, window):
    out = (C.c_int64 * 2)()
    for row0 in range(0, rows, window):
        n = min(window, rows - row0)
        st.tiles(seqs, rows, pad, log, row0, n, out)
        yield row0, n, out[0], out[1]


def test_every_row_of_a_window_has_its_tile_launched(st):
    rng = random.Random(1)
    for _ in range(400):
        seqs, padded = rng.randint(1, 30), rng.random() < 0.4
        if padded:
            pad = rng.randint(1, 40)
            rows = seqs * pad
        else:
            lens = [rng.choice([0, 0, 1, 2, rng.randint(0, 60)]) for _ in range(seqs)]
            before, behind = rng.choice([0, 0, 7]), rng.choice([0, 0, 5])
            off = [before]
            for n in lens:
                off.append(off[-1] + n)
            pad, rows = 0, off[-1] + behind
        if rows == 0:
            continue
        window = rng.randint(1, rows)
        for log in range(5):
            for row0, n, first, count in _windows(st, seqs, rows, pad, log, window):
                for row in range(row0, row0 + n):
                    if pad:
                        unit = row // pad * ((pad + (1 << log) - 1) >> log) + (row % pad >> log)
                    else:
                        s = next((s for s in range(seqs) if off[s] <= row < off[s + 1]), None)
                        if s is None:
                            continue
                        unit = (off[s] >> log) + (s if log else 0) + ((row - off[s]) >> log)
                    assert first <= unit < first + count, (pad, log, row0, n, row)


@pytest.mark.parametrize("seqs,rows,pad", [(4096, 4096, 0), (100, 4096, 0), (1, 100000, 0), (50000, 100000, 0), (3000, 3 * 3000, 3), (7, 7 * 1000, 1000)])
@pytest.mark.parametrize("window", [1, 16, 536, 1 << 20])
@pytest.mark.parametrize("most", [1, 8, 16])
def test_windows_launch_as_many_tiles_as_rows(st, seqs, rows, pad, window, most):
    """All windows together: at most a tile a row, and three more of each window, however many there are."""
    log = st.rows_log(seqs, rows, pad, window, most)
    got = list(_windows(st, seqs, rows, pad, log, window))
    assert sum(count for _, _, _, count in got) <= 2 * rows + 3 * len(got)
    if window >= rows:
        assert sum(count for _, _, _, count in got) <= rows / (1 << log) + seqs + 1
