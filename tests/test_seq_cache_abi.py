"""The paged cache's boundary without a GPU: descriptors, refusals, workspace sizes, rotation fractions (CPU only)."""
import ctypes as C
import os
import subprocess
from decimal import Decimal, getcontext

import pytest
import torch

from paper_2509_20883_amd import recis as R

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
STRUCTS = {"rs_seq_cache": R.CacheDesc, "rs_cache_batch": R.CacheBatch, "rs_cache_rows": R.CacheRows, "rs_cache_query": R.CacheQuery}


def test_structs_match_the_header(tmp_path):
    prog, exe = tmp_path / "layout.c", tmp_path / "layout"
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "recis_mi355x.h"', "int main(void) {"]
    want = []
    for name, cls in STRUCTS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(cls))
        for f in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {f[0]}));')
            want.append(getattr(cls, f[0]).offset)
    prog.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.dirname(R.HEADER), str(prog), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == want


@pytest.mark.parametrize("rotary,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (126, 1.0), (48, 0.5)])
def test_rotation_fractions_of_a_base(rotary, base):
    getcontext().prec = 60
    got = (C.c_uint64 * (rotary // 2))()
    assert R.lib().rs_rotation_turns(None, base, rotary, got) == R.OK
    for i in range(rotary // 2):
        f = (Decimal(base).ln() * Decimal(-2 * i) / Decimal(rotary)).exp() / (2 * PI)
        want = int((f % 1) * 2 ** 64)
        # extended precision carries 64 bits: a few units of the last at a value of a turn or more
        assert abs((got[i] - want + 2 ** 63) % 2 ** 64 - 2 ** 63) <= 64 * max(1, int(f) + 1)


def test_rotation_fractions_of_own_frequencies():
    getcontext().prec = 60
    freqs = [0.0, 1.0, -1.0, 6.25, 100.0, 2.0 ** -60, -3.5]
    got = (C.c_uint64 * len(freqs))()
    assert R.lib().rs_rotation_turns((C.c_double * len(freqs))(*freqs), 0.0, 2 * len(freqs), got) == R.OK
    for f, g in zip(freqs, got):
        want = int(((Decimal(f) / (2 * PI)) * 2 ** 64).to_integral_value()) % 2 ** 64
        assert abs((g - want + 2 ** 63) % 2 ** 64 - 2 ** 63) <= 64 * max(1, int(abs(f)))
    for freqs, base, rotary in ((None, 0.0, 4), (None, float("inf"), 4), (None, float("nan"), 4), (None, 10.0, 3), (None, 10.0, 130),
                                (None, 10.0, -2), ([float("nan"), 1.0], 10.0, 4), ([float("inf"), 1.0], 10.0, 4)):
        own = None if freqs is None else (C.c_double * 2)(*freqs)
        assert R.lib().rs_rotation_turns(own, base, rotary, got) == R.EINVAL


CACHE = dict(codes=1, dtype=R.BF16, heads_kv=2, head_dim=64, page_len=64, reserved=0, pages=100, slots=4, data=4096, scales=8192, open=12288,
             bounds=16384, units=20480)
BATCH = dict(seqs=3, rows=100, pad=0, table_width=40, offsets=4096, lens=8192, table=12288, slots=None)
QUERY = dict(heads_q=8, causal=1, count=0, reserved=0, max_q=0, max_len=0, q_stride=512, q_head_stride=64, scale=0.125, softcap=0.0)
ROWS = dict(k=4096, v=8192, q=12288, q_out=16384, k_stride=128, k_head_stride=64, v_stride=128, v_head_stride=64, q_stride=512,
            q_head_stride=64, heads_q=8, rotary=64, interleaved=0, reserved=0, turns=4096, new_lens=20480)
BAD_CACHE = [dict(codes=2), dict(dtype=7), dict(heads_kv=0), dict(heads_kv=1025), dict(head_dim=4), dict(head_dim=65), dict(head_dim=136),
             dict(page_len=16), dict(page_len=48), dict(page_len=512), dict(reserved=1), dict(pages=-1), dict(pages=1 << 31), dict(slots=-1),
             dict(data=None), dict(scales=None), dict(open=None), dict(units=None), dict(data=4100), dict(open=12290), dict(bounds=16385)]
BAD_BATCH = [dict(seqs=-1), dict(seqs=1 << 24), dict(rows=-1), dict(rows=1 << 31), dict(pad=-1), dict(pad=7), dict(table_width=-1),
             dict(table_width=(1 << 26) + 1), dict(offsets=None), dict(lens=None), dict(table=None)]
BAD_QUERY = [dict(heads_q=1), dict(heads_q=7), dict(heads_q=8194), dict(count=-1), dict(count=65537), dict(reserved=1), dict(max_q=-1),
             dict(max_len=-1), dict(q_stride=4), dict(q_head_stride=-8), dict(q_stride=1 << 31), dict(scale=0.0), dict(scale=-1.0),
             dict(scale=float("nan")), dict(scale=2.0 ** 127), dict(softcap=-1.0), dict(softcap=float("inf")), dict(softcap=1e-39),
             dict(softcap=1e-30, scale=1e20)]
BAD_ROWS = [dict(k=None), dict(v=None), dict(q_out=None), dict(q=None), dict(heads_q=0), dict(heads_q=8193), dict(rotary=3), dict(rotary=66),
            dict(rotary=-2), dict(turns=None), dict(reserved=1), dict(k=4098), dict(q_out=16388), dict(k_stride=4), dict(v_head_stride=-8),
            dict(q_stride=12), dict(new_lens=8192)]


def _all(cache={}, batch={}, query={}, rows={}):
    return R.CacheDesc(**dict(CACHE, **cache)), R.CacheBatch(**dict(BATCH, **batch)), R.CacheQuery(**dict(QUERY, **query)), R.CacheRows(**dict(ROWS, **rows))


def _refused(cache={}, batch={}, query={}, rows={}, calls="arsq"):
    """Every named entry point refuses the call; no pointer of it is ever read."""
    L = R.lib()
    c, b, q, r = (C.byref(x) for x in _all(cache, batch, query, rows))
    if "a" in calls:
        assert L.seq_cache_append(c, b, r, 0, None) == R.EINVAL
    if "r" in calls:
        assert L.seq_cache_read(c, b, None, 4096, 4096, R.F32, 0, None) == R.EINVAL
    if "q" in calls:
        assert L.seq_cache_attention(c, b, q, 4096, None, None, 4096, 4096, 1 << 40, 0, None) == R.EINVAL
    if "s" in calls:
        q1 = R.CacheQuery(**dict(QUERY, **dict(dict(count=4), **query)))
        assert L.seq_cache_select(c, b, C.byref(q1), 4096, 4096, 4096, 1 << 40, 0, None) == R.EINVAL


@pytest.mark.parametrize("bad", BAD_CACHE, ids=str)
def test_caches_that_are_refused(bad):
    _refused(cache=bad)
    c, b, q, _ = _all(cache=bad)
    assert R.lib().seq_cache_attention_workspace_bytes(C.byref(c), C.byref(b), C.byref(q)) == 0


@pytest.mark.parametrize("bad", BAD_BATCH, ids=str)
def test_batches_that_are_refused(bad):
    _refused(batch=bad)


@pytest.mark.parametrize("bad", BAD_QUERY, ids=str)
def test_queries_that_are_refused(bad):
    _refused(query=bad, calls="qs")
    c, b, q, _ = _all(query=bad)
    assert R.lib().seq_cache_select_workspace_bytes(C.byref(c), C.byref(b), C.byref(q)) == 0


@pytest.mark.parametrize("bad", BAD_ROWS, ids=str)
def test_rows_that_are_refused(bad):
    _refused(rows=bad, calls="a")


def test_other_refusals():
    L = R.lib()
    c, b, q, r = _all()
    for args in ((None, C.byref(b), C.byref(r)), (C.byref(c), None, C.byref(r)), (C.byref(c), C.byref(b), None)):
        assert L.seq_cache_append(*args, 0, None) == R.EINVAL
    c, b, q = (C.byref(x) for x in (c, b, q))
    assert L.seq_cache_read(c, b, None, None, 4096, R.F32, 0, None) == R.EINVAL
    assert L.seq_cache_read(c, b, None, 4096, 4097, R.F32, 0, None) == R.EINVAL
    assert L.seq_cache_read(c, b, None, 4096, 4096, 5, 0, None) == R.EINVAL
    _refused(batch=dict(pad=50, seqs=2), calls="r")  # packed only
    assert L.seq_cache_attention(c, b, q, None, None, None, 4096, 4096, 1 << 40, 0, None) == R.EINVAL
    assert L.seq_cache_attention(c, b, q, 4096, None, None, 4098, 4096, 1 << 40, 0, None) == R.EINVAL
    assert L.seq_cache_attention(c, b, q, 4096, 4096, None, 4096, 4096, 1 << 40, 0, None) == R.EINVAL  # a list without a count
    listed = R.CacheQuery(**dict(QUERY, count=3))
    assert L.seq_cache_attention(c, b, C.byref(listed), 4096, None, None, 4096, 4096, 1 << 40, 0, None) == R.EINVAL
    assert L.seq_cache_select(c, b, q, 4096, 4096, 4096, 1 << 40, 0, None) == R.EINVAL  # no count
    _refused(cache=dict(bounds=None, units=None), calls="s")
    # workspaces: missing, too small, not aligned
    long = R.CacheBatch(**dict(BATCH, rows=1, seqs=1, table_width=4000))
    need = L.seq_cache_attention_workspace_bytes(c, C.byref(long), q)
    assert need > 0
    for ws, size in ((None, need), (4096, need - 1), (4096 + 16, need)):
        assert L.seq_cache_attention(c, C.byref(long), q, 4096, None, None, 4096, ws, size, 0, None) == R.EINVAL
    need = L.seq_cache_select_workspace_bytes(c, C.byref(long), C.byref(listed))
    assert need >= 4000 * 2 * 4
    for ws, size in ((None, need), (4096, need - 1), (4096 + 16, need)):
        assert L.seq_cache_select(c, C.byref(long), C.byref(listed), 4096, 4096, ws, size, 0, None) == R.EINVAL


def test_workspaces_stay_bounded():
    """Parts of splits and scores of rows take at most 256 MiB, or one row's."""
    L = R.lib()
    c = R.CacheDesc(**CACHE)
    for rows, seqs, width, count in ((1, 1, 1 << 20, 0), (100000, 10, 20000, 0), (100000, 10, 20000, 64), (300, 256, 64, 0), (7, 3, 1 << 26, 8)):
        b, q = R.CacheBatch(**dict(BATCH, rows=rows, seqs=seqs, table_width=width)), R.CacheQuery(**dict(QUERY, count=count))
        assert L.seq_cache_attention_workspace_bytes(C.byref(c), C.byref(b), C.byref(q)) <= (256 << 20) + 4096
        if count:
            assert L.seq_cache_select_workspace_bytes(C.byref(c), C.byref(b), C.byref(q)) <= max(256 << 20, width * 2 * 4)


def test_binding_refuses_before_the_gpu():
    for kw in (dict(codes="u8"), dict(dtype=torch.float16), dict(page=16), dict(page=100), dict(head_dim=60), dict(heads_kv=0), dict(pages=-1),
               dict(rotary=3), dict(rotary=128), dict(rotary=8, freqs=[1.0])):
        with pytest.raises(R.RecisError):
            R.SeqCache(**dict(dict(pages=4, slots=1, heads_kv=1, head_dim=64), **kw))
