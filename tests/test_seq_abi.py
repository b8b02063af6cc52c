"""The sequence operators' boundary without a GPU: the binding's descriptor, refusals, workspace sizes (CPU only)."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2509_20883_amd import recis as R


def test_attention_descriptor_matches_the_header(tmp_path):
    prog, exe = tmp_path / "layout.c", tmp_path / "layout"
    fields = [f[0] for f in R.AttnDesc._fields_]
    prog.write_text("\n".join(['#include <stdio.h>', '#include <stddef.h>', '#include "recis_mi355x.h"', "int main(void) {",
                               'printf("%zu\\n", sizeof(rs_attn_desc));']
                              + [f'printf("%zu\\n", offsetof(rs_attn_desc, {f}));' for f in fields] + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.dirname(R.HEADER), str(prog), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(R.AttnDesc)] + [getattr(R.AttnDesc, f).offset for f in fields]


def test_host_tensors_are_refused():
    x, off = torch.zeros(4, 2, 16), torch.tensor([0, 4])
    with pytest.raises(R.RecisError, match="on the GPU"):
        R.LayerNorm().forward(torch.zeros(4, 8))
    with pytest.raises(R.RecisError, match="on the GPU"):
        R.SeqAttention().forward(x, x, x, off)


def test_workspace_sizes():
    L = R.lib()
    assert L.layer_norm_bwd_workspace_bytes(1000, 64) >= 2 * 64 * 4
    for rows, dim in ((-1, 64), (1 << 31, 64), (4, 0), (4, (1 << 24) + 1)):
        assert L.layer_norm_bwd_workspace_bytes(rows, dim) == 0
    good = dict(dtype=R.BF16, heads_q=8, heads_kv=2, head_dim=64, causal=1, reserved=0, seqs=3, q_rows=100, kv_rows=100,
                q_pad=0, kv_pad=0, max_q=0, q_stride=512, q_head_stride=64, k_stride=128, k_head_stride=64, v_stride=128,
                v_head_stride=64, scale=0.125, softcap=0.0)
    assert L.seq_attention_workspace_bytes(C.byref(R.AttnDesc(**good)), 1) >= 100 * 8 * 4
    bad = R.AttnDesc(**dict(good, head_dim=65))
    assert L.seq_attention_workspace_bytes(C.byref(bad), 0) == L.seq_attention_workspace_bytes(C.byref(bad), 1) == 0
    assert L.seq_attention_workspace_bytes(None, 1) == 0
