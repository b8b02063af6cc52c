"""The sequence operators' limits without a GPU: what their descriptor refuses, and the kernels that are compiled (CPU only)."""
import ctypes as C
import subprocess

import pytest

from paper_2509_20883_amd import recis as R
from paper_2509_20883_amd.build import LIB


def test_every_compiled_shape_of_the_key_pass_is_launched():
    """fp32 rows of 128 have no shape for few key tiles, and no kernel for one."""
    R.lib()
    names = subprocess.run(["nm", "-C", LIB], capture_output=True, text=True, check=True).stdout
    shapes = {n.split("k_attn_dkdv<")[1].split(">")[0] for n in names.splitlines() if "k_attn_dkdv<" in n}
    want = {f"{t}, {d}, {few}" for t in ("float", "unsigned short") for d in (32, 64, 128) for few in ("true", "false")}
    assert shapes == want - {"float, 128, true"}


@pytest.mark.parametrize("scale,softcap,ok", [
    (0.125, 0.0, True), (0.125, 1e-30, True), (1e-30, 1e-37, True), (0.125, 1e300, True), (1e38, 0.0, True), (1e-300, 5.0, True),
    (3e38, 0.0, False), (1e39, 0.0, False), (1e300, 5.0, False),  # not finite in fp32, in base 2
    (0.125, 1e-46, False), (0.125, 1e-39, False),  # no cap, or half of one, in fp32
    (1e5, 1e-37, False),  # their quotient is not
])
def test_scale_and_cap_hold_in_fp32(scale, softcap, ok):
    d = R.AttnDesc(dtype=R.BF16, heads_q=8, heads_kv=2, head_dim=64, causal=1, reserved=0, seqs=3, q_rows=100, kv_rows=100,
                   q_pad=0, kv_pad=0, max_q=0, q_stride=512, q_head_stride=64, k_stride=128, k_head_stride=64, v_stride=128,
                   v_head_stride=64, scale=scale, softcap=softcap)
    assert (R.lib().seq_attention_workspace_bytes(C.byref(d), 1) > 0) == ok


@pytest.mark.parametrize("dtype,field,value,ok", [
    (R.F32, "k_stride", (1 << 23) - 4, True), (R.F32, "k_stride", 1 << 23, False), (R.BF16, "v_stride", (1 << 23) - 8, True),
    (R.F32, "k_head_stride", (1 << 23) - 4, True), (R.BF16, "q_stride", (1 << 23) - 8, True),
    (R.F32, "q_stride", 5000000, True), (R.F32, "q_stride", (1 << 23) - 4, False),  # 64 rows of q and its heads
    (R.F32, "q_head_stride", (1 << 23) - 4, True), (R.BF16, "q_stride", 12, False), (R.F32, "q_stride", 0, True),
])
def test_strides(dtype, field, value, ok):
    """Rows and heads as far apart as the kernels address them, and no further."""
    d = dict(dtype=dtype, heads_q=2, heads_kv=1, head_dim=64, causal=1, reserved=0, seqs=3, q_rows=200, kv_rows=200, q_pad=0,
             kv_pad=0, max_q=0, q_stride=128, q_head_stride=64, k_stride=64, k_head_stride=64, v_stride=64, v_head_stride=64,
             scale=0.125, softcap=0.0)
    assert (R.lib().seq_attention_workspace_bytes(C.byref(R.AttnDesc(**dict(d, **{field: value}))), 1) > 0) == ok
