"""The sequence operators' limits without a GPU: what their descriptor refuses, and the kernels that are compiled (CPU only)."""
import subprocess

from paper_2509_20883_amd import recis as R
from paper_2509_20883_amd.build import LIB


def test_every_compiled_shape_of_the_key_pass_is_launched():
    """fp32 rows of 128 have no shape for few key tiles, and no kernel for one."""
    R.lib()
    names = subprocess.run(["nm", "-C", LIB], capture_output=True, text=True, check=True).stdout
    shapes = {n.split("k_attn_dkdv<")[1].split(">")[0] for n in names.splitlines() if "k_attn_dkdv<" in n}
    want = {f"{t}, {d}, {few}" for t in ("float", "unsigned short") for d in (32, 64, 128) for few in ("true", "false")}
    assert shapes == want - {"float, 128, true"}
