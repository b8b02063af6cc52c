"""The sequence operators at the limits of their sizes and strides, and what their calls leave to their callers."""
import pytest
import torch

from paper_2509_20883_amd import recis as R
from tests.test_gpu_seq_attention import _close, _offsets, _reference

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("which", ["q", "k", "v"])
@pytest.mark.parametrize("d", [40, 64, 120])
def test_rows_far_apart(which, d):
    """fp32 rows 20 MB apart, so that the 128 rows that a step of the backward loads span more than 2^31 bytes: the same
    results, bit for bit, as from the same rows side by side; the elements between the rows are never read."""
    print("far rows", which, d, flush=True)
    n = 200
    g = torch.Generator(device="cuda").manual_seed(d)
    off = _offsets([n])
    t = {name: torch.randn(n, 1, d, generator=g, device="cuda") for name in ("q", "k", "v", "do")}
    far = torch.full((n, 5000000), float("nan"), device="cuda").view(n, 1, -1)[..., :d]
    far.copy_(t[which])
    op = R.SeqAttention()

    def both(q, k, v):
        out, stats = op.forward(q, k, v, off)
        return (out, stats.lse) + op.backward(t["do"], q, k, v, out, stats, off)[:3]

    want = both(t["q"], t["k"], t["v"])
    got = both(*(far if name == which else t[name] for name in ("q", "k", "v")))
    for name, a, b in zip(("out", "lse", "dq", "dk", "dv"), got, want):
        assert torch.equal(a, b), name
