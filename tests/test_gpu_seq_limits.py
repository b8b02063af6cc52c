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


@pytest.mark.parametrize("dtype,hq,hkv,d", [(torch.bfloat16, 2, 1, 16), (torch.float32, 1, 1, 64), (torch.bfloat16, 2, 2, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_distances_past_2_24_keys(dtype, hq, hkv, d, causal):
    """Three rows at the end of a history longer than the whole numbers of fp32 reach, scores falling by a half a key: the
    keys that count are the last ones, at distances 0, 1, 2, ..., and the rows are as over those keys alone."""
    print("positions", dtype, d, causal, flush=True)
    n, w, rows = (1 << 24) + 3001, 1024, 3
    g = torch.Generator(device="cuda").manual_seed(d)
    k, v = (torch.randn(n, hkv, d, generator=g, device="cuda", dtype=dtype) for _ in range(2))
    q, do = (torch.randn(rows, hq, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    m = torch.full((hq,), 0.5, device="cuda")
    op = R.SeqAttention(causal=causal)
    qo, ko = _offsets([rows]), _offsets([n])
    out, stats = op.forward(q, k, v, qo, kv_offsets=ko, slopes=m, max_q=rows)
    dq, dk, dv, dm = op.backward(do, q, k, v, out, stats, qo, kv_offsets=ko, slopes=m, max_q=rows)
    # keys further back weigh less than e^-500: nothing in fp32
    want, (wm, em) = _reference(q, k[-w:], v[-w:], do, qo, _offsets([w]), causal, 0.0, None, m, d ** -0.5,
                                dtype == torch.bfloat16)
    for name, t in (("out", out), ("lse", stats.lse), ("dq", dq), ("dk", dk[-w:]), ("dv", dv[-w:])):
        _close(t, *want[0][name], name)
    _close(dm, wm, em, "dslopes")
    assert not dk[:-w].any() and not dv[:-w].any()
