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


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 8), (torch.float32, 64)])
def test_last_chunk_of_the_longest_history(dtype, d):
    """One row over nearly 2^31 keys, all of them one row of memory, scores falling by 0.01 a key: the last keys carry
    the sum, and the last chunk of the split ends past the 32-bit whole numbers."""
    print("longest", dtype, d, flush=True)
    n, slope = (1 << 31) - 2048, 0.01
    g = torch.Generator(device="cuda").manual_seed(d)
    row = torch.randn(1, 1, d, generator=g, device="cuda").to(dtype)
    q = torch.randn(1, 1, d, generator=g, device="cuda").to(dtype)
    keys = row.expand(n, -1, -1)
    m = torch.full((1,), slope, device="cuda")
    out, stats = R.SeqAttention().forward(q, keys, keys, _offsets([1]), kv_offsets=_offsets([n]), slopes=m, max_q=1)
    u = 2.0 ** -24
    s = float((q.double() * row.double()).sum()) * d ** -0.5
    want = s - float(torch.log(-torch.expm1(-m.double())))  # sum over t >= 0 of e^(-slope t)
    # the keys that count (e^(-slope t) > u) lie within 1700; their scores and distance terms are at most 17 + |s|, and a
    # lane adds up at most 64 of them in a row before the lanes and the parts are added in trees
    assert abs(float(stats.lse) - want) <= (8 * (17 + abs(s)) + (d + 8) * float((q.double() * row.double()).abs().sum()) + 512) * u
    # probabilities that sum to one over equal rows: v, off by their rounding to bf16 and the result's
    r = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    _close(out, row.double(), row.double().abs() * (r + 600 * u), "out")


def test_more_blocks_than_one_launch_takes():
    """Three million sequences of one row, eight key heads: 24 million blocks, and HIP takes fewer than 2^32 threads."""
    print("many blocks", flush=True)
    n, h, d = 3000000, 8, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, do = (torch.randn(n, h, d, generator=g, device="cuda").bfloat16() for _ in range(4))
    off = torch.arange(n + 1, device="cuda")
    op = R.SeqAttention()
    out, stats = op.forward(q, k, v, off)
    dq, dk, dv, _ = op.backward(do, q, k, v, out, stats, off)
    assert torch.equal(out, v) and torch.equal(dv, do)  # one key: probability 1
    x = (q.float() * k.float()).sum(2) * d ** -0.5
    u = 2.0 ** -24
    lim = (d + 8) * u * (q.float() * k.float()).abs().sum(2) * d ** -0.5 + 8 * u * x.abs() + 1e-6
    assert ((stats.lse - x).abs() <= 2 * lim).all()
    # ds = dP - delta: the same sum of d products taken twice, each off by (d + 8) u of its magnitudes
    ds = 2 * (d + 8) * u * (do.float() * v.float()).abs().sum(2, keepdim=True) * d ** -0.5 * (1 + 2.0 ** -6)
    assert (dq.float().abs() <= ds * k.float().abs() + 1e-30).all() and (dk.float().abs() <= ds * q.float().abs() + 1e-30).all()


def test_more_rows_than_one_launch_takes():
    """Narrow rows, 64 to a block of the layer norm: past 2^30 of them the threads would be more than HIP's 2^32."""
    print("many rows", flush=True)
    rows, dim, part = (1 << 30) + 300, 8, 1 << 20
    g = torch.Generator(device="cuda").manual_seed(1)
    block = torch.randn(part, dim, generator=g, device="cuda").bfloat16()
    x = torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda")
    whole = rows // part * part
    x[:whole].view(-1, part, dim).copy_(block)
    x[whole:] = block[:rows - whole]
    op = R.LayerNorm()
    want, mean, rstd = op.forward(block)
    y, m, s = op.forward(x)
    for got, ref in ((y, want), (m, mean), (s, rstd)):
        assert (got[:whole].view(-1, *ref.shape) == ref).all() and torch.equal(got[whole:], ref[:rows - whole])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d", [(2, 1, 64), (8, 2, 128), (3, 3, 40)])
@pytest.mark.parametrize("bound", [1, 4, 50])
def test_a_bound_of_the_queries_that_does_not_hold(dtype, hq, hkv, d, bound):
    """max_q shapes the launches, the results hold without it: rows past a bound that is too small, over keys that are
    split and keys that are not, masked and not, and padding of the row tiles between them."""
    print("bound", dtype, hq, hkv, d, bound, flush=True)
    ql, kl = [1, 9, 200, 0, 3, 60], [3000, 5000, 900, 40, 100, 20]
    qo, ko = _offsets(ql), _offsets(kl)
    g = torch.Generator(device="cuda").manual_seed(d + bound)
    q = torch.randn(sum(ql), hq, d, generator=g, device="cuda").to(dtype)
    k, v = (torch.randn(sum(kl), hkv, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    m = torch.rand(hq, generator=g, device="cuda") * 0.1
    pre = torch.tensor([5, 0, 950, 1, 50, 3], device="cuda")
    for causal, cap, slopes, prefix in ((True, 0.0, None, None), (False, 4.0, m, None), (True, 0.0, m, pre)):
        op = R.SeqAttention(causal=causal, softcap=cap)
        out = torch.full_like(q, float("nan"))
        _, stats = op.forward(q, k, v, qo, kv_offsets=ko, slopes=slopes, prefix=prefix, max_q=bound, out=out)
        want, _ = _reference(q, k, v, q, qo, ko, causal, cap, prefix, slopes, d ** -0.5, dtype == torch.bfloat16)
        for b, (lo, hi) in enumerate(zip(qo.tolist(), qo.tolist()[1:])):
            _close(out[lo:hi], *want[b]["out"], f"out of sequence {b}")
            _close(stats.lse[lo:hi], *want[b]["lse"], f"lse of sequence {b}")


def _inputs(n):
    g = torch.Generator(device="cuda").manual_seed(n)
    q, do = (torch.randn(n, 2, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn(n, 2, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
    return q, k, v, do, _offsets([n])


def _gradients(op, q, k, v, do, off):
    out, stats = op.forward(q, k, v, off)
    return op.backward(do, q, k, v, out, stats, off)[:3]


def test_a_workspace_that_another_stream_works_on_is_not_handed_out():
    """A call that needs a larger workspace replaces it: the old one, which came from this stream, is not used again while
    the other stream, ordered after this one, still works on it."""
    print("workspace, streams", flush=True)
    small, large = _inputs(300), _inputs(30000)
    want = _gradients(R.SeqAttention(), *small)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _gradients(R.SeqAttention(), *large)  # memory of that stream's own for the calls below
    torch.cuda.synchronize()
    op = R.SeqAttention()
    _gradients(op, *small)
    first, size = op.ws.data_ptr(), op.ws.numel()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200000000)
        got = _gradients(op, *small)
        _gradients(op, *large)
        done = torch.cuda.Event()
        done.record()
    others = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(500)]
    assert not done.query()  # the other stream is still at work
    assert not any(t.data_ptr() < first + size and first < t.data_ptr() + size for t in others)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_workspace_that_a_graph_was_captured_with_is_kept():
    """A larger call after the capture takes another workspace, and the graph's own holds nobody else's values."""
    print("workspace, graph", flush=True)
    small, large = _inputs(300), _inputs(30000)
    want = _gradients(R.SeqAttention(), *small)
    side = torch.cuda.Stream()
    op = R.SeqAttention()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _gradients(op, *small)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _gradients(op, *small)
    size = op.ws.numel()
    _gradients(op, *large)
    assert op.ws.numel() > size
    torch.cuda.synchronize()
    with torch.cuda.stream(side):  # the stream that the first workspace came from
        others = [torch.full((size,), 77, dtype=torch.uint8, device="cuda") for _ in range(500)]
    torch.cuda.synchronize()
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all((t == 77).all() for t in others)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cap", [1e31, 1e38, 1e39, 1e300])
def test_a_cap_past_every_score(dtype, cap):
    """The cap's products with the scores would leave fp32: the same results as without a cap."""
    print("cap", dtype, cap, flush=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    off = _offsets([40, 3, 100])
    q, do = (torch.randn(143, 2, 64, generator=g, device="cuda").to(dtype) for _ in range(2))
    k, v = (torch.randn(143, 2, 64, generator=g, device="cuda").to(dtype) for _ in range(2))
    got = []
    for op in (R.SeqAttention(softcap=cap), R.SeqAttention()):
        out, stats = op.forward(q, k, v, off)
        got.append((out, stats.lse) + op.backward(do, q, k, v, out, stats, off)[:3])
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", TYPES)
def test_lengths_above_the_pad_length_are_cut(dtype):
    """A padded sequence longer than its block is its first pad rows, on either side; its positions go by the cut lengths."""
    print("cut", dtype, flush=True)
    hq, hkv, d, ql, kl = 4, 2, 64, [90, 64, 3, 200], [41, 500, 7, 40]
    for q_pad, kv_pad in ((64, 40), (64, 300), (130, 40)):
        for causal in (True, False):
            g = torch.Generator(device="cuda").manual_seed(q_pad)
            q, do = (torch.randn(4, q_pad, hq, d, generator=g, device="cuda").to(dtype) for _ in range(2))
            k, v = (torch.randn(4, kv_pad, hkv, d, generator=g, device="cuda").to(dtype) for _ in range(2))
            op = R.SeqAttention(causal=causal)
            kw = dict(kv_offsets=_offsets(kl))
            out, stats = op.forward(q, k, v, _offsets(ql), **kw)
            got = dict(zip(("out", "lse", "dq", "dk", "dv"),
                           (out, stats.lse) + op.backward(do, q, k, v, out, stats, _offsets(ql), **kw)[:3]))
            want, _ = _reference(q, k, v, do, _offsets(ql), _offsets(kl), causal, 0.0, None, None, d ** -0.5,
                                 dtype == torch.bfloat16)
            for name, t in got.items():
                for b in range(4):
                    n = want[b][name][0].shape[0]
                    assert n == (min(kl[b], kv_pad) if name in ("dk", "dv") else min(ql[b], q_pad))
                    _close(t[b, :n], *want[b][name], f"{name} of sequence {b}")
                    assert (t[b, n:] == (-float("inf") if name == "lse" else 0)).all()


@pytest.mark.parametrize("hq,hkv,d,ql,kl,max_q", [
    (4, 2, 64, [300, 5, 64], [300, 5, 64], 0),  # one pass over the keys
    (8, 2, 128, [1, 1, 1], [9000, 3, 700], 1),  # split and joined
    (4, 2, 64, [4, 1, 2], [20000, 3, 700], 4),  # few narrow rows, joined by waves and chunks
])
def test_rest_is_what_rounding_took(hq, hkv, d, ql, kl, max_q):
    """out + rest is the output before its rounding, and the backward takes delta from both.  Scores are next to 0, so P is
    1 / Lk with nothing lost as an operand, and v lies around 4: out's rounding is then the largest error of the forward,
    and of dq and dk, whose terms are differences of dP that the 4 does not change."""
    print("rest", hq, d, ql, flush=True)
    qo, ko = _offsets(ql), _offsets(kl)
    g = torch.Generator(device="cuda").manual_seed(d)
    q, do = (torch.randn(sum(ql), hq, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn(sum(kl), hkv, d, generator=g, device="cuda") for _ in range(2))
    k, v = (2 + k).bfloat16(), (4 + 0.1 * v).bfloat16()
    scale = 1e-8
    op = R.SeqAttention(causal=False, scale=scale)
    kw = dict(kv_offsets=ko, max_q=max_q)
    out, stats = op.forward(q, k, v, qo, **kw)
    want, _ = _reference(q, k, v, do, qo, ko, False, 0.0, None, None, scale, True)
    full = torch.cat([want[b]["out"][0] for b in range(len(ql))])
    # rest's own rounding, the sums over the keys and the scores' 1e-7 in P
    lim = (2.0 ** -16 + (max(kl) + 64) * 2.0 ** -24 + 1e-6) * 5
    assert float((out.double() + stats.rest.double() - full).abs().max()) <= lim
    assert float((out.double() - full).abs().max()) > 2 * lim  # without rest it is not
    with_rest = op.backward(do, q, k, v, out, stats, qo, **kw)
    without = op.backward(do, q, k, v, out, R.AttnStats(stats.lse, None), qo, **kw)
    for at, name in ((0, "dq"), (1, "dk")):
        ref = torch.cat([want[b][name][0] for b in range(len(ql))])
        a, b = (float((t[at].double() - ref).norm() / ref.norm()) for t in (with_rest, without))
        assert a < 0.5 * b, (name, a, b)


def test_backward_past_2_31_bytes():
    """A sequence whose q, k and v lie more than 2^32 bytes into their tensors: the gradients of the same sequence alone,
    and zero for the keys of a sequence without queries before it."""
    print("far backward", flush=True)
    lead, n, h, d = 20000000, 300, 1, 128
    g = torch.Generator(device="cuda").manual_seed(4)
    t = [torch.randn(n, h, d, generator=g, device="cuda").bfloat16() for _ in range(4)]
    far = [torch.empty(lead + n, h, d, dtype=torch.bfloat16, device="cuda") for _ in t]
    for a, b in zip(far, t):
        a[:lead], a[lead:] = 0.5, b
    off, alone = _offsets([lead, n]), _offsets([n])
    op = R.SeqAttention()
    m = torch.full((h,), 0.05, device="cuda")
    # the first sequence's queries see no key: it has none
    empty = torch.tensor([0, 0, n], device="cuda")
    out, stats = op.forward(far[0], t[1], t[2], off, kv_offsets=empty, slopes=m)
    ref, rstats = op.forward(t[0], t[1], t[2], alone, slopes=m)
    assert torch.equal(out[lead:], ref) and not out[:lead].any()
    got = op.backward(far[3], far[0], t[1], t[2], out, stats, off, kv_offsets=empty, slopes=m)
    want = op.backward(t[3], t[0], t[1], t[2], ref, rstats, alone, slopes=m)
    assert torch.equal(got[0][lead:], want[0]) and not got[0][:lead].any()
    # and the keys far into theirs, the first sequence without a query
    out, stats = op.forward(t[0], far[1], far[2], empty, kv_offsets=off, slopes=m)
    far_k = op.backward(t[3], t[0], far[1], far[2], out, stats, empty, kv_offsets=off, slopes=m)
    for name, a, b in (("dk", far_k[1], want[1]), ("dv", far_k[2], want[2])):
        # larger key tiles, since there are many: the fp32 sums in another order, rounded once
        assert (a[lead:].double() - b.double()).norm() <= 2.0 ** -8 * b.double().norm() and not a[:lead].any(), name
    for name, a, b in (("dk", got[1], want[1]), ("dv", got[2], want[2])):
        assert torch.equal(a, b), name
