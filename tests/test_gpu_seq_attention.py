"""Attention over ragged sequences, forward and backward, against the formulas in 64 bits.

Tolerances (u = 2^-24; r = 2^-8 in bf16, the rounding of an operand or a result to 8 significant bits, 0 in fp32) follow the arithmetic:
  score      a dot product of d terms, (d + 8) u of its summed magnitudes; the few operations after it, 8 u of the score
             and of the distance term; the capped score in bf16, 4e-7 of the cap (tanh to about 1e-7)
  P          e_ij = its score's error + the largest of its row (the normaliser's) + 16 u, relative
  out        sum_j P |v| (e + r + (Lk + 64) u), and r |out| for the result's rounding
  dP, delta  dot products of d terms; delta also takes out's error and the rounding of out's rest
  ds         P (e |dP - delta| + dP's and delta's error), and r |ds| as an operand
  gradients  those errors through their sums, (terms + 64) u of the magnitudes, r of the result
  dslopes    the same without roundings to bf16: its sums are fp32 throughout
"""
import math

import pytest
import torch

from paper_2509_20883_amd import recis as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _offsets(lens):
    return torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int64, device="cuda")


def _blocks(x, off, pad):
    """Each sequence's rows in float64."""
    o = off.tolist()
    n = len(o) - 1
    if pad:
        return [x[b, :min(o[b + 1] - o[b], pad)].double() for b in range(n)]
    return [x[o[b]:o[b + 1]].double() for b in range(n)]


def _reference(q, k, v, do, q_off, k_off, causal, cap, prefix, slopes, scale, bf16):
    """Per sequence: out, lse, dq, dk, dv (and dslopes of all), each with its error bound."""
    r = 2.0 ** -8 if bf16 else 0.0
    hq, hkv, d = q.shape[-2], k.shape[-2], q.shape[-1]
    G = hq // hkv
    qb, kb, vb, ob = (_blocks(t, off, t.dim() == 4 and t.shape[1]) for t, off in ((q, q_off), (k, k_off), (v, k_off), (do, q_off)))
    res, dsl, edsl = [], torch.zeros(hq, dtype=torch.float64, device="cuda"), torch.zeros(hq, dtype=torch.float64, device="cuda")
    for b, (Q, K, V, O) in enumerate(zip(qb, kb, vb, ob)):
        lq, lk = Q.shape[0], K.shape[0]
        Q, O = Q.transpose(0, 1), O.transpose(0, 1)  # [hq, lq, d]
        K, V = (t.transpose(0, 1).repeat_interleave(G, 0) for t in (K, V))
        p = torch.arange(lq, device="cuda")[:, None] + lk - lq
        j = torch.arange(lk, device="cuda")[None]
        see = torch.ones(lq, lk, dtype=torch.bool, device="cuda")
        if causal:
            see = (j <= p) | (j < (int(prefix[b]) if prefix is not None else 0))
        dist = (p - j).abs().double()
        x = Q @ K.transpose(1, 2) * scale
        es = (d + 8) * U * (Q.abs() @ K.abs().transpose(1, 2)) * scale
        deriv = torch.ones_like(x)
        if cap:
            th = torch.tanh(x / cap)
            x, deriv = cap * th, 1 - th * th
            es = es + (4e-7 if bf16 else 4 * U) * cap
        if slopes is not None:
            m = slopes.double().view(-1, 1, 1)
            x = x - m * dist
            es = es + 8 * U * m.abs() * dist
        es = es + 8 * U * x.abs()
        some = see.any(1, keepdim=True)
        x = torch.where(see, x, -math.inf)
        lse = torch.logsumexp(x, 2) if lk else torch.full((hq, lq), -math.inf, dtype=torch.float64, device="cuda")
        P = torch.where(see & some, torch.exp(x - torch.where(torch.isfinite(lse), lse, 0.0)[..., None]), 0.0)
        es = torch.where(see, es, 0.0)
        e = es + (es.amax(2, keepdim=True) if lk else 0.0) + 16 * U
        out = P @ V
        eout = (P * (e + r + (lk + 64) * U)) @ V.abs() + r * out.abs()
        dP = O @ V.transpose(1, 2)
        edP = (d + 8) * U * (O.abs() @ V.abs().transpose(1, 2))
        delta = (O * out).sum(2, keepdim=True)
        edelta = (O.abs() * (eout + (d + 8) * U * out.abs())).sum(2, keepdim=True)
        dS = P * (dP - delta)
        edS = P * (e * (dP - delta).abs() + edP + edelta)
        if slopes is not None:
            dsl -= (dS * dist).sum((1, 2))
            # sum P dP t - (sum P dP)(sum P t): each sum's error, without delta's
            ePd = P * (e * dP.abs() + edP + (lk + 64) * U * dP.abs())
            ePt = P * (e + (lk + 64) * U)
            edsl += ((ePd * dist).sum(2) + ePd.sum(2) * (P * dist).sum(2) + (P * dP).abs().sum(2) * (ePt * dist).sum(2)
                     ).sum(1)
        dX = dS * deriv
        edX = edS + 4e-7 * dS.abs() * (1 if cap else 0) + (r + 4 * U) * dX.abs()
        if cap:  # the derivative 1 - tanh^2 carries twice the tanh's error
            edX = edX + dS.abs() * 2 * es / cap
        dq = scale * (dX @ K)
        edq = scale * ((edX + (lk + 64) * U * dX.abs()) @ K.abs())
        dk = scale * (dX.transpose(1, 2) @ Q)
        edk = scale * ((edX + (lq * G + 64) * U * dX.abs()).transpose(1, 2) @ Q.abs())
        dv = P.transpose(1, 2) @ O
        edv = (P * (e + r + (lq * G + 64) * U)).transpose(1, 2) @ O.abs()
        fold = lambda t: t.view(hkv, G, *t.shape[1:]).sum(1).transpose(0, 1)  # noqa: E731
        res.append(dict(out=(out.transpose(0, 1), eout.transpose(0, 1)), dq=(dq.transpose(0, 1), edq.transpose(0, 1)),
                        dk=(fold(dk), fold(edk)), dv=(fold(dv), fold(edv)),
                        lse=(lse.transpose(0, 1), ((es.amax(2) if lk else 0.0) + (16 + lk) * U + 8 * U * lse.abs().nan_to_num(posinf=0.0)).transpose(0, 1)
                             if lk else torch.zeros(lq, hq, dtype=torch.float64, device="cuda"))))
    return res, (dsl, edsl)


def _close(got, want, bound, what):
    half_ulp = 2.0 ** -8 if got.dtype == torch.bfloat16 else U
    got = got.double()
    fin = torch.isfinite(want)
    assert torch.equal(got[~fin], want[~fin]), f"{what}: infinities differ"
    err = torch.where(fin, (got - want).abs(), 0.0)
    lim = torch.where(fin, bound + half_ulp * (want.abs() + bound) + 1e-30, 1.0)
    bad = ~(err <= lim)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / lim).max()):.3g} of the bound"


def _case(dtype, hq, hkv, d, q_lens, kv_lens=None, causal=True, cap=0.0, prefix=None, slopes=False, q_pad=0, kv_pad=0,
          max_q=0, seed=0, train=True, scale=None, gap=0, spread=1.0, poison=False):
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    kv_lens_ = q_lens if kv_lens is None else kv_lens
    q_off, k_off = _offsets(q_lens), _offsets(kv_lens_)
    n = len(q_lens)

    def rand(lens, pad, heads):
        lead = (n, pad) if pad else (sum(lens),)
        t = (spread * torch.randn(*lead, heads, d + gap, generator=g, device="cuda")).to(dtype)[..., :d]
        if pad and poison:  # past a sequence's end
            dead = torch.arange(pad, device="cuda") >= torch.tensor(lens, device="cuda")[:, None]
            t[dead] = float("nan")
        return t

    q, do = rand(q_lens, q_pad, hq), rand(q_lens, q_pad, hq)
    k, v = rand(kv_lens_, kv_pad, hkv), rand(kv_lens_, kv_pad, hkv)
    pre = None if prefix is None else torch.tensor(prefix, dtype=torch.int64, device="cuda")
    sl = torch.rand(hq, generator=g, device="cuda") * 0.2 if slopes else None
    op = R.SeqAttention(scale=scale, softcap=cap, causal=causal)
    kw = dict(kv_offsets=k_off if kv_lens is not None else None, prefix=pre, slopes=sl, max_q=max_q)
    out, stats = op.forward(q, k, v, q_off, validate=True, **kw)
    got = dict(out=out, lse=stats.lse)
    if train:
        got["dq"], got["dk"], got["dv"], dsl = op.backward(do, q, k, v, out, stats, q_off, validate=True, **kw)
    want, (wdsl, edsl) = _reference(q, k, v, do, q_off, k_off, causal, cap, pre, sl,
                                    d ** -0.5 if scale is None else scale, dtype == torch.bfloat16)
    qo, ko = q_off.tolist(), k_off.tolist()
    for name, t in got.items():
        off, pad = (ko, kv_pad) if name in ("dk", "dv") else (qo, q_pad)
        for b in range(n):
            m = want[b][name][0].shape[0]
            rows = t[b, :m] if pad else t[off[b]:off[b + 1]]
            _close(rows, *want[b][name], f"{name} of sequence {b} ({q_lens[b]} over {kv_lens_[b]})")
            if pad:
                rest = t[b, m:]
                assert (rest == (-math.inf if name == "lse" else 0)).all(), f"{name}: padding of sequence {b}"
    if train and slopes:
        _close(dsl, wdsl, edsl, "dslopes")
    return got


TYPES = [torch.float32, torch.bfloat16]
RAGGED = [5, 0, 1, 64, 130, 33, 200, 2]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [8, 16, 32, 40, 64, 72, 96, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (6, 2)])
def test_head_layouts(dtype, d, hq, hkv):
    print("heads", dtype, d, hq, hkv, flush=True)
    _case(dtype, hq, hkv, d, RAGGED, seed=d + hq)
    _case(dtype, hq, hkv, d, RAGGED, causal=False, slopes=True, cap=5.0, seed=d + hq + 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("cap", [0.0, 3.0])
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("prefix", [None, [2, 0, 1, 70, 500, 32, 65, 1]])
def test_scores_and_masks(dtype, causal, cap, slopes, prefix):
    print("scores", dtype, causal, cap, slopes, prefix is not None, flush=True)
    _case(dtype, 4, 2, 32, RAGGED, causal=causal, cap=cap, slopes=slopes, prefix=prefix)
    _case(dtype, 2, 2, 64, RAGGED, causal=causal, cap=cap, slopes=slopes, prefix=prefix, q_pad=201, kv_pad=201, poison=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_other_keys_than_queries(dtype, causal):
    """Chunks over a history, more queries than keys (rows that see nothing), empty sides."""
    print("chunks", dtype, causal, flush=True)
    ql, kl = [3, 0, 70, 1, 9, 40, 129, 1], [200, 5, 64, 1, 0, 17, 300, 65]
    for hq, hkv, d in ((2, 2, 32), (8, 2, 128), (5, 1, 64)):
        _case(dtype, hq, hkv, d, ql, kl, causal=causal, seed=d)
        _case(dtype, hq, hkv, d, ql, kl, causal=causal, slopes=True, cap=4.0, prefix=[9, 5, 3, 1, 0, 2, 77, 0], seed=d + 1)
    _case(dtype, 4, 2, 64, ql, kl, causal=causal, q_pad=130, seed=7, poison=True)
    _case(dtype, 4, 2, 64, ql, kl, causal=causal, kv_pad=300, seed=8, poison=True)
    # lengths above the pad length are cut, as the padded copy cuts them: the reference sees the cut rows
    _case(dtype, 4, 2, 64, [64] * 3, [40] * 3, causal=causal, q_pad=64, kv_pad=40, seed=9)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (8, 1, 128), (3, 1, 32)])
def test_chunks_over_long_keys(dtype, hq, hkv, d):
    """Several row tiles over keys long enough to be split, chunks that no row sees, a padded side."""
    print("long chunks", dtype, hq, hkv, d, flush=True)
    ql, kl = [70, 0, 129, 1], [3000, 2000, 257, 5001]
    for causal in (True, False):
        for bound in (129, 0):
            _case(dtype, hq, hkv, d, ql, kl, causal=causal, max_q=bound, seed=d, train=False)
        _case(dtype, hq, hkv, d, ql, kl, causal=causal, slopes=True, cap=5.0, prefix=[100, 3, 300, 2600], max_q=129, seed=1,
              train=False)
    _case(dtype, hq, hkv, d, ql, kl, q_pad=130, kv_pad=5001, seed=2, train=False, poison=True)
    # more queries than keys: the first rows of the sequence see nothing
    _case(dtype, hq, hkv, d, [90, 700], [4000, 600], seed=3, train=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 257, 1000])
def test_lengths_around_the_tiles(dtype, n):
    print("length", dtype, n, flush=True)
    for group in (1, 3):
        _case(dtype, 2 * group, 2, 64, [n], seed=n)
        _case(dtype, 2 * group, 2, 64, [n, 1, n], causal=False, seed=n + 1)
    _case(dtype, 4, 1, 128, [n], prefix=[n // 2], seed=n + 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d", [(1, 1, 64), (8, 2, 128), (16, 1, 32), (40, 1, 64)])
@pytest.mark.parametrize("max_q", [1, 4])
def test_single_tokens(dtype, hq, hkv, d, max_q):
    """One or a few queries over histories of very unequal length, with the bound of their count and without it."""
    print("tokens", dtype, hq, hkv, d, max_q, flush=True)
    kl = [1, 0, 63, 64, 65, 700, 2049, 5000, 3]
    ql = [max_q] * len(kl) if max_q == 1 else [1, 4, 0, 2, 4, 3, 1, 4, 4]
    for bound in (max_q, 0):
        _case(dtype, hq, hkv, d, ql, kl, max_q=bound, seed=hq + d, train=False)
        _case(dtype, hq, hkv, d, ql, kl, max_q=bound, causal=False, cap=9.0, slopes=True, seed=hq + d + 1, train=False)
        _case(dtype, hq, hkv, d, ql, [20000] + kl[1:], max_q=bound, prefix=[30] * len(kl), causal=True, seed=3, train=False)
    _case(dtype, hq, hkv, d, ql, kl, max_q=max_q, seed=5)  # and their gradients
    _case(dtype, hq, hkv, d, ql, [min(x, 900) for x in kl], max_q=max_q, q_pad=max_q, kv_pad=900, seed=6, train=False,
          poison=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_sequences(dtype):
    """More sequences than a wave finds in one step of its search, most of them short, many empty."""
    print("many", dtype, flush=True)
    g = torch.Generator().manual_seed(3)
    for n in (65, 700, 4500):
        lens = torch.randint(0, 12, (n,), generator=g)
        lens[torch.rand(n, generator=g) < 0.4] = 0
        lens[n // 2] = 150
        _case(dtype, 2, 1, 32, lens.tolist(), seed=n, train=n < 4000)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [32, 64, 128])
def test_enough_sequences_for_whole_key_tiles(dtype, d):
    """The backward takes larger key tiles where there are many of them: packed and padded, one and several heads a key head."""
    print("tiles", dtype, d, flush=True)
    g = torch.Generator().manual_seed(d)
    lens = torch.randint(0, 30, (400,), generator=g)
    lens[7], lens[200] = 300, 129
    _case(dtype, 4, 4, d, lens.tolist(), slopes=True, cap=6.0, seed=1)
    _case(dtype, 8, 4, d, lens.clamp(max=40).tolist(), q_pad=40, kv_pad=40, causal=False, seed=2, poison=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv", [(33, 1), (65, 1), (200, 1), (130, 2)])
def test_many_heads_on_a_key_head(dtype, hq, hkv):
    """More query heads on a key head than a step of the backward holds rows."""
    print("groups", dtype, hq, hkv, flush=True)
    _case(dtype, hq, hkv, 32, [3, 0, 1, 40, 70], slopes=True, seed=hq)
    _case(dtype, hq, hkv, 64, [5, 1], [90, 700], max_q=5, cap=3.0, seed=hq + 1)
    _case(dtype, hq, hkv, 128, [2, 9], causal=False, seed=hq + 2)


@pytest.mark.parametrize("dtype", TYPES)
def test_values(dtype):
    """Large scores (one key takes all), equal scores, a scale of one's own."""
    print("values", dtype, flush=True)
    _case(dtype, 2, 2, 64, [100, 70], spread=6.0, seed=1)
    _case(dtype, 2, 2, 64, [100, 70], spread=1e-3, seed=2)
    _case(dtype, 2, 1, 64, [100, 70], scale=0.7, cap=2.0, seed=3)
    # scores far below zero everywhere: the distance term alone is hundreds
    _case(dtype, 2, 2, 32, [1, 700], [700, 700], slopes=True, causal=False, scale=1e-6, seed=4)


@pytest.mark.parametrize("dtype", TYPES)
def test_strided_inputs(dtype):
    """q, k and v as column blocks of one projection, and layouts that are copied."""
    print("strides", dtype, flush=True)
    off = _offsets(RAGGED)
    T, hq, hkv, d = sum(RAGGED), 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(11)
    qkv = torch.randn(T, hq + 2 * hkv, d, generator=g, device="cuda").to(dtype)
    parts = qkv.split([hq, hkv, hkv], 1)
    op = R.SeqAttention()
    do = torch.randn(T, hq, d, generator=g, device="cuda").to(dtype)

    def both(q, k, v, go):
        out, lse = op.forward(q, k, v, off)
        return (out, lse.lse) + op.backward(go, q, k, v, out, lse, off)[:3]

    want = both(*(t.contiguous() for t in parts), do)
    assert all(torch.equal(a, b) for a, b in zip(want, both(*parts, do)))
    heads_first = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in parts]
    assert all(torch.equal(a, b) for a, b in zip(want, both(*heads_first, do)))
    odd = [torch.zeros(t.numel() + 1, dtype=dtype, device="cuda")[1:].view(t.shape).copy_(t) for t in (*parts, do)]
    assert all(torch.equal(a, b) for a, b in zip(want, both(*odd)))
    inner = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in parts]
    assert all(torch.equal(a, b) for a, b in zip(want, both(*inner, do)))
    _case(dtype, 4, 2, 32, RAGGED, gap=8)
    # every row of k the same memory
    out, _ = op.forward(parts[0], parts[1][:1].expand(T, -1, -1), parts[2], off)
    ref, _ = op.forward(parts[0], parts[1][:1].expand(T, -1, -1).contiguous(), parts[2], off)
    assert torch.equal(out, ref)


def test_gradient_against_differences():
    """Central differences of a weighted sum of the fp32 forward along random directions; the step's truncation is
    O(h^2) and the forward's rounding u / h of the sum's magnitudes."""
    print("differences", flush=True)
    g = torch.Generator(device="cuda").manual_seed(4)
    lens, pre = [9, 40], torch.tensor([4, 0], device="cuda")
    off = _offsets(lens)
    q, do = (torch.randn(49, 4, 16, generator=g, device="cuda") for _ in range(2))
    k, v = (torch.randn(49, 2, 16, generator=g, device="cuda") for _ in range(2))
    m = torch.rand(4, generator=g, device="cuda") * 0.1 + 0.05
    op = R.SeqAttention(softcap=2.0)
    f = lambda q, k, v, m: op.forward(q, k, v, off, prefix=pre, slopes=m)  # noqa: E731
    out, lse = f(q, k, v, m)
    grads = op.backward(do, q, k, v, out, lse, off, prefix=pre, slopes=m)
    h = 1e-2
    for at, grad in enumerate(grads):
        u = torch.randn(grad.shape, generator=g, device="cuda")
        u = u / u.norm()
        val = []
        for sign in (1, -1):
            args = [t + sign * h * u if i == at else t for i, t in enumerate((q, k, v, m))]
            val.append(float((f(*args)[0].double() * do.double()).sum()))
        diff, got = (val[0] - val[1]) / (2 * h), float((grad.double() * u.double()).sum())
        assert abs(diff - got) <= 3e-3 * (float(grad.double().norm()) + 1.0), (at, diff, got)


def test_repeats_streams_and_workspace():
    print("repeats", flush=True)
    op = R.SeqAttention(causal=True)
    g = torch.Generator(device="cuda").manual_seed(8)
    for lens in ([300, 20, 500], [7], [1000] * 6, [64, 64]):
        off = _offsets(lens)
        q, do = (torch.randn(sum(lens), 4, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
        k, v = (torch.randn(sum(lens), 2, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
        m = torch.rand(4, generator=g, device="cuda") * 0.1

        def both(o):
            out, lse = o.forward(q, k, v, off, slopes=m)
            return (out, lse.lse) + o.backward(do, q, k, v, out, lse, off, slopes=m)

        first = both(op)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            second = both(R.SeqAttention(causal=True))
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, second))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_outside_every_sequence(dtype):
    """Offsets that start past 0 and end before the last row: the rows outside are neither read nor written."""
    print("outside", dtype, flush=True)
    g = torch.Generator(device="cuda").manual_seed(6)
    op = R.SeqAttention()
    for q_lens, k_lens in (([40, 130], [40, 130]), ([1, 2], [700, 9000])):
        nq, nk, lead = sum(q_lens), sum(k_lens), 300
        q, do = (torch.randn(lead + nq + 9, 4, 64, generator=g, device="cuda").to(dtype) for _ in range(2))
        k, v = (torch.randn(lead + nk + 9, 2, 64, generator=g, device="cuda").to(dtype) for _ in range(2))
        in_q, in_k = slice(lead, lead + nq), slice(lead, lead + nk)
        ref = op.forward(q[in_q], k[in_k], v[in_k], _offsets(q_lens), kv_offsets=_offsets(k_lens), max_q=max(q_lens))
        want = (ref[0],) + op.backward(do[in_q], q[in_q], k[in_k], v[in_k], *ref, _offsets(q_lens),
                                       kv_offsets=_offsets(k_lens))[:3]
        for t, inside in ((q, in_q), (do, in_q), (k, in_k), (v, in_k)):
            t[:lead], t[inside.stop:] = float("nan"), float("nan")
        out = torch.full_like(q, 7.0)
        qo, ko = _offsets(q_lens) + lead, _offsets(k_lens) + lead
        _, stats = op.forward(q, k, v, qo, kv_offsets=ko, max_q=max(q_lens), out=out)
        assert (out[:lead] == 7.0).all() and (out[in_q.stop:] == 7.0).all()
        dq, dk, dv, _ = op.backward(do, q, k, v, out, stats, qo, kv_offsets=ko)
        got = (out[in_q], dq[in_q], dk[in_k], dv[in_k])
        for name, a, b in zip(("out", "dq", "dk", "dv"), got, want):
            # the key chunks of a split start elsewhere: equal up to the order of the fp32 sums
            tol = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -18
            assert (a.double() - b.double()).norm() <= tol * b.double().norm(), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cap, spread", [(100.0, 1.0), (2.0, 1.0), (2.0, 6.0)])
def test_small_and_saturated_caps(dtype, cap, spread):
    """All scores below half the cap, on both sides of it, and far past it."""
    print("caps", dtype, cap, spread, flush=True)
    _case(dtype, 4, 2, 64, [33, 1, 0, 150, 64], cap=cap, spread=spread, slopes=True, causal=False, seed=9)


def test_offsets_past_32_bits():
    """A history whose keys lie more than 2^32 bytes into the tensor, in rows 2 KiB apart."""
    print("far keys", flush=True)
    rows, d, seq = 2200000, 64, 300
    big = torch.zeros(rows, 1, 1024, dtype=torch.bfloat16, device="cuda")[..., :d]
    g = torch.Generator(device="cuda").manual_seed(2)
    tail = torch.randn(seq, 1, d, generator=g, device="cuda").bfloat16()
    big[rows - seq:] = tail
    q = torch.randn(1, 2, d, generator=g, device="cuda").bfloat16()
    op = R.SeqAttention()
    ql, kl = _offsets([0, 1]), _offsets([rows - seq, seq])
    out, _ = op.forward(q, big, big, ql, kl, max_q=1)
    ref, _ = op.forward(q, tail, tail, _offsets([1]), _offsets([seq]), max_q=1)
    _close(out, ref.double(), 2.0 ** -8 * torch.ones_like(ref).double(), "far keys")


def test_refusals():
    off = _offsets([3, 4])
    q, k = torch.randn(7, 4, 16, device="cuda"), torch.randn(7, 2, 16, device="cuda")
    op = R.SeqAttention()
    out, stats = op.forward(q, k, k, off)
    lse = stats.lse
    bad = [lambda: op.forward(q.half(), k.half(), k.half(), off), lambda: op.forward(q, k.bfloat16(), k, off),
           lambda: op.forward(q.cpu(), k, k, off), lambda: op.forward(q, k[:, :, :8], k[:, :, :8], off),
           lambda: op.forward(q, k, k[:6], off), lambda: op.forward(q[:, :3], k, k, off),
           lambda: op.forward(q[..., :12], k[..., :12], k[..., :12], off),
           lambda: op.forward(torch.randn(7, 4, 136, device="cuda"), torch.randn(7, 2, 136, device="cuda"),
                              torch.randn(7, 2, 136, device="cuda"), off),
           lambda: op.forward(q, k, k, off.int()), lambda: op.forward(q, k, k, off, kv_offsets=off[:2]),
           lambda: op.forward(q, k, k, off, prefix=torch.zeros(3, dtype=torch.int64, device="cuda")),
           lambda: op.forward(q, k, k, off, slopes=torch.zeros(3, device="cuda")),
           lambda: op.forward(q, k, k, off, max_q=-1), lambda: op.forward(q, k, k, off, out=torch.empty_like(k)),
           lambda: op.forward(q.view(1, 7, 4, 16), k, k, off),
           lambda: R.SeqAttention(scale=0.0).forward(q, k, k, off), lambda: R.SeqAttention(scale=math.inf).forward(q, k, k, off),
           lambda: R.SeqAttention(softcap=-1.0).forward(q, k, k, off),
           lambda: R.SeqAttention(softcap=math.nan).forward(q, k, k, off),
           lambda: op.forward(q, k, k, torch.tensor([1, 3, 7], device="cuda"), validate=True),
           lambda: op.forward(q, k, k, torch.tensor([0, 5, 3], device="cuda"), validate=True),
           lambda: op.forward(q, k, k, torch.tensor([0, 3, 6], device="cuda"), validate=True),
           lambda: op.forward(q, k, k, off, max_q=3, validate=True),
           lambda: op.backward(q[:6], q, k, k, out, stats, off), lambda: op.backward(q, q, k, k, out.bfloat16(), stats, off),
           lambda: op.backward(q, q, k, k, out, R.AttnStats(lse[:, :2], None), off),
           lambda: op.backward(q, q, k, k, out, R.AttnStats(lse, out.bfloat16()), off)]
    for f in bad:
        with pytest.raises(R.RecisError) as e:
            f()
        assert e.value.status == R.EINVAL
    # the C boundary itself
    import ctypes as C
    L = R.lib()
    good = dict(dtype=R.F32, heads_q=4, heads_kv=2, head_dim=16, causal=1, reserved=0, seqs=2, q_rows=7, kv_rows=7, q_pad=0,
                kv_pad=0, max_q=0, q_stride=64, q_head_stride=16, k_stride=32, k_head_stride=16, v_stride=32,
                v_head_stride=16, scale=0.25, softcap=0.0)
    for field, v in (("dtype", 2), ("heads_q", 3), ("heads_q", 0), ("heads_kv", 0), ("heads_kv", 1025), ("head_dim", 12),
                     ("head_dim", 136), ("head_dim", 0), ("reserved", 1), ("seqs", -1), ("q_rows", -1), ("q_rows", 1 << 30),
                     ("kv_rows", 1 << 31), ("q_pad", 4), ("kv_pad", 5), ("q_pad", -1), ("max_q", -2), ("q_stride", 62),
                     ("k_stride", -4), ("v_head_stride", 1 << 23), ("scale", -1.0), ("softcap", -2.0)):
        d = R.AttnDesc(**dict(good, **{field: v}))
        assert L.seq_attention_workspace_bytes(C.byref(d), 1) == 0
        assert L.seq_attention_fwd(C.byref(d), q.data_ptr(), k.data_ptr(), k.data_ptr(), off.data_ptr(), off.data_ptr(),
                                   None, None, out.data_ptr(), None, lse.data_ptr(), None, 0, 0, None) == R.EINVAL
        assert L.rs_last_error()
    d = R.AttnDesc(**good)
    fwd = [q.data_ptr(), k.data_ptr(), k.data_ptr(), off.data_ptr(), off.data_ptr(), None, None, out.data_ptr(),
           None, lse.data_ptr(), None, 0, 0, None]
    for at, v in ((0, None), (1, None), (2, None), (3, None), (4, None), (7, None), (0, q.data_ptr() + 4),
                  (7, out.data_ptr() + 8), (8, out.data_ptr() + 8)):
        args = list(fwd)
        args[at] = v
        assert L.seq_attention_fwd(C.byref(d), *args) == R.EINVAL
    assert L.seq_attention_fwd(None, *fwd) == R.EINVAL
    need = L.seq_attention_workspace_bytes(C.byref(d), 1)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(k)
    ds = torch.empty(4, device="cuda")
    bwd = [q.data_ptr(), k.data_ptr(), k.data_ptr(), out.data_ptr(), None, lse.data_ptr(), q.data_ptr(),
           off.data_ptr(), off.data_ptr(), None, None, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), None, ws.data_ptr(), need, 0, None]
    for at, v in ((0, None), (3, None), (5, None), (6, None), (7, None), (8, None), (11, None), (12, None), (13, None),
                  (14, ds.data_ptr()), (15, None), (15, ws.data_ptr() + 16), (16, need - 1), (6, q.data_ptr() + 4)):
        args = list(bwd)
        args[at] = v
        assert L.seq_attention_bwd(C.byref(d), *args) == R.EINVAL
    assert L.seq_attention_bwd(C.byref(d), *bwd) == R.OK
    torch.cuda.synchronize()


def test_empty_calls():
    print("empty", flush=True)
    op = R.SeqAttention()
    for lens, n in (([], 0), ([0, 0], 0)):
        off = _offsets(lens) if lens else torch.zeros(1, dtype=torch.int64, device="cuda")
        q, k = torch.empty(0, 4, 16, device="cuda"), torch.empty(0, 2, 16, device="cuda")
        m = torch.ones(4, device="cuda")
        out, lse = op.forward(q, k, k, off, slopes=m)
        dq, dk, dv, dm = op.backward(q, q, k, k, out, lse, off, slopes=m)
        assert out.shape == q.shape and dk.shape == k.shape and not dm.any()
    # queries without any key, keys without any query
    _case(torch.float32, 4, 2, 16, [5, 3], [0, 0])
    _case(torch.float32, 4, 2, 16, [0, 0], [5, 3], slopes=True)
