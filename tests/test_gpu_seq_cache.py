"""The paged cache: append, read, attention and the choice of pages, against the formulas in 64 bits.

Turned rows are off by their rounding to the model's type and by 2^-31 of the pair's length (the angle, to 2^-33 turns below
position 2^31, and the series).  What follows from the turned tokens is exact: codes, scales, bounds, the choice of pages.
The attention's bound stands at cache_reference.attention."""
import math
import random

import pytest
import torch

from paper_2509_20883_amd import recis as R
from tests import cache_reference as ref

pytestmark = pytest.mark.gpu
U = ref.U
BF, F32 = torch.bfloat16, torch.float32


def _cache(pages, slots, hkv, d, page=64, codes="i8", dtype=BF, **kw):
    c = R.SeqCache(pages, slots, hkv, d, page=page, codes=codes, dtype=dtype, **kw)
    c.codes.fill_(0x7F)  # NaN in e4m3
    c.scales.fill_(math.nan)
    c.open.fill_(math.nan)
    if c.bounds is not None:
        c.bounds.fill_(1)
        c.units.fill_(math.nan)
    return c


def _tables(c, pages_per_seq, seed=0, width=None):
    """A table of distinct pages in random order; unused entries are out of range."""
    rng = random.Random(seed)
    ids = list(range(c.codes.shape[0]))
    rng.shuffle(ids)
    width = max([1] + pages_per_seq) if width is None else width
    rows = []
    for n in pages_per_seq:
        rows.append([ids.pop() for _ in range(n)] + [2 ** 30] * (width - n))
    return torch.tensor(rows, dtype=torch.int32, device="cuda").view(len(pages_per_seq), width)


def _slots(n, seed=0, extra=2):
    s = list(range(n + extra))
    random.Random(seed + 1).shuffle(s)
    return torch.tensor(s[:n], dtype=torch.int32, device="cuda")


def _dev(x, dtype=torch.int64):
    return torch.tensor(x, dtype=dtype, device="cuda")


def _half(dtype):
    return 2.0 ** -8 if dtype == BF else U


# ---------------------------------------------------------------------------
# rotation
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,rotary,interleaved", [(64, 64, False), (128, 128, True), (72, 48, False), (72, 6, True), (16, 2, False),
                                                  (8, 8, True), (32, 0, False), (128, 126, False)])
def test_queries_turn_by_their_position(dtype, d, rotary, interleaved):
    g = torch.Generator(device="cuda").manual_seed(rotary)
    lens = [0, 5, 1000003, 2 ** 31 - 2000, 7]
    new = [3, 0, 70, 4, 1]
    c = R.SeqCache(4, 8, 1, d, dtype=dtype, rotary=rotary, interleaved=interleaved, base=500000.0)
    off = ref.offsets(new)
    table = torch.zeros(5, 1, dtype=torch.int32, device="cuda")
    y = torch.randn(sum(new), 7, d, generator=g, device="cuda").to(dtype)
    q = y[:, 1:4]
    assert not q.is_contiguous()
    after, out = c.append(None, None, off, _dev(lens), table, q=q)
    assert after.tolist() == [a + b for a, b in zip(lens, new)]
    pos = torch.cat([torch.arange(a, a + b) for a, b in zip(lens, new)]).cuda()
    want = ref.turned(q, pos, [500000.0 ** (-2.0 * i / rotary) for i in range(rotary // 2)], rotary, interleaved)
    size = ref.turned(q.abs(), pos * 0, [0.0] * (rotary // 2), rotary, interleaved)
    h = rotary // 2
    pair = size.clone()
    if interleaved:
        pair[..., 0:rotary:2] = pair[..., 1:rotary:2] = size[..., 0:rotary:2] + size[..., 1:rotary:2]
    else:
        pair[..., :h] = pair[..., h:rotary] = size[..., :h] + size[..., h:rotary]
    # a frequency as a double is off by 2^-53 of itself: at 2^31, 2^-22 radians in the reference
    slack = pair * (2.0 ** -31 + pos.double()[:, None, None] * 2.0 ** -53)
    slack[..., rotary:] = 0
    bound = _half(dtype) * (want.abs() + slack) + slack
    off_by = (out.double() - want).abs()
    assert bool((off_by <= bound).all()), float((off_by / bound).nan_to_num().max())


def test_own_frequencies_and_padded_rows():
    g = torch.Generator(device="cuda").manual_seed(3)
    freqs = [1.0, 0.25, 7.5, 0.0]
    c = R.SeqCache(1, 3, 2, 16, dtype=F32, rotary=8, freqs=freqs)
    q = torch.randn(3, 5, 4, 16, generator=g, device="cuda")
    q[0, 2:] = math.nan  # past the sequence's end
    off, lens = _dev([0, 2, 7, 14]), _dev([9, 0, 3])  # the last is cut to the pad length
    table = torch.zeros(3, 1, dtype=torch.int32, device="cuda")
    after, out = c.append(None, None, off, lens, table, q=q)
    assert after.tolist() == [11, 5, 8]
    assert (out[0, 2:] == 0).all()
    for b, n in ((0, 2), (1, 5), (2, 5)):
        want = ref.turned(q[b, :n], lens[b] + torch.arange(n, device="cuda"), freqs, 8, False)
        assert float(((out[b, :n].double() - want).abs() - U * want.abs()).max()) <= 2.0 ** -30 * 8


# ---------------------------------------------------------------------------
# append and read
# ---------------------------------------------------------------------------


def _check_pages(c, table, tokens, lens, slots, codes, touched):
    """Pages `touched` [(sequence, page number)] hold the tokens [len, hkv, 2, d] exactly; open pages too."""
    P = c.page
    vals, scales = ref.pages_of(c)
    for b, n in touched:
        x = tokens[b][n * P:(n + 1) * P]
        if x.shape[0] < P:
            got = c.open[int(slots[b]), n % 2, :, :, :x.shape[0]]
            assert torch.equal(got.permute(2, 0, 1, 3), x), (b, n, "open")
            continue
        x = x.permute(1, 2, 0, 3)  # [hkv, 2, P, d]
        want, s = ref.encode(x, codes)
        page = int(table[b, n])
        assert torch.equal(scales[page], s.view(s.shape[:2])), (b, n, "scale")
        assert torch.equal(vals[page], want), (b, n, "codes")
        W = ref.width(c.head_dim)
        raw = c.codes[page]
        if c.head_dim < W:  # columns past the head are 0
            assert (raw[:, 0].view(-1, W // 16, P, 16).transpose(1, 2).reshape(-1, P, W)[..., c.head_dim:] == 0).all()
            assert (raw[:, 1].view(-1, P // 16, W, 16)[:, :, c.head_dim:] == 0).all()
        if c.bounds is not None:
            box, u = ref.bounds(x[:, 0])
            assert torch.equal(c.units[page].double(), u)
            assert torch.equal(c.bounds[page][..., :c.head_dim].double(), box)
            assert (c.bounds[page][..., c.head_dim:] == 0).all()


APPENDS = [
    # hkv, d, page, codes, dtype, rotary, interleaved, lens, new
    (2, 128, 64, "e4m3", BF, 128, False, [0, 0, 63, 64, 5, 127], [64, 65, 1, 1, 0, 300]),
    (2, 64, 64, "i8", BF, 64, True, [0, 1, 62, 60, 100], [1, 62, 2, 5, 28]),
    (1, 32, 32, "i8", F32, 32, False, [0, 31, 0, 17], [31, 1, 97, 15]),
    (3, 72, 32, "e4m3", F32, 48, True, [0, 33, 64, 1], [200, 31, 0, 95]),
    (1, 8, 32, "i8", BF, 2, False, [0, 0, 30], [1, 64, 3]),
    (2, 128, 256, "i8", F32, 128, False, [0, 255, 300], [256, 1, 212]),
    (2, 128, 256, "e4m3", BF, 0, False, [1, 250], [511, 6]),
    (4, 96, 128, "i8", BF, 96, False, [0, 100], [1000, 29]),
    (1, 16, 128, "e4m3", F32, 16, True, [3], [125]),
    # from the middle of one open page to the middle of another at its place
    (2, 64, 32, "e4m3", BF, 64, False, [10, 40, 7], [64, 150, 128]),
]


def _append_case(hkv, d, page, codes, dtype, rotary, interleaved, lens, new, bounds, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ends = [a + b for a, b in zip(lens, new)]
    need = [(e + page - 1) // page for e in ends]
    c = _cache(sum(need) + 2, len(lens) + 2, hkv, d, page, codes, dtype, rotary=rotary, interleaved=interleaved, bounds=bounds)
    table, slots = _tables(c, need, seed), _slots(len(lens), seed)
    tokens = [torch.randn(e, hkv, 2, d, generator=g, device="cuda").to(dtype) for e in ends]
    for b, n in enumerate(lens):  # what the open pages hold already
        first = n // page * page
        c.open[int(slots[b]), n // page % 2, :, :, :n - first] = tokens[b][first:n].permute(1, 2, 0, 3)
    off = ref.offsets(new)
    wide = torch.randn(sum(new), 2 * hkv + 3, d, generator=g, device="cuda").to(dtype)  # column blocks of one projection
    k, v = wide[:, :hkv], wide[:, hkv + 1:2 * hkv + 1]
    for b, n in enumerate(lens):
        k[off[b]:off[b + 1]] = tokens[b][n:, :, 0]
        v[off[b]:off[b + 1]] = tokens[b][n:, :, 1]
    _, kt = c.append(None, None, off, _dev(lens), table, q=k, slots=slots)
    for b, n in enumerate(lens):
        tokens[b][n:, :, 0] = kt[off[b]:off[b + 1]]
    return c, table, slots, tokens, off, k, v


@pytest.mark.parametrize("bounds", [False, True])
@pytest.mark.parametrize("case", APPENDS)
def test_append_writes_exactly_the_codes_of_its_tokens(case, bounds):
    hkv, d, page, codes, dtype, rotary, interleaved, lens, new = case
    c, table, slots, tokens, off, k, v = _append_case(*case, bounds)
    before = c.codes.clone()
    after, none = c.append(k, v, off, _dev(lens), table, slots=slots, validate=True)
    assert none is None and after.tolist() == [a + b for a, b in zip(lens, new)]
    touched = [(b, n) for b, (a, m) in enumerate(zip(lens, new)) if m for n in range(a // page, (a + m - 1) // page + 1)]
    _check_pages(c, table, tokens, after, slots, codes, touched)
    written = {int(table[b, n]) for b, n in touched if (n + 1) * page <= lens[b] + new[b]}
    others = [p for p in range(c.codes.shape[0]) if p not in written]
    assert torch.equal(c.codes[others], before[others])
    # what a read gives
    start = _dev([a // page * page if m else a for a, m in zip(lens, new)])
    count = [e - s for e, s in zip(after.tolist(), start.tolist())]
    for out_type in (dtype, F32, BF):
        gk, gv = c.read(ref.offsets(count), after, table, sum(count), start=start, slots=slots, dtype=out_type, validate=True)
        at = 0
        for b, n in enumerate(count):
            t = tokens[b][start[b]:after[b]]
            for i in range(0, n, page):
                x = t[i:i + page].permute(1, 2, 0, 3)
                if x.shape[2] == page:
                    q, s = ref.encode(x, codes)
                    x = (q.float() * s.float()).to(out_type)
                x = x.permute(1, 2, 0, 3).to(out_type)
                m = x.shape[1]
                assert torch.equal(gk[at + i:at + i + m], x[0]) and torch.equal(gv[at + i:at + i + m], x[1]), (b, i)
            at += n


@pytest.mark.parametrize("dtype,codes,page", [(BF, "i8", 32), (F32, "e4m3", 64)])
def test_the_cache_does_not_depend_on_the_cuts(dtype, codes, page):
    g = torch.Generator(device="cuda").manual_seed(5)
    hkv, d, total = 2, 64, 203
    k, v = (torch.randn(total, hkv, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    caches = []
    for cuts in ([total], [1] * total, [7, 60, 1, 64, 70, 1]):
        c = _cache(total // page + 1, 1, hkv, d, page, codes, dtype, rotary=64, bounds=True)
        table = _tables(c, [total // page + 1])
        lens, at = _dev([0]), 0
        for n in cuts:
            lens, _ = c.append(k[at:at + n], v[at:at + n], _dev([0, n]), lens, table)
            at += n
        assert lens.tolist() == [total]
        caches.append(c)
    pages = table[0, :total // page].long()
    n = total // page
    for c in caches[1:]:
        for name in ("codes", "scales", "bounds", "units"):
            assert torch.equal(getattr(c, name)[pages], getattr(caches[0], name)[pages]), name
        assert torch.equal(c.open[0, n % 2, :, :, :total % page], caches[0].open[0, n % 2, :, :, :total % page])


def test_padded_rows_and_repeated_calls():
    g = torch.Generator(device="cuda").manual_seed(6)
    c = _cache(12, 3, 2, 64, 32, "e4m3", BF, rotary=32)
    c.open.copy_(torch.randn(c.open.shape, generator=g, device="cuda"))  # sequence 2's open page holds 18 tokens
    table = _tables(c, [4, 4, 4])
    k, v = (torch.randn(3, 40, 2, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
    k[0, 33:], v[0, 33:] = math.nan, math.nan  # past the end
    off, lens = _dev([0, 33, 33, 73]), _dev([0, 11, 50])
    for _ in range(2):
        after, _ = c.append(k, v, off, lens, table)
    assert after.tolist() == [33, 11, 90]
    d = _cache(12, 3, 2, 64, 32, "e4m3", BF, rotary=32)
    d.open.copy_(c.open)
    packed = torch.cat([k[0, :33], k[2]]), torch.cat([v[0, :33], v[2]])
    d.append(*packed, off, lens, table)
    for p in (table[0, 0], table[2, 1]):
        assert torch.equal(c.codes[p], d.codes[p]) and torch.equal(c.scales[p], d.scales[p])
    assert torch.equal(c.open[0, 1, :, :, 0], d.open[0, 1, :, :, 0]) and torch.equal(c.open[2, 0, :, :, :26], d.open[2, 0, :, :, :26])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("codes", ["i8", "e4m3"])
def test_extreme_values(codes, dtype):
    """Zeros, the smallest and largest numbers, ties of the codes, infinities and NaN."""
    P, d = 32, 16
    c = _cache(8, 8, 1, d, P, codes, dtype, bounds=True)
    x = torch.zeros(8, P, 1, d, device="cuda")
    x[1] = 2.0 ** -133
    x[2, :, 0] = torch.linspace(-1, 1, d, device="cuda") * 3e38
    x[3, :, 0, :] = torch.arange(d, device="cuda") + 0.5  # ties once the largest is 127
    x[3, 0, 0, 0] = 127.0
    x[4, 3, 0, 2] = math.inf
    x[5, 31, 0, 15] = math.nan
    x[6, :, 0] = 2.0 ** torch.arange(-20, -4, device="cuda").float()  # e4m3's subnormals beside 448
    x[6, 0, 0, 0] = 448.0
    x[7] = -1.0
    x = x.to(dtype)
    k = x.view(8 * P, 1, d)
    off = ref.offsets([P] * 8)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(8, 1)
    c.append(k, k, off, _dev([0] * 8), table)
    for p in (4, 5):
        assert c.scales[p].isnan().all() and (c.codes[p] == 0).all() and c.units[p].isnan().all() and (c.bounds[p] == 0).all()
    tokens = [torch.stack([x[p], x[p]], 2) for p in range(8)]
    good = [0, 1, 2, 3, 6, 7]
    _check_pages(c, table, tokens, None, None, codes, [(p, 0) for p in good])
    gk, _ = c.read(off, _dev([P] * 8), table, 8 * P)
    assert gk.view(8, -1)[4:6].isnan().all() and gk.view(8, -1)[good].isfinite().all()


def test_bad_entries_are_passed_over():
    """Pages and slots outside the cache, lengths past the table: nothing is written for them, they read as 0."""
    g = torch.Generator(device="cuda").manual_seed(8)
    c = _cache(6, 3, 1, 32, 32, "i8", BF)
    table = torch.tensor([[0, -1, 2, 9], [6, 2 ** 31 - 1, -2 ** 31, 9], [3, 4, 5, 9], [1, 1, 1, 9]], dtype=torch.int32, device="cuda")
    slots = torch.tensor([0, 1, 3, -1], dtype=torch.int32, device="cuda")
    k, v = (torch.randn(320, 1, 32, generator=g, device="cuda").bfloat16() for _ in range(2))
    before = c.codes.clone(), c.open.clone()
    off, lens = _dev([0, 100, 200, 300, 320]), _dev([0, 0, 0, 0])
    with pytest.raises(R.RecisError, match="outside the cache|outgrows"):
        c.append(k, v, off, lens, table, slots=slots, validate=True)
    after, _ = c.append(k, v, off, lens, table, slots=slots)
    assert torch.equal(c.codes[1], before[0][1])  # a sequence without a slot and a full page
    gk, gv = c.read(off, after, table, 320, slots=slots)
    assert (gk[32:64] == 0).all() and (gk[100:196] == 0).all() and (gk[296:320] == 0).all()
    assert (gk[96:100] == k[96:100]).all() and (gk[196:200] == k[196:200]).all()
    assert (gk[:32] != 0).any() and (gk[200:296] != 0).any()
    # tokens past the end are 0
    gk, gv = c.read(off, _dev([10, 0, 96, 0]), table, 320, slots=slots)
    assert (gk[10:200] == 0).all() and (gv[296:] == 0).all()


def test_shared_pages_and_slots_are_refused_where_asked():
    c = _cache(4, 3, 1, 32, 32, "i8", BF)
    k = torch.randn(96, 1, 32, device="cuda").bfloat16()
    off, lens = _dev([0, 48, 96]), _dev([0, 0])
    table = torch.tensor([[0, 1], [0, 2]], dtype=torch.int32, device="cuda")
    with pytest.raises(R.RecisError, match="written twice"):
        c.append(k, k, off, lens, table, validate=True)
    table[1, 0] = 3
    with pytest.raises(R.RecisError, match="share a slot"):
        c.append(k, k, off, lens, table, slots=_dev([1, 1], torch.int32), validate=True)
    for bad_off, bad_lens, what in (([0, 60, 50], [0, 0], "nondecreasing|end at"), ([1, 48, 96], [0, 0], "start at 0"),
                                    ([0, 48, 96], [-1, 0], "lens"), ([0, 48, 96], [0, 30], "outgrows"), ([0, 48, 90], [0, 0], "end at")):
        with pytest.raises(R.RecisError, match=what):
            c.append(k, k, _dev(bad_off), _dev(bad_lens), table, validate=True)
    c.append(k, k, off, lens, table, validate=True)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------


def _attend_case(hq, hkv, d, page, codes, dtype, lens, new, causal=True, cap=0.0, slopes=False, padded=0, count=0, seed=0, scale=None,
                 max_q=0, max_len=0, spread=1.0):
    need = [(n + page - 1) // page for n in lens]
    c = _cache(sum(need) + 3, len(lens) + 2, hkv, d, page, codes, dtype, causal=causal, softcap=cap, scale=scale, bounds=count > 0)
    g = ref.fill(c, seed + 1, spread)
    table, slots = _tables(c, need, seed), _slots(len(lens), seed)
    # what no sequence holds may be anything
    unused = [p for p in range(c.codes.shape[0]) if p not in set(table.flatten().tolist())]
    c.scales[unused] = math.nan
    for b, n in enumerate(lens):
        s = int(slots[b])
        c.open[s, n // page % 2, :, :, n % page:] = math.nan
        c.open[s, (n // page + 1) % 2] = math.nan
    if padded:
        q = torch.randn(len(lens), padded, hq, d, generator=g, device="cuda").to(dtype)
        for b, n in enumerate(new):
            q[b, n:] = math.nan
    else:
        q = torch.randn(sum(new), hq + 1, d, generator=g, device="cuda").to(dtype)[:, :hq]
    m = torch.pow(2.0, -1 - 7 * torch.rand(hq, generator=g, device="cuda")) if slopes else None
    off, ln = ref.offsets(new), _dev(lens)
    hold = ref.tokens_of(c, table, lens, slots.tolist())
    at = dict(slots=slots, slopes=m, max_q=max_q, max_len=max_len)
    if count:
        pages = c.select(q, off, ln, table, count, max_q=max_q, max_len=max_len)
        out = c.attend(q, off, ln, table, pages=pages, **at)
    else:
        pages = None
        out = c.attend(q, off, ln, table, validate=True, **at)
    again = c.attend(q, off, ln, table, pages=pages, **at)
    assert torch.equal(out, again)
    sc = scale if scale is not None else d ** -0.5
    for b, n in enumerate(new):
        n = min(n, padded) if padded else n
        rows = out[b, :n] if padded else out[off[b]:off[b + 1]]
        qs = q[b, :n] if padded else q[off[b]:off[b + 1]]
        if padded:
            assert (out[b, n:] == 0).all()
        k, v, there = hold[b]
        pos = torch.arange(n, device="cuda") + lens[b] - n
        key_pos = torch.arange(k.shape[0], device="cuda")
        if not count:
            want, bound = ref.attention(qs, k, v, pos, key_pos, there.long(), causal, cap, m, sc, dtype == BF, hq // hkv)
            _close(rows, want, bound, dtype)
            continue
        closed = lens[b] // page * page
        for i in range(n):
            lists = pages[b, i] if padded else pages[off[b] + i]
            picked = ref.select(qs[i], c, table[b].tolist(), lens[b], int(pos[i]), count, causal)
            for h in range(hkv):
                assert [x for x in lists[h].tolist() if x >= 0] == picked[h], (b, i, h)
                w = torch.zeros_like(key_pos)
                w[closed:] = 1
                for x in picked[h]:
                    w[x * page:(x + 1) * page] += 1
                G = hq // hkv
                want, bound = ref.attention(qs[i:i + 1, h * G:(h + 1) * G], k[:, h:h + 1], v[:, h:h + 1], pos[i:i + 1], key_pos, w, causal, cap,
                                            None if m is None else m[h * G:(h + 1) * G], sc, dtype == BF, G)
                _close(rows[i:i + 1, h * G:(h + 1) * G], want, bound, dtype)


def _close(got, want, bound, dtype):
    lim = bound + _half(dtype) * (want.abs() + bound) + 1e-30
    err = (got.double() - want).abs()
    assert (err <= lim).all(), f"worst {float((err / lim).max()):.3g} of the bound"


LENS = [0, 1, 31, 32, 33, 64, 65, 127, 200, 511, 513]


@pytest.mark.parametrize("dtype,codes", [(BF, "e4m3"), (BF, "i8"), (F32, "e4m3"), (F32, "i8")])
@pytest.mark.parametrize("hq,hkv,d,page,causal", [(8, 2, 128, 64, True), (4, 4, 64, 32, False), (6, 2, 72, 128, True), (3, 1, 16, 256, True),
                                                  (1, 1, 32, 32, True), (40, 1, 8, 64, False), (2, 2, 96, 64, True)])
def test_single_tokens(dtype, codes, hq, hkv, d, page, causal):
    _attend_case(hq, hkv, d, page, codes, dtype, LENS, [1] * len(LENS), causal)
    _attend_case(hq, hkv, d, page, codes, dtype, LENS, [1] * len(LENS), causal, max_q=1, max_len=513, seed=3)


@pytest.mark.parametrize("dtype,codes", [(BF, "e4m3"), (F32, "i8")])
@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 128, 64), (5, 5, 64, 32), (6, 1, 40, 128), (36, 1, 32, 32)])
@pytest.mark.parametrize("causal,cap,slopes", [(True, 0.0, False), (True, 5.0, True), (False, 30.0, False), (False, 0.0, True)])
def test_chunks_of_queries(dtype, codes, hq, hkv, d, page, causal, cap, slopes):
    # more queries than keys among them: rows that see nothing
    _attend_case(hq, hkv, d, page, codes, dtype, [0, 3, 100, 64, 500, 129, 1], [2, 9, 17, 64, 0, 130, 3], causal, cap, slopes, seed=1)


@pytest.mark.parametrize("dtype,codes", [(BF, "i8"), (F32, "e4m3")])
@pytest.mark.parametrize("new,max_q", [([3, 0, 5, 1], 0), ([40, 7, 33, 0], 0), ([40, 7, 33, 0], 2)])
def test_bounds_of_the_sizes_only_shape_the_launches(dtype, codes, new, max_q):
    for max_len in (0, 70):
        _attend_case(8, 2, 64, 64, codes, dtype, [900, 64, 3000, 1], new, True, 0.0, True, max_q=max_q, max_len=max_len, seed=2)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("count", [0, 3])
def test_padded_queries(dtype, count):
    _attend_case(4, 2, 64, 32, "i8", dtype, [40, 0, 300, 77], [5, 3, 0, 7], True, padded=6, count=count, seed=4)
    _attend_case(4, 2, 64, 32, "i8", dtype, [40, 5000, 300, 77], [2, 1, 2, 1], False, padded=2, count=count, seed=5)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_long_history_splits_and_joins(dtype):
    _attend_case(8, 2, 128, 64, "e4m3", dtype, [70001], [4], False, seed=6)
    _attend_case(2, 1, 64, 256, "i8", dtype, [50000, 100, 30017], [1, 1, 2], True, 0.0, True, seed=7, max_q=2, max_len=50000)
    _attend_case(2, 1, 32, 32, "i8", dtype, [20000], [300], True, seed=8)


def test_large_scores_and_small_scales():
    _attend_case(4, 1, 64, 64, "i8", BF, [700], [3], False, scale=20.0, seed=9, spread=3.0)
    _attend_case(4, 1, 64, 64, "e4m3", F32, [700], [3], True, scale=1e-6, seed=9)


@pytest.mark.parametrize("dtype,codes", [(BF, "e4m3"), (F32, "i8")])
@pytest.mark.parametrize("hq,hkv,d,page,count,causal", [(8, 2, 128, 64, 4, True), (4, 4, 64, 32, 1, False), (40, 1, 32, 32, 7, True),
                                                        (6, 3, 24, 128, 300, True), (2, 1, 72, 256, 2, False)])
def test_chosen_pages(dtype, codes, hq, hkv, d, page, count, causal):
    _attend_case(hq, hkv, d, page, codes, dtype, [0, 5, page, 10 * page + 3, 33 * page, 300], [1, 2, 3, 4, 1, 0], causal, 0.0, True,
                 count=count, seed=10)
    _attend_case(hq, hkv, d, page, codes, dtype, [9 * page + 1], [6], causal, 20.0, count=count, seed=11, max_q=6, max_len=page)


def test_lists_with_gaps_and_repeats():
    """-1, numbers past the full pages and pages outside the cache are passed over; a page named twice counts twice."""
    c = _cache(8, 1, 1, 64, 32, "e4m3", BF, causal=False)
    g = ref.fill(c, 1)
    table = torch.tensor([[5, 2, 99, 0, 7]], dtype=torch.int32, device="cuda")
    n = 4 * 32 + 9
    q = torch.randn(2, 4, 64, generator=g, device="cuda").bfloat16()
    pages = torch.tensor([[[3, -1, 0, 3, 2]], [[4, 9, -5, 2 ** 31 - 1, 2]]], dtype=torch.int32, device="cuda")
    out = c.attend(q, _dev([0, 2]), _dev([n]), table, pages=pages)
    k, v, there = ref.tokens_of(c, table, [n], [0])[0]
    pos = torch.arange(2, device="cuda") + n - 2
    for i, picks in enumerate(([3, 0, 3], [])):
        w = torch.zeros(n, dtype=torch.int64, device="cuda")
        w[128:] = 1
        for p in picks:
            w[p * 32:(p + 1) * 32] += 1
        want, bound = ref.attention(q[i:i + 1], k, v, pos[i:i + 1], torch.arange(n, device="cuda"), w, False, 0.0, None, 0.125, True, 4)
        _close(out[i:i + 1], want, bound, BF)
    # nothing at all: no page of the list and no open token
    out = c.attend(q, _dev([0, 2]), _dev([128]), table, pages=torch.full_like(pages, -1))
    assert (out == 0).all()


def test_missing_pages_are_not_seen():
    c = _cache(8, 2, 2, 64, 32, "i8", F32, causal=True)
    g = ref.fill(c, 2)
    table = torch.tensor([[5, -1, 99, 0, 7], [8, 8, 8, 8, 8]], dtype=torch.int32, device="cuda")
    lens, new, slots = [140, 96], [3, 2], [0, 5]
    q = torch.randn(5, 4, 64, generator=g, device="cuda")
    out = c.attend(q, ref.offsets(new), _dev(lens), table, slots=_dev(slots, torch.int32))
    hold = ref.tokens_of(c, table, lens, slots)
    k, v, there = hold[0]
    want, bound = ref.attention(q[:3], k, v, torch.arange(137, 140, device="cuda"), torch.arange(140, device="cuda"), there.long(), True, 0.0, None,
                                0.125, False, 2)
    _close(out[:3], want, bound, F32)
    assert (out[3:] == 0).all()
    # longer than its table: cut to it
    long = c.attend(q, ref.offsets(new), _dev([10 ** 12, 96]), table, slots=_dev(slots, torch.int32))
    assert long.isfinite().all()


def test_ties_go_to_the_lower_page():
    c = _cache(700, 1, 1, 32, 32, "i8", BF, bounds=True, causal=False)
    ref.fill(c, 3)
    c.bounds.copy_(c.bounds[:7].repeat(100, 1, 1, 1))
    c.units.fill_(0.5)
    table = torch.arange(700, dtype=torch.int32, device="cuda").view(1, 700)
    q = torch.randn(3, 2, 32, device="cuda").bfloat16()
    q[1] = 0  # every page alike
    q[2, 0, 3] = math.nan
    q[2, 1] = math.inf
    got = c.select(q, _dev([0, 3]), _dev([700 * 32]), table, 150)
    for i in range(3):
        assert got[i, 0].tolist() == ref.select(q[i], c, list(range(700)), 700 * 32, 0, 150, False)[0]
    assert got[1, 0].tolist() == list(range(150)) == got[2, 0].tolist()
    # a page that is not finite comes first, one that is not there last
    c.units[[13, 600]] = math.nan
    table[0, :20] = -1
    got = c.select(q[:1], _dev([0, 1]), _dev([700 * 32]), table, 690)[0, 0].tolist()
    assert got == ref.select(q[0], c, table[0].tolist(), 700 * 32, 0, 690, False)[0]
    assert 600 in got and got[:10] == list(range(10)) and got[10] == 20


@pytest.mark.parametrize("width", [300, 1024, 1025, 16384, 20000, 65537])
@pytest.mark.parametrize("distinct", [200, 3])
def test_many_pages_are_chosen_exactly(width, distinct):
    """Every way of picking; few distinct pages make nearly every score a tie."""
    c = _cache(distinct, 1, 2, 64, 32, "i8", F32, bounds=True, causal=False)
    g = ref.fill(c, 4)
    table = torch.randint(0, distinct, (1, width), generator=g, device="cuda").to(torch.int32)
    q = torch.randn(2, 6, 64, generator=g, device="cuda")
    for count, max_len in ((1, 0), (64, 0), (width // 4, 1000), (width - 1, 0)):
        got = c.select(q, _dev([0, 2]), _dev([width * 32]), table, count, max_len=max_len)
        for i in range(2):
            assert got[i].tolist() == ref.select(q[i], c, table[0].tolist(), width * 32, 0, count, False)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (5, 1), (8, 1), (18, 2), (40, 1), (12, 3)])
@pytest.mark.parametrize("d,dtype", [(128, BF), (40, F32), (16, BF)])
def test_groups_of_heads_choose_together(hq, hkv, d, dtype):
    """Runs of rows over several sequences, under the causal mask, with rows that see few pages."""
    c = _cache(150, 9, hkv, d, 32, "e4m3", dtype, bounds=True)
    g = ref.fill(c, 6)
    lens, new = [32 * 40 + 5, 3, 32 * 30, 700, 0], [37, 2, 1, 19, 1]
    table = torch.randint(0, 150, (5, 41), generator=g, device="cuda").to(torch.int32)
    q = torch.randn(sum(new), hq, d, generator=g, device="cuda").to(dtype)
    off = ref.offsets(new)
    got = c.select(q, off, _dev(lens), table, 21)
    for b, n in enumerate(new):
        for i in range(n):
            want = ref.select(q[off[b] + i], c, table[b].tolist(), lens[b], lens[b] - n + i, 21, True)
            assert [[x for x in h if x >= 0] for h in got[off[b] + i].tolist()] == want, (b, i)


# ---------------------------------------------------------------------------
# the whole path, streams, graphs, sizes
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("width", [900, 3000])
def test_counts_around_the_threads_of_a_block(width):
    """The range of scores starts at the least of as many groups' largest: counts at and beside powers of two."""
    c = _cache(width, 1, 1, 32, 32, "e4m3", BF, bounds=True, causal=False)
    g = ref.fill(c, 9)
    table = torch.randperm(width, generator=g, device="cuda").to(torch.int32)[None]
    table[0, ::7] = -1  # pages that are not there come last
    q = torch.randn(1, 3, 32, generator=g, device="cuda").bfloat16()
    for count in (1, 2, 3, 4, 5, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 770, 800, 899, 1023, 1024, 1025,
                  2047, 2572, 2999):
        if count < width:
            got = c.select(q, _dev([0, 1]), _dev([width * 32]), table, count)
            assert got[0].tolist() == ref.select(q[0], c, table[0].tolist(), width * 32, 0, count, False), count


@pytest.mark.parametrize("hq,hkv", [(100, 1), (260, 2)])
@pytest.mark.parametrize("d,dtype", [(64, BF), (24, F32)])
def test_many_heads_of_one_key_head(hq, hkv, d, dtype):
    """More heads of a key head than a block holds at once: the choice and both attentions."""
    test_groups_of_heads_choose_together(hq, hkv, d, dtype)
    _attend_case(hq, hkv, d, 32, "i8", dtype, [300, 0, 70], [2, 1, 3], count=3, seed=21)
    _attend_case(hq, hkv, d, 32, "e4m3", dtype, [300, 0, 70], [2, 1, 3], cap=7.0, slopes=True, seed=22)


def test_a_served_history_against_seq_attention():
    """Histories written, read back and attended: the same as SeqAttention over the tokens read, to both sides' roundings."""
    g = torch.Generator(device="cuda").manual_seed(12)
    hq, hkv, d, lens, new = 8, 2, 64, [300, 0, 64, 1000], [5, 3, 64, 1]
    c = _cache(60, 4, hkv, d, 64, "i8", F32, rotary=64, bounds=True)
    table = _tables(c, [8, 8, 8, 20], width=20)
    zero = _dev([0] * 4)

    def tokens(n):
        y = torch.randn(sum(n), hq + 2 * hkv, d, generator=g, device="cuda")
        return y.split([hq, hkv, hkv], 1)

    q, k, v = tokens(lens)
    held, _ = c.append(k, v, ref.offsets(lens), zero, table, q=q, validate=True)
    q, k, v = tokens(new)
    held, turned = c.append(k, v, ref.offsets(new), held, table, q=q, validate=True)
    total = [a + b for a, b in zip(lens, new)]
    assert held.tolist() == total
    rk, rv = c.read(ref.offsets(total), held, table, validate=True)
    look = R.SeqAttention(causal=True)
    want, _ = look.forward(turned, rk, rv, ref.offsets(new), kv_offsets=ref.offsets(total))
    got = c.attend(turned, ref.offsets(new), held, table, validate=True)
    # fp32 on both sides: (6 d + 16) u and (d + 8) u of sum |q| |k| / 8, 10 at most here, twice in a probability: 6e-4 of sum P |v|,
    # which is below 2
    assert (got - want).abs().max() <= 1.2e-3
    # every page chosen: the same again
    pages = c.select(turned, ref.offsets(new), held, table, 16, validate=True)
    again = c.attend(turned, ref.offsets(new), held, table, pages=pages, validate=True)
    assert (again - got).abs().max() <= 1.2e-3


def test_candidates_are_turned_but_not_kept():
    c = _cache(4, 1, 1, 32, 32, "e4m3", BF, rotary=32)
    table = torch.tensor([[2, 1]], dtype=torch.int32, device="cuda")
    k = torch.randn(40, 1, 32, device="cuda").bfloat16()
    held, _ = c.append(k, k, _dev([0, 40]), _dev([0]), table)
    kept = c.codes.clone(), c.open.clone()
    q = torch.randn(5, 2, 32, device="cuda").bfloat16()
    _, turned = c.append(None, None, _dev([0, 5]), held, table, q=q)
    assert torch.equal(kept[0], c.codes) and torch.equal(kept[1].nan_to_num(), c.open.nan_to_num())
    assert turned.shape == q.shape and not torch.equal(turned, q)


def test_captured_steps_replay():
    """append, select and attend in one graph, replayed on changed inputs, beside eager calls of the same object."""
    g = torch.Generator(device="cuda").manual_seed(13)
    hq, hkv, d, seqs = 4, 2, 64, 5
    c = _cache(400, seqs, hkv, d, 32, "i8", BF, rotary=64, bounds=True)
    table = _tables(c, [80] * seqs)
    off, one = ref.offsets([1] * seqs), _dev([0, 1])
    lens0 = [700, 31, 0, 2000, 64]
    y = torch.randn(sum(lens0), 2 * hkv, d, generator=g, device="cuda").bfloat16()
    lens, _ = c.append(y[:, :hkv], y[:, hkv:], ref.offsets(lens0), _dev([0] * seqs), table)
    rows = torch.randn(seqs, hq + 2 * hkv, d, generator=g, device="cuda").bfloat16()

    def step():
        q, k, v = rows.split([hq, hkv, hkv], 1)
        after, turned = c.append(k, v, off, lens, table, q=q)
        pages = c.select(turned, off, after, table, 4)
        return after, pages, c.attend(turned, off, after, table, pages=pages), c.attend(turned, off, after, table, max_q=1)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for i in range(3):
        rows.copy_(torch.randn(rows.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in kept]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
        # a larger call takes a larger workspace; the graph keeps its own
        big = torch.randn(40, hq, d, generator=g, device="cuda").bfloat16()
        c.attend(big, _dev([0, 40]), lens[3:4], table[3:4], slots=_dev([3], torch.int32))


def test_another_stream():
    c = _cache(40, 1, 2, 64, 64, "e4m3", BF, causal=False)
    g = ref.fill(c, 5)
    table = _tables(c, [40])
    q = torch.randn(3, 4, 64, generator=g, device="cuda").bfloat16()
    args = (q, _dev([0, 3]), _dev([2500]), table)
    want = c.attend(*args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = c.attend(*args)
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype,codes", [(BF, "e4m3"), (F32, "i8")])
@pytest.mark.parametrize("new", [[0, 4, 0, 3, 0], [1, 1, 0, 1, 1], [0, 0, 40, 33, 0]])
def test_rows_outside_the_sequences_are_left_as_they_were(dtype, codes, new):
    """Rows before the first and behind the last sequence: untouched, and the others as without them."""
    lens = [700, 2000, 64, 1300, 5]
    c = _cache(150, 5, 2, 64, 32, codes, dtype, causal=True, bounds=True)
    g = ref.fill(c, 4)
    table = _tables(c, [(n + 31) // 32 for n in lens])
    n = sum(new)
    wide = torch.full((n + 13, 6, 64), math.nan, device="cuda", dtype=dtype)
    wide[6:6 + n] = torch.randn(n, 6, 64, generator=g, device="cuda").to(dtype)
    off, ln = ref.offsets(new), _dev(lens)
    pages = c.select(wide[6:6 + n], off, ln, table, 5)
    listed = torch.zeros(n + 13, 2, 5, dtype=torch.int32, device="cuda")
    listed[6:6 + n] = pages
    assert torch.equal(c.select(wide, off + 6, ln, table, 5)[6:6 + n], pages)
    for few, many in ((None, None), (pages, listed)):
        out = torch.full_like(wide, 7.0)
        c.attend(wide, off + 6, ln, table, pages=many, out=out)
        assert (out[:6] == 7).all() and (out[6 + n:] == 7).all()
        for b, (k, v, there) in enumerate(ref.tokens_of(c, table, lens, range(5))):
            pos, key_pos = torch.arange(new[b], device="cuda") + lens[b] - new[b], torch.arange(lens[b], device="cuda")
            for i in range(new[b]):
                at = 6 + int(off[b]) + i
                for h in range(2):
                    w = there.long()
                    if few is not None:
                        w = (key_pos >= lens[b] // 32 * 32).long()
                        for x in pages[at - 6, h].tolist():
                            w[x * 32:(x + 1) * 32] += int(x >= 0)
                    want, bound = ref.attention(wide[at:at + 1, 3 * h:3 * h + 3], k[:, h:h + 1], v[:, h:h + 1], pos[i:i + 1], key_pos, w,
                                                True, 0.0, None, 0.125, dtype == BF, 3)
                    _close(out[at:at + 1, 3 * h:3 * h + 3], want, bound, dtype)


def test_an_output_over_the_queries_is_refused():
    c = _cache(2, 1, 1, 32, 32, "i8", BF)
    ref.fill(c, 7)
    table, off, lens = torch.zeros(1, 2, dtype=torch.int32, device="cuda"), _dev([0, 4]), _dev([40])
    both = torch.randn(4, 4, 32, device="cuda").bfloat16()
    for q, out in ((both, both), (both[:, :2], both.view(8, 2, 32)[4:]), (both.view(8, 2, 32)[:4], both.view(8, 2, 32)[3:7])):
        with pytest.raises(R.RecisError, match="overlap"):
            c.attend(q, off, lens, table, out=out)
    halves = both.view(8, 2, 32)
    want = c.attend(halves[:4].clone(), off, lens, table)
    assert torch.equal(c.attend(halves[:4], off, lens, table, out=halves[4:]), want)


def test_more_rows_than_a_launch_takes():
    """70,001 rows of one sequence and 70,000 sequences of one row each: as in parts."""
    rows = 70001
    c = _cache(12, 70000, 1, 16, 32, "i8", BF, causal=False, bounds=True)
    g = ref.fill(c, 5)
    q = torch.randn(rows, 1, 16, generator=g, device="cuda").bfloat16()
    table, lens = torch.arange(12, dtype=torch.int32, device="cuda")[None], _dev([12 * 32])
    pages = c.select(q, _dev([0, rows]), lens, table, 3)
    out = c.attend(q, _dev([0, rows]), lens, table, pages=pages)
    for a, b in ((0, 40000), (40000, rows)):
        some = c.select(q[a:b], _dev([0, b - a]), lens, table, 3)
        assert torch.equal(some, pages[a:b])
        assert torch.equal(c.attend(q[a:b], _dev([0, b - a]), lens, table, pages=some), out[a:b])
    seqs = 70000
    off, each, tables = torch.arange(seqs + 1, device="cuda"), lens.expand(seqs).contiguous(), table.expand(seqs, 12).contiguous()
    assert torch.equal(c.select(q[:seqs], off, each, tables, 3), pages[:seqs])
    assert torch.equal(c.attend(q[:seqs], off, each, tables, pages=pages[:seqs]), out[:seqs])


def test_empty_calls():
    c = _cache(2, 2, 1, 32, 32, "i8", BF, rotary=32, bounds=True)
    none = torch.zeros(0, 1, 32, dtype=BF, device="cuda")
    table = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    off, lens = _dev([0, 0, 0]), _dev([3, 0])
    after, q = c.append(none, none, off, lens, table, q=none)
    assert after.tolist() == [3, 0] and q.numel() == 0
    assert c.attend(none, off, lens, table).numel() == 0
    assert c.select(none, off, lens, table, 2).shape == (0, 1, 2)
    k, v = c.read(off, lens, table)
    assert k.numel() == 0
    no_seq = _dev([0]), torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, 4, dtype=torch.int32, device="cuda")
    assert c.append(none, none, *no_seq)[0].numel() == 0
    # no table at all: a sequence of its open page
    narrow = torch.zeros(1, 0, dtype=torch.int32, device="cuda")
    q = torch.randn(1, 2, 32, device="cuda").bfloat16()
    assert (c.attend(q, _dev([0, 1]), _dev([0]), narrow) == 0).all()
    assert (c.select(q, _dev([0, 1]), _dev([0]), narrow, 3) == -1).all()


def test_pages_past_2_to_32_bytes():
    """A cache of 4.9 GiB: the first and the last pages, written, read and attended."""
    c = R.SeqCache(80000, 2, 4, 128, page=64, codes="e4m3", bounds=True)
    assert c.codes.numel() > 1 << 32
    table = torch.tensor([[79999, 0, 79998], [70001, 70000, 3]], dtype=torch.int32, device="cuda")
    small = R.SeqCache(6, 2, 4, 128, page=64, codes="e4m3", bounds=True)
    small_table = torch.tensor([[0, 1, 2], [3, 4, 5]], dtype=torch.int32, device="cuda")
    k, v = (torch.randn(380, 4, 128, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(2, 8, 128, device="cuda").bfloat16()
    off, lens, one = _dev([0, 190, 380]), _dev([0, 0]), _dev([0, 1, 2])
    got = []
    for x, t in ((c, table), (small, small_table)):
        held, _ = x.append(k, v, off, lens, t)
        pages = x.select(q, one, held, t, 1)
        got.append((*x.read(off, held, t, 380), x.attend(q, one, held, t), pages, x.attend(q, one, held, t, pages=pages)))
    for a, b in zip(*got):
        assert torch.equal(a, b)
