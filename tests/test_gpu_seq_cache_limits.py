"""The paged cache at its limits: entries outside it, turning alone, extreme magnitudes, large pages, tiles of padded rows.

References and their error bounds: cache_reference."""
import math

import pytest
import torch

from paper_2509_20883_amd import recis as R
from tests import cache_reference as ref
from tests import test_gpu_seq_cache as base

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
_dev, _cache, _close = base._dev, base._cache, base._close


# ---------------------------------------------------------------------------
# slots outside the cache
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("slot", [-1, 2])
@pytest.mark.parametrize("dtype,codes", [(BF, "i8"), (BF, "e4m3"), (F32, "i8"), (F32, "e4m3")])
def test_a_page_whose_first_tokens_had_no_slot_is_passed_over(dtype, codes, slot):
    """Tokens that came for a slot outside the cache are gone when their page fills: the page then stands for nothing, whatever it
    held before.  Its later pages, coded from one call's tokens, are there."""
    P, hq, hkv, d = 32, 4, 2, 64
    c = _cache(8, 2, hkv, d, P, codes, dtype, bounds=True, causal=False)
    g = ref.fill(c, 31)  # of another user
    table = torch.tensor([[4, 2, 5, 0], [1, 3, 6, 7]], dtype=torch.int32, device="cuda")
    slots = torch.tensor([slot, 1], dtype=torch.int32, device="cuda")
    slot_list = [slot, 1]
    k, v = (torch.randn(300, hkv, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    lens, at = _dev([0, 0]), 0
    # pages of the first sequence that are lost after each call: 0 (20 of its tokens), 1 (8 of them)
    for new, lost in ((20, [0]), (20, [0]), (56, [0, 1]), (30, [0, 1, 3])):
        off = _dev([0, new, 2 * new])
        lens, _ = c.append(k[at:at + 2 * new], v[at:at + 2 * new], off, lens, table, slots=slots)
        at += 2 * new
        total = lens.tolist()
        hold = ref.tokens_of(c, table, total, slot_list)
        for p in lost:
            hold[0][2][p * P:(p + 1) * P] = False
        gk, gv = c.read(_dev([0, total[0], 2 * total[0]]), lens, table, 2 * total[0], slots=slots, dtype=F32)
        for b in range(2):
            there = hold[b][2][:, None, None]
            for got, want in ((gk, hold[b][0]), (gv, hold[b][1])):
                assert torch.equal(got[b * total[0]:(b + 1) * total[0]], torch.where(there, want, 0.0).float()), (b, total)
        for rows in (1, 40):  # both kinds of tiles
            q = torch.randn(2 * rows, hq, d, generator=g, device="cuda").to(dtype)
            off = _dev([0, rows, 2 * rows])
            out = c.attend(q, off, lens, table, slots=slots)
            key_pos = torch.arange(total[0], device="cuda")
            for b in range(2):
                pos = torch.arange(rows, device="cuda") + total[b] - rows
                want, bound = ref.attention(q[b * rows:(b + 1) * rows], *hold[b][:2], pos, key_pos, hold[b][2].long(), False, 0.0, None,
                                            d ** -0.5, dtype == BF, hq // hkv)
                _close(out[b * rows:(b + 1) * rows], want, bound, dtype)
            n = total[0] // P
            if n:
                picks = c.select(q, off, lens, table, 1)[:rows]
                seen = [p for p in range(n) if p not in lost]
                assert (picks == 0).all() if not seen else all(x in seen for x in picks.flatten().tolist())
                listed = torch.arange(n, dtype=torch.int32, device="cuda").expand(2 * rows, hkv, n).contiguous()
                again = c.attend(q, off, lens, table, pages=listed, slots=slots)
                for b in range(2):
                    pos = torch.arange(rows, device="cuda") + total[b] - rows
                    want, bound = ref.attention(q[b * rows:(b + 1) * rows], *hold[b][:2], pos, key_pos, hold[b][2].long(), False, 0.0, None,
                                                d ** -0.5, dtype == BF, hq // hkv)
                    _close(again[b * rows:(b + 1) * rows], want, bound, dtype)
    # written again from its slot, the page is there again
    c.append(k[:32], v[:32], _dev([0, 32]), _dev([0]), table[:1], slots=_dev([0], torch.int32))
    gk, _ = c.read(_dev([0, 32]), _dev([32]), table[:1], 32, slots=_dev([0], torch.int32))
    assert (gk != 0).any()


# ---------------------------------------------------------------------------
# pages at 64 KiB of LDS
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("case", [
    # 64 KiB with the block's own LDS, and just below: rows of 120 columns lie 256 (bf16) and 496 bytes apart
    (1, 120, 256, "e4m3", BF, 120, False, [0, 255, 100], [256, 1, 413]),
    (2, 120, 128, "i8", F32, 48, True, [0, 127, 3], [128, 1, 300]),
    (1, 112, 256, "i8", BF, 112, True, [5], [520]),
    (1, 112, 128, "e4m3", F32, 0, False, [5], [260]),
], ids=str)
@pytest.mark.parametrize("bounds", [False, True])
def test_append_of_pages_that_fill_64_kib(case, bounds):
    base.test_append_writes_exactly_the_codes_of_its_tokens(case, bounds)


# ---------------------------------------------------------------------------
# turning alone
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("padded", [False, True])
def test_turning_alone_needs_neither_slots_nor_pages(padded):
    """Queries that are turned and not kept: more sequences than slots, tables that name no page, lengths past them."""
    g = torch.Generator(device="cuda").manual_seed(41)
    c = R.SeqCache(1, 2, 1, 32, page=32, dtype=F32, rotary=32)
    held, new = [5, 0, 10 ** 6, 33, 70], [2, 3, 1, 0, 3]
    off, lens = ref.offsets(new), _dev(held)
    table = torch.full((5, 1), 2 ** 30, dtype=torch.int32, device="cuda")
    q = torch.randn(5, 3, 2, 32, generator=g, device="cuda") if padded else torch.randn(sum(new), 2, 32, generator=g, device="cuda")
    after, out = c.append(None, None, off, lens, table, q=q, validate=True)
    assert after.tolist() == [a + b for a, b in zip(held, new)]
    freqs = [10000.0 ** (-2.0 * i / 32) for i in range(16)]
    for b, n in enumerate(new):
        rows, got = (q[b, :n], out[b, :n]) if padded else (q[off[b]:off[b + 1]], out[off[b]:off[b + 1]])
        pos = held[b] + torch.arange(n, device="cuda")
        want = ref.turned(rows, pos, freqs, 32, False)
        # the reference's frequencies are off by 2^-53 of themselves
        slack = 8 * (2.0 ** -31 + (held[b] + n) * 2.0 ** -53)
        assert bool(((got.double() - want).abs() <= ref.U * (want.abs() + slack) + slack).all()), b
    for bad_off, bad_lens in (([0, 4, 3, 6, 6, 9], held), ([1, 2, 5, 6, 6, 9], held), (off.tolist(), [5, -1, 0, 0, 0])):
        with pytest.raises(R.RecisError):
            c.append(None, None, _dev(bad_off), _dev(bad_lens), table, q=q, validate=True)
    with pytest.raises(R.RecisError):  # and as without queries alone
        c.append(q[..., :1, :].contiguous(), q[..., :1, :].contiguous(), off, lens, table, q=q)


# ---------------------------------------------------------------------------
# more rows than the workspace holds scores of
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("new", [[1] * 1200, [3, 0, 700, 1, 1, 40, 300, 2]])
def test_rows_that_take_several_windows_of_scores(new, padded):
    """Tables so wide that 256 MiB hold the scores of 536 rows: as in parts, and as the formula for some rows."""
    hkv, width, count, P, d = 8, 15625, 9, 32, 32
    c = _cache(60, 1, hkv, d, P, "i8", BF, bounds=True)
    g = ref.fill(c, 51)
    if padded:
        pad, new = max(new[0], 150), [min(n, max(new[0], 150)) for n in new[:8]]
    seqs = len(new)
    table = torch.randint(0, 60, (seqs, width), generator=g, device="cuda").to(torch.int32)
    lens = torch.randint(500, width * P, (seqs,), generator=g, device="cuda")
    lens[0] = width * P
    off = ref.offsets(new)
    q = torch.randn(*((seqs, pad) if padded else (sum(new),)), hkv, d, generator=g, device="cuda").bfloat16()
    got = c.select(q, off, lens, table, count)
    if padded:
        assert seqs * pad > 536 * 2
        for b, n in enumerate(new):
            assert (got[b, n:] == -1).all()
            assert torch.equal(got[b, :n], c.select(q[b, :n], _dev([0, n]), lens[b:b + 1], table[b:b + 1], count))
        return
    assert sum(new) > 536
    for a in range(0, seqs, 2 if seqs < 100 else 300):
        b = min(seqs, a + (2 if seqs < 100 else 300))
        rows = slice(int(off[a]), int(off[b]))
        assert torch.equal(got[rows], c.select(q[rows], off[a:b + 1] - off[a], lens[a:b], table[a:b], count))
    last = int(off[-1]) - 1
    want = ref.select(q[last], c, table[-1].tolist(), int(lens[-1]), int(lens[-1]) - 1, count, True)
    assert got[last].tolist() == want


# ---------------------------------------------------------------------------
# scores and values at the ends of their types' ranges
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("q_by,unit_by", [(2.0 ** -120, 2.0 ** -100), (2.0 ** -40, 2.0 ** -126), (2.0 ** 120, 2.0 ** 100), (2.0 ** 110, 1.0)])
def test_scores_outside_fp32_choose_exactly(dtype, q_by, unit_by):
    """Whole numbers times powers of two: the choice is exact where the scores pass fp32's range, too, and between heads far apart."""
    c = _cache(200, 1, 1, 128, 32, "i8", dtype, bounds=True, causal=False)
    g = ref.fill(c, 61)
    c.units.copy_(unit_by * 2.0 ** torch.randint(0, 4, c.units.shape, generator=g, device="cuda"))
    q = torch.randn(6, 5, 128, generator=g, device="cuda") * q_by
    q[1, 1:] = 0
    q[2, 0] = torch.randn(128, generator=g, device="cuda")
    q[3] *= torch.tensor([1.0, 2.0 ** -2, 0.0, 2.0 ** -5, 1.0], device="cuda")[:, None]
    q[4] = -q[4].abs()
    q = q.to(dtype)
    table = torch.randperm(200, generator=g, device="cuda").to(torch.int32)[None]
    got = c.select(q, _dev([0, 6]), _dev([200 * 32]), table, 17)
    for i in range(6):
        assert got[i].tolist() == ref.select(q[i], c, table[0].tolist(), 200 * 32, 0, 17, False), i


@pytest.mark.parametrize("rows", [1, 70])
def test_fp32_values_past_the_largest_bf16_number(rows):
    """fp32 numbers above bf16's largest are numbers, in queries, keys and values of an open page."""
    d, n = 64, 9
    c = _cache(1, 1, 1, d, 32, "i8", F32, causal=False)
    g = torch.Generator(device="cuda").manual_seed(62)
    top = 3.4e38
    assert torch.tensor(top).bfloat16().isinf()
    c.open[0, 0, 0, :, :n] = torch.randn(2, n, d, generator=g, device="cuda")
    c.open[0, 0, 0, 0, :n, 0] = torch.linspace(-3, 3, n, device="cuda").bfloat16().float() * 2.0 ** -125  # times 3.4e38: -240 to 240
    c.open[0, 0, 0, 0, 2, 0] = 0
    c.open[0, 0, 0, 1, 3, 5] = top
    c.open[0, 0, 0, 1, 4, 6] = -top
    q = torch.randn(rows, 2, d, generator=g, device="cuda")
    q[0, 0, 0], q[-1, 1, 0] = top, -top
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), _dev([n])
    k, v, there = ref.tokens_of(c, table, [n], [0])[0]
    out = c.attend(q, _dev([0, rows]), lens, table)
    pos = torch.arange(rows, device="cuda") + n - rows
    want, bound = ref.attention(q, k, v, pos, torch.arange(n, device="cuda"), there.long(), False, 0.0, None, d ** -0.5, False, 2)
    _close(out, want, bound, F32)
    # a key of its own, past bf16's largest
    c.open[0, 0, 0, 0, 1, 7] = top
    q[:, :, 7] = torch.randn(rows, 2, generator=g, device="cuda").sign() * 2.0 ** -126
    k, v, there = ref.tokens_of(c, table, [n], [0])[0]
    out = c.attend(q, _dev([0, rows]), lens, table)
    want, bound = ref.attention(q, k, v, pos, torch.arange(n, device="cuda"), there.long(), False, 0.0, None, d ** -0.5, False, 2)
    _close(out, want, bound, F32)


# ---------------------------------------------------------------------------
# padded rows in every tile, and more blocks than a launch takes
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,codes", [(BF, "e4m3"), (F32, "i8")])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hkv,d,pad,lens,new", [
    (8, 2, 64, 7, [3000, 5, 64, 20000], [7, 3, 0, 5]),       # 28 rows: tiles of 32
    (6, 2, 40, 9, [300, 0, 31], [9, 1, 12]),                 # 27
    (8, 2, 64, 40, [3000, 0, 64, 500], [40, 3, 0, 17]),      # 160: tiles of 128, waves of absent rows alone
    (4, 2, 128, 70, [70000, 100], [70, 65]),                 # 140, split along the keys
    (5, 1, 24, 33, [0, 40, 200], [33, 40, 2]),               # 165, cut to the pad length
])
def test_padded_rows_in_wider_tiles(dtype, codes, causal, hq, hkv, d, pad, lens, new):
    base._attend_case(hq, hkv, d, 32, codes, dtype, lens, new, causal, padded=pad, seed=71)
    base._attend_case(hq, hkv, d, 64, codes, dtype, lens, new, causal, 9.0, True, padded=pad, seed=72, max_q=pad, max_len=max(lens))


@pytest.mark.parametrize("dtype,codes", [(BF, "i8"), (F32, "e4m3")])
@pytest.mark.parametrize("hq,hkv,pad,new", [(40, 1, 3, [3, 0, 2]), (36, 2, 4, [1, 4, 6]), (4, 2, 40, [40, 3, 17])])
def test_padded_rows_over_listed_pages(dtype, codes, hq, hkv, pad, new):
    base._attend_case(hq, hkv, 64, 32, codes, dtype, [700, 40, 2000], new, True, padded=pad, count=5, seed=73)


@pytest.mark.parametrize("padded", [0, 6])
def test_lists_end_in_minus_one(padded):
    """Whole lists: the chosen pages, ascending, then -1, for rows that see fewer pages than are asked for and for absent ones."""
    c = _cache(90, 5, 2, 64, 32, "i8", F32, bounds=True)
    g = ref.fill(c, 74)
    lens, new = [32 * 12, 0, 5, 700, 33], [6, 2, 3, 4, 0]
    table = torch.randint(0, 90, (5, 25), generator=g, device="cuda").to(torch.int32)
    off = ref.offsets(new)
    q = torch.randn(*((5, padded) if padded else (sum(new),)), 4, 64, generator=g, device="cuda")
    for count in (1, 11, 12, 40):
        got = c.select(q, off, _dev(lens), table, count)
        for b, n in enumerate(new):
            rows, lists = (q[b], got[b]) if padded else (q[off[b]:off[b + 1]], got[off[b]:off[b + 1]])
            for i in range(n):
                want = ref.select(rows[i], c, table[b].tolist(), lens[b], lens[b] - n + i, count, True)
                assert lists[i].tolist() == [h + [-1] * (count - len(h)) for h in want], (b, i, count)
            assert (lists[n:] == -1).all()


def test_more_blocks_than_a_launch_takes():
    """2,200,000 sequences that share one page and one open page: reading, choice and both attentions go in several launches."""
    seqs, d = 2200000, 8
    c = _cache(2, 1, 1, d, 32, "i8", BF, bounds=True, causal=False)
    g = ref.fill(c, 75)
    table = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda").expand(seqs, 2).contiguous()
    slots = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    off, lens = torch.arange(seqs + 1, device="cuda"), torch.full((seqs,), 70, device="cuda")
    start = torch.randint(0, 70, (seqs,), generator=g, device="cuda")
    k, v = c.read(_dev([0, 70]), _dev([70]), table[:1], 70, slots=slots[:1])
    gk, gv = c.read(off, lens, table, seqs, start=start, slots=slots)
    assert torch.equal(gk, k[start]) and torch.equal(gv, v[start])
    q = torch.randn(64, 1, d, generator=g, device="cuda").bfloat16()
    at = torch.randint(0, 64, (seqs,), generator=g, device="cuda")
    few = _dev(list(range(65)))
    pages = c.select(q, few, lens[:64], table[:64], 1)
    out = c.attend(q, few, lens[:64], table[:64], slots=slots[:64], max_q=1)
    listed = c.attend(q, few, lens[:64], table[:64], pages=pages, slots=slots[:64])
    many = q[at]
    assert torch.equal(c.select(many, off, lens, table, 1), pages[at])
    assert torch.equal(c.attend(many, off, lens, table, slots=slots, max_q=1), out[at])
    assert torch.equal(c.attend(many, off, lens, table, pages=pages[at], slots=slots), listed[at])


def test_append_of_more_blocks_than_a_launch_takes():
    """35,000 sequences of 16 key heads, 2.2 million blocks: open pages, turned queries and lengths of the second launch, too."""
    seqs, hkv, d = 35000, 16, 8
    g = torch.Generator(device="cuda").manual_seed(76)
    c = R.SeqCache(4, seqs, hkv, d, page=32, rotary=8)
    table = torch.zeros(seqs, 1, dtype=torch.int32, device="cuda")
    k, v = (torch.randn(seqs, hkv, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    lens = torch.randint(0, 30, (seqs,), generator=g, device="cuda")
    off = torch.arange(seqs + 1, device="cuda")
    after, turned = c.append(k, v, off, lens, table, q=k)
    assert torch.equal(after, lens + 1)
    rows = torch.arange(seqs, device="cuda")
    assert torch.equal(c.open[rows, 0, :, 0, lens], turned) and torch.equal(c.open[rows, 0, :, 1, lens], v)
    some = slice(seqs - 50, seqs)
    want = ref.turned(k[some], lens[some], [10000.0 ** (-i / 4) for i in range(4)], 8, False)
    assert ((turned[some].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -28).all()


# ---------------------------------------------------------------------------
# chunks of queries over listed pages
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,codes", [(BF, "e4m3"), (F32, "i8")])
def test_a_row_sees_its_own_full_page_where_its_list_names_it(dtype, codes):
    """The open page is that after the call: rows of a chunk whose page the chunk filled see it, and themselves, only where it is
    listed; of the open page each sees what is not behind it."""
    hq, hkv, d, P, n = 4, 2, 64, 32, 120
    c = _cache(8, 1, hkv, d, P, codes, dtype, bounds=True)
    g = ref.fill(c, 81)
    table = torch.tensor([[5, 2, 7, 0]], dtype=torch.int32, device="cuda")
    new = 60  # positions 60 .. 119: 4 in page 1, page 2 whole, 24 in the open one
    q = torch.randn(new, hq, d, generator=g, device="cuda").to(dtype)
    off, lens = _dev([0, new]), _dev([n])
    picks = c.select(q, off, lens, table, 1)
    pos = torch.arange(n - new, n, device="cuda")
    own = (pos // P).int()
    own = torch.where((own < 3)[:, None] & (picks[..., 0] != own[:, None]), own[:, None], -1)[..., None]  # named once
    k, v, there = ref.tokens_of(c, table, [n], [0])[0]
    key_pos = torch.arange(n, device="cuda")
    for pages in (picks, torch.cat([picks, own], 2)):
        out = c.attend(q, off, lens, table, pages=pages.contiguous())
        for i in range(new):
            for h in range(hkv):
                w = (key_pos >= 96).long()
                for x in pages[i, h].tolist():
                    if x >= 0:
                        w[x * P:(x + 1) * P] += 1
                G = hq // hkv
                want, bound = ref.attention(q[i:i + 1, h * G:(h + 1) * G], k[:, h:h + 1], v[:, h:h + 1], pos[i:i + 1], key_pos, w, True, 0.0, None,
                                            d ** -0.5, dtype == BF, G)
                _close(out[i:i + 1, h * G:(h + 1) * G], want, bound, dtype)
                assert pages is picks or int(w[pos[i]]) == 1


# ---------------------------------------------------------------------------
# slopes: keys next to a row beside keys far from it
# ---------------------------------------------------------------------------


def _sloped(q, k, v, pos, key_pos, weight, slopes, scale, bf16):
    """One row's attention over its keys, causal, and the bound of cache_reference.attention with the normaliser's error taken as what
    it is, the mean of the keys' errors by their probabilities (there: the largest of the row's, which a far key's distance sets).
    Distances are exact up to 2^24, their terms rounded twice, so 8 u of each score's parts stay.  q [hq, d], k, v [nk, d]."""
    d = q.shape[-1]
    x = q.double() @ k.transpose(0, 1) * scale
    es = (6 * d + 16) * ref.U * (q.double().abs() @ k.abs().transpose(0, 1)) * scale
    dist = (pos - key_pos).abs().double()
    m = slopes.double()[:, None]
    x = x - m * dist
    es = es + 8 * ref.U * (m.abs() * dist + x.abs())
    x = torch.where((weight > 0) & (key_pos <= pos), x + weight.clamp(min=1).double().log(), -math.inf)
    P = torch.softmax(x, 1)
    r = 2.0 ** -8 if bf16 else 0.0
    e = es + (P * es).sum(1, keepdim=True) + 16 * ref.U
    out = P @ v
    return out, (P * (e + r + (2 * k.shape[0] + 128) * ref.U)) @ v.abs() + (r + 4 * ref.U) * out.abs()


@pytest.mark.parametrize("dtype,codes", [(F32, "i8"), (F32, "e4m3"), (BF, "i8")])
@pytest.mark.parametrize("hq,d", [(4, 64), (40, 32)])
@pytest.mark.parametrize("tail", [0, 1, 9])
def test_near_keys_beside_far_ones(dtype, codes, hq, d, tail):
    """Listed pages a million positions back and those next to the row: what the near ones are worth does not depend on how far the
    others lie, in whatever order the list names them."""
    P = 64
    c = _cache(12, 1, 1, d, P, codes, dtype)
    g = ref.fill(c, 91)
    n = 16000 * P + tail
    table = torch.arange(16001, device="cuda").remainder(12).to(torch.int32)[None]
    slopes = torch.linspace(0.03, 0.9, hq, device="cuda")
    q = torch.randn(3, hq, d, generator=g, device="cuda").to(dtype)
    off, lens = _dev([0, 3]), _dev([n])
    pages = torch.tensor([[0, 1, 700, 8000, 15998, 15999], [15999, 3, 15000, 2, 15998, 1], [5, 15999, 4, 15998, 3, 2]], dtype=torch.int32,
                         device="cuda")[:, None]
    out = c.attend(q, off, lens, table, pages=pages, slopes=slopes)
    vals, scales = ref.pages_of(c)
    for i in range(3):
        ids = table[0, pages[i, 0].long()].long()
        kv = (vals[ids, 0] * scales[ids, 0][..., None, None]).transpose(0, 1).reshape(2, -1, d)
        key_pos = (pages[i, 0].long()[:, None] * P + torch.arange(P, device="cuda")).flatten()
        if tail:
            kv = torch.cat([kv, c.open[0, 0, 0, :, :tail].double()], 1)
            key_pos = torch.cat([key_pos, torch.arange(n - tail, n, device="cuda")])
        want, bound = _sloped(q[i], kv[0], kv[1], n - 3 + i, key_pos, torch.ones_like(key_pos), slopes, d ** -0.5, dtype == BF)
        _close(out[i], want, bound, dtype)


@pytest.mark.parametrize("dtype,codes", [(F32, "i8"), (BF, "e4m3")])
@pytest.mark.parametrize("rows", [1, 8, 60])
def test_steep_slopes_over_a_whole_history(dtype, codes, rows):
    """A step of keys after the other, each far above the one before: rows of every tile, one and several parts."""
    hq, d, P, n = 4, 64, 32, 9000
    c = _cache(30, 1, 1, d, P, codes, dtype)
    g = ref.fill(c, 92)
    table = torch.arange(282, device="cuda").remainder(30).to(torch.int32)[None]
    slopes = torch.tensor([0.01, 0.7, 8.0, -0.004], device="cuda")
    q = torch.randn(rows, hq, d, generator=g, device="cuda").to(dtype)
    out = c.attend(q, _dev([0, rows]), _dev([n]), table, slopes=slopes)
    k, v, there = ref.tokens_of(c, table, [n], [0])[0]
    key_pos = torch.arange(n, device="cuda")
    for i in range(rows):
        want, bound = _sloped(q[i], k[:, 0], v[:, 0], n - rows + i, key_pos, there.long(), slopes, d ** -0.5, dtype == BF)
        _close(out[i], want, bound, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale,cap", [(1e-300, 0.0), (1e-300, 5.0), (1e-42, 0.0)])
def test_scales_that_vanish_in_fp32_keep_the_mask(dtype, scale, cap):
    """Every key that a row sees counts alike, and those behind it not at all."""
    for new in ([3, 2], [40, 9]):
        base._attend_case(4, 1, 64, 64, "i8", dtype, [700, 33], new, True, cap, scale=scale, seed=93)
        base._attend_case(4, 1, 64, 64, "e4m3", dtype, [700, 33], new, True, cap, True, scale=scale, count=3, seed=94)


# ---------------------------------------------------------------------------
# rotation is a function of the position
# ---------------------------------------------------------------------------


@pytest.mark.parametrize("d,rotary,interleaved,page", [(128, 128, False, 256), (64, 48, True, 64), (16, 2, False, 32), (32, 32, False, 128)])
@pytest.mark.parametrize("held", [0, 3, 1000003 * 256])
def test_turned_rows_do_not_depend_on_the_cuts(d, rotary, interleaved, page, held):
    """Pairs that turn to nearly nothing show the last bit of their angle: keys and queries are the same however calls cut them, and
    the same as each other."""
    g = torch.Generator(device="cuda").manual_seed(95)
    n, h = page - 1 - held % page, rotary // 2
    freqs = [1.0 + 0.37 * i for i in range(h)]
    pos = held + torch.arange(n, device="cuda")
    w = pos.double()[:, None] * torch.tensor(freqs, dtype=torch.float64, device="cuda")
    x = torch.randn(n, 2, d, generator=g, device="cuda")
    a, b = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, h), slice(h, rotary))
    x[:, 0, a], x[:, 0, b] = torch.sin(w).float(), torch.cos(w).float()
    x[:, 1, a], x[:, 1, b] = torch.cos(w).float(), -torch.sin(w).float()
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    at = held // page % 2, held % page
    got = []
    for cuts in ([n], [1] * n, [5, 1, 2, n - 8], [n // 2, n - n // 2]):
        c = R.SeqCache(1, 1, 2, d, page=page, dtype=F32, rotary=rotary, freqs=freqs, interleaved=interleaved)
        lens, done, rows = _dev([held]), 0, []
        for m in cuts:
            part = x[done:done + m]
            lens, q = c.append(part, part, _dev([0, m]), lens, table, q=part)
            rows.append(q)
            done += m
        got.append((c.open[0, at[0], :, 0, at[1]:at[1] + n].transpose(0, 1), torch.cat(rows)))
    for k, q in got:
        assert torch.equal(k, got[0][0]) and torch.equal(q, got[0][1])
    assert torch.equal(got[0][0], got[0][1])


# ---------------------------------------------------------------------------
# codes and bounds at the ends of fp32
# ---------------------------------------------------------------------------


def _written(x, codes, dtype):
    """Pages of x [pages, P, d] written and looked at: codes, scales, bounds."""
    n, P, d = x.shape
    c = _cache(n, n, 1, d, P, codes, dtype, bounds=True)
    table = torch.arange(n, dtype=torch.int32, device="cuda")[:, None]
    k = x.view(n * P, 1, d)
    c.append(k, k, ref.offsets([P] * n), _dev([0] * n), table)
    tokens = [torch.stack([x[i][:, None], x[i][:, None]], 2) for i in range(n)]
    base._check_pages(c, table, tokens, None, None, codes, [(i, 0) for i in range(n)])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_codes_next_to_ties_under_the_least_scales(dtype):
    """Scales from 2^-126 to 2^-120, whose halves may not be numbers: codes are x / scale to the nearest, ties to even."""
    g = torch.Generator(device="cuda").manual_seed(96)
    x = torch.randn(64, 32, 64, generator=g, device="cuda", dtype=torch.float64) * 2.0 ** -121
    x *= 2.0 ** torch.arange(-4, 4, dtype=torch.float64, device="cuda").repeat(8)[:, None, None]
    x = x.to(dtype)
    s = (x.double().abs().amax((1, 2)) / 127).float().clamp(min=2.0 ** -126).double()
    half = (torch.randint(-100, 100, (64, 8, 64), generator=g, device="cuda") + 0.5) * s[:, None, None]  # next to ties
    x[:, 8:16] = half.to(dtype)
    x[:, 8:16] = torch.where(x[:, 8:16].abs() <= 126 * s[:, None, None], x[:, 8:16], 0)
    _written(x, "i8", dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_bounds_of_columns_far_below_the_largest(dtype):
    """A column whose numbers vanish beside the page's largest is bounded from outside all the same."""
    x = torch.zeros(5, 32, 16, device="cuda")
    x[:, 0, 0] = torch.tensor([3e38, 2e6, 1.0, 1e30, 2.0 ** -20], device="cuda")
    for i, v in enumerate((1e-38, 1e-41, 1e-20, 2.0 ** -133, 1e-10)):
        x[:, :, 2 + 2 * i] = v
        x[:, :, 3 + 2 * i] = -v
    x[:, 5, 13], x[:, 6, 13] = 1e-38, -1e-30
    _written(x.to(dtype), "i8", dtype)
    _written(x.to(dtype), "e4m3", dtype)
