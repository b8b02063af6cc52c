"""Timed cases of the paged history cache: keys and values of behaviour sequences held in 8 bits, in serving.

A user's history is kept as pages of a fixed number of tokens.  A full page is held in 8 bits with one scale for the page,
key head and side (keys or values); the page that is still filling, the open page, in the model's type.

`listed()` names the fixed cases, `draw(rng)` gives others of the same ranges.  A case is a dict of plain values;
`prepare` builds its inputs on the GPU, `run` makes one pass (in plain torch, or through the framework where `own` is
set), `work` counts the bytes and operations that a pass cannot do without, `exact` computes the outputs in 64 bits.

Kinds of case
  append  new tokens of each sequence: queries and keys rotated by their position, keys and values written to the cache,
          then the pages that were touched read back as rows
  attend  out_i = sum_j softmax_j(s_ij) v_j over the keys that query i sees
  sparse  for each query token and key head the `count` pages of the highest score, then attention over those pages and
          the open page

Rotation of token p: columns (a, b) = (i, i + rot / 2), or (2 i, 2 i + 1) interleaved, turn by p base^(-2 i / rot).
Full pages: i8 codes rne(x / s) with s = max |x| / 127 in 32 bits; e4m3 codes of x / s with s the least power of two that keeps
max |x| within 448 s.  Keys are coded after their rotation has been rounded to the model's type.
Attention: head h of hq reads key head h // (hq / hkv); query i of Lq stands at p_i = i + len - Lq;
s_ij = cap(d^-1/2 q_i.k_j) - slope_h |p_i - j|, cap(x) = c tanh(x / c); it sees all keys, or where causal j <= p_i.
Score of a full page: e max over the heads of a key head of sq sum_c max(q8_c mx_c, q8_c mn_c), with q8 = rne(q / sq) and
the page's column maxima mx and minima mn in units of e, all whole numbers up to 127, sq and e powers of two.
"""
import math
import zlib

import torch

own = False

DEV = "cuda"
BASE = 10000.0
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, kind, **kw):
    c = dict(name=name, kind=kind, codes="e4m3", dtype="bf16", hq=8, hkv=2, d=128, page=64, seqs=1, q_lo=1, q_hi=1, kv_lo=0,
             kv_hi=1024, causal=True)
    if kind == "append":
        c.update(rot=c["d"], pairs="half", bounds=False)
    else:
        c.update(cap=0.0, slopes=False, count=0)
    c.update(kw)
    return c


def listed():
    return [
        # one new behaviour for each of 256 users
        _case("append_token_256_users", "append", seqs=256, kv_lo=1, kv_hi=4096),
        # 64 short sessions of a small fp32 encoder, first written: launches and latency count
        _case("append_64_sessions_f32", "append", codes="i8", dtype="f32", hq=2, hkv=2, d=32, page=32, rot=32, seqs=64, q_lo=0,
              q_hi=50, kv_hi=0),
        # histories of a batch of users written in one go, with the bounds that choose pages
        _case("append_24_histories", "append", seqs=24, q_lo=17, q_hi=8191, kv_hi=0, bounds=True),
        # new behaviours of 8 users, part of each head rotated, neighbouring columns paired
        _case("append_chunk_8_users", "append", codes="i8", hq=16, hkv=4, d=72, rot=48, pairs="next", seqs=8, q_lo=33, q_hi=257,
              kv_lo=2000, kv_hi=8191),
        # one new token for each of 256 users with histories of very unequal length
        _case("attend_token_256_users", "attend", seqs=256, kv_lo=1, kv_hi=4096),
        # 64 short sessions through a small fp32 encoder layer, nothing causal
        _case("attend_64_sessions_f32", "attend", codes="i8", dtype="f32", hq=2, hkv=2, d=32, page=32, seqs=64, kv_hi=50,
              causal=False),
        # four candidates against one history of a million behaviours
        _case("attend_4_of_1M", "attend", codes="i8", hq=4, hkv=2, d=64, page=256, q_lo=4, q_hi=4, kv_lo=1000003, kv_hi=1000003,
              causal=False),
        # a chunk of new behaviours of each of 8 users over their histories, capped scores
        _case("attend_chunk_8_users", "attend", seqs=8, q_lo=33, q_hi=257, kv_lo=2000, kv_hi=8191, cap=50.0),
        # the last 4096 behaviours of a lifelong sequence read against all of it
        _case("attend_4096_of_16384", "attend", q_lo=4096, q_hi=4096, kv_lo=16384, kv_hi=16384),
        # four candidates against 64 pages each of a million behaviours
        _case("sparse_4_of_1M", "sparse", hkv=8, hq=32, q_lo=4, q_hi=4, kv_lo=1000003, kv_hi=1000003, causal=False, count=64),
        # one new token for each of 64 users over 32 pages of up to 65536 behaviours, falling off with distance
        _case("sparse_token_64_users", "sparse", codes="i8", seqs=64, kv_lo=1, kv_hi=65536, slopes=True, count=32),
        # a few tokens each of 4 users of a small fp32 model
        _case("sparse_chunk_4_users_f32", "sparse", codes="i8", dtype="f32", hq=4, hkv=4, d=32, page=32, seqs=4, q_lo=1, q_hi=16,
              kv_lo=16, kv_hi=5000, count=20),
    ]


def _logu(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "sparse"])
    group = rng.choice([1, 2, 4, 4, 8])
    hkv = rng.choice([1, 2, 4]) if group > 1 else rng.choice([1, 2, 4, 8])
    d = rng.choice([16, 32, 64, 64, 72, 128, 128])
    c = _case("", kind, codes=rng.choice(["e4m3", "i8"]), dtype=rng.choice(["f32", "bf16", "bf16"]), hq=hkv * group, hkv=hkv, d=d,
              page=rng.choice([32, 64, 64, 128, 256]))
    del c["name"]
    if kind == "append":
        c["rot"] = rng.choice([d, d, d // 2, 0])
        c["pairs"] = rng.choice(["half", "next"])
        c["bounds"] = rng.random() < 0.3
        c["q_hi"] = rng.choice([1, _logu(rng, 2, 16), _logu(rng, 17, 8191)])
        c["q_lo"] = rng.randint(0, c["q_hi"])
        c["kv_hi"] = rng.choice([0, _logu(rng, 1, 100000)])
        c["kv_lo"] = rng.randint(0, c["kv_hi"])
        tokens = 1.3e7 / (hkv * d)
        c["seqs"] = _logu(rng, 1, max(1, min(2000, int(tokens / c["q_hi"]), int(1.5e9 / (hkv * d * (c["kv_hi"] + c["q_hi"] + 256))))))
        if c["seqs"] < 4:  # one to three sequences: not all of them without a new token
            c["q_lo"] = max(1, c["q_lo"])
        return c
    c["causal"] = rng.random() < 0.6
    c["cap"] = rng.choice([0.0, 0.0, 20.0, 50.0])
    c["slopes"] = rng.random() < 0.3
    cells = 1.3e9 / (hkv * d)  # tokens of all caches
    if kind == "attend":
        form = rng.choice(["token", "token", "chunk"])
        c["q_hi"] = _logu(rng, 1, 8) if form == "token" else _logu(rng, 9, 600)
        # scores (query, key, head): fp32 products cost several times more
        scores = 5e8 if c["dtype"] == "bf16" else 1.5e8
        most = min(1000000, int(cells / 8), int(scores / c["hq"] / c["q_hi"]))
    else:
        c["count"] = _logu(rng, 1, 128)
        c["q_hi"] = _logu(rng, 1, max(1, min(40, int(2e8 / (hkv * d * (c["count"] + 1) * c["page"])))))
        scores = 2e8 / (hkv * d) / (c["count"] + 1) / c["page"]  # gathered rows of a pass in plain torch
        most = min(1000000, int(cells / 8))
    c["q_lo"] = rng.randint(0, c["q_hi"])
    c["kv_hi"] = _logu(rng, 16, most)
    c["kv_lo"] = rng.randint(0, c["kv_hi"])
    if kind == "attend":
        seqs = min(scores / c["hq"] / c["kv_hi"] / c["q_hi"], cells / 8 / c["kv_hi"], 2000)
    else:
        seqs = min(scores / c["q_hi"], cells / 8 / c["kv_hi"], 500)
    c["seqs"] = _logu(rng, 1, max(1, int(seqs)))
    if c["seqs"] < 4:
        c["q_lo"], c["kv_lo"] = max(1, c["q_lo"]), max(1, c["kv_lo"])
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------


def _gen(case, seed=None):
    """The case's own random stream, or the stream of a seed."""
    text = repr(sorted((k, v) for k, v in case.items() if k != "name"))
    g = torch.Generator(device=DEV)
    g.manual_seed(zlib.crc32(text.encode()) if seed is None else 1000003 * int(seed) + 17)
    return g


def _lengths(case):
    """New tokens (queries) and tokens held before (append) or in all of each sequence: the case's, not a seed's."""
    g = _gen(case)
    n, P = case["seqs"], case["page"]
    kv = torch.randint(case["kv_lo"], case["kv_hi"] + 1, (n,), generator=g, device=DEV)
    q = torch.randint(case["q_lo"], case["q_hi"] + 1, (n,), generator=g, device=DEV)
    if case["kind"] == "append":
        # An append keeps two open pages of a sequence, by the page number's parity, so that a pass can be repeated unless
        # it goes on by an even number of pages from the middle of one to the middle of another: a page less then.
        step = (kv + q) // P - kv // P
        again = (step >= 2) & (step % 2 == 0) & (kv % P > 0) & ((kv + q) % P > 0)
        q = torch.where(again, q - P, q)
    return q, kv


def _offsets(lens):
    off = torch.zeros(lens.numel() + 1, dtype=torch.int64, device=DEV)
    torch.cumsum(lens, 0, out=off[1:])
    return off


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV).to(TYPES[dtype])


def _width(d):
    return 32 if d <= 32 else 64 if d <= 64 else 128


def _pow2_over(top, most):
    """The least power of two s with top <= most * s (at least 2^-126)."""
    m, e = torch.frexp(top)
    mm, me = math.frexp(most)
    k = torch.where(m <= mm, e - me, e - me + 1)
    k = torch.where(top > 0, k, -126).clamp(min=-126)
    return ((k + 127) << 23).to(torch.int32).view(torch.float32)  # a power function may be off by a bit


def _scale(top, codes):
    return (top / 127).clamp(min=2.0 ** -126) if codes == "i8" else _pow2_over(top, 448.0)


def _encode(x, s, codes):
    y = x / s
    return torch.round(y).clamp(-127, 127).to(torch.int8).view(torch.uint8) if codes == "i8" else y.float().to(
        torch.float8_e4m3fn).view(torch.uint8)


def _decode(c, codes):
    return c.view(torch.int8).float() if codes == "i8" else c.view(torch.float8_e4m3fn).float()


def _column_bounds(x):
    """Column maxima and minima of [..., P, W] in whole units of a power of two, rounded outward, and that unit."""
    e = _pow2_over(x.abs().amax((-1, -2)), 127.0)
    top, low = x.amax(-2) / e[..., None], x.amin(-2) / e[..., None]
    return torch.stack([top.ceil(), low.floor()], -2).to(torch.int8), e


def prepare(case, seed):
    g = _gen(case, seed)
    order = torch.randperm(case["seqs"], generator=g, device=DEV)
    ql, kl = (t[order] for t in _lengths(case))
    n, hq, hkv, d, P, dt = (case[k] for k in ("seqs", "hq", "hkv", "d", "page", "dtype"))
    W, append = _width(d), case["kind"] == "append"
    held = kl + ql if append else kl
    pages = (held + P - 1) // P
    width = max(1, int(pages.max()))
    total = int(pages.sum())
    pool = total + 3
    ids = torch.randperm(pool, generator=g, device=DEV)[:total].to(torch.int32)
    table = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
    table[torch.arange(width, device=DEV) < pages[:, None]] = ids
    s = dict(case=case, lens=kl, table=table, off=_offsets(ql), slots=torch.randperm(n, generator=g, device=DEV).to(torch.int32),
             slopes=None, most_q=case["q_hi"], most=case["kv_hi"],
             codes=torch.zeros(pool, hkv, 2, P * W, dtype=torch.uint8, device=DEV),
             scales=torch.ones(pool, hkv, 2, device=DEV), open=_randn(g, (n, 2, hkv, 2, P, d), dt), bounds=None, units=None)
    if append and case["bounds"] or case["kind"] == "sparse":
        s["bounds"] = torch.zeros(pool, hkv, 2, W, dtype=torch.int8, device=DEV)
        s["units"] = torch.ones(pool, hkv, device=DEV)
    rows = int(ql.sum())
    if append:
        y = _randn(g, (rows, hq + 2 * hkv, d), dt)  # q, k and v as column blocks of one projection
        s["q"], s["k"], s["v"] = y.split([hq, hkv, hkv], 1)
        s["start"] = kl // P * P
        s["back"] = _offsets(torch.where(ql > 0, held - s["start"], 0))
        s["back_rows"] = int(s["back"][-1])
    else:
        # histories drift: the keys of a page share a direction, and a query looks for some page's
        step = max(1, int(1e8 / (hkv * P * W)))
        spread = 0.5 + torch.rand(d, generator=g, device=DEV)
        for i in range(0, pool, step):
            m = min(step, pool - i)
            x = torch.zeros(m, hkv, 2, P, W, device=DEV)
            x[..., :d] = torch.randn(m, hkv, 2, P, d, generator=g, device=DEV) * spread
            x[:, :, 0, :, :d] += torch.randn(m, hkv, 1, d, generator=g, device=DEV)
            sc = _scale(x.abs().amax((3, 4)), case["codes"])
            c = _encode(x, sc[..., None, None], case["codes"])
            s["scales"][i:i + m] = sc
            s["codes"][i:i + m, :, 0] = c[:, :, 0].view(m, hkv, P, W // 16, 16).transpose(2, 3).reshape(m, hkv, P * W)
            s["codes"][i:i + m, :, 1] = c[:, :, 1].view(m, hkv, P // 16, 16, W).transpose(3, 4).reshape(m, hkv, P * W)
            if s["bounds"] is not None:
                s["bounds"][i:i + m], s["units"][i:i + m] = _column_bounds(x[:, :, 0])
        s["q"] = _randn(g, (rows, hq, d), dt)
        if case["slopes"]:
            s["slopes"] = torch.pow(2.0, -1.0 - 7.0 * torch.rand(hq, generator=g, device=DEV))
    if own:
        s["cache"] = _handle(s)
    return s


def _handle(s):
    from paper_2509_20883_amd import recis as R

    case = s["case"]
    c = R.SeqCache(pages=s["codes"].shape[0], slots=case["seqs"], heads_kv=case["hkv"], head_dim=case["d"], page=case["page"],
                   codes=case["codes"], dtype=TYPES[case["dtype"]], bounds=s["bounds"] is not None,
                   rotary=case.get("rot", 0), base=BASE, interleaved=case.get("pairs") == "next", causal=case["causal"],
                   softcap=case.get("cap", 0.0))
    for mine, name in ((c.codes, "codes"), (c.scales, "scales"), (c.open, "open"), (c.bounds, "bounds"), (c.units, "units")):
        if s[name] is not None:
            mine.copy_(s[name].view(mine.shape))
            s[name] = mine
    return c


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------


def run(state):
    if own:
        return _run_own(state)
    return {"append": _plain_append, "attend": _plain_attend, "sparse": _plain_sparse}[state["case"]["kind"]](state)


def _run_own(s):
    case, c = s["case"], s["cache"]
    if case["kind"] == "append":
        lens, q = c.append(s["k"], s["v"], s["off"], s["lens"], s["table"], q=s["q"], slots=s["slots"])
        k, v = c.read(s["back"], lens, s["table"], s["back_rows"], start=s["start"], slots=s["slots"])
        got = dict(q=q, k=k, v=v, lens=lens)
        if case["bounds"]:
            got["bounds"] = (c.bounds * c.units[..., None, None]).to(torch.bfloat16)
        return got
    at = dict(slots=s["slots"], max_q=s["most_q"], max_len=s["most"])
    if case["kind"] == "attend":
        return dict(out=c.attend(s["q"], s["off"], s["lens"], s["table"], slopes=s["slopes"], **at))
    pages = c.select(s["q"], s["off"], s["lens"], s["table"], case["count"], max_q=s["most_q"], max_len=s["most"])
    return dict(pages=pages, out=c.attend(s["q"], s["off"], s["lens"], s["table"], pages=pages, slopes=s["slopes"], **at))


def _turn(x, pos, case):
    """Rows of x [rows, heads, d] turned by their positions, in x's type."""
    r = case["rot"]
    if r == 0 or x.shape[0] == 0:
        return x.clone()
    f = BASE ** (-2.0 * torch.arange(r // 2, dtype=torch.float64, device=DEV) / r)
    angle = pos.double()[:, None] * f
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    y = x.double()  # a key rounded the other way may fall across a border of the codes
    if case["pairs"] == "half":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _plain_append(s):
    case = s["case"]
    n, hkv, d, P, codes, dt = case["seqs"], case["hkv"], case["d"], case["page"], case["codes"], s["q"].dtype
    off, lens, back = s["off"], s["lens"], s["back"]
    rows, total = s["q"].shape[0], s["back_rows"]
    seq = torch.searchsorted(off, torch.arange(rows, device=DEV), right=True) - 1
    pos = lens[seq] + torch.arange(rows, device=DEV) - off[seq]
    q, k = _turn(s["q"], pos, case), _turn(s["k"], pos, case)
    new_lens = lens + off[1:] - off[:-1]
    # every token of the touched pages: those that the open page held, then the new ones
    i = torch.arange(total, device=DEV)
    bs = torch.searchsorted(back, i, right=True) - 1
    p = s["start"][bs] + i - back[bs]
    fresh = (p >= lens[bs])[:, None, None]
    at = (off[bs] + p - lens[bs]).clamp(0, max(rows - 1, 0))
    kept = s["open"][s["slots"][bs].long(), (p // P) % 2, :, :, p % P]  # [total, hkv, 2, d]
    k_rows = torch.where(fresh, k[at], kept[:, :, 0]) if rows else kept[:, :, 0]
    v_rows = torch.where(fresh, s["v"][at], kept[:, :, 1]) if rows else kept[:, :, 1]
    # page by page: [units, hkv, P, d]
    per = (back[1:] - back[:-1] + P - 1) // P
    first = _offsets(per)
    unit, full = first[bs] + (p - s["start"][bs]) // P, ((p // P + 1) * P <= new_lens[bs])[:, None, None]
    units = int(first[-1])
    got = dict(q=q, lens=new_lens)
    for name, x in (("k", k_rows), ("v", v_rows)):
        grid = torch.zeros(units, P, hkv, d, device=DEV)
        grid[unit, p % P] = x.float()
        sc = _scale(grid.abs().amax((1, 3), keepdim=True), codes)
        coded = _decode(_encode(grid.double(), sc.double(), codes), codes) * sc  # values next to a border of the codes
        got[name] = torch.where(full, coded[unit, p % P].to(dt), x)
        if name == "k" and case["bounds"]:
            box = torch.zeros(s["bounds"].shape, device=DEV)
            whole = torch.zeros(units, dtype=torch.bool, device=DEV)
            whole[unit] = full[:, 0, 0]
            us = torch.searchsorted(first, torch.arange(units, device=DEV), right=True) - 1
            page = s["table"][us, s["start"][us] // P + torch.arange(units, device=DEV) - first[us]].long()
            b, e = _column_bounds(grid.transpose(1, 2))
            box[page[whole], :, :, :d] = (b * e[..., None, None])[whole]
            got["bounds"] = box.to(torch.bfloat16)
    return got


def _dense(s):
    """Keys and values of every sequence in 32 bits, [seqs, tokens, hkv, d], zero past its end."""
    case = s["case"]
    n, hkv, d, P, W = case["seqs"], case["hkv"], case["d"], case["page"], _width(case["d"])
    lens, width = s["lens"], s["table"].shape[1]
    ids = s["table"].clamp(min=0).long()
    nf, seqs = lens // P, torch.arange(n, device=DEV)
    live = (torch.arange((width + 1) * P, device=DEV) < lens[:, None])[:, :, None, None]
    got = []
    for side in (0, 1):
        x = _decode(s["codes"][:, :, side][ids], case["codes"]) * s["scales"][:, :, side][ids][..., None]
        if side == 0:
            x = x.view(n, width, hkv, W // 16, P, 16).permute(0, 1, 4, 2, 3, 5).reshape(n, width, P, hkv, W)
        else:
            x = x.view(n, width, hkv, P // 16, W, 16).permute(0, 1, 3, 5, 2, 4).reshape(n, width, P, hkv, W)
        x = torch.cat([x[..., :d], torch.zeros(n, 1, P, hkv, d, device=DEV)], 1)
        x[seqs, nf] = s["open"][s["slots"].long(), nf % 2, :, side].float().transpose(1, 2)
        got.append(torch.where(live, x.view(n, (width + 1) * P, hkv, d), 0.0))
    return got


def _soft(sc, sees, v):
    sc.masked_fill_(~sees, -math.inf)
    top = sc.amax(-1, keepdim=True).clamp_(min=-3e38)
    e = sc.sub_(top).exp_()
    return e.div_(e.sum(-1, keepdim=True).clamp_(min=1e-38)) @ v


def _plain_attend(s):
    case = s["case"]
    n, hq, hkv, d, lq = case["seqs"], case["hq"], case["hkv"], case["d"], s["most_q"]
    group, off, lens = hq // hkv, s["off"], s["lens"]
    rows = s["q"].shape[0]
    if rows == 0:
        return dict(out=torch.zeros_like(s["q"]))
    k, v = _dense(s)
    lk = k.shape[1]
    ql = off[1:] - off[:-1]
    i, j = torch.arange(lq, device=DEV), torch.arange(lk, device=DEV)
    q = torch.where((i < ql[:, None])[:, :, None, None], s["q"][(off[:-1, None] + i).clamp_(max=rows - 1)].float(), 0.0)
    q = q.view(n, lq, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, group * lq, d)
    k, v = (x.permute(0, 2, 1, 3).contiguous() for x in (k, v))
    p = i + (lens - ql)[:, None]  # [seqs, lq]
    sees = (j < lens[:, None])[:, None, :].expand(n, lq, lk)
    if case["causal"]:
        sees = sees & (j <= p[:, :, None])
    sc = (q @ k.transpose(2, 3)).mul_(d ** -0.5)
    if case["cap"]:
        sc = sc.div_(case["cap"]).tanh_().mul_(case["cap"])
    sc = sc.view(n, hkv, group, lq, lk)
    if s["slopes"] is not None:
        sc = sc - s["slopes"].view(hkv, group, 1, 1) * (p[:, :, None] - j).abs().float()[:, None, None]
    o = _soft(sc, sees[:, None, None], v[:, :, None])  # [n, hkv, group, lq, d]
    t = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(off, t, right=True) - 1
    return dict(out=o.permute(0, 3, 1, 2, 4)[seq, t - off[seq]].reshape(rows, hq, d).to(s["q"].dtype))


def _plain_sparse(s):
    case = s["case"]
    hq, hkv, d, P, count = (case[k] for k in ("hq", "hkv", "d", "page", "count"))
    W = _width(d)
    group, off, lens, dt = hq // hkv, s["off"], s["lens"], s["q"].dtype
    rows, width = s["q"].shape[0], s["table"].shape[1]
    t = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(off, t, right=True) - 1
    pos = lens[seq] - (off[seq + 1] - off[seq]) + t - off[seq]
    q = s["q"].float().view(rows, hkv, group, d)
    # scores of every page, whole numbers times powers of two
    sq = _pow2_over(q.abs().amax(-1), 127.0)
    q8 = torch.round(q / sq[..., None])
    score = torch.empty(rows, hkv, width, device=DEV)
    step = max(1, int(2e8 / (width * hkv * d)))
    for r in range(0, rows, step):
        ids = s["table"][seq[r:r + step]].clamp(min=0).long()  # [step, width]
        b = s["bounds"][ids].float()[..., :d]  # [step, width, hkv, 2, d]
        x = q8[r:r + step]
        whole = (x.clamp(min=0) @ b[..., 0, :].permute(0, 2, 3, 1).contiguous() +
                 x.clamp(max=0) @ b[..., 1, :].permute(0, 2, 3, 1).contiguous())
        score[r:r + step] = (whole * sq[r:r + step, ..., None]).amax(2) * s["units"][ids].transpose(1, 2)
    page = torch.arange(width, device=DEV)
    seen = page < (lens // P)[seq][:, None]
    if case["causal"]:
        seen = seen & (page * P <= pos[:, None])
    score.masked_fill_(~seen[:, None], -math.inf)
    if width < count:
        score = torch.cat([score, torch.full((rows, hkv, count - width), -math.inf, device=DEV)], 2)
    best, at = torch.sort(score, dim=2, descending=True, stable=True)
    none = 1 << 30
    at = torch.where(best[..., :count] > -math.inf, at[..., :count], none).sort(2).values
    pages = torch.where(at < none, at, -1).to(torch.int32)
    # the chosen pages and the open page of each token and key head: [rows, hkv, (count + 1) P, d]
    ids = torch.where(pages >= 0, s["table"][seq[:, None, None], pages.clamp(min=0).long()], 0).long()
    head = torch.arange(hkv, device=DEV)[None, :, None]
    nf = lens[seq] // P
    kv = []
    for side in (0, 1):
        x = _decode(s["codes"][ids, head, side], case["codes"]) * s["scales"][ids, head, side][..., None]
        if side == 0:
            x = x.view(rows, hkv, count, W // 16, P, 16).transpose(3, 4).reshape(rows, hkv, count * P, W)
        else:
            x = x.view(rows, hkv, count, P // 16, W, 16).transpose(4, 5).reshape(rows, hkv, count * P, W)
        tail = s["open"][s["slots"][seq].long(), nf % 2, :, side].float()
        live = (torch.arange(P, device=DEV) < (lens[seq] - nf * P)[:, None])[:, None, :, None]
        kv.append(torch.cat([x[..., :d], torch.where(live, tail, 0.0)], 2))
    k, v = kv
    j = torch.arange(P, device=DEV)
    j = torch.cat([(torch.where(pages >= 0, pages, none // P)[..., None] * P + j).flatten(2),
                   (nf[:, None] * P + j)[:, None].expand(rows, hkv, P)], 2)
    sees = (j < lens[seq][:, None, None])
    if case["causal"]:
        sees = sees & (j <= pos[:, None, None])
    sc = (q @ k.transpose(2, 3).contiguous()).mul_(d ** -0.5)
    if case["cap"]:
        sc = sc.div_(case["cap"]).tanh_().mul_(case["cap"])
    if s["slopes"] is not None:
        sc = sc - s["slopes"].view(hkv, group, 1) * (pos[:, None, None] - j).abs().float()[:, :, None]
    o = _soft(sc, sees[:, :, None], v)
    return dict(pages=pages, out=o.reshape(rows, hq, d).to(dt))


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# ---------------------------------------------------------------------------


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    ql, kl = (t.double() for t in _lengths(case))
    hq, hkv, d, P = case["hq"], case["hkv"], case["d"], case["page"]
    rows = float(ql.sum())
    if case["kind"] == "append":
        start = torch.floor(kl / P) * P
        touched = float(torch.where(ql > 0, kl + ql - start, 0.0).sum())
        full = float(torch.where(ql > 0, torch.floor((kl + ql) / P) * P - start, 0.0).sum())
        kept = float(torch.where(ql > 0, kl - start, 0.0).sum())
        b = rows * (2 * hq + 2 * hkv) * d * es  # q in and out, k and v in
        b += 2 * kept * hkv * d * es  # what the open pages held
        b += 2 * hkv * d * (2 * full + 2 * (touched - full) * es)  # codes and open rows, written and read
        b += 2 * touched * hkv * d * es  # rows read back
        if case["bounds"]:
            b += full / P * hkv * 2 * d * 3
        return {"bytes": int(b + 32 * case["seqs"]), "flops": int(rows * (hq + hkv) * case["rot"] * 3 + touched * hkv * d * 6)}
    nf = torch.floor(kl / P) * P
    cache = float((nf * 2 * hkv * d + (kl - nf) * 2 * hkv * d * es).sum())
    ends = 2 * rows * hq * d * es + 24 * case["seqs"]
    if case["kind"] == "attend":
        if not case["causal"]:
            pairs = float((ql * kl).sum())
        else:
            i = torch.arange(int(ql.max()) if ql.numel() else 0, device=DEV, dtype=torch.float64)
            pairs = float(((kl - ql)[:, None] + i + 1).clamp_(min=0).minimum(kl[:, None]).mul(i < ql[:, None]).sum())
        return {"bytes": int(cache * (rows > 0) + ends), "flops": int(4 * d * hq * pairs)}
    pages = nf / P
    chosen = torch.minimum(pages, ql * case["count"])
    b = float((pages * (ql > 0)).sum()) * hkv * 2 * d + float(chosen.sum()) * P * 2 * hkv * d + ends
    b += float(((kl - nf) * (ql > 0)).sum()) * 2 * hkv * d * es + rows * hkv * case["count"] * 4
    pairs = float((ql * (torch.minimum(pages, torch.full_like(pages, case["count"])) * P + kl - nf)).sum())
    return {"bytes": int(b), "flops": int(4 * d * hq * (float((ql * pages).sum()) + pairs))}


def _two_to(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_unit(a, most):
    """The least power of two s, from 2^-126 on, with a <= most s."""
    s = _two_to(torch.ceil(torch.log2(a.clamp(min=2.0 ** -200) / most)).clamp(min=-126))
    s = torch.where(a > most * s, 2 * s, s)
    return torch.where(a <= most * s / 2, s / 2, s).clamp(min=2.0 ** -126)


def _exact_codes(x, codes):
    """[hkv, P, d] in 64 bits as the page stands for it."""
    a = x.abs().amax((1, 2), keepdim=True)
    if codes == "i8":
        s = (a / 127).clamp(min=2.0 ** -126).float().double()  # held in 32 bits
        return torch.round(x / s) * s
    s = _exact_unit(a, 448)
    y = x / s
    # e4m3: three bits after the leading one, down to 2^-6, and steps of 2^-9 below
    step = _two_to(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))) / 8
    step = torch.where(y.abs() < 8 * step.clamp(min=2.0 ** -8), step / 2, step).clamp(min=2.0 ** -9)
    step = torch.where(y.abs() >= 16 * step, 2 * step, step)
    return torch.round(y / step) * step * s


def _exact_turn(x, pos, case):
    r = case["rot"]
    y = x.double()
    out = y.clone()
    for i in range(r // 2):
        a, b = (i, i + r // 2) if case["pairs"] == "half" else (2 * i, 2 * i + 1)
        w = pos.double() * BASE ** (-2.0 * i / r)
        c, s = torch.cos(w)[:, None], torch.sin(w)[:, None]
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., a] * s + y[..., b] * c
    return out


def _exact_append(s):
    case = s["case"]
    P, dt = case["page"], s["q"].dtype
    off, lens, back = s["off"].tolist(), s["lens"].tolist(), s["back"].tolist()
    slots, table = s["slots"].tolist(), s["table"].tolist()
    total = back[-1]
    got = {k: torch.zeros(total, case["hkv"], case["d"], dtype=torch.float64, device=DEV) for k in ("k", "v")}
    seq = torch.repeat_interleave(torch.arange(case["seqs"], device=DEV), s["off"][1:] - s["off"][:-1])
    pos = s["lens"][seq] + torch.arange(off[-1], device=DEV) - s["off"][seq]
    q, k = _exact_turn(s["q"], pos, case), _exact_turn(s["k"], pos, case).to(dt)
    box = torch.zeros(s["bounds"].shape, dtype=torch.float64, device=DEV) if case["bounds"] else None
    for b in range(case["seqs"]):
        start, end = lens[b] // P * P, lens[b] + off[b + 1] - off[b]
        if off[b + 1] == off[b]:
            continue
        for name, new, side in (("k", k, 0), ("v", s["v"], 1)):
            old = s["open"][slots[b], (lens[b] // P) % 2, :, side, :lens[b] - start].double().transpose(0, 1)
            x = torch.cat([old, new[off[b]:off[b + 1]].double()])
            for t in range(start, end - P + 1, P):
                y = x[t - start:t - start + P].transpose(0, 1)
                if side == 0 and box is not None:
                    u = _exact_unit(y.abs().amax((1, 2)), 127)[:, None]
                    page = table[b][t // P]
                    box[page, :, 0, :case["d"]] = torch.ceil(y.amax(1) / u) * u
                    box[page, :, 1, :case["d"]] = torch.floor(y.amin(1) / u) * u
                x[t - start:t - start + P] = _exact_codes(y, case["codes"]).transpose(0, 1)
            got[name][back[b]:back[b + 1]] = x
    res = dict(q=q, k=got["k"], v=got["v"], lens=s["lens"] + s["off"][1:] - s["off"][:-1])
    if box is not None:
        res["bounds"] = box
    return res


def _exact_page(s, page, head, side):
    """[P, d] of a full page, as it stands, in 64 bits."""
    case = s["case"]
    P, W = case["page"], _width(case["d"])
    c = s["codes"][page, head, side]
    x = (c.view(torch.int8) if case["codes"] == "i8" else c.view(torch.float8_e4m3fn)).double() * s["scales"][page, head, side].double()[..., None]
    if side == 0:
        x = x.view(-1, W // 16, P, 16).transpose(1, 2).reshape(-1, W)
    else:
        x = x.view(-1, P // 16, W, 16).transpose(2, 3).reshape(-1, W)
    return x[:, :case["d"]]


def _exact_rows(s, b, h, q, keys, k, v, pos):
    """Attention of one sequence's rows q [group, nq, d] over keys at positions `keys` [nk] or [nq, nk]."""
    case = s["case"]
    logits = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(case["d"])
    if case["cap"]:
        logits = case["cap"] * torch.tanh(logits / case["cap"])
    if s["slopes"] is not None:
        m = s["slopes"].view(case["hkv"], -1)[h].double()
        logits = logits - m[:, None, None] * (pos[:, None] - keys).abs()
    seen = (keys <= pos[:, None]) if case["causal"] else torch.ones_like(keys <= pos[:, None])
    logits = torch.where(seen, logits, -1e300)
    return torch.matmul(torch.softmax(logits, -1) * seen.any(-1, keepdim=True), v)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    hq, hkv, d, P, count = case["hq"], case["hkv"], case["d"], case["page"], case["count"]
    group = hq // hkv
    off, lens, slots = s["off"].tolist(), s["lens"].tolist(), s["slots"].tolist()
    sparse = case["kind"] == "sparse"
    if sparse and off[-1] * hkv > 6000 or case["seqs"] * hkv > 20000:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    pages = torch.full((off[-1], hkv, count), -1, dtype=torch.int32, device=DEV)
    for b in range(case["seqs"]):
        nq, nk = off[b + 1] - off[b], lens[b]
        if nq == 0 or nk == 0:
            continue
        nf = nk // P
        rows = slice(off[b], off[b + 1])
        pos = torch.arange(nq, device=DEV) + nk - nq
        ids = s["table"][b, :nf].long()
        q = s["q"][rows].double().view(nq, hkv, group, d)
        for h in range(hkv):
            tail = [s["open"][slots[b], nf % 2, h, side, :nk - nf * P].double() for side in (0, 1)]
            if not sparse:
                k, v = (torch.cat([_exact_page(s, ids, h, side), tail[side]]) for side in (0, 1))
                step = max(1, int(2e8 / (nq * nk)))  # query heads at a time
                for g in range(0, group, step):
                    one = slice(g, min(g + step, group))
                    if s["slopes"] is not None and step < group:
                        return None
                    o = _exact_rows(s, b, h, q[:, h, one].transpose(0, 1), torch.arange(nk, device=DEV)[None], k, v, pos)
                    out[rows, h * group + g:h * group + one.stop] = o.transpose(0, 1)
                continue
            for i in range(nq):
                p = int(pos[i])
                n = nf if not case["causal"] else max(0, min(nf, p // P + 1))
                pick = torch.zeros(0, dtype=torch.int64, device=DEV)
                if n:
                    x = q[i, h]
                    u = _exact_unit(x.abs().amax(-1), 127)
                    x = torch.round(x / u[:, None])
                    box = s["bounds"][ids[:n], h, :, :d].double()
                    whole = torch.maximum(x[:, None] * box[:, 0], x[:, None] * box[:, 1]).sum(-1)  # [group, n]
                    score = (whole * u[:, None]).amax(0) * s["units"][ids[:n], h].double()
                    pick = torch.sort(score, descending=True, stable=True).indices[:count].sort().values
                    pages[off[b] + i, h, :pick.numel()] = pick.to(torch.int32)
                keys = torch.cat([(pick[:, None] * P + torch.arange(P, device=DEV)).flatten(),
                                  torch.arange(nf * P, nk, device=DEV)])
                if keys.numel() == 0:
                    continue
                k, v = (torch.cat([_exact_page(s, ids[pick], h, side), tail[side]]) for side in (0, 1))
                o = _exact_rows(s, b, h, q[i:i + 1, h].transpose(0, 1), keys[None], k, v, pos[i:i + 1])
                out[off[b] + i, h * group:(h + 1) * group] = o[:, 0]
    return dict(pages=pages, out=out) if sparse else dict(out=out)
