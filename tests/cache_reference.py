"""The paged cache's formulas in 64 bits, from its memory as the header describes it."""
import math

import torch

U = 2.0 ** -24


def width(d):
    return 32 if d <= 32 else 64 if d <= 64 else 128


def offsets(lens, device="cuda"):
    return torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int64, device=device)


def unit(top, most):
    """The least power of two s >= 2^-126 with top <= most s, elementwise in float64."""
    m, e = math.frexp(most)
    out = []
    for x in top.flatten().tolist():
        k = -126
        if x > 0:
            xm, xe = math.frexp(x)
            k = max(-126, xe - e + (1 if xm > m else 0))
        out.append(2.0 ** k)
    return torch.tensor(out, dtype=torch.float64, device=top.device).view(top.shape)


def encode(x, codes):
    """Codes' values (whole numbers, or e4m3 numbers) and scale of [..., P, d], over the last two axes."""
    top = x.double().abs().amax((-1, -2), keepdim=True)
    if codes == "i8":
        # in 64 bits first: a float32 tensor over a number may be taken as a product by its reciprocal, off by a bit
        s = torch.clamp((top / 127).float(), min=2.0 ** -126).double()
        return torch.round(x.double() / s), s
    s = unit(top, 448)
    return (x.double() / s).float().to(torch.float8_e4m3fn).double(), s


def bounds(x):
    """[..., 2, d] whole numbers and the unit of [..., P, d]."""
    u = unit(x.double().abs().amax((-1, -2)), 127)
    y = x.double() / u[..., None, None]
    return torch.stack([y.amax(-2).ceil(), y.amin(-2).floor()], -2), u


def pages_of(c):
    """Code values of every page, [pages, hkv, 2, P, d], and scales [pages, hkv, 2], both in float64."""
    n, h, P, d, W = c.codes.shape[0], c.heads_kv, c.page, c.head_dim, width(c.head_dim)
    raw = c.codes.view(torch.float8_e4m3fn).float() if c._desc.codes else c.codes.view(torch.int8)
    raw = raw.double()
    k = raw[:, :, 0].view(n, h, W // 16, P, 16).transpose(2, 3).reshape(n, h, P, W)
    v = raw[:, :, 1].view(n, h, P // 16, W, 16).transpose(3, 4).reshape(n, h, P, W)
    return torch.stack([k, v], 2)[..., :d], c.scales.double()


def fill(c, seed, spread=1.0):
    """Random pages and open pages, as an append would leave them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, h, P, d, W = c.codes.shape[0], c.heads_kv, c.page, c.head_dim, width(c.head_dim)
    codes = "e4m3" if c._desc.codes else "i8"
    x = torch.randn(n, h, 2, P, d, generator=g, device="cuda") * spread
    x[:, :, 0] += torch.randn(n, h, 1, d, generator=g, device="cuda")
    q, s = encode(x, codes)
    raw = torch.zeros(n, h, 2, P, W, device="cuda")
    raw[..., :d] = q.float()
    raw = raw.to(torch.float8_e4m3fn).view(torch.uint8) if c._desc.codes else raw.to(torch.int8).view(torch.uint8)
    c.codes[:, :, 0] = raw[:, :, 0].view(n, h, P, W // 16, 16).transpose(2, 3).reshape(n, h, P * W)
    c.codes[:, :, 1] = raw[:, :, 1].view(n, h, P // 16, 16, W).transpose(3, 4).reshape(n, h, P * W)
    c.scales.copy_(s.view(n, h, 2))
    c.open.copy_(torch.randn(c.open.shape, generator=g, device="cuda") * spread)
    if c.bounds is not None:
        b, u = bounds(x[:, :, 0])
        c.bounds.zero_()
        c.bounds[..., :d] = b.to(torch.int8)
        c.units.copy_(u)
    return g


def tokens_of(c, table, lens, slots):
    """Per sequence: keys, values [len, hkv, d] in float64, and for each token whether its page is there."""
    vals, scales = pages_of(c)
    out = []
    for b, n in enumerate(lens):
        P = c.page
        n = min(max(n, 0), table.shape[1] * P)
        nf = n // P
        ids = table[b, :nf].tolist()
        there = [0 <= i < c.codes.shape[0] for i in ids]
        x = torch.zeros(2, n, c.heads_kv, c.head_dim, dtype=torch.float64, device="cuda")
        seen = torch.zeros(n, dtype=torch.bool, device="cuda")
        for i, (p, ok) in enumerate(zip(ids, there)):
            if ok:
                y = vals[p] * scales[p][..., None, None]  # [hkv, 2, P, d]
                x[:, i * P:(i + 1) * P] = y.permute(1, 2, 0, 3)
                seen[i * P:(i + 1) * P] = True
        if n > nf * P and 0 <= slots[b] < c.open.shape[0]:
            x[:, nf * P:] = c.open[slots[b], nf % 2, :, :, :n - nf * P].double().permute(1, 2, 0, 3)
            seen[nf * P:] = True
        out.append((x[0], x[1], seen))
    return out


def attention(q, k, v, pos, key_pos, weight, causal, cap, slopes, scale, bf16, group):
    """out and its error bound, [nq, hq, d]: q [nq, hq, d], k, v [nk, hkv, d], weight [nk]: how often a key counts (0: not).

    The bound: a score is a dot product of d terms in up to six products of pieces, (6 d + 16) u of its summed magnitudes;
    cap 4e-7 of it in bf16 (tanh to about 1e-7) and 4 u in fp32; the other operations 8 u of the score and the distance term.
    A probability is off by its score's error and the largest of its row (the normaliser's), relative, and 16 u; as an operand
    by 2^-8 in bf16.  The sums take (nk + 64) u of their magnitudes, twice where splits are joined."""
    r = 2.0 ** -8 if bf16 else 0.0
    d, nk = q.shape[-1], k.shape[0]
    Q = q.double().transpose(0, 1)
    K, V = (t.transpose(0, 1).repeat_interleave(group, 0) for t in (k, v))
    x = Q @ K.transpose(1, 2) * scale
    es = (6 * d + 16) * U * (Q.abs() @ K.abs().transpose(1, 2)) * scale
    if cap:
        x = cap * torch.tanh(x / cap)
        es = es + (4e-7 if bf16 else 4 * U) * cap
    dist = (pos[:, None] - key_pos[None]).abs().double()
    if slopes is not None:
        m = slopes.double().view(-1, 1, 1)
        x = x - m * dist
        es = es + 8 * U * m.abs() * dist
    es = es + 8 * U * x.abs()
    see = (weight > 0)[None] & ((key_pos[None] <= pos[:, None]) if causal else torch.ones(1, 1, dtype=torch.bool, device=q.device))
    x = torch.where(see, x, -math.inf)
    some = see.any(1)
    lse = torch.logsumexp(x + weight.clamp(min=1).double().log(), 2) if nk else torch.zeros(Q.shape[:2], dtype=torch.float64, device=q.device)
    P = torch.where(see & some[:, None], torch.exp(x - torch.where(torch.isfinite(lse), lse, 0.0)[..., None]), 0.0) * weight
    es = torch.where(see, es, 0.0)
    e = es + (es.amax(2, keepdim=True) if nk else 0.0) + 16 * U
    out = P @ V
    eout = (P * (e + r + (2 * nk + 128) * U)) @ V.abs() + (r + 4 * U) * out.abs()
    return out.transpose(0, 1), eout.transpose(0, 1)


def turned(x, pos, freqs, rotary, interleaved):
    """Rows [rows, heads, d] turned by their positions, float64."""
    y = x.double().clone()
    w = pos.double()[:, None] * torch.tensor(freqs, dtype=torch.float64, device=x.device)
    c, s = torch.cos(w)[:, None], torch.sin(w)[:, None]
    h = rotary // 2
    a, b = (y[..., 0:rotary:2].clone(), y[..., 1:rotary:2].clone()) if interleaved else (y[..., :h].clone(), y[..., h:rotary].clone())
    p, q = a * c - b * s, b * c + a * s
    if interleaved:
        y[..., 0:rotary:2], y[..., 1:rotary:2] = p, q
    else:
        y[..., :h], y[..., h:rotary] = p, q
    return y


def select(q, c, table_row, lens, pos, count, causal):
    """Page numbers of one row, [hkv][<= count], by whole numbers in Python's order; q [hq, d]."""
    P, hkv = c.page, c.heads_kv
    group = q.shape[0] // hkv
    n = min(max(lens, 0), len(table_row) * P) // P
    if causal:
        n = min(n, 0 if pos < 0 else pos // P + 1)
    res = []
    for h in range(hkv):
        x = q[h * group:(h + 1) * group].double()
        finite = torch.isfinite(x).all(1, keepdim=True)
        x = torch.where(finite, x, 0.0)
        sq = unit(x.abs().amax(1), 127)
        sq = torch.where(finite[:, 0], sq, 1.0)
        q8 = torch.round(x / sq[:, None])
        ids = torch.tensor(table_row[:n], dtype=torch.int64, device=q.device)
        ok = (ids >= 0) & (ids < c.codes.shape[0])
        box = c.bounds[ids.clamp(0, c.codes.shape[0] - 1), h, :, :c.head_dim].double()  # [n, 2, d]
        whole = torch.maximum(q8[:, None] * box[None, :, 0], q8[:, None] * box[None, :, 1]).sum(2)  # [group, n]
        score = (whole * sq[:, None]).amax(0) * c.units[ids.clamp(0, c.codes.shape[0] - 1), h].double()
        score = torch.where(score.isnan(), math.inf, score)
        score = torch.where(ok, score, -math.inf).tolist()
        best = sorted(range(n), key=lambda i: (-score[i], i))[:count]
        res.append(sorted(best))
    return res
