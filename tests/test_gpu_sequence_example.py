"""The sequence operators together with the embedding step, as the example runs them."""
import pytest
import torch

from examples import sequence_encoder as E
from paper_2509_20883_amd import recis as R

pytestmark = pytest.mark.gpu


def test_training_learns_and_serving_agrees_with_the_formula():
    print("example", flush=True)
    model, table, losses = E.train(steps=25, bags=128, pad=64, dim=32, heads=4, vocab=2000)
    assert all(x == x for x in losses) and sum(losses[-5:]) < 0.6 * sum(losses[:5]), losses
    # a candidate's score from the same rows in plain torch: bf16 operands of three products in a row, each rounded
    history = torch.randint(0, 2000, (700,), generator=torch.Generator().manual_seed(1)).cuda()
    candidates = torch.arange(5, device="cuda")
    got = E.serve(model, table, history, candidates)
    ids = torch.cat([history, candidates])
    rows = table.read_rows(table.find(ids))[0].double()
    c = rows - rows.mean(1, keepdim=True)
    x = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * model.gain.detach().double() + model.shift.detach().double()
    h, kv, d, n = model.heads, model.kv_heads, model.d, history.numel()
    q, k, v = (x @ model.qkv.detach().double()).view(-1, h + 2 * kv, d).split([h, kv, kv], 1)
    k, v = (t[:n].repeat_interleave(h // kv, 1).transpose(0, 1) for t in (k, v))
    p = torch.softmax(q[n:].transpose(0, 1) @ k.transpose(1, 2) / d ** 0.5, 2)
    out = (p @ v).transpose(0, 1).reshape(candidates.numel(), -1)
    want = ((rows[n:] + out @ model.proj.detach().double()) @ model.head.detach().double()).squeeze(1)
    # each of the six bf16 roundings on the way is off by at most 2^-8 of its value; their magnitudes reach the score
    # through |proj| and |head|
    mag = ((rows[n:].abs() + out.abs() @ model.proj.detach().double().abs()) @ model.head.detach().double().abs()).squeeze(1)
    assert ((got.double() - want).abs() <= 6 * 2.0 ** -8 * mag + 1e-3).all(), (got, want)
    table.close()


def test_gradient_reaches_the_rows():
    """The padded copy's gradient through norm, attention and projection is zero past each sequence's end and otherwise
    what autograd gives for the same block in float64 (three bf16 roundings of operands on the way)."""
    print("gradient", flush=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    model = E.Encoder(32, 2, 1)
    lens = torch.tensor([5, 0, 17, 9], device="cuda")
    offsets = torch.zeros(5, dtype=torch.int64, device="cuda")
    torch.cumsum(lens, 0, out=offsets[1:])
    mask = (torch.arange(17, device="cuda") < lens[:, None]).to(torch.uint8)
    rows = (torch.randn(4, 17, 32, generator=g, device="cuda") * mask[..., None]).bfloat16().requires_grad_()
    model.scores(rows, mask, offsets).sum().backward()
    assert not rows.grad[mask == 0].any()
    x = rows.detach().double().requires_grad_()
    total = 0.0
    for b, n in enumerate(lens.tolist()):
        if n == 0:
            continue
        r = x[b, :n]
        c = r - r.mean(1, keepdim=True)
        y = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5)
        q, k, v = (y @ model.qkv.detach().double()).view(n, 4, 16).split([2, 1, 1], 1)
        i = torch.arange(n, device="cuda")
        s = q.transpose(0, 1) @ k.transpose(0, 1).transpose(1, 2) / 4 - model.slopes.detach().double()[:, None, None] * (
            i[:, None] - i).abs()
        p = torch.softmax(s.masked_fill(i[None, :] > i[:, None], -torch.inf), 2)
        h = r + (p @ v.transpose(0, 1)).transpose(0, 1).reshape(n, -1) @ model.proj.detach().double()
        total = total + (h.mean(0) @ model.head.detach().double()).sum()
    total.backward()
    diff = (rows.grad.double() - x.grad).norm() / x.grad.norm()
    assert diff < 12 * 2.0 ** -8, float(diff)
