"""Layer norm, forward and backward, against the formulas in 64 bits.

Tolerances (u = 2^-24, the rounding of one fp32 operation).  A sum of D terms is taken by at most 256 threads of at most
D / 256 + 32 consecutive terms each and a tree, so its error is at most (D / 256 + 48) u times the summed magnitudes;
`depth` is that count with room for the few operations around it.
  xhat    depth u (max|x - 0| rstd + |xhat|): the error of the mean and of the difference, against the row's spread
  y       |w| times that, 4 u (|xhat w| + |b|) for the products; bf16 adds half an ulp, 2^-8 of |y|
  dx      the magnitudes of its three terms times depth u, and the error of xhat through them
  dweight the rows are added in parts of at most rows / 1024 + 64 rows and the parts in a tree of 64 + 16
"""
import pytest
import torch

from paper_2509_20883_amd import recis as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5


def _ref(x, w, b, dy, mask, eps=EPS):
    """y, dx, dw, db and the error bounds of each, in float64."""
    x, dy = x.double(), dy.double()
    rows, dim = x.shape
    live = torch.ones(rows, 1, dtype=torch.bool, device=x.device) if mask is None else mask.view(-1, 1) != 0
    x, dy = torch.where(live, x, 0.0), torch.where(live, dy, 0.0)
    w = torch.ones(dim, device=x.device).double() if w is None else w.double()
    b = torch.zeros(dim, device=x.device).double() if b is None else b.double()
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    xhat = (x - mean) * rstd
    y = torch.where(live, xhat * w + b, 0.0)
    g = dy * w
    mg, mgx = g.mean(1, keepdim=True), (g * xhat).mean(1, keepdim=True)
    dx = torch.where(live, rstd * (g - mg - xhat * mgx), 0.0)
    dw, db = (dy * xhat).sum(0), dy.sum(0)
    depth = dim / 256 + 64
    exh = depth * U * (x.abs().amax(1, keepdim=True) * rstd + xhat.abs())
    ey = w.abs() * exh + 4 * U * ((xhat * w).abs() + b.abs())
    ag, agx = g.abs().mean(1, keepdim=True), (g * xhat).abs().mean(1, keepdim=True)
    edx = rstd * depth * U * (g.abs() + ag + xhat.abs() * agx)
    edx = edx + rstd * (exh * agx + xhat.abs() * (g.abs() * exh).mean(1, keepdim=True))
    rdepth = rows / 1024 + 64 + 80
    edw = (dy.abs() * exh).sum(0) + rdepth * U * (dy * xhat).abs().sum(0)
    edb = rdepth * U * dy.abs().sum(0)
    return dict(y=y, dx=dx, dw=dw, db=db, mean=mean.view(-1) * live.view(-1), rstd=rstd.view(-1) * live.view(-1)), \
        dict(y=ey, dx=edx, dw=edw, db=edb, mean=depth * U * x.abs().amax(1), rstd=2 * depth * U * rstd.view(-1) *
             (1 + (x.abs().amax(1, keepdim=True) * rstd).view(-1)))


def _close(got, want, bound, what):
    half_ulp = 2.0 ** -8 if got.dtype == torch.bfloat16 else U
    err = (got.double() - want).abs()
    lim = bound + half_ulp * (want.abs() + bound) + 1e-37
    bad = ~(err <= lim)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / lim).max()):.3g} of the bound"


def _inputs(rows, dim, dtype, ptype, seed, gap=0, scale=1.0, shift=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def mat():
        t = torch.empty(rows, dim + gap, device="cuda", dtype=dtype)
        t.copy_(torch.randn(rows, dim + gap, generator=g, device="cuda"))
        return t[:, :dim]

    x = mat()
    x.mul_(scale).add_(shift)
    dy = mat()
    w = (1 + 0.3 * torch.randn(dim, generator=g, device="cuda")).to(ptype)
    b = torch.randn(dim, generator=g, device="cuda").to(ptype)
    return x, dy, w, b


def _check(x, dy, w, b, mask=None, op=None):
    op = op or R.LayerNorm(EPS)
    y, mean, rstd = op.forward(x, w, b, mask=mask)
    dx, dw, db = op.backward(dy, x, mean, rstd, w, mask=mask)
    assert y.dtype == dx.dtype == x.dtype and dw.dtype == (w.dtype if w is not None else torch.float32)
    want, bound = _ref(x, w, b, dy, mask)
    for name, got in (("y", y), ("mean", mean), ("rstd", rstd), ("dx", dx), ("dw", dw), ("db", db)):
        _close(got, want[name], bound[name], name)
    return y, dx, dw, db


DIMS = [1, 2, 3, 7, 8, 16, 31, 64, 100, 128, 256, 257, 264, 512, 1000, 1024, 1032, 2040, 2047, 2048, 2049, 2056, 4096, 4104,
        5000, 8191, 8192, 8193, 8200, 20000]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", DIMS)
def test_widths(dim, dtype):
    print("layer norm", dim, dtype, flush=True)
    for rows, ptype in ((1, torch.float32), (37, torch.bfloat16), (301, dtype)):
        x, dy, w, b = _inputs(rows, dim, dtype, ptype, dim * 7 + rows)
        _check(x, dy, w, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim,gap", [(64, 8), (64, 1), (128, 65), (129, 7), (1024, 1), (1025, 7), (2048, 3), (4096, 8)])
def test_strided_rows(dim, gap, dtype):
    print("strided", dim, gap, dtype, flush=True)
    x, dy, w, b = _inputs(77, dim, dtype, torch.float32, dim + gap, gap=gap)
    _check(x, dy, w, b)
    # an offset of one element moves every row off the wide accesses' alignment
    flat = torch.randn(77 * dim + 1, device="cuda").to(dtype)
    _check(flat[1:].view(77, dim), dy, w, b)
    # transposed memory is copied
    _check(torch.randn(dim, 77, device="cuda").to(dtype).t(), dy, w, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [7, 16, 64, 128, 1024, 2047, 8192, 9000])
def test_masked_rows_are_not_read(dim, dtype):
    print("masked", dim, dtype, flush=True)
    bags, pad = 23, 19
    x, dy, w, b = _inputs(bags * pad, dim, dtype, torch.float32, dim)
    lens = torch.randint(0, pad + 1, (bags,), device="cuda")
    lens[0], lens[1] = 0, pad
    mask = (torch.arange(pad, device="cuda") < lens[:, None]).to(torch.uint8)
    dead = mask.view(-1) == 0
    x[dead] = float("nan")
    dy[dead] = float("inf")
    y, dx, dw, db = _check(x, dy, w, b, mask=mask)
    assert not y[dead].any() and not dx[dead].any()
    # the same in the padded copy's own shape, and with a bool mask
    op = R.LayerNorm(EPS)
    y3, mean, rstd = op.forward(x.view(bags, pad, dim), w, b, mask=mask != 0)
    dx3, _, _ = op.backward(dy.view(bags, pad, dim), x.view(bags, pad, dim), mean, rstd, w, mask=mask != 0)
    assert y3.shape == (bags, pad, dim) and mean.shape == (bags, pad)
    assert torch.equal(y3.view(-1, dim), y) and torch.equal(dx3.view(-1, dim), dx)
    # every row masked
    none = torch.zeros(bags * pad, dtype=torch.uint8, device="cuda")
    y, mean, rstd = op.forward(x, w, b, mask=none)
    dx, dw, db = op.backward(dy, x, mean, rstd, w, mask=none)
    assert not y.any() and not dx.any() and not dw.any() and not db.any() and not mean.any() and not rstd.any()


@pytest.mark.parametrize("rows", [0, 1, 15, 16, 17, 63, 65, 1023, 4097, 70001])
def test_row_counts(rows):
    print("rows", rows, flush=True)
    for dim, dtype in ((32, torch.float32), (128, torch.bfloat16), (33, torch.float32)):
        x, dy, w, b = _inputs(rows, dim, dtype, torch.float32, rows + dim)
        if rows == 0:
            op = R.LayerNorm(EPS)
            y, mean, rstd = op.forward(x, w, b)
            dx, dw, db = op.backward(dy, x, mean, rstd, w)
            assert y.shape == dx.shape == (0, dim) and not dw.any() and not db.any()
        else:
            _check(x, dy, w, b)


@pytest.mark.parametrize("dim", [64, 1000, 4096, 10000])
def test_values(dim):
    """Rows far from zero, of one value, of very large and very small values; no weight or no bias."""
    print("values", dim, flush=True)
    x, dy, w, b = _inputs(64, dim, torch.float32, torch.float32, dim)
    _check(x * 1e-3 + 1000.0, dy, w, b)
    _check(x * 1e15, dy, w, b)
    x2 = x * 1e-20
    x2[5] = 3.25  # constant: xhat 0, rstd 1 / sqrt(eps)
    _check(x2, dy, w, b)
    _check(x, dy, None, b)
    _check(x, dy, w, None)
    _check(x, dy, None, None)
    # NaN and infinity stay in their row of y and dx
    x3 = x.clone()
    x3[3, dim // 2], x3[9, 0] = float("nan"), float("inf")
    op = R.LayerNorm(EPS)
    y, mean, rstd = op.forward(x3, w, b)
    dx, _, _ = op.backward(dy, x3, mean, rstd, w)
    keep = torch.ones(64, dtype=torch.bool, device="cuda")
    keep[3] = keep[9] = False
    assert torch.isfinite(y[keep]).all() and torch.isfinite(dx[keep]).all()
    assert torch.isnan(y[3]).all() and torch.isnan(dx[3]).all() and torch.isnan(y[9, 0])


@pytest.mark.parametrize("dim", [5, 64, 2050])
def test_gradient_against_differences(dim):
    """Central differences of a weighted sum of the forward's fp32 output along random directions.  With step h the
    truncation is O(h^2) and the outputs' rounding enters as u / h: h = 1e-2 keeps both below 2e-3 of the magnitudes."""
    print("differences", dim, flush=True)
    x, dy, w, b = _inputs(6, dim, torch.float32, torch.float32, dim)
    op = R.LayerNorm(EPS)
    y, mean, rstd = op.forward(x, w, b)
    grads = op.backward(dy, x, mean, rstd, w)
    h = 1e-2
    g = torch.Generator(device="cuda").manual_seed(dim)
    for at, grad in enumerate(grads):
        v = torch.randn(grad.shape, generator=g, device="cuda")
        v = v / v.norm()
        args = [x, w, b]
        val = []
        for sign in (1, -1):
            moved = [t + sign * h * v if k == at else t for k, t in enumerate(args)]
            val.append((op.forward(*moved)[0].double() * dy.double()).sum())
        diff = float(val[0] - val[1]) / (2 * h)
        got = float((grad.double() * v.double()).sum())
        mag = float((grad.double() ** 2).sum().sqrt()) + 1.0
        assert abs(diff - got) <= 2e-3 * mag, (at, diff, got)


def test_repeats_streams_and_workspace():
    """Bit-equal repeats; one object's workspace over sizes that shrink and grow; a stream of its own."""
    op = R.LayerNorm(EPS)
    for rows, dim in ((5000, 128), (70, 1024), (9000, 2048), (3, 9), (20000, 64)):
        x, dy, w, b = _inputs(rows, dim, torch.float32, torch.float32, rows)
        first = _check(x, dy, w, b, op=op)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            own = R.LayerNorm(EPS)
            y, mean, rstd = own.forward(x, w, b)
            second = (y, *own.backward(dy, x, mean, rstd, w))
        s.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(first, second))


def test_more_than_2_31_elements():
    rows, dim = 17000003, 128
    print("large", rows, dim, flush=True)
    x = torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    block = torch.randn(1 << 16, dim, generator=g, device="cuda").to(torch.bfloat16)
    for r in range(0, rows, 1 << 16):
        x[r:r + (1 << 16)] = block[:min(1 << 16, rows - r)]
    w, b = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
    op = R.LayerNorm(EPS)
    y, mean, rstd = op.forward(x, w, b)
    dx, dw, db = op.backward(x, x, mean, rstd, w)
    want, bound = _ref(block, w, b, block, None)
    for r in (0, 16777216 - 65536, 16777216, rows // 65536 * 65536):
        n = min(65536, rows - r)
        _close(y[r:r + n], want["y"][:n], bound["y"][:n], "y")
        _close(dx[r:r + n], want["dx"][:n], bound["dx"][:n], "dx")
    copies, tail = divmod(rows, 65536)
    t_want, _ = _ref(block[:tail], w, b, block[:tail], None)
    total = want["dw"] * copies + t_want["dw"]
    mag = (block.double().abs() * ((block.double() - 0).abs() + 1) * 1.5).sum(0) * (copies + 1)
    _close(dw, total, (rows / 1024 + 64 + 80) * U * mag, "dw")


def test_refusals():
    x = torch.randn(4, 8, device="cuda")
    w = torch.ones(8, device="cuda")
    op = R.LayerNorm(EPS)
    y, mean, rstd = op.forward(x, w, w)
    for bad in (lambda: op.forward(x.half(), w, w), lambda: op.forward(x, w[:7], w), lambda: op.forward(x, w.half(), w),
                lambda: op.forward(x, w.bfloat16(), w), lambda: op.forward(x.cpu(), w, w),
                lambda: op.forward(x, w, w, mask=torch.ones(3, dtype=torch.uint8, device="cuda")),
                lambda: op.forward(x, w, w, mask=torch.ones(4, dtype=torch.int64, device="cuda")),
                lambda: op.forward(x, w, w, out=torch.empty(4, 9, device="cuda")),
                lambda: op.forward(torch.empty(4, 0, device="cuda")),
                lambda: R.LayerNorm(-1.0).forward(x, w, w), lambda: R.LayerNorm(float("nan")).forward(x, w, w),
                lambda: op.backward(x.bfloat16(), x, mean, rstd, w), lambda: op.backward(x[:3], x, mean, rstd, w),
                lambda: op.backward(x, x, mean[:2], rstd, w), lambda: op.backward(x, x, mean.double(), rstd, w)):
        with pytest.raises(R.RecisError) as e:
            bad()
        assert e.value.status == R.EINVAL
    # the C boundary itself
    L, p = R.lib(), x.data_ptr()
    fwd = [p, 4, 8, 8, R.F32, None, None, R.F32, 1e-5, None, y.data_ptr(), 8, None, None, None]
    for at, v in ((0, None), (1, -1), (1, 1 << 31), (2, 0), (2, (1 << 24) + 1), (3, 7), (4, 2), (7, 5), (8, -1.0),
                  (10, None), (11, 7), (3, 1 << 32)):
        args = list(fwd)
        args[at] = v
        assert L.layer_norm_fwd(*args) == R.EINVAL and L.rs_last_error()
    ws = torch.empty(L.layer_norm_bwd_workspace_bytes(4, 8), dtype=torch.uint8, device="cuda")
    dp = torch.empty(2, 8, device="cuda")
    bwd = [p, 8, p, 4, 8, 8, R.F32, None, R.F32, None, mean.data_ptr(), rstd.data_ptr(), y.data_ptr(), 8,
           dp.data_ptr(), dp[1].data_ptr(), ws.data_ptr(), ws.numel(), None]
    for at, v in ((0, None), (1, 7), (2, None), (3, -1), (4, 0), (5, 3), (6, 9), (8, 9), (10, None), (11, None), (13, 7),
                  (16, None), (16, ws.data_ptr() + 4), (17, ws.numel() - 1)):
        args = list(bwd)
        args[at] = v
        assert L.layer_norm_bwd(*args) == R.EINVAL and L.rs_last_error()
    assert L.layer_norm_bwd_workspace_bytes(-1, 8) == 0 and L.layer_norm_bwd_workspace_bytes(4, 0) == 0
    # gradients that are not wanted need no workspace
    args = list(bwd)
    args[14] = args[15] = args[16] = None
    args[17] = 0
    assert L.layer_norm_bwd(*args) == R.OK
    torch.cuda.synchronize()
