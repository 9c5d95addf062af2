"""Layer norm and its gradient against the formulas in 64 bits.

Tolerances (u = 2^-24): a row's sums are taken in at most A = 40 + d / 256 roundings one after the other, so
mu is within A u mean|x|, the sum of squares within (A + 2) u of itself plus what mu's error moves, 1/r likewise;
outputs add one rounding of their type.  The weight's gradient adds n terms: n u sum|terms|.
"""
import pytest
import torch

from paper_2311_14908_amd import svmx

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-5
# lanes of a wave (one to 64), 2 and 4 units a lane, a workgroup a row, rows read again
DIMS = [1, 2, 3, 5, 8, 31, 64, 100, 256, 301, 513, 784, 1023, 1024, 1025, 2049, 4095, 4100, 8191, 8200, 20001]
KINDS = [(F32, F32, F32), (BF16, BF16, F32), (BF16, F32, BF16), (F16, F16, F16), (F16, F32, F32), (BF16, BF16, BF16)]  # x, y, weight


def inputs(n, d, kind, seed, shift=0.5):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, d, generator=g) * (0.5 + torch.rand(n, 1, generator=g)) + shift).to(kind[0])
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(kind[2])
    b = torch.randn(d, generator=g).to(kind[2])
    dy = torch.randn(n, d, generator=g).to(kind[1])
    return x, w, b, dy


def stats64(x):
    x = x.double()
    mu = x.mean(1, keepdim=True)
    var = (x - mu).square().mean(1, keepdim=True)
    return x, mu, 1 / torch.sqrt(var + EPS)


def stat_errors(x):
    """Bounds on mu and, relative, on r."""
    x, mu, r = stats64(x)
    A = 40 + x.shape[1] / 256
    emu = A * U * x.abs().mean(1, keepdim=True) + U * mu.abs()
    c = (x - mu).abs()
    er = ((A + 4) * U * c.square().mean(1, keepdim=True) + 2 * emu * (emu + U * x.abs().mean(1, keepdim=True))
          + 2 * U * (c * x.abs()).mean(1, keepdim=True)) * r * r + 4 * U
    return x, mu, r, emu, er


def close(got, ref, err):
    got64 = got.cpu().double()
    lim = err + HALF_ULP[got.dtype] * (ref.abs() + err) * (1 + 2 ** -6) + (2.0 ** -24 if got.dtype == F16 else 1e-44)
    worst = ((got64 - ref).abs() - lim).max().item() if ref.numel() else 0.0
    assert worst <= 0, worst


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", DIMS)
def test_forward(d, kind):
    for n in (1, 3, 70):
        x, w, b, _ = inputs(n, d, kind, d + n)
        y, mean, rstd = svmx.svm_layernorm(x.cuda(), w.cuda(), b.cuda(), EPS, out_dtype=kind[1])
        x64, mu, r, emu, er = stat_errors(x)
        h = (x64 - mu) * r
        ref = h * w.double() + b.double()
        err = (r * (emu + U * (x64.abs() + mu.abs())) + h.abs() * (er + 3 * U)) * w.double().abs() + U * ref.abs()
        assert y.dtype == kind[1]
        close(y, ref, err)
        close(mean, mu[:, 0], emu[:, 0])
        close(rstd, r[:, 0], (r * er)[:, 0])


def grad64(dy, x, mean, rstd, w):
    """In 64 bits from the kept mean and rstd, and each result's size for the bound."""
    dy, w = dy.double(), w.double()
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    q = dy * w
    r = rstd.double()[:, None]
    m1, m2 = q.mean(1, keepdim=True), (q * h).mean(1, keepdim=True)
    a1, a2 = q.abs().mean(1, keepdim=True), (q * h).abs().mean(1, keepdim=True)
    dx = r * (q - m1 - h * m2)
    A = 40 + x.shape[1] / 256
    # h itself is within 2 u of x - mu's parts
    eh = 3 * U * r * (x.double().abs() + mean.double().abs()[:, None])
    a3 = (q.abs() * eh).mean(1, keepdim=True)
    ex = r * (4 * U * q.abs() + A * U * (a1 + h.abs() * a2) + h.abs() * a3 + eh * a2 + 4 * U * (m1.abs() + (h * m2).abs()))
    return dx, ex, dy, h, eh


def check_grad(dy, x, mean, rstd, w, got):
    dx, dw, db = got
    refx, ex, dy64, h, eh = grad64(dy, x, mean, rstd, w)
    n = x.shape[0]
    close(dx, refx, ex)
    close(dw, (dy64 * h).sum(0), (n + 4) * U * (dy64 * h).abs().sum(0) + (dy64.abs() * eh).sum(0))
    close(db, dy64.sum(0), (n + 4) * U * dy64.abs().sum(0))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", DIMS)
def test_gradient(d, kind):
    for n in (1, 2, 37, 400 if d <= 4100 else 50):
        x, w, _, dy = inputs(n, d, kind, 7 * d + n)
        _, mu, r = stats64(x)
        mean, rstd = mu[:, 0].float(), r[:, 0].float()
        args = [t.cuda() for t in (dy, x, mean, rstd, w)]
        got = svmx.svm_layernorm_grad(*args)
        assert [t.dtype for t in got] == [kind[0], kind[2], kind[2]]
        check_grad(dy, x, mean, rstd, w, got)
        assert all(torch.equal(a, b) for a, b in zip(got, svmx.svm_layernorm_grad(*args)))


def test_many_rows_of_few_features():
    for d, n in ((3, 50001), (64, 33000), (784, 9000)):
        x, w, _, dy = inputs(n, d, KINDS[0], d)
        _, mu, r = stats64(x)
        mean, rstd = mu[:, 0].float(), r[:, 0].float()
        check_grad(dy, x, mean, rstd, w, svmx.svm_layernorm_grad(*[t.cuda() for t in (dy, x, mean, rstd, w)]))
        y, m2, _ = svmx.svm_layernorm(x.cuda(), w.cuda(), None, EPS)
        assert (y.cpu().double() - (x.double() - mu) * r * w.double()).abs().max() <= 1e-5 * 20  # |h w| < 20, u x 100
        assert (m2.cpu() - mean).abs().max() <= 1e-5


def test_no_weight_no_rows_and_constants():
    x = torch.full((5, 40), 3.25)
    y, mean, rstd = svmx.svm_layernorm(x.cuda())
    assert bool((y == 0).all()) and bool((mean == 3.25).all())
    assert (rstd.cpu().double() - EPS ** -0.5).abs().max() <= 4 * U * EPS ** -0.5
    dx, dw, db = svmx.svm_layernorm_grad(torch.ones(5, 40).cuda(), x.cuda(), mean, rstd)
    assert dw.dtype == F32 and bool((dw == 0).all()) and bool((db == 5).all()) and bool((dx.abs() <= 1e-3).all())
    e = torch.empty(0, 40).cuda()
    y, mean, rstd = svmx.svm_layernorm(e, torch.ones(40).cuda())
    assert y.shape == (0, 40) and mean.shape == (0,)
    dx, dw, db = svmx.svm_layernorm_grad(e, e, mean, rstd, torch.ones(40).cuda())
    assert dx.shape == (0, 40) and bool((dw == 0).all()) and bool((db == 0).all())


def test_large_mean():
    """A mean a thousand times the spread: the variance is a sum of squared differences, not a difference of sums."""
    x = 1000.0 + torch.randn(9, 500, generator=torch.Generator().manual_seed(3))
    y, _, _ = svmx.svm_layernorm(x.cuda())
    x64, mu, r, emu, er = stat_errors(x)
    close(y, (x64 - mu) * r, r * (emu + U * (x64.abs() + mu.abs())) + ((x64 - mu) * r).abs() * (er + 3 * U))


def test_rows_are_their_own():
    """Infinities and NaN of one row stay in it."""
    for d in (40, 300, 2000, 9000):
        x = torch.randn(6, d, generator=torch.Generator().manual_seed(d))
        clean, _, _ = svmx.svm_layernorm(x.cuda())
        x[1, 3], x[4, d - 1] = float("nan"), float("inf")
        y, mean, rstd = svmx.svm_layernorm(x.cuda())
        keep = torch.tensor([0, 2, 3, 5])
        assert torch.equal(y.cpu()[keep], clean.cpu()[keep]) and bool(y[1].isnan().all()) and bool(y[4].isnan().any())


def test_pitch_and_alignment():
    for kind in KINDS:
        for d in (37, 301, 1100):
            x, w, b, dy = inputs(33, d, kind, d)
            wide = [torch.zeros(33, d + 9, dtype=t.dtype).cuda() for t in (x, dy)]
            wide[0][:, 3:3 + d], wide[1][:, 5:5 + d] = x.cuda(), dy.cuda()
            y0, m0, r0 = svmx.svm_layernorm(x.cuda(), w.cuda(), b.cuda(), EPS, out_dtype=kind[1])
            y1, m1, r1 = svmx.svm_layernorm(wide[0][:, 3:3 + d], w.cuda(), b.cuda(), EPS, out_dtype=kind[1])
            assert torch.equal(y0, y1) and torch.equal(m0, m1) and torch.equal(r0, r1)
            g0 = svmx.svm_layernorm_grad(dy.cuda(), x.cuda(), m0, r0, w.cuda())
            g1 = svmx.svm_layernorm_grad(wide[1][:, 5:5 + d], wide[0][:, 3:3 + d], m0, r0, w.cuda())
            assert all(torch.equal(a, c) for a, c in zip(g0, g1))


def test_gradient_is_the_difference_quotient():
    """Central differences of the formula in 64 bits (step 1e-5: within 1e-8 of the derivative)."""
    x, w, b, dy = inputs(3, 19, KINDS[0], 2)
    f = lambda x, w, b: ((x - x.mean(1, keepdim=True)) / torch.sqrt(x.var(1, correction=0, keepdim=True) + EPS) * w + b)
    args = [t.double() for t in (x, w, b)]
    _, mean, rstd = svmx.svm_layernorm(x.cuda(), w.cuda(), b.cuda(), EPS)
    got = svmx.svm_layernorm_grad(dy.cuda(), x.cuda(), mean, rstd, w.cuda())
    for k in range(3):
        flat = args[k].reshape(-1)
        for i in range(flat.numel()):
            old = flat[i].item()
            flat[i] = old + 1e-5
            up = (f(*args) * dy.double()).sum()
            flat[i] = old - 1e-5
            down = (f(*args) * dy.double()).sum()
            flat[i] = old
            num = (up - down) / 2e-5
            assert abs(num - got[k].reshape(-1)[i].item()) <= 1e-5 * (1 + abs(num))  # sums of 57 terms near 1, 2^-24 each


def test_on_another_stream_and_in_a_graph():
    x, w, b, dy = (t.cuda() for t in inputs(300, 784, KINDS[0], 1))
    want, mean, rstd = svmx.svm_layernorm(x, w, b)
    wantg = svmx.svm_layernorm_grad(dy, x, mean, rstd, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _, _ = svmx.svm_layernorm(x, w, b, stream=side)
    gotg = svmx.svm_layernorm_grad(dy, x, mean, rstd, w, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and all(torch.equal(p, q) for p, q in zip(gotg, wantg))
    graph = torch.cuda.CUDAGraph()
    x0 = x.clone()
    with torch.cuda.graph(graph):
        y, m, r = svmx.svm_layernorm(x, w, b)
        gs = svmx.svm_layernorm_grad(dy, x, m, r, w)
    for k in range(3):
        x.copy_(x0 * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        y2, m2, r2 = svmx.svm_layernorm(x, w, b)
        assert torch.equal(y, y2) and all(torch.equal(p, q) for p, q in zip(gs, svmx.svm_layernorm_grad(dy, x, m2, r2, w)))


def test_binding_refusals():
    x, w = torch.randn(4, 8).cuda(), torch.ones(8).cuda()
    for bad in (lambda: svmx.svm_layernorm(x.cpu()), lambda: svmx.svm_layernorm(x.t()), lambda: svmx.svm_layernorm(x, w[:7]),
                lambda: svmx.svm_layernorm(x, w, w.half()), lambda: svmx.svm_layernorm(x.double()),
                lambda: svmx.svm_layernorm_grad(x[:3], x, w[:4], w[:4]), lambda: svmx.svm_layernorm_grad(x, x, w[:3], w[:4])):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad in (lambda: svmx.svm_layernorm(x, w.half()), lambda: svmx.svm_layernorm(x, out_dtype=torch.float16),
                lambda: svmx.svm_layernorm(x, w, None, 0.0)):
        with pytest.raises(svmx.SvmError):
            bad()
