"""AdamW steps against the formula in 64 bits.

Tolerances (u = 2^-24): m and v are two products and a sum, their constants rounded once: 5 u of the parts; the
step a quotient with a square root: 12 u of itself plus what v's error moves; parameters one more rounding.  An
8-bit state is within half a step of its code, 2^-4 of the value or 2^-10 of the scale, of the unrounded one.
"""
import math

import pytest
import torch

from paper_2311_14908_amd import svmx

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, F16, F8 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn
HALF_ULP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
SIZES = [1, 3, 4, 255, 256, 257, 1000, 4096, 4097, 9001, 0, 70000]
HYPER = dict(beta1=0.9, beta2=0.999, eps=1e-8)


def make(sizes, ptype, gtype, seed):
    g = torch.Generator().manual_seed(seed)
    p = [torch.randn(s, generator=g).to(ptype) for s in sizes]
    gr = [(torch.randn(s, generator=g) * 0.1).to(gtype) for s in sizes]
    m = [torch.randn(s, generator=g) * 0.03 for s in sizes]
    v = [torch.rand(s, generator=g) ** 4 * 0.01 for s in sizes]
    return p, gr, m, v


def step64(p, g, m, v, t, lr, wd, gs, beta1, beta2, eps):
    g = g.double() * gs
    m1 = beta1 * m.double() + (1 - beta1) * g
    v1 = beta2 * v.double() + (1 - beta2) * g * g
    em = 5 * U * (beta1 * m.double().abs() + (1 - beta1) * g.abs()) * 2
    ev = 6 * U * v1 * 2
    den = torch.sqrt(v1 / (1 - beta2 ** t)) + eps
    upd = lr / (1 - beta1 ** t) * m1 / den
    eu = lr / (1 - beta1 ** t) * em / den + upd.abs() * (12 * U + 6 * U)
    p1 = p.double() * (1 - lr * wd) - upd
    return p1, m1, v1, eu + 3 * U * p.double().abs() + U * p1.abs(), em, ev


def cuda(lists):
    return [[t.cuda() for t in x] for x in lists]


def within(got, ref, err):
    got64 = got.cpu().double()
    lim = err + HALF_ULP[got.dtype] * (ref.abs() + err) * (1 + 2 ** -6) + (2.0 ** -24 if got.dtype == F16 else 1e-44)
    assert not ref.numel() or ((got64 - ref).abs() - lim).max().item() <= 0


@pytest.mark.parametrize("ptype,gtype,master", [(F32, F32, False), (F32, BF16, False), (BF16, BF16, True), (F16, F32, True),
                                                (BF16, F16, False)])
def test_step(ptype, gtype, master):
    p, g, m, v = make(SIZES, ptype, gtype, 1)
    decay = [0.01 * (i % 3) for i in range(len(SIZES))]
    pd, gd, md, vd = cuda((p, g, m, v))
    ma = [t.float() + 1e-4 for t in p] if master else None
    mad = [t.cuda() for t in ma] if master else None
    svmx.svm_adamw(pd, gd, md, vd, 3, 1e-2, weight_decay=decay, grad_scale=0.5, master=mad, **HYPER)
    for i in range(len(SIZES)):
        p1, m1, v1, ep, em, ev = step64((ma or p)[i], g[i], m[i], v[i], 3, 1e-2, decay[i], 0.5, **HYPER)
        within(md[i], m1, em)
        within(vd[i], v1, ev)
        within(mad[i] if master else pd[i], p1, ep)
        if master:
            assert torch.equal(pd[i], mad[i].to(ptype))


def decoded(codes, scale):
    n = codes.numel()
    return codes.float().cpu().double() * scale.cpu().double().repeat_interleave(256)[:n]


def block_max(x):
    n = -(-x.numel() // 256) * 256
    return torch.nn.functional.pad(x.abs(), (0, n - x.numel())).view(-1, 256).amax(1)


@pytest.mark.parametrize("ptype,gtype", [(F32, F32), (F32, BF16), (BF16, BF16)])
def test_eight_bit_states(ptype, gtype):
    p, g, _, _ = make(SIZES, ptype, gtype, 2)
    pd, gd = cuda((p, g))
    md, vd, ms, vs = svmx.svm_adamw_states(pd, F8)
    master = [t.float().cuda() for t in p] if ptype != F32 else None
    for t in range(1, 4):
        before = [(decoded(md[i], ms[i]), decoded(vd[i], vs[i]), (master or pd)[i].cpu().clone()) for i in range(len(SIZES))]
        svmx.svm_adamw(pd, gd, md, vd, t, 1e-2, weight_decay=0.1, m_scale=ms, v_scale=vs, master=master, **HYPER)
        for i in range(len(SIZES)):
            m0, v0, p0 = before[i]
            p1, m1, v1, ep, em, ev = step64(p0, g[i], m0, v0, t, 1e-2, 0.1, 1.0, **HYPER)
            within((master or pd)[i], p1, ep + 4 * U * p1.abs())
            for x, codes, scale, e in ((m1, md[i], ms[i], em), (v1, vd[i], vs[i], ev)):
                top = block_max(x) / 448
                assert ((scale.cpu().double() - top).abs() <= 8 * U * top + block_max(e) / 448).all()
                step = top.repeat_interleave(256)[:x.numel()]
                assert ((decoded(codes, scale) - x).abs() <= (2.0 ** -4 * x.abs() + 2.0 ** -10 * step) * (1 + 1e-5) + e
                        + (2.0 ** -10 * step if codes is vd[i] else 0)).all()  # (the smallest code holds all below it)
            assert (decoded(vd[i], vs[i])[v1 > 1e-25] > 0).all()


def test_codes_of_a_block():
    """Every code of e4m3 is kept as it is, ties go to even, and a block's largest value is exact."""
    codes = torch.arange(0, 127, dtype=torch.uint8).view(F8).float()  # 0 .. 448
    x = torch.zeros(512)
    x[:127], x[127:254] = codes, -codes
    x[256] = 448.0
    odd = (codes[8:126] + codes[9:127]) / 2  # half way between neighbours
    x[257:257 + 118] = odd
    p, g = [torch.zeros(512).cuda()], [(x * 10).cuda()]
    m, v, ms, vs = svmx.svm_adamw_states(p, F8)
    svmx.svm_adamw(p, g, m, v, 1, 1e-3, beta1=0.9, m_scale=ms, v_scale=vs)  # m = 0.1 x 10 x, near x
    got = decoded(m[0], ms[0])
    assert (ms[0].cpu() - 1.0).abs().max() <= 4 * U
    assert ((got - x.double())[:256].abs() <= 8 * U * x[:256].abs()).all()
    step = (codes[9:127] - codes[8:126]).double()
    assert ((got[257:375] - odd.double()).abs() <= step / 2 * (1 + 1e-5)).all()
    assert got[256].item() == pytest.approx(448.0, rel=8 * U)


def test_second_moments_never_vanish():
    """A gradient 2^-14 of its block's largest has a second moment 2^-28 of it, below the smallest code: it is kept
    as that code, so the next step stays of the order of lr."""
    g = torch.full((256,), 2.0 ** -14)
    g[7] = 1.0
    p = [torch.zeros(256).cuda()]
    m, v, ms, vs = svmx.svm_adamw_states(p, F8)
    for t in range(1, 6):
        before = p[0].clone()
        svmx.svm_adamw(p, [g.cuda()], m, v, t, 1e-3, m_scale=ms, v_scale=vs)
        assert (p[0] - before).abs().max().item() <= 1.1e-3
    assert (decoded(v[0], vs[0]) > 0).all()


def test_not_finite():
    """NaN and infinities stay with their parameter; a block's other values keep their scale."""
    g = torch.randn(700, generator=torch.Generator().manual_seed(1))
    clean = g.clone()
    g[5], g[300], g[600] = float("nan"), float("inf"), -float("inf")
    bad = torch.zeros(700, dtype=torch.bool)
    bad[[5, 300, 600]] = True
    clean[bad] = 0.0
    for dtype in (F32, F8):
        out = []
        for grad in (g, clean):
            p = [torch.ones(700).cuda()]
            m, v, ms, vs = svmx.svm_adamw_states(p, dtype)
            for t in (1, 2):
                svmx.svm_adamw(p, [grad.cuda()], m, v, t, 1e-2, m_scale=ms, v_scale=vs)
            out.append((p[0].cpu(), m[0].float().cpu(), [s[0].cpu() for s in (ms, vs)] if ms else None))
        assert bool(out[0][0][bad].isnan().all()) and torch.equal(out[0][0][~bad], out[1][0][~bad])
        if dtype == F8:
            assert bool(out[0][1][bad].isnan().all()) and torch.equal(out[0][1][~bad], out[1][1][~bad])
            assert torch.equal(out[0][2][0], out[1][2][0])


def test_huge_gradient_with_eight_bits():
    """A squared gradient past fp32 is kept as the largest fp32; the block's others shrink their steps, none blows up."""
    g = torch.full((256,), 1e-2)
    g[3] = 1e25
    p = [torch.zeros(256).cuda()]
    m, v, ms, vs = svmx.svm_adamw_states(p, F8)
    for t in (1, 2, 3):
        svmx.svm_adamw(p, [g.cuda()], m, v, t, 1e-3, m_scale=ms, v_scale=vs)
    assert bool(p[0].isfinite().all()) and p[0].abs().max().item() <= 4e-3
    assert bool(vs[0].isfinite().all())


def test_zero_gradients_and_eps():
    for dtype in (F32, F8):
        p = [torch.ones(300).cuda()]
        m, v, ms, vs = svmx.svm_adamw_states(p, dtype)
        svmx.svm_adamw(p, [torch.zeros(300).cuda()], m, v, 1, 0.1, weight_decay=0.5, m_scale=ms, v_scale=vs)
        assert (p[0].cpu().double() - 0.95).abs().max() <= 2 * U


def test_more_tensors_than_a_launch_holds_and_mixed_lists():
    sizes = [1 + (37 * i) % 900 for i in range(131)]
    p, g, m, v = make(sizes, F32, F32, 5)
    g = [t.to(BF16) if i % 3 == 0 else t for i, t in enumerate(g)]
    pd, gd, md, vd = cuda((p, g, m, v))
    m8, v8, ms, vs = svmx.svm_adamw_states(pd, F8)
    for i in range(0, 131, 2):  # every other tensor with 8-bit states that start as zeros
        md[i], vd[i], m[i], v[i] = m8[i], v8[i], torch.zeros(sizes[i]), torch.zeros(sizes[i])
    scale = torch.tensor([0.25]).cuda()
    svmx.svm_adamw(pd, gd, md, vd, 1, 1e-2, grad_scale=scale, m_scale=ms, v_scale=vs, **HYPER)
    for i in range(131):
        p1, m1, v1, ep, em, ev = step64(p[i], g[i], m[i], v[i], 1, 1e-2, 0.0, 0.25, **HYPER)
        within(pd[i], p1, ep)
        if i % 2:
            within(md[i], m1, em)
            within(vd[i], v1, ev)


def test_views_at_odd_places():
    """Tensors anywhere in a flat buffer; what lies between them is left alone."""
    for ptype, dtype in ((F32, F32), (BF16, F8)):
        flat = torch.randn(4000, generator=torch.Generator().manual_seed(4)).to(ptype)
        cut = [(1, 700), (703, 300), (1004, 2995)]
        dev = flat.cuda()
        p = [dev[a:a + n] for a, n in cut]
        alone = [t.clone() for t in p]
        g = [torch.randn(n, generator=torch.Generator().manual_seed(a)).to(ptype).cuda() for a, n in cut]
        for lst in (p, alone):
            m, v, ms, vs = svmx.svm_adamw_states(lst, dtype)
            if dtype == F8:  # codes at odd addresses too
                room = [torch.zeros(1 + t.numel(), dtype=torch.uint8).cuda() for t in m]
                m = [r[1:].view(F8) for r in room]
            svmx.svm_adamw(lst, g, m, v, 1, 1e-2, m_scale=ms, v_scale=vs)
        assert all(torch.equal(a, b) for a, b in zip(p, alone))
        gaps = torch.ones(4000, dtype=torch.bool)
        for a, n in cut:
            gaps[a:a + n] = False
        assert torch.equal(dev.cpu()[gaps], flat[gaps])


def test_descends():
    """With the gradient of a quadratic, either state reaches its minimum."""
    target = torch.randn(1000, generator=torch.Generator().manual_seed(6)).cuda()
    for dtype in (F32, F8):
        p = [torch.zeros(1000).cuda()]
        m, v, ms, vs = svmx.svm_adamw_states(p, dtype)
        for t in range(1, 401):
            svmx.svm_adamw(p, [p[0] - target], m, v, t, 0.05 * math.cos(t / 401 * math.pi / 2), m_scale=ms, v_scale=vs)
        assert (p[0] - target).abs().max().item() <= 0.1


def test_on_another_stream_and_in_a_graph():
    p, g, m, v = make([5000, 300], F32, F32, 8)
    a, b = cuda((p, g, m, v)), cuda((p, g, m, v))
    svmx.svm_adamw(a[0], a[1], a[2], a[3], 2, 1e-2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    svmx.svm_adamw(b[0], b[1], b[2], b[3], 2, 1e-2, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for k in (0, 2, 3) for x, y in zip(a[k], b[k]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        svmx.svm_adamw(b[0], b[1], b[2], b[3], 2, 1e-2)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        svmx.svm_adamw(a[0], a[1], a[2], a[3], 2, 1e-2)
        assert all(torch.equal(x, y) for k in (0, 2, 3) for x, y in zip(a[k], b[k]))


def test_binding_refusals():
    p, g, m, v = cuda(make([10, 20], F32, F32, 1))
    m8, v8, ms, vs = svmx.svm_adamw_states(p, F8)
    for bad in (lambda: svmx.svm_adamw(p, g[:1], m, v, 1, 1e-3), lambda: svmx.svm_adamw(p, g[::-1], m, v, 1, 1e-3),
                lambda: svmx.svm_adamw(p, g, m8, v8, 1, 1e-3), lambda: svmx.svm_adamw(p, g, m8, v, 1, 1e-3, m_scale=ms, v_scale=vs),
                lambda: svmx.svm_adamw([t.double() for t in p], g, m, v, 1, 1e-3),
                lambda: svmx.svm_adamw(p, g, m8, v8, 1, 1e-3, m_scale=ms, v_scale=[s[:0] for s in vs]),
                lambda: svmx.svm_adamw(p, [t.cpu() for t in g], m, v, 1, 1e-3),
                lambda: svmx.svm_adamw(p, g, m, v, 1, 1e-3, weight_decay=[0.1])):
        with pytest.raises((TypeError, ValueError)):
            bad()
    with pytest.raises(svmx.SvmError):
        svmx.svm_adamw(p, g, m, v, 0, 1e-3)
    svmx.svm_adamw([], [], [], [], 1, 1e-3)


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-15, 1e-8, 1.0, 1e25])
@pytest.mark.parametrize("dtype", [F32, F8])
def test_any_eps(eps, dtype):
    """Tiny second moments with an eps that does or does not hide them: below it the step is as exact."""
    sizes = [2048, 5000]
    g = torch.Generator().manual_seed(9)
    p = [torch.randn(s, generator=g) * 1e-3 for s in sizes]
    gr = [torch.randn(s, generator=g) * torch.exp(torch.randn(s, generator=g) * 3 - 20) for s in sizes]
    pd, gd = cuda((p, gr))
    md, vd, ms, vs = svmx.svm_adamw_states(pd, dtype)
    svmx.svm_adamw(pd, gd, md, vd, 1, 1e-3, eps=eps, m_scale=ms, v_scale=vs)
    for i in range(len(sizes)):
        zero = torch.zeros(sizes[i])
        p1, m1, v1, ep, _, _ = step64(p[i], gr[i], zero, zero, 1, 1e-3, 0.0, 1.0, 0.9, 0.999, eps)
        # v is held in fp32: what is denormal there has an error of half the smallest number
        vmin = 2.0 ** -149
        moved = 1e-3 * gr[i].double().abs() / (torch.sqrt(((v1 - vmin).clamp_min(0)) / 1e-3) + eps) - 1e-3 * gr[i].double().abs() / (
            torch.sqrt(v1 / 1e-3) + eps)
        within(pd[i], p1, ep + moved.nan_to_num(nan=1.0, posinf=1.0))


def test_blocks_at_every_place_step_alike():
    """A value's step does not depend on where in its tensor it stands, in whole chunks or behind them."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn(256, generator=g)
    for dtype in (F32, F8):
        p = [x.repeat(21).cuda()]
        gr = [(x.flip(0) * 0.1).repeat(21).cuda()]
        m, v, ms, vs = svmx.svm_adamw_states(p, dtype)
        for t in range(1, 4):
            svmx.svm_adamw(p, gr, m, v, t, 1e-2, m_scale=ms, v_scale=vs)
        rows = p[0].view(21, 256)
        assert torch.equal(rows, rows[:1].expand_as(rows))
