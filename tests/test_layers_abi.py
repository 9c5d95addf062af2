"""Refusals of the operators for learned rows that need no GPU: every check runs before any device access."""
import ctypes as C

import pytest

from paper_2311_14908_amd import svmx

P = C.c_void_p(4096)  # never read: each call is refused before
EINVAL, EWORKSPACE, ENOMEM = svmx.SVM_EINVAL, svmx.SVM_EWORKSPACE, svmx.SVM_ENOMEM


def embed(**kw):
    a = dict(table=P, tt=0, V=10, d=8, ld=8, tok=P, tb=4, T=5, bags=P, B=2, scale=1.0, mean=0, pad=-1, out=P, ot=0, ldo=8,
             inv=None, ws=None, wsb=0, o=None)
    a.update(kw)
    return svmx.load().svm_embed(*a.values())


def embed_grad(**kw):
    a = dict(tok=P, tb=4, T=5, bags=P, B=2, scale=1.0, mean=0, pad=-1, dy=P, yt=0, ldy=8, de=P, et=0, V=10, d=8, lde=8, acc=0,
             inv=None, ws=None, wsb=0, o=None)
    a.update(kw)
    return svmx.load().svm_embed_grad(*a.values())


def norm(**kw):
    a = dict(x=P, xt=0, n=4, d=8, ld=8, w=P, b=P, wt=0, eps=1e-5, y=P, yt=0, ldy=8, mean=None, rstd=None, o=None)
    a.update(kw)
    return svmx.load().svm_layernorm(*a.values())


def norm_grad(**kw):
    a = dict(dy=P, yt=0, ldy=8, x=P, xt=0, n=4, d=8, ld=8, mean=P, rstd=P, w=P, wt=0, dx=P, ldx=8, dw=P, db=P, ws=None, wsb=0, o=None)
    a.update(kw)
    return svmx.load().svm_layernorm_grad(*a.values())


def adamw(count=1, params=None, null=False, **kw):
    t = dict(param=4096, master=None, grad=4096, m=4096, v=4096, m_scale=None, v_scale=None, count=7, weight_decay=0.0,
             param_type=0, grad_type=0, state_type=0, reserved=0)
    t.update(kw)
    p = dict(struct_size=C.sizeof(svmx.svm_adamw_params), step=1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0)
    p.update(params or {})
    arr = (svmx.svm_adamw_tensor * 1)(svmx.svm_adamw_tensor(**t))
    return svmx.load().svm_adamw(None if null else arr, count, C.byref(svmx.svm_adamw_params(**p)), None)


def predict_grad(**kw):
    a = dict(X=P, y=P, alpha=P, n=9, d=3, gamma=0.5, T=P, m=2, up=None, out=P, ws=None, wsb=0, o=None)
    a.update(kw)
    return svmx.load().svm_predict_grad(*a.values())


def objective_grad(**kw):
    a = dict(X=P, y=P, alpha=P, n=9, d=3, gamma=0.5, out=P, ws=None, wsb=0, o=None)
    a.update(kw)
    return svmx.load().svm_objective_grad(*a.values())


NAN, INF = float("nan"), float("inf")
BIG = 2 ** 31 - 1


@pytest.mark.parametrize("kw", [dict(V=0), dict(d=0), dict(T=-1), dict(B=-1), dict(tt=3), dict(tt=-1), dict(ot=9), dict(ld=7),
                                dict(ldo=7), dict(tb=2), dict(tok=None), dict(table=None), dict(out=None), dict(scale=NAN),
                                dict(scale=INF), dict(bags=None), dict(B=0), dict(V=BIG), dict(T=BIG), dict(B=BIG), dict(d=BIG),
                                dict(ld=2 ** 60)])
def test_embed_refusals(kw):
    assert embed(**kw) == EINVAL and svmx.load().svm_last_error()


def test_embed_workspace_is_asked_for():
    lib = svmx.load()
    assert embed() == EWORKSPACE
    assert embed(ws=P, wsb=lib.svm_embed_workspace_bytes(5, 8, 2, 1) - 1) == EWORKSPACE
    assert lib.svm_embed_workspace_bytes(5, 8, 5, 0) == 0
    assert lib.svm_embed_workspace_bytes(-1, 8, 2, 1) == -1 and lib.svm_embed_workspace_bytes(5, 0, 2, 1) == -1
    assert lib.svm_embed_grad_workspace_bytes(5, 0, 2) == -1 and lib.svm_embed_grad_workspace_bytes(5, 8, -2) == -1
    assert embed(T=0, B=0) == svmx.SVM_OK  # nothing to write


@pytest.mark.parametrize("kw", [dict(V=0), dict(d=0), dict(T=-1), dict(B=-1), dict(yt=3), dict(et=7), dict(ldy=7), dict(lde=7),
                                dict(tb=3), dict(tok=None), dict(dy=None), dict(de=None), dict(scale=NAN), dict(bags=None), dict(B=0)])
def test_embed_grad_refusals(kw):
    assert embed_grad(**kw) == EINVAL and svmx.load().svm_last_error()


def test_embed_grad_workspace_is_asked_for():
    assert embed_grad() == EWORKSPACE
    assert embed_grad(ws=P, wsb=svmx.load().svm_embed_grad_workspace_bytes(5, 8, 2) - 1) == EWORKSPACE


@pytest.mark.parametrize("kw", [dict(n=-1), dict(d=0), dict(xt=5), dict(yt=1), dict(yt=2), dict(wt=1), dict(wt=3), dict(ld=7),
                                dict(ldy=7), dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(eps=1e-60),
                                dict(x=None), dict(y=None), dict(d=BIG, ld=BIG, ldy=BIG), dict(ld=2 ** 60)])
def test_norm_refusals(kw):
    assert norm(**kw) == EINVAL and svmx.load().svm_last_error()


@pytest.mark.parametrize("kw", [dict(n=-1), dict(d=0), dict(xt=5), dict(yt=1), dict(wt=2), dict(ld=7), dict(ldy=7), dict(ldx=7),
                                dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None)])
def test_norm_grad_refusals(kw):
    assert norm_grad(**kw) == EINVAL and svmx.load().svm_last_error()


def test_norm_grad_workspace_is_asked_for():
    lib = svmx.load()
    assert norm_grad() == EWORKSPACE
    assert lib.svm_layernorm_grad_workspace_bytes(4, 0, 0) == -1 and lib.svm_layernorm_grad_workspace_bytes(4, 8, 3) == -1


@pytest.mark.parametrize("kw", [dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(count=-1), dict(null=True),
                                dict(param_type=3), dict(grad_type=4), dict(state_type=1), dict(state_type=3), dict(reserved=1),
                                dict(weight_decay=-0.1), dict(weight_decay=NAN)]
                         + [dict(params=p) for p in (dict(step=0), dict(lr=-1.0), dict(lr=NAN), dict(beta1=1.0), dict(beta1=-0.1),
                                                     dict(beta2=1.0), dict(beta2=NAN), dict(eps=-1.0), dict(eps=INF),
                                                     dict(grad_scale=NAN), dict(struct_size=0), dict(reserved=1))])
def test_adamw_refusals(kw):
    kw = dict(kw)
    if kw.pop("null", False):
        assert adamw(null=True) == EINVAL
    else:
        assert adamw(**kw) == EINVAL
    assert svmx.load().svm_last_error()


def test_adamw_struct_sizes():
    assert C.sizeof(svmx.svm_adamw_tensor) == 88 and C.sizeof(svmx.svm_adamw_params) == 64


@pytest.mark.parametrize("call", [predict_grad, objective_grad])
@pytest.mark.parametrize("kw", [dict(n=0), dict(d=0), dict(gamma=0.0), dict(gamma=-1.0), dict(gamma=NAN), dict(gamma=INF), dict(X=None),
                                dict(y=None), dict(alpha=None), dict(out=None), dict(d=2 ** 60)])
def test_machine_gradient_refusals(call, kw):
    assert call(**kw) == EINVAL and svmx.load().svm_last_error()


def test_machine_gradient_limits():
    lib = svmx.load()
    assert predict_grad(m=-1) == EINVAL and predict_grad(T=None) == EINVAL
    assert predict_grad(n=BIG) == ENOMEM and objective_grad(n=BIG) == ENOMEM
    assert predict_grad(m=0, T=None, out=None) == svmx.SVM_OK
    assert lib.svm_predict_grad_workspace_bytes(0, 3, 2) == -1 and lib.svm_objective_grad_workspace_bytes(9, 0) == -1


def test_bad_options_are_refused():
    o = svmx.svm_options()
    svmx.load().svm_default_options(C.byref(o))
    o.struct_size = 3
    r = C.byref(o)
    assert {embed(o=r), embed_grad(o=r), norm(o=r), norm_grad(o=r), predict_grad(o=r), objective_grad(o=r)} == {EINVAL}
