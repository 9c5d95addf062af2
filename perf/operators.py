"""Performance cases of the operators around a kernel SVM whose rows are learned from tokens.

tokens -> embedding bags -> layer norm -> rows X of the machine -> its loss -> gradient of the rows ->
layer norm's gradient -> gradient of the table -> AdamW.  ``listed()`` names the standing cases, ``draw(rng)``
adds one of the same ranges, ``prepare`` makes the device arrays that a program holds before the call and ``run``
is one call: of the library where ``own`` is true, else of the plain form (elementary torch operations in 32
bits, rounded once at the end).

Recipes (drawn on the device from the seed):
  tokens   frequencies 1/rank over a shuffled vocabulary (natural text is close to that)
  bags     cut at uniformly drawn places of the token list, so lengths spread from 0 to several means
  blobs    two overlapping Gaussian classes, means +-shift, unit variance        gamma 1/d
  sparse   U[0,1] features, 80% zeroed                                           gamma 15.68/d
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BETA1, BETA2, ADAM_EPS, LR, DECAY, STEP = 0.9, 0.999, 1e-8, 1e-3, 0.01, 10
NORM_EPS = 1e-5
BLOCK, F8MAX = 256, 448.0  # values an 8-bit state's scale stands for; largest e4m3 value
CLIP = 0.7  # factor on every gradient, as clipping by the norm gives it


def listed():
    return [
        # Serving: the tokens of one short text to one row.  Launches and host work are all there is.
        dict(name="embed-one", kind="embed", V=50000, d=128, T=37, B=1, bags=True, mean=True, pad=False, dtype="f32", out="f32"),
        # A training set's texts to rows in one go: ragged bags, padded, 16-bit table, rows in 32 bits for the machine.
        dict(name="embed-corpus", kind="embed", V=65537, d=784, T=1000003, B=20000, bags=True, mean=True, pad=True, dtype="bf16", out="f32"),
        # The gradient of one small batch in a small vocabulary: 64 texts.
        dict(name="embed-grad-batch", kind="embed_grad", V=2000, d=64, T=5000, B=64, bags=True, mean=True, pad=True, dtype="f32", out="f32"),
        # A long batch of single tokens (one row a token), 16-bit gradients, odd vocabulary: sort and sums.
        dict(name="embed-grad-tokens", kind="embed_grad", V=65537, d=256, T=1000003, B=1000003, bags=False, mean=False, pad=False, dtype="bf16", out="f32"),
        # The rows of the standard binary problem, normalised before they go to the machine.
        dict(name="norm-rows", kind="norm", n=20000, d=784, dtype="f32", wtype="f32", out="f32"),
        # Its gradient at a length that divides nothing.
        dict(name="norm-grad-ragged", kind="norm_grad", n=60001, d=301, dtype="f32", wtype="f32", out="f32"),
        # Long 16-bit rows, many of them: bound by memory.
        dict(name="norm-grad-wide", kind="norm_grad", n=65536, d=4096, dtype="bf16", wtype="f32", out="bf16"),
        # The optimiser on a small feature model (table, two vectors of the norm): one launch's latency.
        dict(name="adamw-small", kind="adamw", V=2000, d=64, layers=0, state="f32", dtype="f32", grad="f32"),
        # 146 tensors, 195 million parameters, 8-bit states, gradients in 16 bits.
        dict(name="adamw-8bit", kind="adamw", V=50001, d=1000, layers=12, state="f8", dtype="f32", grad="bf16"),
        # Serving: how one sample's decision value moves with its features (15,000 support vectors).
        dict(name="predict-grad-one", kind="predict_grad", recipe="sparse", n=20000, d=784, m=1, sv=0.75),
        # The loss gradient in all rows of the standard binary problem: two large matrix products.
        dict(name="objective-grad-784", kind="objective_grad", recipe="sparse", n=20000, d=784, sv=0.75),
        # The same on short rows and many samples, nothing a multiple of a tile: exponentials and products.
        dict(name="objective-grad-short", kind="objective_grad", recipe="blobs", n=99999, d=31, sv=0.3),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + 1 if v == 3072 else v


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm_grad", "norm_grad", "adamw", "adamw", "predict_grad",
                       "objective_grad", "objective_grad"])
    if kind in ("embed", "embed_grad"):
        V, d, T = _log(rng, 100, 200000), _log(rng, 8, 2000), _log(rng, 1, 1000000)
        T = max(1, min(T, 800000000 // d // 3))
        V = max(10, min(V, 200000000 // d))
        bags = rng.random() < 0.6
        B = max(1, min(T, _log(rng, 1, 30000))) if bags else T
        dtype = rng.choice(["f32", "bf16", "f16"])
        return dict(kind=kind, V=V, d=d, T=T, B=B, bags=bags, mean=bags and rng.random() < 0.7, pad=rng.random() < 0.4, dtype=dtype,
                    out=rng.choice(["f32", dtype]))
    if kind in ("norm", "norm_grad"):
        d = _log(rng, 8, 9000)
        n = max(1, min(_log(rng, 1, 100000), 268435456 // d))
        dtype = rng.choice(["f32", "bf16", "f16"])
        return dict(kind=kind, n=n, d=d, dtype=dtype, wtype=rng.choice(["f32", dtype]), out=rng.choice(["f32", dtype]))
    if kind == "adamw":
        return dict(kind=kind, V=_log(rng, 100, 50000), d=_log(rng, 16, 900) | 1, layers=rng.randint(0, 12), state=rng.choice(["f32", "f8"]),
                    dtype=rng.choice(["f32", "bf16"]), grad=rng.choice(["f32", "bf16"]))
    recipe = rng.choice(["blobs", "sparse"])
    if kind == "predict_grad":
        return dict(kind=kind, recipe=recipe, n=_log(rng, 500, 50000), d=_log(rng, 8, 784), m=_log(rng, 1, 4000), sv=round(rng.uniform(0.1, 0.75), 3))
    d = _log(rng, 8, 784)
    n = min(_log(rng, 500, 60000), int(15000 / 0.75 * math.sqrt(784 / max(d, 64))))
    return dict(kind=kind, recipe=recipe, n=n, d=d, sv=round(rng.uniform(0.1, 0.5), 3))


def _normal(g, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(dtype)


def _tokens(case, g):
    """int32 tokens of frequency 1/rank; with padding one in ten is the padding id 0."""
    V, T = case["V"], case["T"]
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    tok = torch.randperm(V, generator=g, device="cuda")[rank].to(torch.int32)
    if case["pad"]:
        tok[torch.rand(T, generator=g, device="cuda") < 0.1] = 0
    return tok


def _bag_starts(case, g):
    cuts = torch.randint(0, case["T"] + 1, (case["B"] - 1,), generator=g, device="cuda").sort().values
    return torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), case["T"])])


def _sizes(case):
    """Tensors of a small transformer's shape, or (no layers) of a table and a norm."""
    d = case["d"]
    layer = [d * d] * 4 + [4 * d * d] * 2 + [4 * d] + [d] * 5
    return [case["V"] * d] + layer * case["layers"] + [d, d]


def _views(flat, sizes, blocks=1):
    """One view a tensor of a buffer in which every tensor starts on a multiple of BLOCK values."""
    ends = np.cumsum([-(-s // BLOCK) for s in sizes]) * (BLOCK // blocks)
    starts = np.concatenate([[0], ends[:-1]])
    lens = [-(-s // blocks) for s in sizes]
    return [flat[int(a):int(a) + n] for a, n in zip(starts, lens)]


def _rows(case, n, g):
    d = case["d"]
    if case["recipe"] == "sparse":
        X = torch.rand(n, d, generator=g, device="cuda")
        return X.masked_fill_(torch.rand(n, d, generator=g, device="cuda") < 0.8, 0.0)
    sign = 1.0 - 2.0 * (torch.arange(n, device="cuda") % 2).float()
    return torch.randn(n, d, generator=g, device="cuda").add_(sign[:, None] * (1.7 / math.sqrt(d)))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, st = case["kind"], dict(case=case)
    if kind in ("embed", "embed_grad"):
        st["tokens"] = _tokens(case, g)
        st["bags"] = _bag_starts(case, g) if case["bags"] else None
        st["scale"] = 1.0 if case["mean"] else math.sqrt(case["d"])
        st["padding"] = 0 if case["pad"] else -1
        if kind == "embed":
            st["table"] = _normal(g, (case["V"], case["d"]), TYPES[case["dtype"]], 1.0 / math.sqrt(case["d"]))
        else:
            st["dY"] = _normal(g, (case["B"], case["d"]), TYPES[case["dtype"]], 0.01)
        return st
    if kind in ("norm", "norm_grad"):
        n, d, t = case["n"], case["d"], TYPES[case["dtype"]]
        st["x"] = _normal(g, (n, d), torch.float32).mul_(torch.rand(n, 1, generator=g, device="cuda") + 0.5).add_(0.3).to(t)
        st["w"] = (1.0 + _normal(g, (d,), torch.float32, 0.2)).to(TYPES[case["wtype"]])
        st["b"] = _normal(g, (d,), TYPES[case["wtype"]], 0.2)
        if kind == "norm_grad":
            st["dy"] = _normal(g, (n, d), TYPES[case["out"]], 0.01)
            x = st["x"].float()
            st["mean"] = x.mean(1)  # what the forward pass has kept
            st["rstd"] = torch.rsqrt((x - st["mean"][:, None]).square().mean(1) + NORM_EPS)
        return st
    if kind == "adamw":
        sizes = _sizes(case)
        total = sum(-(-s // BLOCK) * BLOCK for s in sizes)
        zero = torch.ones(total // BLOCK, BLOCK, device="cuda")  # 0 in the gaps behind the tensors
        last = np.cumsum([-(-s // BLOCK) for s in sizes]) - 1
        rest = torch.tensor([s - (-(-s // BLOCK) - 1) * BLOCK for s in sizes], device="cuda")
        zero[torch.from_numpy(last).cuda()] = (torch.arange(BLOCK, device="cuda")[None, :] < rest[:, None]).float()
        zero = zero.reshape(-1)
        st["sizes"] = sizes
        st["p"] = _normal(g, (total,), torch.float32, 0.05).mul_(zero).to(TYPES[case["dtype"]])
        st["g"] = _normal(g, (total,), torch.float32, 0.01).mul_(zero).to(TYPES[case["grad"]])
        m = _normal(g, (total,), torch.float32, 0.003).mul_(zero)
        v = _normal(g, (total,), torch.float32, 0.01).square_().mul_(zero)
        del zero
        if case["state"] == "f8":
            st["m"], st["ms"] = _to_f8(m, False)
            st["v"], st["vs"] = _to_f8(v, True)
            st["lists"] = [_views(st[k], sizes, 1) for k in "pgmv"] + [_views(st[k], sizes, BLOCK) for k in ("ms", "vs")]
        else:
            st["m"], st["v"] = m, v
            st["lists"] = [_views(st[k], sizes, 1) for k in "pgmv"] + [None, None]
        if case["dtype"] != "f32":  # 32-bit copy that the 16-bit parameters are rounded from
            st["master"] = st["p"].float()
            st["masters"] = _views(st["master"], sizes, 1)
        return st
    gamma = (15.68 if case["recipe"] == "sparse" else 1.0) / case["d"]
    C = 10.0 if case["recipe"] == "sparse" else 1.0
    n = case["n"]
    st.update(gamma=gamma, X=_rows(case, n, g))
    st["y"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, 1, -1).to(torch.int32)
    # a trained model's multipliers: a share `sv` above zero, a third of those at the bound
    a = (C * 1.5 * torch.rand(n, generator=g, device="cuda", dtype=torch.float64)).clamp_(max=C)
    a[torch.rand(n, generator=g, device="cuda") >= case["sv"]] = 0.0
    st["alpha"] = a
    if kind == "predict_grad":
        st["T"] = _rows(case, case["m"], g)
        st["up"] = torch.randn(case["m"], generator=g, device="cuda", dtype=torch.float64)
    return st


# ---------------------------------------------------------------------------------- plain forms

def _bag_weights(st):
    """Every token's bag, 1 or 0 by padding, and every bag's weight."""
    case, tok = st["case"], st["tokens"].long()
    used = (tok != st["padding"]).float()
    if not case["bags"]:
        return tok, torch.arange(case["T"], device="cuda"), used, torch.full((case["B"],), st["scale"], device="cuda")
    lens = st["bags"][1:] - st["bags"][:-1]
    bag = torch.repeat_interleave(torch.arange(case["B"], device="cuda"), lens, output_size=case["T"])
    if not case["mean"]:
        return tok, bag, used, torch.full((case["B"],), st["scale"], device="cuda")
    count = torch.zeros(case["B"], device="cuda").index_add_(0, bag, used)
    return tok, bag, used, st["scale"] / count.clamp_(min=1.0)


def _plain_embed(st):
    case = st["case"]
    tok, bag, used, w = _bag_weights(st)
    rows = st["table"][tok].float() * used[:, None]
    if case["bags"]:
        rows = torch.zeros(case["B"], case["d"], device="cuda").index_add_(0, bag, rows)
    return (rows * w[:, None]).to(TYPES[case["out"]])


def _plain_embed_grad(st):
    case = st["case"]
    tok, bag, used, w = _bag_weights(st)
    rows = st["dY"].float()
    if case["bags"]:
        rows = (rows * w[:, None])[bag] * used[:, None]
    else:
        rows = rows * (w * used)[:, None]
    return torch.zeros(case["V"], case["d"], device="cuda").index_add_(0, tok, rows).to(TYPES[case["out"]])


def _plain_norm(st):
    x = st["x"].float()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = torch.rsqrt(c.square().mean(1) + NORM_EPS)
    y = c * rstd[:, None] * st["w"].float() + st["b"].float()
    return y.to(TYPES[st["case"]["out"]]), mean, rstd


def _plain_norm_grad(st):
    dy, w = st["dy"].float(), st["w"]
    h = (st["x"].float() - st["mean"][:, None]) * st["rstd"][:, None]
    q = dy * w.float()
    dx = (q - q.mean(1, keepdim=True) - h * (q * h).mean(1, keepdim=True)) * st["rstd"][:, None]
    return dx.to(st["x"].dtype), (dy * h).sum(0).to(w.dtype), dy.sum(0).to(w.dtype)


def _to_f8(x, positive):
    """Codes and scales: blocks of BLOCK values over their largest magnitude / 448 (a block below 2^-100: zeros);
    a positive second moment is never rounded to zero."""
    x = x.view(-1, BLOCK)
    top = x.abs().amax(1, keepdim=True)
    top = torch.where(top < 2.0 ** -100, torch.zeros_like(top), top)
    r = torch.where(top > 0, x * (F8MAX / top), torch.zeros_like(x)).clamp_(-F8MAX, F8MAX)
    if positive:
        r = torch.where(r > 0, r.clamp(min=2.0 ** -9), r)
    return r.to(torch.float8_e4m3fn).view(-1), (top / F8MAX).view(-1)


def _plain_adamw(st):
    case = st["case"]
    f8 = case["state"] == "f8"
    g = st["g"].float() * CLIP
    m, v = st["m"], st["v"]
    if f8:
        m = (m.float().view(-1, BLOCK) * st["ms"][:, None]).view(-1)
        v = (v.float().view(-1, BLOCK) * st["vs"][:, None]).view(-1)
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * g * g
    w = st["master"] if "master" in st else st["p"]
    w.mul_(1.0 - LR * DECAY)
    w.sub_(LR / (1.0 - BETA1 ** STEP) * m / (v.sqrt() * (1.0 / math.sqrt(1.0 - BETA2 ** STEP)) + ADAM_EPS))
    if "master" in st:
        st["p"].copy_(w)
    if f8:
        m8, ms = _to_f8(m, False)
        v8, vs = _to_f8(v, True)
        st["m"].copy_(m8), st["v"].copy_(v8), st["ms"].copy_(ms), st["vs"].copy_(vs)
    else:
        st["m"].copy_(m), st["v"].copy_(v)
    return _adamw_out(st)


def _adamw_out(st):
    return {k: st[k] for k in ("p", "m", "v", "ms", "vs", "master") if k in st}


def _kernel32(A, B, gamma):
    d2 = A.square().sum(1)[:, None] + B.square().sum(1)[None, :] - 2.0 * (A @ B.T)
    return torch.exp(-gamma * d2.clamp_(min=0.0))


def _plain_predict_grad(st):
    sv = st["alpha"].nonzero()[:, 0]
    X, T = st["X"][sv], st["T"]
    c = (st["alpha"][sv] * st["y"][sv]).float()
    K = _kernel32(T, X, st["gamma"]) * c
    return (K @ X - K.sum(1)[:, None] * T) * (2.0 * st["gamma"] * st["up"].float())[:, None]


def _plain_objective_grad(st):
    sv = st["alpha"].nonzero()[:, 0]
    X = st["X"][sv]
    c = (st["alpha"][sv] * st["y"][sv]).float()
    K = _kernel32(X, X, st["gamma"]) * c
    dX = torch.zeros_like(st["X"])
    dX[sv] = (K.sum(1)[:, None] * X - K @ X) * (2.0 * st["gamma"] * c)[:, None]
    return dX


PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad,
         "adamw": _plain_adamw, "predict_grad": _plain_predict_grad, "objective_grad": _plain_objective_grad}


# ---------------------------------------------------------------------------------- the calls

def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return PLAIN[kind](st)
    from paper_2311_14908_amd import svmx
    if kind == "embed":  # the data set's tokens have been checked when it was loaded
        return svmx.svm_embed(st["table"], st["tokens"], bags=st["bags"], scale=st["scale"], mean=case["mean"],
                              padding=st["padding"], out_dtype=TYPES[case["out"]], check=False)
    if kind == "embed_grad":
        return svmx.svm_embed_grad(st["tokens"], st["dY"], case["V"], bags=st["bags"], scale=st["scale"], mean=case["mean"],
                                   padding=st["padding"], out_dtype=TYPES[case["out"]], check=False)
    if kind == "norm":
        return svmx.svm_layernorm(st["x"], st["w"], st["b"], NORM_EPS, out_dtype=TYPES[case["out"]])
    if kind == "norm_grad":
        return svmx.svm_layernorm_grad(st["dy"], st["x"], st["mean"], st["rstd"], st["w"])
    if kind == "adamw":
        p, g, m, v, ms, vs = st["lists"]
        svmx.svm_adamw(p, g, m, v, STEP, LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY, grad_scale=CLIP,
                       m_scale=ms, v_scale=vs, master=st.get("masters"))
        return _adamw_out(st)
    if kind == "predict_grad":
        return svmx.svm_predict_grad(st["X"], st["y"], st["alpha"], st["gamma"], st["T"], st["up"])
    return svmx.svm_objective_grad(st["X"], st["y"], st["alpha"], st["gamma"])


def work(case):
    kind = case["kind"]
    if kind in ("embed", "embed_grad"):
        V, d, T, B = case["V"], case["d"], case["T"], case["B"]
        edges = np.log(np.arange(1, V + 2)) / math.log(V + 1.0)
        distinct = float(np.sum(-np.expm1(T * np.log1p(-np.minimum(np.diff(edges), 1.0 - 1e-12)))))
        index = 4.0 * T + (8.0 * (B + 1) if case["bags"] else 0.0)
        if kind == "embed":
            return {"bytes": index + distinct * d * SIZE[case["dtype"]] + 1.0 * B * d * SIZE[case["out"]], "flops": 1.0 * T * d}
        return {"bytes": index + 1.0 * B * d * SIZE[case["dtype"]] + 1.0 * V * d * SIZE[case["out"]], "flops": 2.0 * T * d}
    if kind in ("norm", "norm_grad"):
        n, d = case["n"], case["d"]
        x, y, w = SIZE[case["dtype"]], SIZE[case["out"]], SIZE[case["wtype"]]
        if kind == "norm":
            return {"bytes": 1.0 * n * d * (x + y) + 8.0 * n + 2.0 * d * w, "flops": 8.0 * n * d}
        return {"bytes": 1.0 * n * d * (2 * x + y) + 8.0 * n + 3.0 * d * w, "flops": 14.0 * n * d}
    if kind == "adamw":
        count = float(sum(_sizes(case)))
        state = 16.0 if case["state"] == "f32" else 4.0 + 16.0 / BLOCK
        param = 8.0 if case["dtype"] == "f32" else 10.0  # 16-bit parameters: their 32-bit copy read and written, themselves written
        return {"bytes": count * (state + param + SIZE[case["grad"]]), "flops": 14.0 * count}
    n, d = case["n"], case["d"]
    nsv = case["sv"] * n
    if kind == "predict_grad":
        m = case["m"]
        return {"bytes": 4.0 * d * (nsv + 2 * m) + 12.0 * n + 8.0 * m, "flops": 4.0 * m * nsv * d}
    # K is symmetric: half a product for it, a whole one with X
    return {"bytes": 4.0 * d * (nsv + n) + 12.0 * n, "flops": 3.0 * nsv * nsv * d}


# ---------------------------------------------------------------------------------- in 64 bits

def _exact_bags(st):
    """Sorted by bag as given: starts, lengths, and the weight of every token (0 for padding)."""
    case, tok = st["case"], st["tokens"].long()
    start = st["bags"] if case["bags"] else torch.arange(case["T"] + 1, device="cuda")
    live = torch.where(tok == st["padding"], 0.0, 1.0).double()
    bag = torch.searchsorted(start, torch.arange(case["T"], device="cuda"), right=True) - 1
    w = torch.full((case["B"],), float(st["scale"]), dtype=torch.float64, device="cuda")
    if case["mean"]:
        run_sum = torch.cat([live.new_zeros(1), live.cumsum(0)])
        count = run_sum[start[1:]] - run_sum[start[:-1]]
        w = torch.where(count > 0, w / count.clamp(min=1.0), torch.zeros_like(w))
    return tok, bag, live * w[bag]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "embed":
        tok, bag, w = _exact_bags(st)
        out = torch.zeros(case["B"], case["d"], dtype=torch.float64, device="cuda")
        for i in range(0, case["T"], 1 << 17):
            j = slice(i, i + (1 << 17))
            out.index_add_(0, bag[j], w[j, None] * st["table"][tok[j]].double())
        return out
    if kind == "embed_grad":
        tok, bag, w = _exact_bags(st)
        out = torch.zeros(case["V"], case["d"], dtype=torch.float64, device="cuda")
        for i in range(0, case["T"], 1 << 17):
            j = slice(i, i + (1 << 17))
            out.index_add_(0, tok[j], w[j, None] * st["dY"][bag[j]].double())
        return out
    if kind == "norm":
        x = st["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        sd = torch.sqrt(var + NORM_EPS)
        return (x - mean[:, None]) / sd[:, None] * st["w"].double() + st["b"].double(), mean, 1.0 / sd
    if kind == "norm_grad":
        n, d = case["n"], case["d"]
        dx = torch.empty(n, d, dtype=torch.float64, device="cuda")
        dw = torch.zeros(d, dtype=torch.float64, device="cuda")
        db = torch.zeros(d, dtype=torch.float64, device="cuda")
        for i in range(0, n, 8192):
            j = slice(i, i + 8192)
            dy, r = st["dy"][j].double(), st["rstd"][j].double()[:, None]
            h = (st["x"][j].double() - st["mean"][j].double()[:, None]) * r
            dw += (dy * h).sum(0)
            db += dy.sum(0)
            q = dy * st["w"].double()
            dx[j] = r / d * (d * q - q.sum(1, keepdim=True) - h * (q * h).sum(1, keepdim=True))
        return dx, dw, db
    if kind == "adamw":
        g = CLIP * st["g"].double()
        m, v = st["m"].to(torch.float32).double(), st["v"].to(torch.float32).double()
        if case["state"] == "f8":
            m *= st["ms"].double().repeat_interleave(BLOCK)
            v *= st["vs"].double().repeat_interleave(BLOCK)
        m.mul_(BETA1).add_(g, alpha=1.0 - BETA1)
        v.mul_(BETA2).addcmul_(g, g, value=1.0 - BETA2)
        del g
        p = (st["master"] if "master" in st else st["p"]).double()
        p = p - LR * (m / (1.0 - BETA1 ** STEP) / (torch.sqrt(v / (1.0 - BETA2 ** STEP)) + ADAM_EPS) + DECAY * p)
        out = {"p": p}
        if "master" in st:
            out["master"] = p
        if case["state"] == "f8":  # the scales; which code a value is rounded to has no 64-bit answer
            out.update(m=None, v=None, ms=m.view(-1, BLOCK).abs().amax(1) / F8MAX, vs=v.view(-1, BLOCK).amax(1) / F8MAX)
        else:
            out.update(m=m, v=v)
        return out
    X, a, gamma = st["X"].double(), st["alpha"] * st["y"], st["gamma"]
    sv = torch.nonzero(a)[:, 0]
    A, c = X[sv], a[sv]
    if kind == "predict_grad":
        Q, up = st["T"].double(), st["up"]
    else:
        Q, up = A, -c
    out = torch.empty_like(Q)
    for i in range(0, Q.shape[0], 2048):
        q = Q[i:i + 2048]
        d2 = (q * q).sum(1)[:, None] + (A * A).sum(1)[None, :]
        K = torch.exp(-gamma * torch.addmm(d2, q, A.T, alpha=-2.0).clamp_(min=0.0)) * c
        out[i:i + 2048] = 2.0 * gamma * up[i:i + 2048, None] * (K @ A - K.sum(1, keepdim=True) * q)
    if kind == "predict_grad":
        return out
    full = torch.zeros_like(X)
    full[sv] = out
    return full
