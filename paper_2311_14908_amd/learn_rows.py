"""A kernel SVM on texts, with the rows learned together with the machine.

A text is a bag of tokens; its row is the layer norm of the mean of its tokens' vectors.  Every step embeds and
normalises the training texts, trains the machine on the rows (from the last step's multipliers), takes the
gradient of the machine's objective in the rows back through both, and steps the table and the norm by AdamW.

    python -m paper_2311_14908_amd.learn_rows --texts 4000 --steps 20
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import svmx


def synthetic_texts(n: int, vocabulary: int, seed: int, mean_length: int = 24):
    """Texts of two classes: tokens of frequency 1/rank, and a tenth of a text from its class's own share of the
    vocabulary.  NumPy: tokens int32 [T], starts int64 [n + 1], y int32 [n]; token 0 is padding and does not occur."""
    rng = np.random.default_rng(seed)
    y = np.where(np.arange(n) % 2 == 0, 1, -1).astype(np.int32)
    lens = 1 + rng.geometric(1.0 / mean_length, size=n)
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    total = int(starts[-1])
    tok = np.minimum(np.exp(rng.random(total) * np.log(vocabulary - 1.0)).astype(np.int64), vocabulary - 1)
    own = rng.random(total) < 0.1
    side = np.repeat((y < 0).astype(np.int64), lens)
    marked = vocabulary // 10  # the last tenth of the vocabulary, even tokens for one class and odd ones for the other
    pick = vocabulary - marked + 2 * rng.integers(0, marked // 2, size=total) + side
    return np.where(own, np.minimum(pick, vocabulary - 1), tok).astype(np.int32), starts, y


class RowModel:
    """Table, norm and their optimiser; everything on the current device."""

    def __init__(self, vocabulary: int, d: int, *, state=torch.float32, padding: int = 0, seed: int = 0):
        g = torch.Generator().manual_seed(seed)
        self.table = torch.randn(vocabulary, d, generator=g).mul_(0.5).cuda()
        self.weight, self.bias = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
        self.padding, self.steps = padding, 0
        self.params = [self.table, self.weight, self.bias]
        self.m, self.v, self.m_scale, self.v_scale = svmx.svm_adamw_states(self.params, state)

    def rows(self, tokens, bags, check: bool = True):
        """Rows [texts, d], and what the gradient needs of the way there."""
        e = svmx.svm_embed(self.table, tokens, bags=bags, mean=True, padding=self.padding, check=check)
        x, mean, rstd = svmx.svm_layernorm(e, self.weight, self.bias)
        return x, (tokens, bags, e, mean, rstd)

    def step(self, dX, kept, lr: float, weight_decay: float = 0.01):
        """One step against the rows' gradient dX."""
        tokens, bags, e, mean, rstd = kept
        de, dw, db = svmx.svm_layernorm_grad(dX, e, mean, rstd, self.weight)
        dtable = svmx.svm_embed_grad(tokens, de, self.table.shape[0], bags=bags, mean=True, padding=self.padding, check=False)
        self.steps += 1
        svmx.svm_adamw(self.params, [dtable, dw, db], self.m, self.v, self.steps, lr, weight_decay=[weight_decay, 0.0, 0.0],
                       m_scale=self.m_scale, v_scale=self.v_scale)


def fit(model: RowModel, tokens, bags, y, *, C: float = 1.0, gamma: float | None = None, tol: float = 1e-3, steps: int = 20,
        lr: float = 0.02, report=None):
    """Learn the rows of the texts; returns (machine, rows, objective of every step's machine)."""
    gamma = 0.5 / model.table.shape[1] if gamma is None else gamma
    alpha, objective = None, []
    for s in range(steps + 1):
        X, kept = model.rows(tokens, bags, check=s == 0)
        machine = svmx.svm_train(X, y, C, gamma, tol, alpha_init=alpha)
        objective.append(machine.stats["dual_obj"])
        if report:
            report(s, machine)
        if s == steps:
            return machine, X, objective
        model.step(svmx.svm_objective_grad(X, y, machine.alpha, gamma), kept, lr)
        alpha = machine.alpha


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--texts", type=int, default=4000)
    p.add_argument("--vocabulary", type=int, default=2000)
    p.add_argument("--features", type=int, default=64)
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--states", choices=("f32", "f8"), default="f32", help="optimiser states in 32 or 8 bits")
    a = p.parse_args(argv)
    tok, starts, y = (torch.from_numpy(t).cuda() for t in synthetic_texts(a.texts, a.vocabulary, 1))
    ttok, tstarts, ty = (torch.from_numpy(t).cuda() for t in synthetic_texts(a.texts, a.vocabulary, 2))
    model = RowModel(a.vocabulary, a.features, state=torch.float8_e4m3fn if a.states == "f8" else torch.float32)
    gamma = 0.5 / a.features

    def accuracy(machine, X):
        T, _ = model.rows(ttok, tstarts)
        dec = svmx.svm_predict(X, y, machine.alpha, machine.b, gamma, T)
        return float(((dec > 0) == (ty > 0)).double().mean())

    def report(s, machine):
        print(f"step {s:3d}: objective {machine.stats['dual_obj']:10.3f}, {machine.stats['n_sv']} support vectors, "
              f"{machine.stats['iterations']} pair steps", flush=True)

    first = fit(model, tok, starts, y, gamma=gamma, steps=0)
    print(f"before: {100 * accuracy(first[0], first[1]):.1f}% of the test texts")
    machine, X, _ = fit(model, tok, starts, y, gamma=gamma, steps=a.steps, report=report)
    print(f"after:  {100 * accuracy(machine, X):.1f}% of the test texts")


if __name__ == "__main__":
    main()
