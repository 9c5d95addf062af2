"""The operators together: rows of texts learned with the machine that is trained on them."""
import numpy as np
import pytest
import torch

from paper_2311_14908_amd import learn_rows, svmx

pytestmark = pytest.mark.gpu


def texts(n, seed):
    return [torch.from_numpy(t).cuda() for t in learn_rows.synthetic_texts(n, 400, seed)]


def accuracy(model, machine, X, y, gamma, test):
    T, _ = model.rows(test[0], test[1])
    dec = svmx.svm_predict(X, y, machine.alpha, machine.b, gamma, T)
    return float(((dec > 0) == (test[2] > 0)).double().mean())


@pytest.mark.parametrize("state", [torch.float32, torch.float8_e4m3fn])
def test_rows_become_separable(state):
    tok, starts, y = texts(1000, 1)
    test = texts(1000, 2)
    model = learn_rows.RowModel(400, 32, state=state)
    gamma = 0.5 / 32
    machine, X, first = learn_rows.fit(model, tok, starts, y, gamma=gamma, steps=0)
    before = accuracy(model, machine, X, y, gamma, test)
    machine, X, objective = learn_rows.fit(model, tok, starts, y, gamma=gamma, steps=15)
    assert objective[0] == first[0]
    assert objective[-1] < 0.5 * objective[0]  # the loss that is descended
    assert np.mean(np.diff(objective) < 0) >= 0.8
    assert accuracy(model, machine, X, y, gamma, test) >= before + 0.02  # and what it is for


def test_repeats_bit_for_bit():
    tok, starts, y = texts(300, 3)
    runs = []
    for _ in range(2):
        model = learn_rows.RowModel(400, 20)
        _, X, objective = learn_rows.fit(model, tok, starts, y, steps=3)
        runs.append((X, model.table.clone(), objective))
    assert torch.equal(runs[0][0], runs[1][0]) and torch.equal(runs[0][1], runs[1][1]) and runs[0][2] == runs[1][2]


def test_gradient_of_the_table_is_the_difference_quotient():
    """The whole way, multipliers fixed: W of rows made from the table by the formulas in 64 bits."""
    tok, starts, y = texts(60, 5)
    model = learn_rows.RowModel(400, 6, seed=2)
    gamma, C = 0.3, 1.0
    X, kept = model.rows(tok, starts)
    alpha = svmx.svm_train(X, y, C, gamma, 1e-6).alpha
    dX = svmx.svm_objective_grad(X, y, alpha, gamma)
    de, dw, db = svmx.svm_layernorm_grad(dX, kept[2], kept[3], kept[4], model.weight)
    dtable = svmx.svm_embed_grad(tok, de, 400, bags=starts, mean=True, padding=0).cpu().double()
    c = (alpha * y).cpu()
    t, s = tok.cpu().long(), starts.cpu()
    bag = torch.repeat_interleave(torch.arange(60), s[1:] - s[:-1])
    lens = (s[1:] - s[:-1]).double()

    def W(E):
        rows = torch.zeros(60, 6, dtype=torch.float64).index_add_(0, bag, E[t]) / lens[:, None]
        h = (rows - rows.mean(1, keepdim=True)) / torch.sqrt(rows.var(1, correction=0, keepdim=True) + 1e-5)
        K = torch.exp(-gamma * torch.cdist(h, h, compute_mode="donot_use_mm_for_euclid_dist").square())
        return alpha.cpu().sum() - 0.5 * c @ K @ c

    E = model.table.cpu().double()
    g = torch.Generator().manual_seed(1)
    for _ in range(5):
        D = torch.randn(E.shape, generator=g, dtype=torch.float64)
        num = (W(E + 1e-5 * D) - W(E - 1e-5 * D)) / 2e-5
        want = (D * dtable).sum()
        # 2,400 products of fp32 gradients, each good to about 1e-5 of the largest
        assert abs(num - want) <= 1e-4 * (D * dtable).abs().sum()
    assert bool((dtable[0] == 0).all())  # no token is the padding


def test_command(capsys):
    learn_rows.main(["--texts", "200", "--vocabulary", "300", "--features", "16", "--steps", "2", "--states", "f8"])
    assert "after:" in capsys.readouterr().out
