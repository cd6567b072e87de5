"""The mini-batch operators where the other tests do not reach.

U = 2^-24 is fp32's largest relative rounding error; every bound below is the sum of the roundings that its comment
counts, to first order, and 1.01 for the orders above."""
import numpy as np
import pytest

from test_gpu_operators import COUNTS, U, make_model, w2v, within  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ losses near zero
@pytest.mark.parametrize("tree", ["two", "zipf", "deep"])
@pytest.mark.parametrize("n", [1, 130, 20481])
def test_loss_of_likely_words_keeps_its_digits(w2v, tree, n):  # noqa: F811
    """s z from 14 to 50 at every node, by products that are exact: losses of 1e-6 down to 1e-22, against a bound that is
    relative to them. One row a wavefront, and four sorted rows that share the whole path."""
    import torch
    counts = COUNTS[tree]()
    word = counts.size - 1
    model, otree = make_model(w2v, counts, 3)
    k, code = int(otree.codelen[word]), int(otree.code[word])
    nodes = otree.points[otree.point_off[word]:otree.point_off[word] + k]
    model.syn1[:, :3] = 0
    for j, node in enumerate(nodes):
        model.syn1[int(node), 0] = (1 - 2 * ((code >> j) & 1)) * (1 + (j % 5) / 8)
    x = torch.zeros(n, 3, device="cuda")
    x[:, 0] = 14 + (torch.arange(n, device="cuda") % 76) / 4
    z = x[:, :1].double().cpu().numpy() * (1 + (np.arange(k) % 5) / 8)
    loss = np.log1p(np.exp(-z)).sum(1)
    # e: the exponent rounded twice and the power (2 |z| + 4); 2 roundings a node and at 4 joins; log1p 2 ulp
    bound = 1.01 * ((2 * z + 4) * U * np.exp(-z)).sum(1) + (2 * k + 12) * U * loss
    t = torch.full((n,), word, dtype=torch.int32, device="cuda")
    for grads in (True, False):
        got = w2v.hs_loss(model, x, t, grads=grads)[0]
        within(got, torch.from_numpy(loss), torch.from_numpy(bound), f"loss, grads={grads}")
