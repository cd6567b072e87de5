"""The mini-batch operators where the other tests do not reach.

U = 2^-24 is fp32's largest relative rounding error; every bound below is the sum of the roundings that its comment
counts, to first order, and 1.01 for the orders above."""
import numpy as np
import pytest

from test_gpu_operators import COUNTS, U, draw_targets, half_step, hidden, kind, make_model, w2v, within  # noqa: F401

pytestmark = pytest.mark.gpu


def fibonacci(v):
    """Counts whose tree is a chain: the two rarest words have codes of v - 1 turns, one of them all ones."""
    f = [1, 1]
    while len(f) < v:
        f.append(f[-1] + f[-2])
    return np.array(f[::-1], dtype=np.int64)


def tree_of(name):
    return fibonacci(int(name[3:])) if name.startswith("fib") else COUNTS[name]()


def softmax_reference(otree, syn1, x, targets, weights=None, x_off=None):
    """loss, dx and dsyn1 in 64 bits, word by word, and how far fp32 kernels may be off (x_off: how far x itself is).

    z: ceil(d / 64) products of a lane, added as they are formed, and 6 levels of lanes.
    e = exp(-|z|): z log2(e) rounded twice (2 |z| U ln 2 log2(e) of e), its power within 2 ulp (4 U).
    The loss: prod (1 + e) - 1 takes two roundings a node and two a join of lanes, log1p 2 ulp, the terms -s z one
    rounding a node; all of them relative, q / (1 + q) <= log1p(q) and e / (1 + e) <= log1p(e).
    sigmoid: e's error, 1 + e, its reciprocal (1 ulp) and two products.
    dx: a multiply-add a node. dsyn1: 32 rows of a block, 16 blocks of a wavefront, 16 wavefronts, 9 of those in a slab of
    67,584 rows and a slab: 75 additions at most in a row."""
    v, d = otree.codelen.size, x.shape[1]
    x, y = np.asarray(x, dtype=np.float64), np.asarray(syn1, dtype=np.float64)[:, :d]
    x_off = np.zeros_like(x) if x_off is None else x_off
    n = x.shape[0]
    out = dict(loss=np.zeros(n), dx=np.zeros((n, d)), d1=np.zeros((v - 1, d)), loss_b=np.zeros(n), dx_b=np.zeros((n, d)),
               d1_b=np.zeros((v - 1, d)))
    targets = np.asarray(targets)
    for t in np.unique(targets[targets >= 0]):
        at = np.nonzero(targets == t)[0]
        k, code = int(otree.codelen[t]), int(otree.code[t])
        nodes = otree.points[otree.point_off[t]:otree.point_off[t] + k]
        s = np.array([1.0 - 2.0 * ((code >> j) & 1) for j in range(k)])
        rows, xs = y[nodes], x[at]
        sz = (xs @ rows.T) * s
        z_off = (-(-d // 64) + 7) * U * (np.abs(xs) @ np.abs(rows).T) + x_off[at] @ np.abs(rows).T
        e = np.exp(-np.abs(sz))
        f = np.where(sz < 0, 1.0, e) / (1 + e)
        e_rel = (2 * np.abs(sz) + 4) * U
        loss = np.logaddexp(0, -sz).sum(1)
        out["loss"][at] = loss
        out["loss_b"][at] = 1.01 * ((f * z_off + e_rel * e / (1 + e)).sum(1) + (2 * k + 16) * U * loss) + k * 2.0**-126
        w = np.ones((at.size, 1)) if weights is None else np.asarray(weights, dtype=np.float64)[at, None]
        g = -w * s * f
        g_off = 1.01 * np.abs(w) * (f * (1 - f) * z_off + f * (e_rel * np.where(sz < 0, e, 1.0) + 6 * U))
        out["dx"][at] = g @ rows
        out["dx_b"][at] = 1.01 * (g_off + (k + 2) * U * np.abs(g)) @ np.abs(rows)
        out["d1"][nodes] += g.T @ xs
        out["d1_b"][nodes] += 1.01 * (g_off + 76 * U * np.abs(g)).T @ np.abs(xs) + np.abs(g).T @ x_off[at]
    return out


def check(w2v, model, otree, x, targets, weights=None, name="f32"):  # noqa: F811
    import torch
    t = torch.from_numpy(np.asarray(targets, dtype=np.int32)).cuda()
    w = None if weights is None else torch.from_numpy(weights).cuda()
    loss, dx, dsyn1 = w2v.hs_loss(model, x, t, w)
    alone = w2v.hs_loss(model, x, t, grads=False)[0]
    ref = softmax_reference(otree, model.syn1.double().cpu().numpy(), x.double().cpu().numpy(), targets, weights)
    as_t = torch.from_numpy
    within(loss, as_t(ref["loss"]), as_t(ref["loss_b"]), "loss")
    within(alone, as_t(ref["loss"]), as_t(ref["loss_b"]), "loss without gradients")
    want, b = as_t(ref["dx"]), as_t(ref["dx_b"])
    within(dx, want, b + (want.abs() + b) * half_step(kind(name)) + 2.0**-25 * (name == "f16"), "dx")
    within(dsyn1[:, :model.dim], as_t(ref["d1"]), as_t(ref["d1_b"]), "dsyn1")


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


# ------------------------------------------------------------------ codes of 64 turns
@pytest.mark.parametrize("v", [64, 65])
@pytest.mark.parametrize("n", [4, 300, 2500, 20481])
def test_loss_of_the_deepest_codes(w2v, v, n):  # noqa: F811
    """Codes of 63 and 64 turns, all ones among them, with rows without a target before, between and behind the deepest
    words: such a row has no part in any run, nor in what four sorted rows share."""
    import torch
    counts = fibonacci(v)
    model, otree = make_model(w2v, counts, 10)
    assert int(otree.codelen.max()) == model.tree.max_len == v - 1
    rng = np.random.default_rng(n)
    targets = np.array([0, v - 2, -1, v - 2], dtype=np.int32) if n == 4 else rng.integers(-1, v, n).astype(np.int32)
    if n > 4:
        deep = rng.random(n) < 0.5
        targets[deep] = rng.choice([-1, v - 2, v - 1, v - 3], size=int(deep.sum()))
    x = hidden(n, 10, torch.float32)
    check(w2v, model, otree, x, targets, rng.random(n, dtype=np.float32))
    loss, dx, _ = w2v.hs_loss(model, x, torch.from_numpy(targets).cuda())
    none = torch.from_numpy(targets < 0).cuda()
    assert not loss[none].any() and not dx[none].any()


# ------------------------------------------------------------------ the gradient that hs_loss makes itself
@pytest.mark.parametrize("dim,stride", [(64, 64), (50, 64), (33, 64), (32, 64), (20, 64), (300, 320), (4, 4)])
@pytest.mark.parametrize("n", [0, 1, 3000])
def test_loss_makes_its_own_gradient(w2v, monkeypatch, dim, stride, n):  # noqa: F811
    """Without a dsyn1 of the caller's: its columns as in one that is given, zeros in the padding whatever lay in the
    memory before, and the zeros written once, by the kernels (torch fills padding of 32 columns and more alone)."""
    import torch
    counts = COUNTS["zipf"]()
    model, _ = make_model(w2v, counts, dim, stride=stride)
    x = hidden(n, dim, torch.float32)
    t = torch.from_numpy(draw_targets(np.random.default_rng(n), counts, n)).cuda()
    want = w2v.hs_loss(model, x, t, dsyn1=torch.full_like(model.syn1, 3.0))[2][:, :dim].clone()
    filled = []
    zero_ = torch.Tensor.zero_
    monkeypatch.setattr(torch, "zeros_like", lambda *a, **k: pytest.fail("the gradient's zeros, twice"))
    monkeypatch.setattr(torch.Tensor, "zero_", lambda self: filled.append(tuple(self.shape)) or zero_(self))
    for _ in range(3):
        stale = torch.full_like(model.syn1, float("nan"))
        del stale   # the next tensor of this size takes its memory
        got = w2v.hs_loss(model, x, t)[2]
        assert got.shape == model.syn1.shape and torch.equal(got[:, :dim], want) and not got[:, dim:].any()
        del got
    assert set(filled) <= ({(model.V - 1, stride - dim)} if stride - dim >= 32 else set())
