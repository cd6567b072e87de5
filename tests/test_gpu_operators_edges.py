"""The mini-batch operators where the other tests do not reach.

U = 2^-24 is fp32's largest relative rounding error; every bound below is the sum of the roundings that its comment
counts, to first order, and 1.01 for the orders above."""
import numpy as np
import pytest

from test_gpu_operators import (B1, B2, COUNTS, EPS, U, adam_reference, draw_targets, guarded, half_step, hidden,  # noqa: F401
                                kind, make_model, narrow_reference, untouched, w2v, within)

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
    The loss: q = prod (1 + e) - 1 takes two roundings a node and at each of three joins (2 k + 6), log(1 + q) a logarithm and
    a reciprocal of 1 ulp each (4 U), u - 1, two products and what the ratio log(u) / (u - 1) moves with u's rounding (4 U),
    the terms -s z one rounding a node (fewer than q), their sum one; all of them relative, q / (1 + q) <= log(1 + q) and
    e / (1 + e) <= log(1 + e).
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
    # e: the exponent rounded twice and the power (2 |z| + 4); 2 roundings a node, or at a quarter of the nodes and 2 joins
    # (2 k + 4); log(1 + q) 8 U
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


@pytest.mark.parametrize("dim,stride", [(50, 64), (20, 64)])
def test_a_captured_loss_makes_its_own_gradient(w2v, dim, stride):  # noqa: F811
    """The same in a graph: every replay writes all of it again, whatever became of it in between."""
    import torch
    counts = COUNTS["zipf"]()
    model, _ = make_model(w2v, counts, dim, stride=stride)
    x = hidden(2500, dim, torch.float32)
    t = torch.from_numpy(draw_targets(np.random.default_rng(1), counts, 2500)).cuda()
    w2v.hs_loss(model, x, t)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loss, dx, dsyn1 = w2v.hs_loss(model, x, t)
    for k in range(4):
        for out in (loss, dx, dsyn1):
            out.fill_(float("nan"))
        x.mul_(0.9)
        g.replay()
        want = w2v.hs_loss(model, x, t)
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(dx, want[1]) and torch.equal(dsyn1, want[2]), k


# ------------------------------------------------------------------ sums of many rows
@pytest.mark.parametrize("tree,n,dim,name", [("zipf", 257, 100, "f32"), ("zipf", 4096, 200, "f32"), ("wide", 9000, 65, "f32"),
                                             ("zipf", 8191, 520, "bf16"), ("wide", 33000, 300, "f16"), ("two", 67584, 5, "f32"),
                                             ("zipf", 67584 + 4097, 20, "f32")])
def test_loss_within_its_longest_chain(w2v, tree, n, dim, name):  # noqa: F811
    """Every output against the roundings that the kernels' arrangement has (see softmax_reference), from one block of the
    sums to two slabs of them."""
    counts = COUNTS[tree]()
    rng = np.random.default_rng(n)
    model, otree = make_model(w2v, counts, dim)
    check(w2v, model, otree, hidden(n, dim, kind(name), dim + 3, 1), draw_targets(rng, counts, n), rng.random(n, dtype=np.float32),
          name)


# ------------------------------------------------------------------ layer norm, several rows a group of lanes
@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,d", [(15, 300), (17, 50), (8193, 50), (8195, 300), (20001, 100), (16400, 200), (9001, 255), (5003, 512),
                                 (1100, 700), (1027, 4100)])
def test_norm_backward_of_many_rows(w2v, n, d, name):  # noqa: F811
    """From 8,192 narrow rows on a group of sixteen lanes takes several, the next one on its way; wide rows have the same
    from 512 (of a workgroup each) on. dx of its own, in dy's place and in x's: equal bits."""
    import torch
    t = kind(name)
    stride = d + 5
    g = torch.Generator().manual_seed(n)
    x, xbuf = guarded(n, d, t, stride, 3)
    dy, dybuf = guarded(n, d, t, stride, 3)
    x.copy_(torch.randn(n, d, generator=g) * 1.5 + 0.5)
    dy.copy_(torch.randn(n, d, generator=g))
    w = (1 + 0.3 * torch.randn(d, generator=g)).cuda()
    _, mean, rstd = w2v.layer_norm(x, w)
    out, buf = guarded(n, d, t, d + 1, 2)
    dx, dw, db = w2v.layer_norm_backward(dy, x, w, mean, rstd, dx=out)
    assert untouched(buf, out, n, d, d + 1, 2)
    x64, dy64, w64 = x.double().cpu(), dy.double().cpu(), w.double().cpu()
    r = rstd.double().cpu()[:, None]
    h = (x64 - mean.double().cpu()[:, None]) * r
    a = dy64 * w64
    c0, c1 = a.mean(1, keepdim=True), (a * h).mean(1, keepdim=True)
    want = r * (a - c0 - h * c1)
    # h: two roundings, a: one. A row's sums: 20 elements a lane, 6 levels, 16 wavefronts (42), their terms' own, 1 / d and
    # its product (2). dx: three products and two subtractions.
    c0_b = 45 * U * a.abs().mean(1, keepdim=True)
    c1_b = 48 * U * (a * h).abs().mean(1, keepdim=True)
    bound = 1.01 * r * (4 * U * (a.abs() + c0.abs() + (h * c1).abs()) + c0_b + h.abs() * c1_b + 2 * U * (h * c1).abs())
    within(dx, want, bound + (want.abs() + bound) * half_step(t) + 2.0**-25 * (name == "f16"), "dx")
    # columns: a lane's rows, 2 levels and 4 wavefronts, 32 workgroups one after the other and 16 wavefronts
    chain = -(-n // 512) + 2 + 4 + 32 + 16
    within(dw, (dy64 * h).sum(0), 1.01 * (chain + 3) * U * (dy64 * h).abs().sum(0), "dweight")
    within(db, dy64.sum(0), 1.01 * chain * U * dy64.abs().sum(0), "dbias")
    first = [q.clone() for q in (dx, dw, db)]
    for place, place_buf in ((dy, dybuf), (x, xbuf)):
        kept = place.clone()
        again = w2v.layer_norm_backward(dy, x, w, mean, rstd, dx=place)
        assert all(torch.equal(p, q) for p, q in zip(first, again)) and untouched(place_buf, place, n, d, stride, 3)
        place.copy_(kept)


# ------------------------------------------------------------------ AdamW, rows with gaps over several chunks
GAPPED = [(1000, 50), (301, 301), (3001, 3), (5000, 2), (9000, 1), (130, 64), (700, 7), (2, 5001)]


def gapped_case(p_kind, g_kind, seed):
    """Parameters and gradients whose rows lie differently far apart, and the parameters' buffers."""
    import torch
    g = torch.Generator().manual_seed(seed)
    ps, gs, bufs = [], [], []
    for i, (rows, cols) in enumerate(GAPPED):
        p, buf = guarded(rows, cols, p_kind, cols + 1 + 2 * i, i % 3)
        q, _ = guarded(rows, cols, g_kind, cols + 5 - i % 5, i % 2)
        p.copy_(torch.randn(rows, cols, generator=g) * 0.5)
        q.copy_(torch.randn(rows, cols, generator=g) * 0.1)
        ps.append(p)
        gs.append(q)
        bufs.append((buf, cols + 1 + 2 * i, i % 3))
    return ps, gs, bufs


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_name,g_name", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "f16")])
def test_adamw_of_rows_with_gaps(w2v, bits, p_name, g_name):  # noqa: F811
    """Tensors of more than one chunk of 4,096 elements whose rows have gaps, any number of columns: parameters and moments
    against 64 bits, 8-bit codes and scales bit for bit, the gaps as they were."""
    import torch
    ps, gs, bufs = gapped_case(kind(p_name), kind(g_name), 5)
    opt = w2v.AdamW(ps, gs, bits=bits, betas=(B1, B2), eps=EPS, weight_decay=0.02, seed=9)
    for step in (1, 2, 3):
        old = [p.clone() for p in ps]
        m0, v0 = (a.clone() for a in opt.moments())
        opt.step(step, 0.02, grad_scale=0.5)
        for i, (p, g) in enumerate(zip(ps, gs)):
            n, at = p.numel(), opt.offsets[i]
            cut, blocks = slice(at, at + n), slice(at // 256, at // 256 + -(-n // 256))
            p1, m1, v1, p_b, m_b, v_b = adam_reference(old[i].flatten(), g.flatten(), m0[cut], v0[cut], step, 0.02, 0.02, 0.5)
            within(p.flatten(), p1, p_b + (p1.abs() + p_b) * half_step(kind(p_name)) + 2.0**-25 * (p_name == "f16"), f"p {i}")
            assert untouched(bufs[i][0], p, *GAPPED[i], *bufs[i][1:]), i
            if bits == 32:
                within(opt.m[cut], m1, m_b, f"m {i}")
                within(opt.v[cut], v1, v_b, f"v {i}")
                continue
            scaled = (g.float() * 0.5).flatten().cpu().numpy()
            mc, vc, ms, rs = narrow_reference(scaled, m0[cut].cpu().numpy(), v0[cut].cpu().numpy(), at, step, 9)
            assert np.array_equal(opt.m_scale[blocks].cpu().numpy(), ms) and np.array_equal(opt.v_scale[blocks].cpu().numpy(), rs), (i, step)
            assert np.array_equal(opt.m[cut].cpu().numpy(), mc) and np.array_equal(opt.v[cut].cpu().numpy(), vc), (i, step)
        for g in gs:
            g.mul_(-0.7)


@pytest.mark.parametrize("g_name", ["bf16", "f16"])
def test_adamw_eight_bits_of_narrow_gradients(w2v, g_name):  # noqa: F811
    """8-bit moments with 16-bit parameters and gradients, packed tensors whose last chunk is full, short and ragged."""
    import torch
    gen = torch.Generator().manual_seed(4)
    t = kind(g_name)
    sizes = [1, 255, 256, 4096, 4097, 8192, 12289, 20000]
    ps = [(torch.randn(n, generator=gen) * 0.5).to(t).cuda() for n in sizes]
    gs = [(torch.randn(n, generator=gen) * 0.1).to(t).cuda() for n in sizes]
    opt = w2v.AdamW(ps, gs, bits=8, betas=(B1, B2), eps=EPS, weight_decay=0.1, seed=3)
    for step in (1, 2, 3):
        old = [p.clone() for p in ps]
        m0, v0 = (a.clone() for a in opt.moments())
        opt.step(step, 0.01)
        for i, (p, g) in enumerate(zip(ps, gs)):
            n, at = p.numel(), opt.offsets[i]
            cut, blocks = slice(at, at + n), slice(at // 256, at // 256 + -(-n // 256))
            p1, _, _, p_b, _, _ = adam_reference(old[i], g, m0[cut], v0[cut], step, 0.01, 0.1)
            within(p, p1, p_b + (p1.abs() + p_b) * half_step(t) + 2.0**-25 * (g_name == "f16"), f"p {i}")
            mc, vc, ms, rs = narrow_reference(g.float().cpu().numpy(), m0[cut].cpu().numpy(), v0[cut].cpu().numpy(), at, step, 3)
            assert np.array_equal(opt.m_scale[blocks].cpu().numpy(), ms) and np.array_equal(opt.v_scale[blocks].cpu().numpy(), rs), (i, step)
            assert np.array_equal(opt.m[cut].cpu().numpy(), mc) and np.array_equal(opt.v[cut].cpu().numpy(), vc), (i, step)
        for g in gs:
            g.mul_(-0.5)
