"""The mini-batch operators (layer norm, the hierarchical softmax as a loss, AdamW) against plain 64-bit
implementations on the same inputs.

Tolerances follow from the kernels' arithmetic. U = 2^-24 is fp32's largest relative rounding error; a sum whose
longest chain of additions has D links is off by at most about D U times the sum of the terms' magnitudes; a result
stored in a type of fewer bits is off by half a step of it (eps / 2) more."""
import math

import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

U = 2.0**-24


@pytest.fixture(scope="module")
def w2v():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1606_07822_amd as w2v
    w2v.lib()
    return w2v


def kind(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def half_step(t):
    import torch
    return 0.0 if t == torch.float32 else torch.finfo(t).eps / 2


def within(got, want, bound, what):
    """Every element off by at most its bound (64-bit tensors on the CPU)."""
    got, want, bound = got.double().cpu(), want.double().cpu(), bound.double().cpu()
    off = (got - want).abs() - bound
    worst = int(off.argmax()) if off.numel() else 0
    assert off.numel() == 0 or bool((off <= 0).all()), (
        what, worst, got.flatten()[worst].item(), want.flatten()[worst].item(), bound.flatten()[worst].item())


CANARY = 12345.0


def guarded(rows, dim, t, stride=None, lead=0):
    """A [rows, dim] view into a buffer that is filled with a value nothing else has, `lead` elements in, rows `stride`
    apart; and the buffer."""
    import torch
    stride = dim if stride is None else stride
    buf = torch.full((lead + max(rows, 1) * stride + 8,), CANARY, dtype=torch.float32, device="cuda").to(t)
    return buf[lead:lead + rows * stride].view(rows, stride)[:, :dim] if rows else buf[:0].view(0, dim), buf


def untouched(buf, view, rows, dim, stride, lead):
    """Whether the buffer outside the view still holds the guard value."""
    import torch
    mask = torch.ones(buf.numel(), dtype=torch.bool, device="cuda")
    if rows:
        mask[lead:lead + rows * stride].view(rows, stride)[:, :dim] = False
    return bool((buf[mask] == torch.tensor(CANARY).to(buf.dtype).cuda()).all())


# ------------------------------------------------------------------ layer norm
NORM_SIZES = [(1, 1), (1, 300), (3, 2), (5, 7), (33, 64), (257, 100), (64, 300), (19, 321), (130, 513), (37, 1023), (9, 2048),
              (12, 2049), (17, 4096), (3, 8191), (2, 8193), (5, 16384), (1, 16383)]


def norm_inputs(n, d, t, stride, lead, seed=1):
    import torch
    g = torch.Generator().manual_seed(seed)
    x, _ = guarded(n, d, t, stride, lead)
    dy, _ = guarded(n, d, t, stride, lead)
    x.copy_(torch.randn(n, d, generator=g) * 1.5 + 0.5)
    dy.copy_(torch.randn(n, d, generator=g))
    return x, dy, (1 + 0.3 * torch.randn(d, generator=g)).cuda(), (0.2 * torch.randn(d, generator=g)).cuda()


def norm_reference(x, w, b, eps):
    x = x.double().cpu()
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    rstd = 1 / (var + eps).sqrt()
    h = (x - mean[:, None]) * rstd[:, None]
    y = h if w is None else h * w.double().cpu()
    return (y if b is None else y + b.double().cpu()), mean, rstd, h


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,d", NORM_SIZES)
def test_norm_forward(w2v, n, d, name):
    import torch
    t = kind(name)
    for stride, lead, w_kind in ((d, 0, torch.float32), (d + 5, 3, t)):
        x, _, w, b = norm_inputs(n, d, t, stride, lead)
        w, b = w.to(w_kind), b.to(w_kind)
        out, buf = guarded(n, d, t, stride, lead)
        y, mean, rstd = w2v.layer_norm(x, w, b, 1e-5, out=out)
        want, m64, r64, h = norm_reference(x, w, b, 1e-5)
        # a lane adds at most 32 elements one after the other, then 10 levels of lanes and wavefronts
        a = x.double().cpu().abs().mean(1)
        mean_off = 45 * U * a
        within(mean, m64, mean_off, "mean")
        # the centred values carry the mean's error, which enters the variance with their sum, about zero: second order
        rel = (24 + 4) * U + (mean_off * r64) ** 2
        within(rstd, r64, r64 * rel, "rstd")
        w64, b64 = w.double().cpu().abs(), b.double().cpu().abs()
        bound = w64 * ((mean_off * r64)[:, None] + h.abs() * (rel + 4 * U)[:, None]) + 2 * U * (want.abs() + b64)
        within(y, want, bound + (want.abs() + bound) * half_step(t) + 2.0**-25 * (name == "f16"), "y")
        assert untouched(buf, out, n, d, stride, lead)


def test_norm_without_affine_in_place_and_empty(w2v):
    import torch
    x, _, w, b = norm_inputs(70, 96, torch.float32, 96, 0)
    want = w2v.layer_norm(x)[0].clone()
    within(want, norm_reference(x, None, None, 1e-5)[0], torch.full_like(want, 1e-5), "y")
    only_bias = w2v.layer_norm(x, None, b)[0]
    within(only_bias, norm_reference(x, None, b, 1e-5)[0], torch.full_like(want, 1e-5), "y with a bias alone")
    assert torch.equal(w2v.layer_norm(x, out=x)[0], want)
    y, mean, rstd = w2v.layer_norm(torch.empty(0, 96, device="cuda"), w, b)
    assert y.shape == (0, 96) and mean.numel() == 0 and rstd.numel() == 0
    dx, dw, db = w2v.layer_norm_backward(torch.empty(0, 96, device="cuda"), torch.empty(0, 96, device="cuda"), w, mean, rstd)
    assert dx.shape == (0, 96) and not dw.any() and not db.any()


def test_norm_of_equal_and_of_far_columns(w2v):
    """A row of one value has no variance: y is the bias. A mean of 1e4 with a deviation of 1: the variance survives."""
    import torch
    x = torch.full((3, 300), 7.25, device="cuda")
    b = torch.randn(300, device="cuda")
    y, mean, rstd = w2v.layer_norm(x, torch.ones(300, device="cuda"), b)
    assert torch.equal(y, b.expand(3, 300)) and torch.equal(mean, x[:, 0])
    x = torch.randn(5, 1000, device="cuda") + 1e4
    y, mean, rstd = w2v.layer_norm(x)
    want, m64, r64, h = norm_reference(x, None, None, 1e-5)
    off = (45 * U * x.double().cpu().abs().mean(1) * r64)[:, None]
    within(y, want, off + h.abs() * (off**2 + 30 * U), "y")


def test_norm_keeps_rows_that_are_not_finite_to_themselves(w2v):
    import torch
    x, dy, w, b = norm_inputs(40, 300, torch.float32, 320, 0)
    clean = w2v.layer_norm(x, w, b)[0].clone()
    x[7, 3], x[21, 299] = float("nan"), float("inf")
    y, mean, rstd = w2v.layer_norm(x, w, b)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[7, 21]] = True
    assert torch.equal(y[~bad], clean[~bad]) and bool(y[bad].isnan().any(1).all())


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,d", NORM_SIZES + [(4099, 300), (1500, 1100)])
def test_norm_backward(w2v, n, d, name):
    import torch
    t = kind(name)
    for stride, lead, w_kind in ((d, 0, torch.float32), (d + 3, 1, t)):
        x, dy, w, b = norm_inputs(n, d, t, stride, lead)
        w = w.to(w_kind)
        _, mean, rstd = w2v.layer_norm(x, w, b.to(w_kind))
        out, buf = guarded(n, d, t, stride, lead)
        dx, dw, db = w2v.layer_norm_backward(dy, x, w, mean, rstd, dx=out)
        x64, dy64, w64 = x.double().cpu(), dy.double().cpu(), w.double().cpu()
        r = rstd.double().cpu()[:, None]
        h = (x64 - mean.double().cpu()[:, None]) * r
        a = dy64 * w64
        c0, c1 = a.mean(1, keepdim=True), (a * h).mean(1, keepdim=True)
        want = r * (a - c0 - h * c1)
        bound = r * (5 * U * a.abs() + 46 * U * a.abs().mean(1, keepdim=True)
                     + h.abs() * (50 * U * (a * h).abs().mean(1, keepdim=True) + 5 * U * c1.abs()) + 3 * U * c0.abs())
        within(dx, want, bound + (want.abs() + bound) * half_step(t) + 2.0**-25 * (name == "f16"), "dx")
        # rows of a lane (16 or so), lanes and wavefronts (6), then the workgroups' sums: 64 in a chain and 16 wavefronts
        within(dw, (dy64 * h).sum(0), 120 * U * (dy64 * h).abs().sum(0), "dweight")
        within(db, dy64.sum(0), 120 * U * dy64.abs().sum(0), "dbias")
        assert untouched(buf, out, n, d, stride, lead)
        again = w2v.layer_norm_backward(dy, x, w, mean, rstd)
        assert torch.equal(again[1], dw) and torch.equal(again[2], db) and torch.equal(again[0], dx)


def test_norm_of_more_than_2_to_32_elements(w2v):
    """The last rows of an array whose elements need 33 bits to count."""
    import torch
    n, d = 2**32 // 16384 + 64, 16384
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    x[-80:].normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    x[:-80].fill_(1.0)
    y, mean, rstd = w2v.layer_norm(x, out=x.clone())
    want, m64, r64, h = norm_reference(x[-80:], None, None, 1e-5)
    off = (45 * U * x[-80:].double().cpu().abs().mean(1) * r64)[:, None]
    fp32 = off + h.abs() * (off**2 + 30 * U)
    within(y[-80:], want, fp32 + (want.abs() + fp32) * 2.0**-8, "y")
    dx, _, _ = w2v.layer_norm_backward(x, x, None, mean, rstd, dx=y)
    a = x[-80:].double().cpu()
    want = r64[:, None] * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
    # the kernel's own mean and rstd, off by 45 U and 28 U, and the bounds of the backward pass's sums
    fp32 = 200 * U * r64[:, None] * (1 + a.abs()) * (1 + h.abs())
    within(dx[-80:], want, fp32 + (want.abs() + fp32) * 2.0**-8, "dx")


def test_norm_outputs_one_by_one(w2v):
    """The C calls without statistics, with one of the two weight gradients."""
    import torch
    x, dy, w, b = norm_inputs(50, 130, torch.float32, 130, 0)
    y, mean, rstd = w2v.layer_norm(x, w, b)
    dx, dw, db = w2v.layer_norm_backward(dy, x, w, mean, rstd)
    s, L = torch.cuda.current_stream().cuda_stream, w2v.lib()
    alone = torch.zeros_like(x)
    assert L.w2v_layer_norm(x.data_ptr(), 0, 50, 130, 130, w.data_ptr(), b.data_ptr(), 0, 1e-5, alone.data_ptr(), 130, None,
                            None, s) == w2v.W2V_OK
    assert torch.equal(alone, y)
    ws = torch.empty(L.w2v_layer_norm_backward_workspace_bytes(50, 130), dtype=torch.uint8, device="cuda")
    for which in (0, 1, 2):
        out, sums = torch.zeros_like(x), torch.zeros(2, 130, device="cuda")
        rc = L.w2v_layer_norm_backward(
            dy.data_ptr(), 130, x.data_ptr(), 0, 50, 130, 130, w.data_ptr(), 0, mean.data_ptr(), rstd.data_ptr(), out.data_ptr(),
            130, sums[0].data_ptr() if which == 1 else None, sums[1].data_ptr() if which == 2 else None,
            ws.data_ptr() if which else None, ws.numel() if which else 0, s)
        assert rc == w2v.W2V_OK and torch.equal(out, dx)
        assert torch.equal(sums[0], dw) if which == 1 else not sums[0].any()
        assert torch.equal(sums[1], db) if which == 2 else not sums[1].any()


def test_norm_backward_against_differences(w2v):
    """dx, dweight and dbias as slopes of sum(dy y): a central difference of the forward kernel, h = 2^-5."""
    import torch
    x, dy, w, b = norm_inputs(6, 50, torch.float32, 50, 0)
    g = torch.Generator().manual_seed(5)
    _, mean, rstd = w2v.layer_norm(x, w, b)
    dx, dw, db = w2v.layer_norm_backward(dy, x, w, mean, rstd)
    h = 2.0**-5
    for i, grad in ((0, dx), (1, dw), (2, db)):
        args = [x, w, b]
        v = torch.randn(args[i].shape, generator=g).cuda()
        sides, sides64 = [], []
        for s in (h, -h):
            moved = [a + s * v if k == i else a for k, a in enumerate(args)]
            sides.append((w2v.layer_norm(*moved)[0].double() * dy.double()).sum().item())
            sides64.append((norm_reference(moved[0], moved[1], moved[2], 1e-5)[0] * dy.double().cpu()).sum().item())
        slope = (grad.double() * v.double()).sum().item()
        exact = (sides64[0] - sides64[1]) / (2 * h)
        # the kernel's quotient carries both sides' roundings (each y off by less than 100 U (|x| + 1) at these sizes);
        # what the quotient itself lacks of the slope is third order in h
        rounding = 100 * U * (dy.abs() * (x.abs() + 1)).sum().item() / h
        assert abs((sides[0] - sides[1]) / (2 * h) - exact) <= rounding
        assert abs(slope - exact) <= rounding + 8 * h * h * (dy.abs().sum() * v.abs().max() ** 3).item()


# ------------------------------------------------------------------ the tree
def zipf_counts(v):
    return np.sort((1e6 / np.arange(1, v + 1) ** 1.0).astype(np.int64) + 1)[::-1].copy()


COUNTS = {
    "two": lambda: np.array([5, 3], dtype=np.int64),
    "three": lambda: np.array([5, 3, 1], dtype=np.int64),
    "equal": lambda: np.full(64, 9, dtype=np.int64),
    "zipf": lambda: zipf_counts(1000),
    "deep": lambda: (2 ** np.arange(46, dtype=np.int64))[::-1].copy(),      # a chain: codes of 1 to 45 turns
    "wide": lambda: zipf_counts(20011),
}


def make_model(w2v, counts, dim, stride=None, seed=3, scale=1.0):
    import torch
    rng = np.random.default_rng(seed)
    c = torch.from_numpy(counts).cuda()
    tree = w2v.build_huffman(c)
    v = counts.size
    syn0 = (rng.standard_normal((v, dim)) * scale / math.sqrt(dim)).astype(np.float32)
    syn1 = (rng.standard_normal((v - 1, dim)) * 2 * scale / math.sqrt(dim)).astype(np.float32)
    voc = w2v.Vocab(None, None, c, None, v, int(counts.sum()), None)
    return w2v.make_model(syn0, syn1, voc, tree, stride=stride, pad_value=float("nan")), oracle.build_huffman(counts)


def loss_reference(otree, syn1, x, targets, weights, dim):
    """Row by row in 64 bits: loss, dx, dsyn1 and the magnitudes that their bounds go by."""
    n, v = x.shape[0], otree.codelen.size
    x, y = x.double().cpu().numpy(), syn1[:, :dim].double().cpu().numpy()
    out = dict(loss=np.zeros(n), dx=np.zeros((n, dim)), d1=np.zeros((v - 1, dim)), loss_b=np.zeros(n),
               dx_b=np.zeros((n, dim)), d1_b=np.zeros((v - 1, dim)))
    for i, t in enumerate(targets):
        if t < 0:
            continue
        k = int(otree.codelen[t])
        nodes = otree.points[otree.point_off[t]:otree.point_off[t] + k]
        s = 1.0 - 2.0 * ((int(otree.code[t]) >> np.arange(k)) & 1)
        rows = y[nodes]
        z = rows @ x[i]
        z_off = 24 * U * (np.abs(rows) @ np.abs(x[i]))           # 16 elements a lane, 6 levels of lanes, the product
        out["loss"][i] = np.logaddexp(0, -s * z).sum()
        # exp(-|z|) is off by 3 U (|z| e^-|z| < 0.4), the product of 1 + e by U a node
        out["loss_b"][i] = (z_off + 8 * U).sum() + 6 * U * out["loss"][i]
        w = 1.0 if weights is None else float(weights[i])
        g = -w * s / (1 + np.exp(s * z))
        g_off = abs(w) * (z_off / 4 + 8 * U)
        out["dx"][i] = g @ rows
        out["dx_b"][i] = (g_off + (k + 2) * U * np.abs(g)) @ np.abs(rows)
        np.add.at(out["d1"], nodes, g[:, None] * x[i])
        # 64 rows in a block, 64 blocks in a join, 16 joins; a slab's sum is one more
        np.add.at(out["d1_b"], nodes, (g_off + 160 * U * np.abs(g))[:, None] * np.abs(x[i]))
    return out


def check_loss(w2v, model, otree, x, targets, weights, name="f32", **given):
    import torch
    t = torch.from_numpy(np.asarray(targets, dtype=np.int32)).cuda()
    w = None if weights is None else torch.from_numpy(weights).cuda()
    loss, dx, dsyn1 = w2v.hs_loss(model, x, t, w, **given)
    d = model.dim
    ref = loss_reference(otree, model.syn1, x, targets, weights, d)
    as_t = torch.from_numpy
    within(loss, as_t(ref["loss"]), as_t(ref["loss_b"]), "loss")
    want, b = as_t(ref["dx"]), as_t(ref["dx_b"])
    within(dx, want, b + (want.abs() + b) * half_step(kind(name)) + 2.0**-25 * (name == "f16"), "dx")
    within(dsyn1[:model.V - 1, :d], as_t(ref["d1"]), as_t(ref["d1_b"]), "dsyn1")
    return loss, dx, dsyn1


def hidden(n, d, t, stride=None, lead=0, seed=11):
    import torch
    g = torch.Generator().manual_seed(seed)
    x, _ = guarded(n, d, t, stride, lead)
    x.copy_(torch.randn(n, d, generator=g))
    return x


def draw_targets(rng, counts, n, masked=0.1):
    p = counts / counts.sum()
    t = rng.choice(counts.size, size=n, p=p).astype(np.int32)
    t[rng.random(n) < masked] = -1
    return t


@pytest.mark.parametrize("tree", sorted(COUNTS))
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 130])
def test_loss_trees_and_row_counts(w2v, tree, n):
    counts = COUNTS[tree]()
    rng = np.random.default_rng(n)
    model, otree = make_model(w2v, counts, 20)
    targets = rng.integers(0, counts.size, n).astype(np.int32) if n % 2 else draw_targets(rng, counts, n)
    import torch
    check_loss(w2v, model, otree, hidden(n, 20, torch.float32), targets, rng.random(n, dtype=np.float32))


@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [1, 3, 50, 64, 65, 100, 128, 200, 257, 300, 321, 511, 513, 1024])
def test_loss_widths_and_types(w2v, dim, name):
    counts = COUNTS["zipf"]()
    rng = np.random.default_rng(dim)
    model, otree = make_model(w2v, counts, dim, stride=(dim + 3) // 4 * 4 + 4)
    check_loss(w2v, model, otree, hidden(97, dim, kind(name), dim + 7, 1), draw_targets(rng, counts, 97),
               rng.random(97, dtype=np.float32), name)


@pytest.mark.parametrize("n", [2047, 2048, 2049, 4096, 4097, 9000])
def test_loss_many_rows(w2v, n):
    """More than one block of the sort, more than one join."""
    import torch
    counts = COUNTS["wide"]()
    rng = np.random.default_rng(n)
    model, otree = make_model(w2v, counts, 6)
    check_loss(w2v, model, otree, hidden(n, 6, torch.float32), draw_targets(rng, counts, n), None)


@pytest.mark.parametrize("n,dim,name", [(8192, 130, "bf16"), (8195, 300, "f32"), (8193, 65, "f16"), (8200, 700, "f16")])
def test_loss_thousands_of_rows(w2v, n, dim, name):
    """Rows in thousands, at the widths of a lane's columns."""
    counts = COUNTS["zipf"]()
    rng = np.random.default_rng(n)
    model, otree = make_model(w2v, counts, dim)
    check_loss(w2v, model, otree, hidden(n, dim, kind(name), dim + 3, 1), draw_targets(rng, counts, n),
               rng.random(n, dtype=np.float32) / n, name)


@pytest.mark.parametrize("tree,n,dim,name", [("zipf", 20479, 70, "f32"), ("zipf", 20480, 130, "bf16"), ("wide", 20483, 300, "f32"),
                                             ("zipf", 20481, 65, "f16"), ("zipf", 20490, 700, "f16"), ("wide", 32768, 6, "f32"),
                                             ("wide", 32769, 50, "bf16"), ("deep", 20493, 10, "f32"), ("deep", 40001, 9, "f32")])
def test_loss_large_batches(w2v, tree, n, dim, name):
    """From 20,480 rows on four sorted ones a wavefront, their common levels together, then each row's own (not where they
    are too wide for that); past 32,768 more rows a workgroup in the sort."""
    counts = COUNTS[tree]()
    rng = np.random.default_rng(n)
    model, otree = make_model(w2v, counts, dim)
    check_loss(w2v, model, otree, hidden(n, dim, kind(name), dim + 3, 1), draw_targets(rng, counts, n),
               rng.random(n, dtype=np.float32) / n, name)


@pytest.mark.parametrize("n", [65, 1023, 1025, 2049, 5000])
def test_loss_many_rows_of_a_deep_tree(w2v, n):
    """Codes of up to 45 turns, every word as likely as the next: keys of 64 bits, runs that are cut at every level."""
    import torch
    counts = COUNTS["deep"]()
    rng = np.random.default_rng(n)
    model, otree = make_model(w2v, counts, 10)
    targets = rng.integers(-1, counts.size, n).astype(np.int32)
    check_loss(w2v, model, otree, hidden(n, 10, torch.float32), targets, rng.random(n, dtype=np.float32))


@pytest.mark.parametrize("tree", ["two", "zipf"])
def test_loss_more_rows_than_a_slab(w2v, tree):
    """67,584 rows are summed together; what comes after them is added."""
    import torch
    counts = COUNTS[tree]()
    n = 67584 + 77
    rng = np.random.default_rng(4)
    model, otree = make_model(w2v, counts, 4)
    x = hidden(n, 4, torch.float32)
    targets = draw_targets(rng, counts, n)
    loss, dx, dsyn1 = w2v.hs_loss(model, x, torch.from_numpy(targets).cuda())
    ref = loss_reference(otree, model.syn1, x, targets, None, 4)
    as_t = torch.from_numpy
    within(loss, as_t(ref["loss"]), as_t(ref["loss_b"]), "loss")
    within(dx, as_t(ref["dx"]), as_t(ref["dx_b"]), "dx")
    within(dsyn1[:, :4], as_t(ref["d1"]), as_t(ref["d1_b"]), "dsyn1")


@pytest.mark.parametrize("which", ["one", "none", "every", "rarest"])
def test_loss_target_patterns(w2v, which):
    """All rows the same word; none with a target; each word once; the two deepest words."""
    import torch
    counts = COUNTS["zipf"]()
    v = counts.size
    targets = {"one": np.full(3000, 5), "none": np.full(130, -1), "every": np.arange(v), "rarest": v - 1 - np.arange(300) % 2}
    targets = targets[which].astype(np.int32)
    model, otree = make_model(w2v, counts, 12)
    loss, dx, dsyn1 = check_loss(w2v, model, otree, hidden(targets.size, 12, torch.float32), targets, None)
    if which == "none":
        assert not loss.any() and not dx.any() and not dsyn1[:, :12].any()


def test_loss_of_rows_without_a_target_reads_nothing_of_them(w2v):
    """Values that are not finite in rows without a target change nothing."""
    import torch
    counts = COUNTS["zipf"]()
    rng = np.random.default_rng(8)
    model, otree = make_model(w2v, counts, 40)
    targets = torch.from_numpy(draw_targets(rng, counts, 200, 0.4)).cuda()
    x = hidden(200, 40, torch.float32)
    clean = [t.clone() for t in w2v.hs_loss(model, x, targets)]
    x[targets < 0] = float("nan")
    for a, b in zip(clean, w2v.hs_loss(model, x, targets)):
        assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))
    assert bool(torch.isfinite(clean[2][:, :40]).all())


def test_loss_keeps_a_row_that_is_not_finite_to_its_path(w2v):
    import torch
    counts = COUNTS["zipf"]()
    rng = np.random.default_rng(9)
    model, otree = make_model(w2v, counts, 40)
    targets = draw_targets(rng, counts, 200, 0.0)
    t = torch.from_numpy(targets).cuda()
    x = hidden(200, 40, torch.float32)
    clean = [c.clone() for c in w2v.hs_loss(model, x, t)]
    x[17] = float("nan")
    loss, dx, dsyn1 = w2v.hs_loss(model, x, t)
    others = torch.arange(200, device="cuda") != 17
    assert torch.equal(loss[others], clean[0][others]) and bool(loss[17].isnan())
    assert torch.equal(dx[others], clean[1][others])
    word = targets[17]
    path = torch.zeros(model.V - 1, dtype=torch.bool, device="cuda")
    path[torch.from_numpy(otree.points[otree.point_off[word]:otree.point_off[word + 1]].astype(np.int64)).cuda()] = True
    assert torch.equal(dsyn1[~path][:, :40], clean[2][~path][:, :40]) and bool(dsyn1[path][:, :40].isnan().all())


def test_loss_of_targets_outside_the_tree(w2v):
    """A word past the vocabulary, and one whose code is longer than the caller said: NaN, and no gradient."""
    import torch
    counts = COUNTS["deep"]()
    model, otree = make_model(w2v, counts, 8)
    x = hidden(5, 8, torch.float32)
    t = torch.tensor([0, counts.size, 2**31 - 1, -2**31, 3], dtype=torch.int32, device="cuda")
    loss, dx, dsyn1 = w2v.hs_loss(model, x, t)
    assert loss.isnan().tolist() == [False, True, True, False, False] and loss[3].item() == 0
    assert not dx[1:4].any() and bool(torch.isfinite(dsyn1[:, :8]).all())
    import dataclasses
    short = dataclasses.replace(model, tree=dataclasses.replace(model.tree, max_len=3))
    loss, dx, dsyn1 = w2v.hs_loss(short, x, torch.tensor([0, 1, 2, 3, 40], dtype=torch.int32, device="cuda"))
    assert loss.isnan().tolist() == [False, False, False, True, True] and not dx[3:].any()


def test_loss_far_out(w2v):
    """Products of +-1e4: a loss of 0 or of the product, a gradient of 0 or of the whole row."""
    import torch
    model, otree = make_model(w2v, COUNTS["two"](), 4)
    model.syn1[0, :4] = 100.0
    x = torch.tensor([[25.0] * 4, [-25.0] * 4], device="cuda")
    for word in (0, 1):
        loss, dx, _ = w2v.hs_loss(model, x, torch.tensor([word, word], dtype=torch.int32, device="cuda"))
        s = 1 - 2 * (int(otree.code[word]) & 1)
        assert loss.tolist() == ([0.0, 1e4] if s > 0 else [1e4, 0.0])
        right = 0 if s > 0 else 1
        assert not dx[right].any() and torch.equal(dx[1 - right], torch.full((4,), -100.0 * s, device="cuda"))


def test_loss_padding_and_repeatability(w2v):
    """Columns between rows stay as they are (a dsyn1 of syn1's layout may get zeros there); two calls give equal bits;
    without gradients the same loss."""
    import torch
    counts = COUNTS["wide"]()
    rng = np.random.default_rng(2)
    model, otree = make_model(w2v, counts, 50, stride=64)
    n = 5000
    x = hidden(n, 50, torch.float32, 64)
    t = torch.from_numpy(draw_targets(rng, counts, n)).cuda()
    dx, dbuf = guarded(n, 50, torch.float32, 56, 2)
    wide = torch.full((counts.size - 1, 80), CANARY, device="cuda")
    ds = wide[:, :64]
    ws = w2v.hs_loss_workspace(model, x)
    ws.fill_(255)
    first = w2v.hs_loss(model, x, t, dx=dx, dsyn1=ds, workspace=ws)
    assert untouched(dbuf, dx, n, 50, 56, 2) and bool((wide[:, 50:] == CANARY).all())
    kept = [first[0].clone(), dx.clone(), ds.clone()]
    ws.fill_(0)
    again = w2v.hs_loss(model, x, t, dx=dx, dsyn1=ds, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(kept, again))
    own = w2v.hs_loss(model, x, t, dsyn1=torch.full_like(model.syn1, CANARY))[2]
    assert torch.equal(own[:, :50], kept[2][:, :50]) and bool(((own[:, 50:] == 0) | (own[:, 50:] == CANARY)).all())
    alone, none1, none2 = w2v.hs_loss(model, x, t, grads=False)
    assert torch.equal(alone, kept[0]) and none1 is None and none2 is None


def test_loss_empty_batch(w2v):
    import torch
    model, _ = make_model(w2v, COUNTS["zipf"](), 10)
    loss, dx, dsyn1 = w2v.hs_loss(model, torch.empty(0, 10, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"),
                                  dsyn1=torch.full_like(model.syn1, 3.0))
    assert loss.numel() == 0 and dx.shape == (0, 10) and not dsyn1[:, :10].any()


def test_loss_against_differences(w2v):
    """dx and dsyn1 as slopes of sum(w loss): central differences of the kernel's loss, h = 2^-5."""
    import torch
    counts = COUNTS["zipf"]()
    rng = np.random.default_rng(6)
    model, otree = make_model(w2v, counts, 30)
    n, h = 80, 2.0**-5
    targets = draw_targets(rng, counts, n)
    t = torch.from_numpy(targets).cuda()
    weights = rng.random(n, dtype=np.float32)
    w = torch.from_numpy(weights).cuda()
    x = hidden(n, 30, torch.float32)
    _, dx, dsyn1 = w2v.hs_loss(model, x, t, w)
    base = model.syn1.clone()
    g = torch.Generator().manual_seed(1)
    for which in ("x", "syn1"):
        v = torch.randn((n, 30) if which == "x" else (counts.size - 1, 30), generator=g).cuda()
        total, exact, rounding = [], [], 0.0
        for s in (h, -h):
            model.syn1.copy_(base)
            moved = x
            if which == "x":
                moved = x + s * v
            else:
                model.syn1[:, :30] += s * v
            total.append((w2v.hs_loss(model, moved, t, grads=False)[0].double() * w.double()).sum().item())
            ref = loss_reference(otree, model.syn1, moved, targets, weights, 30)
            exact.append(float((ref["loss"] * weights).sum()))
            rounding += float((ref["loss_b"] * weights).sum()) / (2 * h)
        model.syn1.copy_(base)
        slope = ((dx if which == "x" else dsyn1[:, :30]).double() * v.double()).sum().item()
        quotient = (exact[0] - exact[1]) / (2 * h)
        assert abs((total[0] - total[1]) / (2 * h) - quotient) <= rounding
        # a node's third derivative is at most 1/8 of the cube of its slope along v, below 12 here; h^2 / 6 of it
        nodes = float(otree.codelen[targets[targets >= 0]].sum())
        assert abs(slope - quotient) <= rounding + h * h / 6 * 12**3 / 8 * nodes * 0.5


def test_loss_of_a_table_past_4_gigabytes(w2v):
    """Inner nodes whose rows lie more than 2^32 bytes into the tables (the root's is the last of all)."""
    import torch
    v, dim, n = 1_100_000, 1000, 150
    counts = torch.full((v,), 7, dtype=torch.int64, device="cuda")
    tree = w2v.build_huffman(counts)
    g = torch.Generator(device="cuda").manual_seed(1)
    syn1 = torch.empty(v - 1, 1024, device="cuda").normal_(generator=g).mul_(0.05)
    model = w2v.Model(torch.empty(v, 1024, device="cuda"), syn1, dim, counts, 7 * v, tree)
    x = torch.randn(n, dim, generator=g, device="cuda")
    targets = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    loss, dx, dsyn1 = w2v.hs_loss(model, x, targets)
    off, length = tree.point_off.cpu().numpy(), tree.codelen.cpu().numpy()
    code, points = tree.code.cpu().numpy(), tree.points.cpu().numpy()
    want = torch.zeros(v - 1, dtype=torch.bool, device="cuda")
    total = torch.zeros(dim, dtype=torch.float64, device="cuda")
    for i, t in enumerate(targets.tolist()):
        nodes = torch.from_numpy(points[off[t]:off[t] + length[t]].astype(np.int64)).cuda()
        s = torch.from_numpy(1.0 - 2.0 * ((code[t] >> np.arange(length[t])) & 1)).cuda()
        rows, row = syn1[nodes, :dim].double(), x[i].double()
        z = rows @ row
        z_off = 24 * U * (rows.abs() @ row.abs())
        value = torch.nn.functional.softplus(-s * z).sum()
        within(loss[i], value, (z_off + 8 * U).sum() + 6 * U * value, "loss")
        grad = -s * torch.sigmoid(-s * z)
        within(dx[i], grad @ rows, (z_off / 4 + 30 * U) @ rows.abs(), "dx")
        want[nodes] = True
        root = int((nodes == v - 2).nonzero()[0])
        total += grad[root] * row
    within(dsyn1[v - 2, :dim], total, 400 * U * x.double().abs().sum(0), "the root's gradient")
    assert bool((dsyn1[:, :dim].abs().amax(1) > 0).eq(want).all())


def test_loss_outputs_one_by_one(w2v):
    """Each of the C call's outputs may be left out; the others are the same bits."""
    import ctypes
    import torch
    counts = COUNTS["zipf"]()
    rng = np.random.default_rng(12)
    model, _ = make_model(w2v, counts, 24)
    x, t = hidden(300, 24, torch.float32), torch.from_numpy(draw_targets(rng, counts, 300)).cuda()
    loss, dx, dsyn1 = w2v.hs_loss(model, x, t)
    cm, ws = model.c(), w2v.hs_loss_workspace(model, x)
    for keep in (0, 1, 2, 3, 4, 5, 6):
        a, b, c = torch.zeros_like(loss), torch.zeros_like(dx), torch.zeros_like(dsyn1)
        rc = w2v.lib().w2v_hs_loss(
            ctypes.byref(cm), model.tree.max_len, x.data_ptr(), 0, 300, 24, t.data_ptr(), None, a.data_ptr() if keep & 1 else None,
            b.data_ptr() if keep & 2 else None, 24, c.data_ptr() if keep & 4 else None, c.stride(0),
            ws.data_ptr() if keep & 4 else None, ws.numel() if keep & 4 else 0, torch.cuda.current_stream().cuda_stream)
        assert rc == w2v.W2V_OK, w2v.last_error()
        for bit, got, full in ((1, a, loss), (2, b, dx), (4, c[:, :24], dsyn1[:, :24])):
            assert torch.equal(got, full) if keep & bit else not got.any(), (keep, bit)


# ------------------------------------------------------------------ AdamW
B1, B2, EPS = 0.9, 0.999, 1e-8


def adam_reference(p, g, m, v, step, lr, wd, scale=1.0):
    """New p, m, v in 64 bits, and their bounds for fp32 steps."""
    p, m, v = p.double().cpu(), m.double().cpu(), v.double().cpu()
    g = g.double().cpu() * scale
    m1 = B1 * m + (1 - B1) * g
    m_b = 4 * U * (B1 * m.abs() + (1 - B1) * g.abs())
    v1 = B2 * v + (1 - B2) * g * g
    v_b = 5 * U * v1
    size = lr / (1 - B1**step)
    den = (v1 / (1 - B2**step)).sqrt() + EPS
    upd = size * m1 / den
    p1 = p * (1 - lr * wd) - upd
    p_b = 3 * U * (p.abs() + p1.abs()) + size * m_b / den + 10 * U * upd.abs()
    return p1, m1, v1, p_b, m_b, v_b


def adam_case(shapes, p_kind, g_kind, seed=0, stride_extra=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    ps, gs = [], []
    for s in shapes:
        for to, t, scale in ((ps, p_kind, 0.5), (gs, g_kind, 0.1)):
            if len(s) == 2 and stride_extra:
                view, _ = guarded(s[0], s[1], t, s[1] + stride_extra)
                to.append(view)
            else:
                to.append(torch.empty(*s, dtype=t, device="cuda"))
            to[-1].copy_((torch.randn(*s, generator=g) * scale))
    return ps, gs


SHAPES = [(1,), (3,), (255,), (256,), (257,), (50, 20), (7, 301), (4096,), (4097,), (64, 128), (0,), (5, 1), (3, 5, 7), (9001,)]


@pytest.mark.parametrize("g_name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("p_name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("extra", [0, 3])
def test_adamw_three_steps(w2v, p_name, g_name, extra):
    import torch
    ps, gs = adam_case(SHAPES, kind(p_name), kind(g_name), 1, extra)
    decay = [0.0 if i % 3 == 0 else 0.05 * i for i in range(len(ps))]
    opt = w2v.AdamW(ps, gs, betas=(B1, B2), eps=EPS, weight_decay=decay)
    for step in (1, 2, 3):
        old = [p.clone() for p in ps]
        m0, v0 = opt.m.clone(), opt.v.clone()
        opt.step(step, 0.01 * step, grad_scale=0.5)
        for i, (p, g) in enumerate(zip(ps, gs)):
            n, at = p.numel(), opt.offsets[i]
            cut = slice(at, at + n)
            p1, m1, v1, p_b, m_b, v_b = adam_reference(old[i].flatten(), g.flatten(), m0[cut], v0[cut], step, 0.01 * step,
                                                      decay[i], 0.5)
            within(opt.m[cut], m1, m_b, "m")
            within(opt.v[cut], v1, v_b, "v")
            within(p.flatten(), p1, p_b + (p1.abs() + p_b) * half_step(kind(p_name)) + 2.0**-25 * (p_name == "f16"), "p")
            assert not opt.m[at + n:at + -(-n // 256) * 256].any()
        for g in gs:
            g.mul_(-0.7)


def test_adamw_strided_rows_leave_the_gaps(w2v):
    import torch
    p, buf = guarded(37, 50, torch.float32, 64, 0)
    p.normal_()
    g = torch.randn(37, 50, device="cuda")
    q, packed = p.clone(), g.clone()
    w2v.AdamW([p], [g]).step(1, 0.1)
    w2v.AdamW([q], [packed]).step(1, 0.1)
    assert torch.equal(p, q) and untouched(buf, p, 37, 50, 64, 0)


def mix(h):
    h = h.astype(np.uint64)
    m = np.uint64(0xFFFFFFFF)
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x85EBCA6B)) & m
    h = ((h ^ (h >> np.uint64(13))) * np.uint64(0xC2B2AE35)) & m
    return h ^ (h >> np.uint64(16))


R_VALUES = np.array([c * 2.0**-18 if c < 16 else (1 + (c % 16) / 16) * 2.0 ** (c // 16 - 15) for c in range(256)])


def narrow_reference(g, m, v, offset, step, seed):
    """fp32 steps of one tensor with 8-bit moments, numpy's fp32: (m codes, v codes, m scales, v scales) after it."""
    import torch
    f = np.float32
    n = g.size
    m = m * f(B1) + g * f(1 - B1)
    v = v * f(B2) + (g * g) * f(1 - B2)
    r = np.sqrt(v)
    pad = -n % 256
    blocks = lambda a: np.pad(a, (0, pad)).reshape(-1, 256)  # noqa: E731
    ms = np.abs(blocks(m)).max(1) * f(1 / 448)
    ms = np.where(ms < f(2.0**-126), f(0), ms)
    rs = blocks(r).max(1) * f(16 / 31)
    with np.errstate(divide="ignore"):
        mi, ri = np.where(ms > 0, f(1) / ms, f(0)), np.where(rs > 0, f(1) / rs, f(0))
    mc = torch.from_numpy((blocks(m) * mi[:, None]).astype(f)).to(torch.float8_e4m3fn).view(torch.uint8).numpy().ravel()[:n]
    t = (blocks(r) * ri[:, None]).astype(f).ravel()[:n]
    at = np.arange(offset, offset + n, dtype=np.uint64)
    key = mix(np.array([(seed ^ (step * 0x9E3779B9)) & 0xFFFFFFFF], dtype=np.uint64))
    h = mix(((at >> np.uint64(1)) & np.uint64(0xFFFFFFFF)) ^ key)
    h = np.where(at & np.uint64(1), h >> np.uint64(16), h & np.uint64(0xFFFF)).astype(np.int64)
    # a code is the exponent and fraction bits of t 2^-112 in fp32, subnormal numbers among them
    c = np.minimum(((t * f(2.0**-112)).view(np.int32).astype(np.int64) + h * 8 + 4) >> 19, 255)
    return mc, np.where((r > 0) & (c == 0), 1, c).astype(np.uint8), ms, rs


@pytest.mark.parametrize("p_name", ["f32", "bf16"])
@pytest.mark.parametrize("extra", [0, 3])
def test_adamw_eight_bits(w2v, p_name, extra):
    """Codes and scales bit for bit over four steps, parameters within an fp32 step's roundings of the moments that the
    codes stand for; values over thirty orders of magnitude in one tensor."""
    import torch
    ps, gs = adam_case(SHAPES, kind(p_name), torch.float32, 2, extra)
    gs[-1].mul_(torch.logspace(-20, 3, gs[-1].numel(), device="cuda"))
    gs[4].zero_()
    opt = w2v.AdamW(ps, gs, bits=8, betas=(B1, B2), eps=EPS, weight_decay=0.02, seed=77)
    for step in (1, 2, 3, 4):
        old = [p.clone() for p in ps]
        m0, v0 = (a.clone() for a in opt.moments())
        assert torch.equal(v0.cpu(), torch.from_numpy(
            ((R_VALUES[opt.v.cpu().numpy()].astype(np.float32).reshape(-1, 256) * opt.v_scale.cpu().numpy()[:, None]) ** 2
             ).astype(np.float32).ravel()))
        opt.step(step, 0.02)
        for i, (p, g) in enumerate(zip(ps, gs)):
            n, at = p.numel(), opt.offsets[i]
            if n == 0:
                continue
            cut, blocks = slice(at, at + n), slice(at // 256, at // 256 + -(-n // 256))
            mc, vc, ms, rs = narrow_reference(g.flatten().cpu().numpy(), m0[cut].cpu().numpy(), v0[cut].cpu().numpy(), at, step, 77)
            assert np.array_equal(opt.m_scale[blocks].cpu().numpy(), ms), (i, step)
            assert np.array_equal(opt.v_scale[blocks].cpu().numpy(), rs), (i, step)
            assert np.array_equal(opt.m[cut].cpu().numpy(), mc), (i, step)
            assert np.array_equal(opt.v[cut].cpu().numpy(), vc), (i, step)
            p1, _, _, p_b, _, _ = adam_reference(old[i].flatten(), g.flatten(), m0[cut], v0[cut], step, 0.02, 0.02)
            within(p.flatten(), p1, p_b + (p1.abs() + p_b) * half_step(kind(p_name)), "p")
        for g in gs:
            g.mul_(0.9)


def test_adamw_eight_bits_root_is_unbiased_and_never_lost(w2v):
    """The rounded root's mean over 65,536 equal elements lies within five standard deviations of the root (a code's
    width times sqrt(q (1-q) / n)), and a tiny gradient beside a large one keeps a second moment."""
    import torch
    n = 65536
    g = torch.full((n,), 0.37, device="cuda")
    g[::256] = 1.0
    p = torch.zeros(n, device="cuda")
    opt = w2v.AdamW([p], [g], bits=8, betas=(B1, B2), weight_decay=0.0, seed=5)
    opt.step(1, 0.0)
    root = opt.moments()[1].double().sqrt()
    plain = (torch.arange(n, device="cuda") % 256) != 0
    want = 0.37 * math.sqrt(1 - B2)
    width = root[plain].max() - root[plain].min()
    assert width > 0 and abs(root[plain].mean().item() - want) <= 5 * 0.5 * width.item() / math.sqrt(n)
    g.fill_(1e-9)
    g[::256] = 1.0
    opt = w2v.AdamW([p], [g], bits=8)
    opt.step(1, 1e-3)
    assert bool((opt.v > 0).all()) and p.abs().max().item() <= 1.01e-3


def test_adamw_of_more_than_2_to_32_elements(w2v):
    """The last elements of a tensor that needs 33 bits to count them, moments in 8 bits."""
    import torch
    n = 2**32 + 5000
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    lo = n // 256 * 256 - 4096
    g[lo:].normal_(generator=torch.Generator(device="cuda").manual_seed(9))
    p[lo:].normal_(generator=torch.Generator(device="cuda").manual_seed(8))
    old = p[lo:].clone()
    opt = w2v.AdamW([p], [g], bits=8, betas=(B1, B2), eps=EPS, weight_decay=0.1, seed=4)
    opt.step(1, 0.01)
    zero = np.zeros(n - lo, dtype=np.float32)
    mc, vc, ms, rs = narrow_reference(g[lo:].float().cpu().numpy(), zero, zero, lo, 1, 4)
    assert np.array_equal(opt.m[lo:n].cpu().numpy(), mc) and np.array_equal(opt.v[lo:n].cpu().numpy(), vc)
    assert np.array_equal(opt.m_scale[lo // 256:].cpu().numpy(), ms) and not opt.m[:1000].any()
    p1, _, _, p_b, _, _ = adam_reference(old, g[lo:], torch.zeros(n - lo), torch.zeros(n - lo), 1, 0.01, 0.1)
    within(p[lo:], p1, p_b + (p1.abs() + p_b) * half_step(torch.bfloat16), "p")


def test_adamw_of_memory_that_is_no_plan_does_nothing(w2v):
    import ctypes
    import torch
    p, g = torch.ones(512, device="cuda"), torch.ones(512, device="cuda")
    opt = w2v.AdamW([p], [g])
    opt._plan = torch.zeros_like(opt._plan)
    opt.step(1, 0.1)
    opt.step(torch.ones(1, dtype=torch.int64, device="cuda"), 0.1)
    assert bool((p == 1).all()) and not opt.m.any() and not opt._plan.any()


def test_adamw_not_finite_stays_in_its_block(w2v):
    import torch
    for bits in (8, 32):
        p, g = torch.ones(1024, device="cuda"), torch.ones(1024, device="cuda")
        g[300] = float("nan")
        g[700] = float("inf")
        opt = w2v.AdamW([p], [g], bits=bits)
        opt.step(1, 0.1)
        good = torch.ones(1024, dtype=torch.bool, device="cuda")
        good[[300, 700]] = False
        assert bool(torch.isfinite(p[good]).all()) and not bool(torch.isfinite(p[~good]).any())
        g.fill_(1.0)
        m, v = opt.moments()
        if bits == 8:
            assert bool(torch.isfinite(m[:256]).all()) and bool(torch.isfinite(m[768:]).all())
            assert not bool(torch.isfinite(m[256:512]).any()) and not bool(torch.isfinite(v[256:512]).any())


def test_adamw_resumes_from_its_state(w2v):
    import torch
    for bits in (8, 32):
        p, g = torch.randn(5000, device="cuda"), torch.randn(5000, device="cuda")
        q = p.clone()
        a = w2v.AdamW([p], [g], bits=bits, seed=3)
        for s in (1, 2, 3):
            a.step(s, 0.01)
        b = w2v.AdamW([q], [g], bits=bits, seed=3)
        b.step(1, 0.01)
        state = [t for t in (b.m, b.v, b.m_scale, b.v_scale) if t is not None]
        c = w2v.AdamW([q], [g], bits=bits, seed=3, state=state)
        for s in (2, 3):
            c.step(s, 0.01)
        assert torch.equal(p, q) and torch.equal(a.m, c.m) and torch.equal(a.v, c.v)


def test_adamw_keeps_its_buffers(w2v):
    """A parameter or gradient that gets other storage later: a step goes to the memory that the plan was made for, not to
    whatever has taken its place. The moments are the optimizer's own."""
    import torch
    n = 1 << 20
    p, g = torch.ones(n, device="cuda"), torch.ones(n, device="cuda")
    opt = w2v.AdamW([p], [g])
    p.data, g.data = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    opt.params.clear()
    opt.grads.clear()
    taken = [torch.full((n,), 7.0, device="cuda") for _ in range(4)]
    opt.step(1, 0.1)
    assert not p.any() and all(bool((t == 7).all()) for t in taken) and bool((opt.m != 0).all())
    with pytest.raises(AttributeError):
        opt.m = torch.zeros(256, device="cuda")


# ------------------------------------------------------------------ streams, graphs, a step of them together
def small_step(w2v, bits=32, seed=0, n=300):
    """hidden -> layer norm -> loss -> gradients -> AdamW on syn1, weight and bias, buffers kept."""
    import torch
    counts = COUNTS["zipf"]()
    model, otree = make_model(w2v, counts, 48, stride=64, seed=seed)
    rng = np.random.default_rng(seed)
    x = hidden(n, 48, torch.float32, seed=seed)
    targets = torch.from_numpy(draw_targets(rng, counts, n)).cuda()
    w, b = torch.ones(48, device="cuda"), torch.zeros(48, device="cuda")
    dsyn1 = torch.zeros_like(model.syn1)
    dw, db = torch.zeros(48, device="cuda"), torch.zeros(48, device="cuda")
    params = [model.vectors()[1], w, b]
    opt = w2v.AdamW(params, [dsyn1[:, :48], dw, db], bits=bits, weight_decay=[0.01, 0.0, 0.0])
    y, dy, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    loss = torch.empty(n, device="cuda")
    weights = torch.full((n,), 1.0 / n, device="cuda")
    ws = w2v.hs_loss_workspace(model, x)

    def run(step, lr):
        _, mean, rstd = w2v.layer_norm(x, w, b, out=y)
        w2v.hs_loss(model, y, targets, weights, loss=loss, dx=dy, dsyn1=dsyn1, workspace=ws)
        w2v.layer_norm_backward(dy, x, w, mean, rstd, dx=dx, dweight=dw, dbias=db)
        opt.step(step, lr)

    return dict(run=run, model=model, otree=otree, params=params, x=x, dx=dx, dw=dw, db=db, dsyn1=dsyn1, loss=loss, w=w, b=b,
                opt=opt, targets=targets, weights=weights, y=y)


def test_a_step_of_them_together(w2v):
    """The whole step against 64 bits: the chain's gradients, then AdamW on them (the first step: an update of nearly lr
    wherever the gradient is not tiny, so it is compared through AdamW's formula on the kernel's own gradients)."""
    import torch
    s = small_step(w2v)
    model, x = s["model"], s["x"]
    before = [p.clone() for p in s["params"]]
    s["run"](1, 0.01)
    targets, weights = s["targets"].cpu().numpy(), s["weights"].cpu().numpy()
    y64, mean, rstd, h = norm_reference(x, before[1], before[2], 1e-5)
    ref = loss_reference(s["otree"], before[0], y64, targets, weights, 48)
    dy = torch.from_numpy(ref["dx"])
    a = dy * before[1].double().cpu()
    dx = rstd[:, None] * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
    # y carries about 60 U (|y| + 1) into the loss: twenty times the loss's own bounds covers the chain at this size
    scale = dy.abs().max()
    within(s["dx"], dx, torch.full_like(dx, 1000 * U) * scale * rstd[:, None], "dx")
    within(s["dw"], (dy * h).sum(0), 1000 * U * scale * h.abs().sum(0), "dweight")
    within(s["db"], dy.sum(0), torch.full_like(dy[0], 1000 * U * 300) * scale, "dbias")
    within(s["dsyn1"][:, :48], torch.from_numpy(ref["d1"]), torch.from_numpy(20 * ref["d1_b"]), "dsyn1")
    opt = s["opt"]
    grads = [s["dsyn1"][:, :48], s["dw"], s["db"]]
    for i, (p, g, wd) in enumerate(zip(s["params"], grads, (0.01, 0.0, 0.0))):
        zero = torch.zeros(p.numel())
        p1, m1, v1, p_b, m_b, v_b = adam_reference(before[i].flatten(), g.flatten(), zero, zero, 1, 0.01, wd)
        within(p.flatten(), p1, p_b, f"parameter {i}")


@pytest.mark.parametrize("bits", [8, 32])
def test_a_captured_step_replays(w2v, bits):
    """A graph of the whole step, the step's number and learning rate in device memory, replayed beside eager work: the
    same bits as eager steps."""
    import torch
    eager, graph = small_step(w2v, bits, 3), small_step(w2v, bits, 3)
    step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
    graph["run"](1, 0.01)   # before the capture: every buffer is there
    eager["run"](1, 0.01)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        graph["run"](step, lr)
    for k in range(2, 7):
        step.fill_(k)
        lr.fill_(0.01 / k)
        g.replay()
        eager["run"](k, float(torch.tensor(0.01 / k, dtype=torch.float32)))
        torch.cuda.synchronize()
        for a, b in zip(eager["params"], graph["params"]):
            assert torch.equal(a, b), k
        assert torch.equal(eager["loss"], graph["loss"]) and torch.equal(eager["opt"].m, graph["opt"].m)
        _ = torch.randn(1000, device="cuda").sum().item()


def test_calls_on_other_streams(w2v):
    """Two steps at once on two streams, each with its own buffers, give what they give alone."""
    import torch
    alone = [small_step(w2v, 32, k, 2500) for k in (1, 2)]
    both = [small_step(w2v, 32, k, 2500) for k in (1, 2)]
    for s in alone:
        for k in (1, 2, 3):
            s["run"](k, 0.01)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    for k in (1, 2, 3):
        for s, st in zip(both, streams):
            with torch.cuda.stream(st):
                s["run"](k, 0.01)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for p, q in zip(a["params"], b["params"]):
            assert torch.equal(p, q)
        assert torch.equal(a["loss"], b["loss"]) and torch.equal(a["dx"], b["dx"])


# ------------------------------------------------------------------ refusals of the binding
def test_binding_refuses(w2v):
    import torch
    x = torch.randn(4, 8, device="cuda")
    w = torch.ones(8, device="cuda")
    with pytest.raises(ValueError):
        w2v.layer_norm(x.cpu())
    with pytest.raises(ValueError):
        w2v.layer_norm(x.double())
    with pytest.raises(ValueError):
        w2v.layer_norm(x[0])
    with pytest.raises(ValueError):
        w2v.layer_norm(x.t())
    with pytest.raises(ValueError):
        w2v.layer_norm(x, w[:4])
    with pytest.raises(ValueError):
        w2v.layer_norm(x, w, w.half())
    with pytest.raises(ValueError):
        w2v.layer_norm(x, w, out=torch.empty(4, 8, dtype=torch.float16, device="cuda"))
    with pytest.raises(w2v.W2VError):
        w2v.layer_norm(x, eps=-1.0)
    with pytest.raises(w2v.W2VError):
        w2v.layer_norm(x[:1].expand(4, 8))                       # rows on top of each other
    with pytest.raises(w2v.W2VError):
        w2v.layer_norm(torch.empty(1, 16385, device="cuda"))
    with pytest.raises(ValueError):
        w2v.layer_norm_backward(x, x, w, torch.zeros(3, device="cuda"), torch.zeros(4, device="cuda"))
    model, _ = make_model(w2v, COUNTS["zipf"](), 8)
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        w2v.hs_loss(model, x[:, :4], t)
    with pytest.raises(ValueError):
        w2v.hs_loss(model, x, t.long())
    with pytest.raises(ValueError):
        w2v.hs_loss(model, x, t[:3])
    with pytest.raises(w2v.W2VError):
        w2v.hs_loss(model, x, t, dx=x)
    with pytest.raises(w2v.W2VError):
        w2v.hs_loss(model, x, t, dsyn1=model.syn1)
    with pytest.raises(ValueError):
        w2v.AdamW([x], [x.cpu()])
    with pytest.raises(ValueError):
        w2v.AdamW([x], [x[:2]])
    with pytest.raises(ValueError):
        w2v.AdamW([x.t()], [x.t()])
    with pytest.raises(ValueError):
        w2v.AdamW([x], [x], bits=4)
    with pytest.raises(w2v.W2VError):
        w2v.AdamW([x, x], [x.clone(), x.clone()])                # the same parameter twice
    opt = w2v.AdamW([x], [x.clone()])
    with pytest.raises(w2v.W2VError):
        opt.step(0, 0.1)
    with pytest.raises(w2v.W2VError):
        opt.step(1, float("nan"))
    with pytest.raises(ValueError):
        opt.step(1, torch.zeros(1, dtype=torch.float64, device="cuda"))
