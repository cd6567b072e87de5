"""A batch's gradients at every width, with moments in 8 and 32 bits over several steps, and training's edges.

U = 2^-24 is fp32's largest relative rounding error; bounds are carried through the step to first order (1.01 for the
orders above)."""
import copy

import numpy as np
import pytest

from test_gpu_batch import text
from test_gpu_operators import B1, B2, U, make_model, narrow_reference, w2v, within, zipf_counts  # noqa: F401
from test_gpu_operators_edges import softmax_reference

pytestmark = pytest.mark.gpu

ROWS = 76   # additions one after the other in a sum over sorted rows (see softmax_reference)


def batch_gradients(otree, syn0, syn1, gain, bias, centres, window, norm_eps):
    """Gradients of the batch's mean loss in 64 bits, [(gradient, bound)] of syn0, syn1, gain and bias, and the summed
    loss with its bound.

    The window's mean: a sum of at most 2 window rows and a division. The norm: 20 elements a lane and 10 levels (30 U)
    for each mean, the variance's second sum and a division (34 U, halved by the root), 3 U for the root's reciprocal.
    dgain and dbias: 8 rows of a lane, 2 levels and 4 wavefronts, then 32 rows and 16 wavefronts (62, and 3 for h)."""
    n, d = len(centres), syn0.shape[1]
    norm = gain is not None
    live = np.array([len(w) > 0 for _, w in centres])
    targets = np.array([c if len(w) else -1 for c, w in centres])
    h, h_b = np.zeros((n, d)), np.zeros((n, d))
    for i, (_, w) in enumerate(centres):
        if len(w):
            h[i], h_b[i] = syn0[w].mean(0), (len(w) + 1) * U * np.abs(syn0[w]).mean(0)
    y, y_b = h, h_b
    if norm:
        mu, mu_b = h.mean(1, keepdims=True), (30 * U * np.abs(h) + h_b).mean(1, keepdims=True)
        c = h - mu
        c_b = h_b + mu_b + U * np.abs(c)
        var = (c * c).mean(1, keepdims=True) + norm_eps
        var[~live] = 1.0   # no part in anything
        r = 1 / np.sqrt(var)
        r_rel = ((np.abs(c) * c_b).mean(1, keepdims=True) * 2 / var + 34 * U) / 2 + 3 * U
        hat = c * r
        hat_b = c_b * r + np.abs(hat) * (r_rel + U)
        y = hat * gain + bias
        y_b = np.abs(gain) * (hat_b + U * np.abs(hat)) + U * np.abs(y)
    ref = softmax_reference(otree, syn1, y, targets, None, y_b)
    dy, dy_b = ref["dx"], ref["dx_b"]
    out = [None, (ref["d1"], ref["d1_b"])]
    dh, dh_b = dy, dy_b
    if norm:
        out.append(((dy * hat)[live].sum(0), (dy_b * np.abs(hat) + np.abs(dy) * hat_b + 65 * U * np.abs(dy * hat))[live].sum(0)))
        out.append((dy.sum(0), (dy_b + 62 * U * np.abs(dy)).sum(0)))
        a, a_b = dy * gain, dy_b * np.abs(gain) + U * np.abs(dy * gain)
        c0, c0_b = a.mean(1, keepdims=True), (a_b + 32 * U * np.abs(a)).mean(1, keepdims=True)
        c1 = (a * hat).mean(1, keepdims=True)
        c1_b = (a_b * np.abs(hat) + np.abs(a) * hat_b + 33 * U * np.abs(a * hat)).mean(1, keepdims=True)
        dh = r * (a - c0 - hat * c1)
        dh_b = r_rel * np.abs(dh) + r * (a_b + c0_b + hat_b * np.abs(c1) + np.abs(hat) * c1_b
                                         + 4 * U * (np.abs(a) + np.abs(c0) + np.abs(hat * c1)))
    g0, g0_b = np.zeros_like(syn0), np.zeros_like(syn0)
    for (_, w), row, off in zip(centres, dh, dh_b):
        if len(w):
            np.add.at(g0, w, row / len(w))
            np.add.at(g0_b, w, (off + (2 * window + 2 + ROWS) * U * np.abs(row)) / len(w))
    out[0] = (g0, g0_b)
    return ([(g / n, (1.01 * b + 3 * U * np.abs(g)) / n) for g, b in out], ref["loss"].sum(),
            1.01 * (ref["loss_b"].sum() + 2 * U * ref["loss"].sum()))


def windows(w2v, tok, counts, p):  # noqa: F811
    """Kept centres in order, (word, window words), from the sampler's listing of pairs (places in the whole text)."""
    import torch
    s = w2v.sample_pairs(torch.from_numpy(tok).cuda(), counts.size, torch.from_numpy(counts).cuda(), int(counts.sum()), p,
                         cap=40 * tok.size, want_mask=True)
    keep = np.nonzero(s.keep_mask.cpu().numpy())[0]
    centre, context = s.centre.cpu().numpy() - p.first_raw_index, s.context.cpu().numpy() - p.first_raw_index
    order = np.argsort(centre, kind="stable")
    cut = np.searchsorted(centre[order], np.append(keep, tok.size))
    words = tok[context[order]]
    return [(int(tok[k]), words[a:b]) for k, a, b in zip(keep, cut[:-1], cut[1:])]


def clone(model):
    return type(model)(model.syn0.clone(), model.syn1.clone(), model.dim, model.vocab_counts, model.train_words, model.tree)


def clone_state(state):
    import torch
    s = copy.copy(state)
    for name, t in vars(state).items():
        if isinstance(t, torch.Tensor):
            setattr(s, name, t.clone())
    return s


def parameters(model, state):
    return [model.syn0[:, :model.dim], model.syn1[:model.V - 1, :model.dim]] + (
        [state.gain, state.bias] if state.gain is not None else [])


def gradients_of(w2v, model, tok, p, state):  # noqa: F811
    """A batch's gradients as the kernels take them: with beta1 = 0 the first moment after a step is the gradient.
    The moments' array of it, and where each parameter's part begins."""
    m, s = clone(model), w2v.BatchState(model, norm=state.gain is not None, betas=(0.0, 0.0), eps=1.0, norm_eps=state.norm_eps)
    if state.gain is not None:
        s.gain, s.bias = state.gain.clone(), state.bias.clone()
    _, total, terms = w2v.train_batch_epoch(m, tok, p, s)
    assert s.steps == 1
    starts, at = [], 0
    for q in parameters(model, state):
        starts.append(at)
        at += -(-q.numel() // 256) * 256
    return s.m, starts, total, terms


def adam_step(p, g, m, v, step, lr, wd, eps):
    """New p, m and v in 64 bits, and their bounds for fp32 steps: m two products and their sum (4 U of the terms), v three
    and its terms positive (5 U), the update those, the root, three constants rounded once, three products and a hardware
    reciprocal (1 ulp) (10 U), p a product and the update's subtraction."""
    p, g, m, v = (t.double().cpu() for t in (p, g, m, v))
    m1, v1 = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
    m_b = 4 * U * (B1 * m.abs() + (1 - B1) * g.abs())
    size, den = lr / (1 - B1**step), (v1 / (1 - B2**step)).sqrt() + eps
    upd = size * m1 / den
    p1 = p * (1 - lr * wd) - upd
    return p1, m1, v1, 1.01 * (3 * U * (p.abs() + p1.abs()) + size * m_b / den + 10 * U * upd.abs()), m_b, 5 * U * v1


def check_gradients(w2v, model, otree, tok, counts, p, state):  # noqa: F811
    import torch
    centres = windows(w2v, tok, counts, p)
    q = [t.double().cpu().numpy() for t in parameters(model, state)] + [None, None]
    want, loss, loss_b = batch_gradients(otree, q[0], q[1], q[2], q[3], centres, p.window, state.norm_eps)
    m, starts, total, terms = gradients_of(w2v, model, torch.from_numpy(tok).cuda(), p, state)
    assert terms == sum(len(w) > 0 for _, w in centres) and abs(total + loss) <= loss_b
    for k, ((g, b), lo) in enumerate(zip(want, starts)):
        within(m[lo:lo + g.size].view(g.shape), torch.from_numpy(g), torch.from_numpy(b), f"gradient {k}")
    return m, starts


def with_norm(model, state, seed):
    """A gain and a bias that are no ones and zeros."""
    import torch
    g = torch.Generator().manual_seed(seed)
    state.gain.copy_(1 + 0.3 * torch.randn(model.dim, generator=g))
    state.bias.copy_(0.2 * torch.randn(model.dim, generator=g))
    return state


# ------------------------------------------------------------------ centres without a window, and no eps
def test_an_empty_window_has_no_part_in_the_norm(w2v):  # noqa: F811
    """Documents with one kept word have a centre without a window, whose hidden vector is zeros. With norm_eps = 0 that
    row has no finite deviation; the batch's gradients and the model are those of the other centres."""
    import torch
    counts = zipf_counts(60)
    rng = np.random.default_rng(4)
    tok = text(counts, 600, 9)
    tok[rng.random(600) < 0.5] = -1
    for dim, norm_eps in ((20, 0.0), (300, 0.0), (20, 1e-5)):
        model, otree = make_model(w2v, counts, dim)
        p = w2v.Params(window=3, arch=1, doc_len=3, corpus_tokens=600, sync_batch=1 << 12, alpha0=0.01)
        state = with_norm(model, w2v.BatchState(model, norm_eps=norm_eps, eps=1e-3), dim)
        centres = windows(w2v, tok, counts, p)
        alone = sum(len(w) == 0 for _, w in centres)
        assert 50 < alone < len(centres) - 50
        check_gradients(w2v, model, otree, tok, counts, p, state)
        t = torch.from_numpy(tok).cuda()
        before = w2v.batch_loglik(model, t, p, state)
        _, total, terms = w2v.train_batch_epoch(model, t, p, state)
        assert (total, terms) == before and np.isfinite(total)
        for q in parameters(model, state):
            assert bool(torch.isfinite(q).all())
        after = w2v.batch_loglik(model, t, p, state)
        assert np.isfinite(after[0]) and after[0] > before[0]


# ------------------------------------------------------------------ steps that were taken
def test_a_failed_epoch_keeps_its_steps(w2v, monkeypatch):  # noqa: F811
    """An error after some updates: the state counts those, as its moments hold them."""
    import torch
    counts = zipf_counts(40)
    model, _ = make_model(w2v, counts, 8)
    tok = torch.from_numpy(text(counts, 300, 1)).cuda()
    p = w2v.Params(window=3, arch=1, doc_len=50, corpus_tokens=300, sync_batch=64)
    state = w2v.BatchState(model)
    w2v.train_batch_epoch(model, tok, p, state)
    once = state.steps
    assert once > 1
    real = w2v.lib()

    class Failing:
        def __getattr__(self, name):
            return getattr(real, name)

        def w2v_train_batch_epoch(self, *args):
            assert real.w2v_train_batch_epoch(*args) == w2v.W2V_OK
            return w2v.W2V_E_ARG

    monkeypatch.setattr(w2v, "lib", Failing)
    with pytest.raises(w2v.W2VError):
        w2v.train_batch_epoch(model, tok, p, state)
    assert state.steps == 2 * once


def test_a_state_belongs_to_its_models_sizes(w2v):  # noqa: F811
    """Moments are laid out by the tables' rows and columns: a model of others is refused, though its number of moments
    (whole blocks of 256) may be the same. A model of the same sizes is taken."""
    import torch
    tok = torch.zeros(20, dtype=torch.int32, device="cuda")
    p = w2v.Params(window=2, arch=1, sync_batch=16)
    for norm, (v, dim), (v2, dim2) in ((True, (16, 16), (15, 16)), (False, (16, 16), (31, 8)), (False, (16, 16), (16, 15))):
        model, _ = make_model(w2v, zipf_counts(v), dim)
        other, _ = make_model(w2v, zipf_counts(v2), dim2)
        state = w2v.BatchState(model, norm=norm)
        assert w2v.BatchState(other, norm=norm).n_moments == state.n_moments
        kept = other.syn0.clone()
        for call in (w2v.train_batch_epoch, w2v.batch_loglik):
            with pytest.raises(ValueError, match="other sizes"):
                call(other, tok, p, state)
        assert torch.equal(other.syn0.nan_to_num(7.0), kept.nan_to_num(7.0)) and state.steps == 0
        same, _ = make_model(w2v, zipf_counts(v), dim, seed=5)
        w2v.train_batch_epoch(same, tok, p, state)


# ------------------------------------------------------------------ widths and steps
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dim", [1, 64, 130, 200, 256, 300, 320, 400, 512, 513, 700, 1000, 1024])
def test_gradients_at_every_width(w2v, norm, dim):  # noqa: F811
    """All widths of a lane's columns: window means, norm, loss, the gradients' way back to syn0 and syn1."""
    counts = zipf_counts(60)
    tok = text(counts, 700, dim)
    model, otree = make_model(w2v, counts, dim)
    p = w2v.Params(window=5, sample=1e-2, arch=1, doc_len=100, corpus_tokens=700, sync_batch=1 << 12)
    state = w2v.BatchState(model, norm=norm)
    check_gradients(w2v, model, otree, tok, counts, p, with_norm(model, state, dim) if norm else state)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dim,norm", [(300, True), (300, False), (50, True), (600, True)])
def test_steps_one_by_one_and_together(w2v, bits, dim, norm):  # noqa: F811
    """Four batches of whole documents. One call a batch: each step's gradients against 64 bits, the moments (8 bits: codes
    and scales bit for bit) and parameters against AdamW of the gradients as the kernels took them. One call for all: the
    same bits."""
    import torch
    counts = zipf_counts(60)
    rng = np.random.default_rng(dim)
    per, batches, rate = 150, 4, 0.01
    tok = rng.choice(60, size=per * batches, p=counts / counts.sum()).astype(np.int32)
    model, otree = make_model(w2v, counts, dim)
    decay, seed, eps = 0.1, 11, 1e-3
    state = w2v.BatchState(model, norm=norm, bits=bits, eps=eps, weight_decay=decay, seed=seed)
    if norm:
        with_norm(model, state, dim)
    together, state_together = clone(model), clone_state(state)

    def settings(k):   # no token is dropped: a batch is three documents
        return w2v.Params(window=5, arch=1, doc_len=50, corpus_tokens=per * batches, sync_batch=per, alpha0=rate, first_raw_index=k * per)

    for k in range(batches):
        part = tok[k * per:(k + 1) * per]
        p = settings(k)
        grads, starts = check_gradients(w2v, model, otree, part, counts, p, state)
        before = [q.clone().flatten() for q in parameters(model, state)]
        if bits == 8:
            opt_m = (state.m.view(torch.float8_e4m3fn).float().view(-1, 256) * state.m_scale[:, None]).flatten()
            c = state.v.long()
            root = torch.where(c < 16, c * 2.0**-18, (1 + (c % 16) / 16) * 2.0 ** (c // 16 - 15).double()).float()
            opt_v = ((root.view(-1, 256) * state.v_scale[:, None]) ** 2).flatten()
        else:
            opt_m, opt_v = state.m.clone(), state.v.clone()
        w2v.train_batch_epoch(model, torch.from_numpy(part).cuda(), p, state)
        assert state.steps == k + 1
        for i, (q, old, lo) in enumerate(zip(parameters(model, state), before, starts)):
            n = old.numel()
            g, m0, v0 = grads[lo:lo + n], opt_m[lo:lo + n], opt_v[lo:lo + n]
            p1, m1, v1, p_b, m_b, v_b = adam_step(old, g, m0, v0, k + 1, rate, decay if i < 2 else 0.0, eps)
            within(q.flatten(), p1, p_b, f"parameter {i} after step {k + 1}")
            if bits == 8:
                mc, vc, ms, rs = narrow_reference(g.cpu().numpy(), m0.cpu().numpy(), v0.cpu().numpy(), lo, k + 1, seed)
                blocks = slice(lo // 256, lo // 256 + -(-n // 256))
                assert np.array_equal(state.m_scale[blocks].cpu().numpy(), ms), (i, k)
                assert np.array_equal(state.v_scale[blocks].cpu().numpy(), rs), (i, k)
                assert np.array_equal(state.m[lo:lo + n].cpu().numpy(), mc), (i, k)
                assert np.array_equal(state.v[lo:lo + n].cpu().numpy(), vc), (i, k)
            else:
                within(state.m[lo:lo + n], m1, m_b, "m")
                within(state.v[lo:lo + n], v1, v_b, "v")
    w2v.train_batch_epoch(together, torch.from_numpy(tok).cuda(), settings(0), state_together)
    assert state_together.steps == batches
    for a, b in zip(parameters(model, state), parameters(together, state_together)):
        assert torch.equal(a, b)
    assert torch.equal(state.m, state_together.m) and torch.equal(state.v, state_together.v)
    if bits == 8:
        assert torch.equal(state.m_scale, state_together.m_scale) and torch.equal(state.v_scale, state_together.v_scale)


def test_a_large_batch_through_the_norm(w2v):  # noqa: F811
    """Some 21,000 centres: each group of sixteen lanes of the norm's backward pass has several rows, four sorted rows a
    wavefront share their path, the words' sums have many blocks."""
    import torch
    counts = zipf_counts(50)
    n, dim = 22_500, 36
    tok = text(counts, n, 7)
    model, otree = make_model(w2v, counts, dim)
    state = with_norm(model, w2v.BatchState(model), 3)
    p = w2v.Params(window=2, arch=1, doc_len=1000, corpus_tokens=n, sync_batch=1 << 17)
    centres = windows(w2v, tok, counts, p)
    q = [t.double().cpu().numpy() for t in parameters(model, state)]
    want, loss, loss_b = batch_gradients(otree, *q, centres, p.window, state.norm_eps)
    m, starts, total, terms = gradients_of(w2v, model, torch.from_numpy(tok).cuda(), p, state)
    assert terms == sum(len(w) > 0 for _, w in centres) and len(centres) > 20_480 and abs(total + loss) <= loss_b
    for k, ((g, b), lo) in enumerate(zip(want, starts)):
        within(m[lo:lo + g.size].view(g.shape), torch.from_numpy(g), torch.from_numpy(b), f"gradient {k}")
