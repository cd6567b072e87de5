"""Training in mini-batches (train_batch_epoch, batch_loglik) against a step-by-step 64-bit computation from the
sampler's pairs, and against the framework's CBOW score."""
import numpy as np
import pytest

import oracle
import synth
from test_gpu_operators import B1, B2, U, half_step, kind, loss_reference, make_model, w2v, within, zipf_counts  # noqa: F401

pytestmark = pytest.mark.gpu


def text(counts, n, seed, doc_len=100):
    """Token indices drawn from the counts, with a few that are dropped."""
    rng = np.random.default_rng(seed)
    t = rng.choice(counts.size, size=n, p=counts / counts.sum()).astype(np.int32)
    t[rng.random(n) < 0.05] = -1
    return t


def windows(w2v, tok, counts, p):
    """Kept centres in order: (word, window words), from the sampler's listing of pairs."""
    import torch
    s = w2v.sample_pairs(torch.from_numpy(tok).cuda(), counts.size, torch.from_numpy(counts).cuda(), int(counts.sum()), p,
                         cap=40 * tok.size, want_mask=True)
    keep = np.nonzero(s.keep_mask.cpu().numpy())[0]
    c, x = s.centre.cpu().numpy(), s.context.cpu().numpy()
    return [(int(tok[k]), tok[x[c == k]]) for k in keep]


def reference(model0, otree, centres, batch, lr_of, norm, eps, decay, dim):
    """Parameters [syn0, syn1, gain, bias] after one pass, in 64 bits, the summed log-likelihood, and the largest
    gradient seen."""
    import torch
    p = [a.astype(np.float64) for a in model0] + [np.ones(dim), np.zeros(dim)]
    m, v = [np.zeros_like(a) for a in p], [np.zeros_like(a) for a in p]
    total, terms, biggest, t = 0.0, 0, 0.0, 0
    for lo in range(0, len(centres), batch):
        part = centres[lo:lo + batch]
        n = len(part)
        t += 1
        h = np.stack([p[0][w].mean(0) if len(w) else np.zeros(dim) for _, w in part])
        targets = [c if len(w) else -1 for c, w in part]
        mean, r, y, hat = 0, 0, h, h
        if norm:
            mean = h.mean(1, keepdims=True)
            r = 1 / np.sqrt(((h - mean) ** 2).mean(1, keepdims=True) + 1e-5)
            hat = (h - mean) * r
            y = hat * p[2] + p[3]
        ref = loss_reference(otree, torch.from_numpy(p[1]), torch.from_numpy(y), targets, None, dim)
        total -= ref["loss"].sum()
        terms += sum(c >= 0 for c in targets)
        g = [np.zeros_like(a) for a in p]
        g[1] = ref["d1"]
        dy = ref["dx"]
        dh = dy
        if norm:
            g[2], g[3] = (dy * hat).sum(0), dy.sum(0)
            a = dy * p[2]
            dh = r * (a - a.mean(1, keepdims=True) - hat * (a * hat).mean(1, keepdims=True))
        for (c, w), d in zip(part, dh):
            if len(w):
                np.add.at(g[0], w, d / len(w))
        lr = lr_of(lo)
        for k in range(4):
            gk = g[k] / n
            biggest = max(biggest, np.abs(gk).max())
            m[k] = B1 * m[k] + (1 - B1) * gk
            v[k] = B2 * v[k] + (1 - B2) * gk * gk
            keep = 1 - lr * (decay if k < 2 else 0.0)
            p[k] = p[k] * keep - lr / (1 - B1**t) * m[k] / (np.sqrt(v[k] / (1 - B2**t)) + eps)
    return p, total, terms, biggest, t


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dim,batch,n,window", [(20, 64, 600, 3), (50, 1000, 700, 5), (65, 33, 150, 10), (3, 1, 12, 1)])
def test_epoch_against_64_bits(w2v, norm, dim, batch, n, window):  # noqa: F811
    """AdamW's eps is a tenth of a gradient's size, so that an update is smooth in its gradient: an error of it enters by
    lr / eps at most, a batch's errors by as many steps as follow."""
    import torch
    counts = zipf_counts(60)
    tok = text(counts, n, dim)
    model, otree = make_model(w2v, counts, dim)
    start = [model.syn0[:, :dim].cpu().numpy(), model.syn1[:counts.size - 1, :dim].cpu().numpy()]
    p = w2v.Params(window=window, sample=1e-2, arch=1, doc_len=100, corpus_tokens=n, alpha0=0.01, sync_batch=batch)
    state = w2v.BatchState(model, norm=norm, betas=(B1, B2), eps=1e-3, weight_decay=0.1)
    centres = windows(w2v, tok, counts, p)
    stats, total, terms = w2v.train_batch_epoch(model, torch.from_numpy(tok).cuda(), p, state)
    want, total64, terms64, biggest, steps = reference(start, otree, centres, batch, lambda lo: 0.01, norm, 1e-3, 0.1, dim)
    assert terms == terms64 and state.steps == steps
    assert stats.tolist()[:2] == [n, int((tok >= 0).sum())] and stats[2].item() == len(centres)
    assert stats[3].item() == sum(len(w) for _, w in centres)
    assert stats[4].item() == sum(int(otree.codelen[c]) for c, w in centres if len(w))
    # a gradient is off by about 1000 U of the largest (sums of a few hundred terms through the layer norm)
    off = steps * 0.01 / 1e-3 * 1000 * U * biggest + 20 * U
    got = [model.syn0[:, :dim], model.syn1[:counts.size - 1, :dim]] + ([state.gain, state.bias] if norm else [])
    for k, (a, b) in enumerate(zip(got, want)):
        b = torch.from_numpy(b)
        within(a, b, torch.full_like(b, off) + 4 * steps * U * b.abs(), f"parameter {k}")
    assert abs(total - total64) <= abs(total64) * 1e-5 + terms * off * 100


def test_score_is_the_cbow_objective(w2v):  # noqa: F811
    """Without a layer norm, batch_loglik is hs_loglik's CBOW objective (fp64 there, fp32 products here), whatever the
    batch."""
    import torch
    counts = zipf_counts(500)
    tok = torch.from_numpy(text(counts, 20_000, 1)).cuda()
    model, _ = make_model(w2v, counts, 100)
    for batch in (100, 4096, 1 << 20):
        p = w2v.Params(window=5, sample=1e-3, arch=1, doc_len=100, corpus_tokens=20_000, sync_batch=batch)
        want, terms, _ = w2v.hs_loglik(model, tok, p)
        got, n = w2v.batch_loglik(model, tok, p, w2v.BatchState(model, norm=False))
        assert n == terms and abs(got - want) <= 1e-6 * abs(want)


def test_first_batch_is_the_score_and_bits_repeat(w2v):  # noqa: F811
    """An epoch of one batch scores the untouched model; two epochs from one start give equal bits; moments in 8 bits
    change nothing in the first step."""
    import torch
    counts = zipf_counts(300)
    tok = torch.from_numpy(text(counts, 5_000, 2)).cuda()
    p = w2v.Params(window=4, sample=1e-2, arch=1, doc_len=250, corpus_tokens=5_000, sync_batch=1 << 16, alpha0=0.01)
    ends = []
    for bits in (32, 32, 8):
        model, _ = make_model(w2v, counts, 40)
        state = w2v.BatchState(model, bits=bits)
        before = w2v.batch_loglik(model, tok, p, state)
        _, total, terms = w2v.train_batch_epoch(model, tok, p, state)
        assert (total, terms) == before and state.steps == 1
        ends.append([model.syn0[:, :40].clone(), model.syn1[:, :40].clone(), state.gain, state.bias, state])
    for a, b, c in zip(*[e[:4] for e in ends]):
        assert torch.equal(a, b) and torch.equal(a, c)
    m, narrow = ends[0][4].m, ends[2][4]
    wide = (narrow.m.view(torch.float8_e4m3fn).float().view(-1, 256) * narrow.m_scale[:, None]).flatten()
    most = m.view(-1, 256).abs().amax(1, keepdim=True).expand(-1, 256).flatten()
    # e4m3: half a step of three fraction bits, or of the smallest normal number (2^-6 of 448) times that
    within(wide, m, m.abs() * 2.0**-4 * 1.01 + most * 2.0**-10 / 448 * 1.01, "8-bit m")


def test_documents_and_batches_that_cut_windows(w2v):  # noqa: F811
    """A step's change does not depend on how far the batch's words lie from its border: one batch over the whole text
    equals the sum of its centres' gradients whatever the document length (here through the moments: m after one step is
    (1 - b1) times the gradient)."""
    import torch
    counts = zipf_counts(40)
    tok = text(counts, 900, 3)
    for doc_len in (1, 7, 64, 900):
        model, otree = make_model(w2v, counts, 8)
        start = [model.syn0[:, :8].cpu().numpy(), model.syn1[:counts.size - 1, :8].cpu().numpy()]
        p = w2v.Params(window=6, arch=1, doc_len=doc_len, corpus_tokens=900, sync_batch=1000, alpha0=1e-3)
        state = w2v.BatchState(model, norm=False, eps=1e-3)
        centres = windows(w2v, tok, counts, p)
        _, total, terms = w2v.train_batch_epoch(model, torch.from_numpy(tok).cuda(), p, state)
        want, total64, terms64, biggest, _ = reference(start, otree, centres, 1000, lambda lo: 1e-3, False, 1e-3, 0.0, 8)
        assert terms == terms64 and (doc_len > 1 or terms == 0)
        off = 1e-3 / 1e-3 * 1000 * U * max(biggest, 1e-3) + 20 * U
        within(model.syn0[:, :8], torch.from_numpy(want[0]), torch.full((counts.size, 8), off, dtype=torch.float64), "syn0")


def test_a_batch_of_many_blocks(w2v):  # noqa: F811
    """One batch of some 76,000 centres (more than one slab of the sums, by word and by node): m after one step is
    (1 - b1) times the gradient."""
    import torch
    counts = zipf_counts(50)
    n, dim = 80_000, 4
    tok = text(counts, n, 7)
    model, otree = make_model(w2v, counts, dim)
    syn0, syn1 = model.syn0[:, :dim].double().cpu().numpy(), model.syn1[:, :dim].double().cpu().numpy()
    p = w2v.Params(window=2, arch=1, doc_len=1000, corpus_tokens=n, sync_batch=1 << 17, alpha0=1e-3)
    s = w2v.sample_pairs(torch.from_numpy(tok).cuda(), counts.size, torch.from_numpy(counts).cuda(), int(counts.sum()), p,
                         cap=4 * n, want_mask=True)
    centre, context = s.centre.cpu().numpy(), s.context.cpu().numpy()
    rows, first, size = np.unique(centre, return_index=True, return_counts=True)
    place = np.repeat(np.arange(rows.size), size)
    h = np.zeros((rows.size, dim))
    np.add.at(h, place, syn0[tok[context]])
    h /= size[:, None]
    g1, dh, mag1 = np.zeros_like(syn1), np.zeros_like(h), np.zeros_like(syn1)
    word = tok[rows]
    for t in np.unique(word):
        at = np.nonzero(word == t)[0]
        for j, node in enumerate(otree.points[otree.point_off[t]:otree.point_off[t + 1]]):
            turn = (int(otree.code[t]) >> j) & 1
            g = 1 / (1 + np.exp(-(h[at] @ syn1[node]))) - (1 - turn)
            dh[at] += g[:, None] * syn1[node]
            g1[node] += g @ h[at]
            mag1[node] += np.abs(g) @ np.abs(h[at])
    g0, mag0 = np.zeros_like(syn0), np.zeros_like(syn0)
    np.add.at(g0, tok[context], (dh / size[:, None])[place])
    np.add.at(mag0, tok[context], np.abs(dh / size[:, None])[place])
    state = w2v.BatchState(model, norm=False, betas=(B1, B2))
    _, total, terms = w2v.train_batch_epoch(model, torch.from_numpy(tok).cuda(), p, state)
    kept = int(s.keep_mask.sum())
    assert terms == rows.size > 67584 and state.steps == 1
    # a term is off by 60 U or so, the sums (32 rows, 16 and 256 blocks, two slabs) by 400 U of their magnitude at most
    as_t = torch.from_numpy
    for lo, want, mag in ((0, g0, mag0), (-(-g0.size // 256) * 256, g1, mag1)):
        got = state.m[lo:lo + want.size].view(want.shape).double().cpu() / (1 - B1) * kept
        within(got, as_t(want), as_t(500 * U * mag), "gradient")


def test_empty_and_all_dropped_texts(w2v):  # noqa: F811
    import torch
    counts = zipf_counts(40)
    model, _ = make_model(w2v, counts, 8)
    kept = model.syn0.clone()
    p = w2v.Params(window=3, arch=1, doc_len=10, sync_batch=16)
    state = w2v.BatchState(model)
    for tok in (torch.empty(0, dtype=torch.int32, device="cuda"), torch.full((95,), -1, dtype=torch.int32, device="cuda")):
        stats, total, terms = w2v.train_batch_epoch(model, tok, p, state)
        assert total == 0 and terms == 0 and stats.tolist() == [tok.numel(), 0, 0, 0, 0] and state.steps == 0
        assert w2v.batch_loglik(model, tok, p, state) == (0.0, 0)
    assert torch.equal(model.syn0.nan_to_num(7.0), kept.nan_to_num(7.0))


def test_learning_rate_is_the_schedules(w2v):  # noqa: F811
    """The rate of a batch is that of its first centre: in the last epoch of two it starts at half of alpha0. With one
    step, a tiny eps and no decay, a parameter with a gradient moves by the rate."""
    import torch
    counts = zipf_counts(200)
    tok = torch.from_numpy(text(counts, 2_000, 5)).cuda()
    for epoch, rate in ((0, 0.02), (1, 0.02 * max(1e-4, 1 - 10_000 / (2 * 10_000 + 1)))):
        model, _ = make_model(w2v, counts, 16)
        before = model.syn0[:, :16].clone()
        p = w2v.Params(window=3, arch=1, doc_len=100, corpus_tokens=10_000, n_epochs=2, epoch=epoch, alpha0=0.02,
                       sync_batch=4096)
        w2v.train_batch_epoch(model, tok, p, w2v.BatchState(model, eps=1e-30))
        moved = (model.syn0[:, :16] - before).abs()
        moved = moved[torch.isfinite(moved) & (moved > 0)]
        # the step's root and quotient are off by a few roundings, the stored value by one of its own size
        assert moved.numel() > 1000 and bool(((moved - rate).abs() <= rate * 12 * U + 4 * U).all())


def test_binding_refuses(w2v):  # noqa: F811
    import torch
    counts = zipf_counts(40)
    model, _ = make_model(w2v, counts, 8)
    other, _ = make_model(w2v, counts, 12)
    tok = torch.zeros(50, dtype=torch.int32, device="cuda")
    state = w2v.BatchState(model)
    with pytest.raises(w2v.W2VError, match="arch 1"):
        w2v.train_batch_epoch(model, tok, w2v.Params(window=3), state)
    with pytest.raises(w2v.W2VError, match="sync_batch"):
        w2v.train_batch_epoch(model, tok, w2v.Params(window=3, arch=1, sync_batch=0), state)
    with pytest.raises(ValueError):
        w2v.train_batch_epoch(other, tok, w2v.Params(window=3, arch=1), state)
    with pytest.raises(ValueError):
        w2v.train_batch_epoch(model, tok.long(), w2v.Params(window=3, arch=1), state)
    with pytest.raises(ValueError):
        w2v.BatchState(model, bits=16)


@pytest.mark.parametrize("bits", (8, 32))
def test_state_of_other_sizes_is_refused(w2v, bits):  # noqa: F811
    """Moments that were put in place of the state's own ones: of its sizes and types, or refused."""
    import torch
    counts = zipf_counts(40)
    model, _ = make_model(w2v, counts, 8)
    tok = torch.from_numpy(text(counts, 300, 1)).cuda()
    p = w2v.Params(window=3, arch=1, sync_batch=64)
    names = ("m", "v", "m_scale", "v_scale") if bits == 8 else ("m", "v")
    for name in names:
        for bad in (lambda t: t[:-1], lambda t: t.double(), lambda t: t.cpu()):
            state = w2v.BatchState(model, bits=bits)
            setattr(state, name, bad(getattr(state, name)))
            for call in (w2v.train_batch_epoch, w2v.batch_loglik):
                with pytest.raises(ValueError):
                    call(model, tok, p, state)
    a, b = w2v.BatchState(model, bits=bits), w2v.BatchState(model, bits=bits)
    for name in names:
        setattr(b, name, getattr(a, name).clone())
    w2v.train_batch_epoch(model, tok, p, b)
    assert b.steps > 0 and b.m.any()
