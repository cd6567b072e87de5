"""The gated feed-forward block, orthogonalize and Muon against plain 64-bit implementations.

U = 2^-24 is fp32's largest relative rounding error and R a type's (half a step). A product over k is off by at most
(k + 70) U times the product of the absolute values: one rounding an addition, up to 64 more where k is cut into parts, and
less than U a term for what three bf16 parts leave out (2 * 2^-27 of it)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0**-24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def w2v():
    import paper_1606_07822_amd as w2v
    return w2v


def step_of(kind):
    return 0.0 if kind == torch.float32 else torch.finfo(kind).eps / 2


def least(kind):
    """Half of the smallest step of all."""
    return {torch.float32: 2.0**-150, torch.bfloat16: 2.0**-134, torch.float16: 2.0**-25}[kind]


def rounded(v, kind):
    """How far a result of this size may be off by being stored."""
    return torch.finfo(kind).eps / 2 * v.abs() + least(kind)


def rows_of(g, n, d, kind, scale=1.0, pad=0, shift=0):
    """[n, d] inside rows of d + pad elements, starting `shift` elements into its memory; what surrounds it is NaN."""
    mem = torch.full((shift + n * (d + pad) + 8,), float("nan"), dtype=kind, device="cuda")
    v = mem[shift:shift + n * (d + pad)].view(n, d + pad)[:, :d]
    v.copy_((torch.randn(n, d, generator=g, device="cuda") * scale).to(kind))
    return v


def untouched(v):
    """What surrounds rows_of's array is still NaN."""
    mem = torch.empty(0, dtype=v.dtype, device=v.device).set_(v.untyped_storage())
    inside = torch.zeros_like(mem, dtype=torch.bool)
    inside.as_strided(v.shape, v.stride(), v.storage_offset()).fill_(True)
    return bool(mem[~inside].isnan().all())


def act64(act, g):
    """Value and slope."""
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * torch.sigmoid(-g))
    p = 0.5 * torch.special.erfc(-g / math.sqrt(2))
    return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def act_off(g, a):
    """Errors of the activation's value and slope in fp32: the sigmoid's exponential loses |g| U of itself to its argument,
    and it, the sum, the reciprocal and the products two U each; erf is off by 2 ulp of 1 at most."""
    return (a.abs() * (g.abs() + 7) + 6 * g.abs()) * U, (12 + 4 * g.abs()) * U


def block64(x, wg, wu, wd, act, kind):
    """((y, g, u), bounds)."""
    x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
    d, h = wg.shape[1], wg.shape[0]
    g, u = x @ wg.T, x @ wu.T
    eg, eu = ((d + 70) * U * (x.abs() @ w.abs().T) for w in (wg, wu))
    a, _ = act64(act, g)
    ea = 1.13 * eg + act_off(g, a)[0]            # no slope of either is above 1.13
    v = a * u
    ev = ea * u.abs() + (a.abs() + ea) * eu + (U + step_of(kind)) * v.abs() + least(kind)
    y = v @ wd.T
    ey = ev @ wd.abs().T + (h + 70) * U * ((v.abs() + ev) @ wd.abs().T)
    return (y, g, u), [1.01 * (e + rounded(t, kind)) for e, t in ((ey, y), (eg, g), (eu, u))]


def back64(dy, x, wg, wu, wd, g, u, act, kind):
    """((dx, dwg, dwu, dwd), bounds) for g and u as they are."""
    dy, x, wg, wu, wd, g, u = (t.double() for t in (dy, x, wg, wu, wd, g, u))
    n, d, h = x.shape[0], x.shape[1], wg.shape[0]
    r = step_of(kind)
    dh = dy @ wd
    eh = (d + 70) * U * (dy.abs() @ wd.abs())
    a, s = act64(act, g)
    ea, es = act_off(g, a)
    du, dg, v = dh * a, dh * u * s, a * u
    edu = eh * a.abs() + dh.abs() * ea + (2 * U + r) * du.abs() + least(kind)
    edg = eh * (u * s).abs() + (dh * u).abs() * es + (3 * U + r) * dg.abs() + least(kind)
    ev = ea * u.abs() + (U + r) * v.abs() + least(kind)
    dx = dg @ wg + du @ wu
    edx = edg @ wg.abs() + edu @ wu.abs() + (2 * h + 140) * U * ((dg.abs() + edg) @ wg.abs() + (du.abs() + edu) @ wu.abs())
    out, off = [dx], [edx]
    for t, e, z in ((dg, edg, x), (du, edu, x)):
        out.append(t.T @ z)
        off.append(e.T @ z.abs() + (n + 70) * U * ((t.abs() + e).T @ z.abs()))
    out.append(dy.T @ v)
    off.append(dy.abs().T @ ev + (n + 70) * U * (dy.abs().T @ (v.abs() + ev)))
    return out, [1.01 * (e + rounded(t, kind)) for e, t in zip(off, out)]


def within(got, want, bound, name):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (name, int(bad.sum()), ((got.double() - want).abs() / bound).max().item())


# one row to tiles of every size, odd widths, k that ends inside a step, k cut into parts
SIZES = [(1, 1, 1), (1, 300, 800), (3, 7, 5), (16, 64, 130), (17, 33, 65), (64, 129, 77), (65, 64, 64), (129, 72, 136),
         (257, 100, 400), (600, 520, 1100), (130, 1023, 2731), (2100, 72, 640), (4099, 40, 90)]


def inputs(n, d, h, kind, seed, pad=0, shift=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = rows_of(g, n, d, kind, 1.0, pad, shift)
    wg, wu = (rows_of(g, h, d, kind, d**-0.5, p, shift) for p in (pad, 2 * pad))
    return g, x, wg, wu, rows_of(g, d, h, kind, h**-0.5, pad, shift)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("n,d,h", SIZES)
def test_gated_ffn(w2v, n, d, h, kind, act):
    """With what it saves, and without."""
    _, x, wg, wu, wd = inputs(n, d, h, kind, n + d + h)
    want, bounds = block64(x, wg, wu, wd, act, kind)
    got = w2v.gated_ffn(x, wg, wu, wd, act, save=True)
    for name, g, w, b in zip(("y", "gate", "up"), got, want, bounds):
        within(g, w, b, name)
    alone, gate, up = w2v.gated_ffn(x, wg, wu, wd, act)
    assert gate is None and up is None and torch.equal(alone, got[0])


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("n,d,h", SIZES)
def test_gated_ffn_backward(w2v, n, d, h, kind, act):
    rng, x, wg, wu, wd = inputs(n, d, h, kind, n + d + h)
    gate, up = ((x.double() @ w.double().T).to(kind) for w in (wg, wu))
    dy = rows_of(rng, n, d, kind, 0.3)
    want, bounds = back64(dy, x, wg, wu, wd, gate, up, act, kind)
    got = w2v.gated_ffn_backward(dy, x, wg, wu, wd, gate, up, act)
    for name, g, w, b in zip(("dx", "dw_gate", "dw_up", "dw_down"), got, want, bounds):
        within(g, w, b, name)


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (40, 8), (5, 3)])
@pytest.mark.parametrize("n", [5, 200])
def test_strides_and_alignment(w2v, n, pad, shift, kind):
    """Rows with gaps, rows off any vector's border, gate and up weights of different strides; nothing is written, and no NaN
    read, around the arrays."""
    d, h = 72, 104
    rng, x, wg, wu, wd = inputs(n, d, h, kind, 3, pad, shift)
    want, bounds = block64(x, wg, wu, wd, "silu", kind)
    y, gate, up = (rows_of(rng, n, c, kind, 1.0, pad, shift) for c in (d, h, h))
    w2v.gated_ffn(x, wg, wu, wd, save=True, out=y, gate=gate, up=up)
    for name, g, w, b in zip(("y", "gate", "up"), (y, gate, up), want, bounds):
        within(g, w, b, name)
        assert untouched(g), name
    dy = rows_of(rng, n, d, kind, 0.3, pad, shift)
    want, bounds = back64(dy, x, wg, wu, wd, gate, up, "silu", kind)
    outs = [rows_of(rng, *t.shape, kind, 1.0, pad, shift) for t in (x, wg, wu, wd)]
    w2v.gated_ffn_backward(dy, x, wg, wu, wd, gate, up, dx=outs[0], dw_gate=outs[1], dw_up=outs[2], dw_down=outs[3])
    for name, g, w, b in zip(("dx", "dw_gate", "dw_up", "dw_down"), outs, want, bounds):
        within(g, w, b, name)
        assert untouched(g), name


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("n", [7, 300])
def test_in_place(w2v, n, kind):
    """y over x; dx over dy, and over x."""
    rng, x, wg, wu, wd = inputs(n, 64, 96, kind, 5)
    y, gate, up = w2v.gated_ffn(x, wg, wu, wd, save=True)
    z = x.clone()
    assert w2v.gated_ffn(z, wg, wu, wd, out=z)[0] is z and torch.equal(z, y)
    dy = rows_of(rng, n, 64, kind)
    want = w2v.gated_ffn_backward(dy, x, wg, wu, wd, gate, up)
    for over in ("dy", "x"):
        a = dict(dy=dy.clone(), x=x.clone())
        got = w2v.gated_ffn_backward(a["dy"], a["x"], wg, wu, wd, gate, up, dx=a[over])
        assert got[0] is a[over]
        for g, w in zip(got, want):
            assert torch.equal(g, w)


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("n,d,h", [(6, 40, 56), (200, 72, 104), (513, 33, 95)])
def test_inputs_that_are_one_array(w2v, n, d, h, kind):
    """Tied weights, an upstream gradient that is x, g and u in one place: inputs may be each other."""
    _, x, w, _, wd = inputs(n, d, h, kind, 31)
    want, bounds = block64(x, w, w, wd, "silu", kind)
    y, gate, up = w2v.gated_ffn(x, w, w, wd, save=True)
    for name, g, t, b in zip(("y", "gate", "up"), (y, gate, up), want, bounds):
        within(g, t, b, name)
    assert torch.equal(gate, up)
    want, bounds = back64(x, x, w, w, wd, gate, gate, "silu", kind)
    got = w2v.gated_ffn_backward(x, x, w, w, wd, gate, gate)
    for name, g, t, b in zip(("dx", "dw_gate", "dw_up", "dw_down"), got, want, bounds):
        within(g, t, b, name)


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
def test_no_rows(w2v, kind):
    _, x, wg, wu, wd = inputs(0, 12, 20, kind, 1)
    y, gate, up = w2v.gated_ffn(x, wg, wu, wd, save=True)
    assert y.shape == (0, 12) and gate.shape == up.shape == (0, 20)
    dws = [rows_of(torch.Generator(device="cuda"), *t.shape, kind, 1.0, 3, 1) for t in (wg, wu, wd)]
    w2v.gated_ffn_backward(y, x, wg, wu, wd, gate, up, dw_gate=dws[0], dw_up=dws[1], dw_down=dws[2])
    for t in dws:
        assert not t.any() and untouched(t)


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("n", [9, 150, 700])
def test_a_row_that_is_not_finite_stays_alone(w2v, n, kind):
    _, x, wg, wu, wd = inputs(n, 72, 136, kind, 2)
    clean, _, _ = w2v.gated_ffn(x, wg, wu, wd)
    for value in (float("nan"), float("inf")):
        z = x.clone()
        z[n // 2, 3] = value
        y, _, _ = w2v.gated_ffn(z, wg, wu, wd)
        rest = torch.arange(n, device="cuda") != n // 2
        assert torch.equal(y[rest], clean[rest]) and not y[n // 2].isfinite().any()


@pytest.mark.parametrize("kind", TYPES[1:], ids=IDS[1:])
@pytest.mark.parametrize("n", [1, 5, 16, 20, 33, 64, 300])
def test_h_beyond_the_range_of_its_type(w2v, n, kind):
    """Row n // 2's first h is finite in fp32 and past the type's largest number; it meets weights that bring it back. Few rows
    keep h in fp32. In tiles it is rounded to the type, an infinity, which the weights' signs hand on."""
    _, x, wg, wu, wd = inputs(n, 24, 40, kind, 9)
    at = n // 2
    wg[0], wu[0], x[:, :2], x[at] = 0, 0, 0, 0   # the other rows' first h is 0
    if kind == torch.float16:                  # 300 * 300
        x[at, 0], wg[0, 0], wu[0, 0] = 1, 300, 300
        wd[:, 0] = torch.linspace(-0.01, 0.01, 24, device="cuda").to(kind)
    else:                                      # 2^64 (2^64 - 2^53), between bf16's largest number and fp32's
        x[at, :2] = 1
        wg[0, 0], wg[0, 1], wu[0, 0] = 2.0**64, -2.0**53, 2.0**64
        wd[:, 0] = torch.linspace(-1, 1, 24, device="cuda").to(kind) * 2.0**-120
    h = x[at].double() @ wg[0].double() * (x[at].double() @ wu[0].double())
    assert torch.finfo(kind).max < h < torch.finfo(torch.float32).max
    (want, gate, up), (off, _, _) = block64(x, wg, wu, wd, "silu", kind)
    y, g, u = w2v.gated_ffn(x, wg, wu, wd, save=True)
    rest = torch.arange(n, device="cuda") != at
    if n <= 64:
        within(y, want, off, "y")
    else:
        within(y[rest], want[rest], off[rest], "y")
        assert torch.equal(y[at], wd[:, 0] * float("inf"))


@pytest.mark.parametrize("n", [1, 7, 40])
def test_an_infinite_h_of_few_rows(w2v, n):
    """g u past fp32's range: an infinity of the weight's sign in that row alone, as the sum over h has it."""
    _, x, wg, wu, wd = inputs(n, 24, 40, torch.bfloat16, 9)
    clean = w2v.gated_ffn(x, wg, wu, wd)[0]
    at = n // 2
    wg[0], wu[0], wg[0, 0], wu[0, 0] = 0, 0, 2.0**70, 2.0**70
    x[:, 0] = 0
    base = w2v.gated_ffn(x, wg, wu, wd)[0]
    x[at, 0] = 1
    y = w2v.gated_ffn(x, wg, wu, wd)[0]
    rest = torch.arange(n, device="cuda") != at
    assert clean.isfinite().all() and torch.equal(y[rest], base[rest])
    assert torch.equal(y[at], wd[:, 0] * float("inf"))


@pytest.mark.parametrize("scale", [1e-18, 1e15])
def test_small_and_large_fp32_values(w2v, scale):
    """Parts of 8 bits have fp32's range."""
    rng, x, wg, wu, wd = inputs(130, 96, 160, torch.float32, 8)
    x.mul_(scale)
    want, bounds = block64(x, wg, wu, wd, "silu", torch.float32)
    got = w2v.gated_ffn(x, wg, wu, wd, save=True)
    for name, g, w, b in zip(("y", "gate", "up"), got, want, bounds):
        within(g, w, b, name)


@pytest.mark.parametrize("n", [3, 100])
def test_fp32_near_its_largest(w2v, n):
    """fp32's largest number has no bf16 beside it; its parts are still its own."""
    x = torch.full((n, 8), torch.finfo(torch.float32).max, device="cuda")
    w = torch.zeros(16, 8, device="cuda")
    w[:, 0] = 2.0**-127
    _, gate, up = w2v.gated_ffn(x, w, w, torch.zeros(8, 16, device="cuda"), save=True)
    want = torch.finfo(torch.float32).max * 2.0**-127
    assert ((gate.double() - want).abs() <= 80 * U * want).all() and torch.equal(gate, up)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activation_at_its_ends(w2v, act):
    """Arguments from far below to far above: the identity, zero, and slopes one and zero."""
    g = torch.tensor([-1e30, -200.0, -90.0, -30.0, -5.0, -1e-3, 0.0, 1e-3, 5.0, 30.0, 90.0, 200.0, 1e30], device="cuda")
    n = g.numel()
    eye = torch.eye(n, device="cuda")
    gate, up = eye * g, torch.ones(n, n, device="cuda")
    dx, dwg, dwu, dwd = w2v.gated_ffn_backward(eye, eye, eye, torch.zeros_like(eye), eye, gate, up, act)
    a, s = act64(act, g.double())
    # dy = Wd = 1: dh = 1; dw_down is h, its diagonal act(g); dx = dg its slope
    off, slope_off = act_off(g.double(), a)
    assert ((torch.diag(dwd).double() - a).abs() <= 1.01 * off + 1e-38).all()
    clear = g.abs() < 1e29                     # there a product of g with a share of zero or one is all
    assert ((torch.diag(dx).double() - s).abs() <= 1.01 * slope_off + 1e-38)[clear].all()
    assert torch.isfinite(dx).all()


def gelu_share_off(g):
    """The relative error of Phi(g) for g < 0, and of the density beside it, in fp32: one U for the polynomial; 1 + c |g| and
    its reciprocal 4 U, a polynomial whose terms cancel to no less than a third of their sum 9, three products and the
    hardware's power 5; the exponent g^2 log2(e) / 2 three roundings, 1.5 g^2 U of the power. For g > 0, one less it: U more."""
    return (20 + 2 * g * g) * U


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
def test_gelu_of_negative_arguments(w2v, kind):
    """Phi(g) to its last digits down to where a fp32 product of it is no longer normal: g Phi(g) forward, by few rows and by
    tiles; value and slope in the backward pass."""
    g = torch.linspace(-12.5, 4.0, 331, device="cuda").to(kind)
    n = g.numel()
    a, s = act64("gelu", g.double())
    share = gelu_share_off(g.double())
    off = (share + 2 * U) * a.abs() + rounded(a, kind)
    one = torch.eye(2, dtype=kind, device="cuda")
    x = torch.stack([g, torch.ones_like(g)], 1)
    for rows in (slice(0, n), slice(10, 50), slice(30, 31), slice(150, 151)):
        # rounded twice: h, and the product with one
        y = w2v.gated_ffn(x[rows], one[:1], one[1:], one[:, :1], "gelu")[0]
        within(y[:, 0], a[rows], 1.01 * (off + rounded(a, kind))[rows], "y")
    eye = torch.eye(n, dtype=kind, device="cuda")
    dx, _, _, dwd = w2v.gated_ffn_backward(eye, eye, eye, torch.zeros_like(eye), eye, eye * g, torch.ones_like(eye), "gelu")
    within(torch.diag(dwd), a, 1.01 * (off + rounded(a, kind)), "dw_down")
    g = g.double()
    phi, density = 0.5 * torch.special.erfc(-g / math.sqrt(2)), torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    off = (share + 4 * U) * (phi + g.abs() * density) + 2 * rounded(s, kind)
    within(torch.diag(dx), s, 1.01 * off, "dx")


def test_gradients_against_differences(w2v):
    """The gradients along random directions against differences of the 64-bit forward pass."""
    n, d, h, kind = 40, 24, 56, torch.float32
    rng, x, wg, wu, wd = inputs(n, d, h, kind, 11)
    dy = rows_of(rng, n, d, kind)
    for act in ("silu", "gelu"):
        (_, g64, u64), _ = block64(x, wg, wu, wd, act, kind)
        got = w2v.gated_ffn_backward(dy, x, wg, wu, wd, g64.float(), u64.float(), act)
        _, bounds = back64(dy, x, wg, wu, wd, g64, u64, act, kind)
        args = [t.double() for t in (x, wg, wu, wd)]

        def total(a):
            gate, up = a[0] @ a[1].T, a[0] @ a[2].T
            return ((act64(act, gate)[0] * up) @ a[3].T * dy.double()).sum()
        for i, (grad, bound) in enumerate(zip(got, bounds)):
            v = torch.randn(args[i].shape, generator=rng, device="cuda", dtype=torch.float64)
            e = 1e-6                           # a third derivative of some 1e3 at most leaves 1e-9; rounding 1e-16 / 1e-6 of the sum
            up_, down = ([t + s * e * v if k == i else t for k, t in enumerate(args)] for s in (1, -1))
            want = (total(up_) - total(down)) / (2 * e)
            size = total([t.abs() for t in args]).abs()
            # g and u were rounded to fp32: U of them, which moves a gradient less than the bound's (k + 70) U
            assert abs((grad.double() * v).sum() - want) <= 2 * (bound * v.abs()).sum() + 1e-8 * size + 1e-8


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
def test_the_same_twice_and_with_a_kept_workspace(w2v, kind):
    rng, x, wg, wu, wd = inputs(333, 200, 520, kind, 4)
    ws, back = w2v.gated_ffn_workspace(x, 520), w2v.gated_ffn_workspace(x, 520, grads=True)
    y, gate, up = w2v.gated_ffn(x, wg, wu, wd, save=True)
    ws.fill_(0xFF)
    back.fill_(0xFF)                           # NaN wherever it is read before it is written
    again = w2v.gated_ffn(x, wg, wu, wd, save=True, workspace=ws)
    for a, b in zip((y, gate, up), again):
        assert torch.equal(a, b)
    dy = rows_of(rng, 333, 200, kind)
    one = w2v.gated_ffn_backward(dy, x, wg, wu, wd, gate, up)
    two = w2v.gated_ffn_backward(dy, x, wg, wu, wd, gate, up, workspace=back)
    for a, b in zip(one, two):
        assert torch.equal(a, b)


def test_more_than_four_gigabytes_of_rows(w2v):
    """Rows past 2^32 bytes, and a stride of more than a product's 32-bit offsets."""
    n, d, h = (1 << 20) + 77, 2048, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, 1 << 19, n - 78, n - 1], device="cuda")
    x[at] = torch.randn(5, d, generator=g, device="cuda").bfloat16()
    wg, wu = (torch.randn(h, d, generator=g, device="cuda").mul_(d**-0.5).bfloat16() for _ in range(2))
    wd = torch.randn(d, h, generator=g, device="cuda").mul_(h**-0.5).bfloat16()
    y, gate, up = w2v.gated_ffn(x, wg, wu, wd, save=True)
    want, bounds = block64(x[at], wg, wu, wd, "silu", torch.bfloat16)
    for t, w, b in zip((y, gate, up), want, bounds):
        within(t[at], w, b, "y")
    dy = x
    got = w2v.gated_ffn_backward(dy, x, wg, wu, wd, gate, up, dx=y)
    want, bounds = back64(dy[at], x[at], wg, wu, wd, gate[at], up[at], "silu", torch.bfloat16)
    bounds[1:] = [b + 1.01 * n * U * w.abs() for b, w in zip(bounds[1:], want[1:])]   # all rows' additions, of zeros here
    within(got[0][at], want[0], bounds[0], "dx")
    for a, w, b in zip(got[1:], want[1:], bounds[1:]):
        within(a, w, b, "dw")
    del x, y, gate, up, dy, got
    wide = torch.zeros(70 * ((1 << 23) + 8), dtype=torch.bfloat16, device="cuda").view(70, -1)[:, :64]
    wide.copy_(torch.randn(70, 64, generator=g, device="cuda"))
    out = w2v.gated_ffn(wide, wg[:, :64], wu[:, :64], wd[:64])[0]
    assert torch.equal(out, w2v.gated_ffn(wide.contiguous(), wg[:, :64].contiguous(), wu[:, :64].contiguous(), wd[:64])[0])


# ------------------------------------------------------------------ Newton-Schulz
# tiles of every size, in each product: whole ones, cut along k into equal pieces and into pieces that start and end anywhere
CUTS = [(1100, 66, 3041), (1946, 2431, 40), (4097, 212, 1815), (2535, 871, 1768), (510, 1544, 2384), (3619, 376, 2700),
        (799, 2643, 631), (2293, 200, 3691), (11614, 344, 960), (7257, 323, 1670), (19978, 83, 45), (16649, 386, 72),
        (7353, 1941, 67)]


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("n,d,h", CUTS)
def test_gated_ffn_cuts(w2v, n, d, h, kind):
    act = "silu" if n % 2 else "gelu"
    rng, x, wg, wu, wd = inputs(n, d, h, kind, n + d + h, pad=8)
    dy = rows_of(rng, n, d, kind, 0.3)
    want, bounds = block64(x, wg, wu, wd, act, kind)
    y, gate, up = w2v.gated_ffn(x, wg, wu, wd, act, save=True)
    for name, g, w, b in zip(("y", "gate", "up"), (y, gate, up), want, bounds):
        within(g, w, b, name)
    assert torch.equal(w2v.gated_ffn(x, wg, wu, wd, act)[0], y)
    want, bounds = back64(dy, x, wg, wu, wd, gate, up, act, kind)
    got = w2v.gated_ffn_backward(dy, x, wg, wu, wd, gate, up, act)
    for name, g, w, b in zip(("dx", "dw_gate", "dw_up", "dw_down"), got, want, bounds):
        within(g, w, b, name)


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("n,d,h", [(1, 2**20, 3), (2, 5, 2**20), (90, 2**20, 2), (70, 3, 2**20)])
def test_gated_ffn_widest(w2v, n, d, h, kind):
    """The widest sizes that are taken, with few rows and with tiles; one more is refused."""
    rng, x, wg, wu, wd = inputs(n, d, h, kind, 21)
    dy = rows_of(rng, n, d, kind, 0.3)
    want, bounds = block64(x, wg, wu, wd, "gelu", kind)
    y, gate, up = w2v.gated_ffn(x, wg, wu, wd, "gelu", save=True)
    for name, g, w, b in zip(("y", "gate", "up"), (y, gate, up), want, bounds):
        within(g, w, b, name)
    want, bounds = back64(dy, x, wg, wu, wd, gate, up, "gelu", kind)
    got = w2v.gated_ffn_backward(dy, x, wg, wu, wd, gate, up, "gelu")
    for name, g, w, b in zip(("dx", "dw_gate", "dw_up", "dw_down"), got, want, bounds):
        within(g, w, b, name)
    sizes = (d + 1, h) if d == 2**20 else (d, h + 1)
    a = [torch.zeros(s, dtype=kind, device="cuda") for s in ((1, sizes[0]), (sizes[1], sizes[0]), (sizes[1], sizes[0]), sizes)]
    with pytest.raises(w2v.W2VError):
        w2v.gated_ffn(*a)


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("n,d,h", [(7, 60, 130), (130, 70, 300), (1100, 66, 3041), (700, 520, 1100)])
def test_some_outputs_only(w2v, n, d, h, kind):
    """NULL outputs through the C interface: those that are wanted are within the bounds, g and u one at a time, every set of
    gradients, none of them."""
    rng, x, wg, wu, wd = inputs(n, d, h, kind, 11)
    lib, stream, t = w2v.lib(), torch.cuda.current_stream().cuda_stream, TYPES.index(kind)
    y, gate, up = w2v.gated_ffn(x, wg, wu, wd, save=True)
    none = w2v.CRows(None, 0)

    def rows(a):
        return none if a is None else w2v.CRows(a.data_ptr(), a.stride(0))
    ws = w2v.gated_ffn_workspace(x, h)
    want, bounds = block64(x, wg, wu, wd, "silu", kind)
    for on in range(4):
        outs = [torch.full_like(y, float("nan"))] + [torch.full_like(gate, float("nan")) if on >> i & 1 else None
                                                     for i in range(2)]
        assert lib.w2v_gated_ffn(rows(x), rows(wg), rows(wu), rows(wd), n, d, h, t, 0, *map(rows, outs), ws.data_ptr(),
                                 ws.numel(), stream) == 0
        for name, g, w, b in zip(("y", "gate", "up"), outs, want, bounds):
            if g is not None:
                within(g, w, b, (on, name))
    dy = rows_of(rng, n, d, kind, 0.3)
    ws = w2v.gated_ffn_workspace(x, h, grads=True)
    want, bounds = back64(dy, x, wg, wu, wd, gate, up, "silu", kind)
    for on in range(16):
        outs = [torch.full_like(a, float("nan")) if on >> i & 1 else None for i, a in enumerate((x, wg, wu, wd))]
        assert lib.w2v_gated_ffn_backward(rows(dy), rows(x), rows(wg), rows(wu), rows(wd), rows(gate), rows(up), n, d, h, t, 0,
                                          *map(rows, outs), ws.data_ptr(), ws.numel(), stream) == 0
        for name, g, w, b in zip(("dx", "dw_gate", "dw_up", "dw_down"), outs, want, bounds):
            if g is not None:
                within(g, w, b, (on, name))


def steps64(x, steps=5, eps=1e-7, keep=lambda x: x):
    """In 64 bits; keep: what becomes of each matrix that the kernels store between products."""
    a, b, c = COEFFICIENTS
    x = x.double()
    x = x / (x.pow(2).sum().sqrt() + eps)
    tall = x.shape[0] > x.shape[1]
    x = keep(x.T if tall else x)
    eye = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for i in range(steps):
        q = keep(x @ x.T)
        p = keep(a * eye + b * q + c * (q @ q))
        x = p @ x
        x = x if i == steps - 1 else keep(x)
    return x.T if tall else x


def orth_bound(x, kind, **kw):
    """The largest relative error (in norm) that is allowed: four times what rounding each matrix between products to 11
    bits (bf16) or 20 (others: 22 are kept, and the sums' roundings are as large) costs in 64 bits, and the result's
    rounding. A step multiplies an error by 3.9 at most, which makes no smaller bound for 11 bits than this."""
    bits = 11 if kind == torch.bfloat16 else 20

    def keep(t):
        m, e = torch.frexp(t)
        return torch.ldexp((m * 2**bits).round(), e - bits)
    want = steps64(x, **kw)
    off = (steps64(x, keep=keep, **kw) - want).norm()
    return want, 4 * off + torch.finfo(kind).eps / 2 * want.norm() + 1e-30


def near(got, want, bound):
    off = (got.double() - want).norm()
    assert off <= bound, (off.item(), bound.item())


SHAPES = [(1, 1), (1, 50), (50, 1), (7, 5), (64, 64), (100, 400), (400, 100), (130, 77), (77, 131), (300, 300), (257, 1023),
          (1023, 257), (129, 2000), (700, 900)]


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("m,n", SHAPES)
def test_orthogonalize(w2v, m, n, kind):
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n)
    x = rows_of(g, m, n, kind, 1e-3)
    out = w2v.orthogonalize(x)
    near(out, *orth_bound(x, kind))
    if min(m, n) >= 50:
        s = torch.linalg.svdvals(out.double())
        assert s.max() < 1.25 and s.median() > 0.6


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("m,n", [(1, 2**20), (2**20, 3), (130, 2**18 + 5), (2**17 - 1, 200)])
def test_orthogonalize_longest(w2v, m, n, kind):
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n)
    x = torch.randn(m, n, generator=g, device="cuda").to(kind)
    near(w2v.orthogonalize(x), *orth_bound(x, kind))
    with pytest.raises(w2v.W2VError):
        w2v.orthogonalize(torch.zeros(2**20 + 1, 1, dtype=kind, device="cuda"))


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("count,m,n", [(1, 1500, 1600), (1, 2300, 2000), (1, 2300, 5000), (5, 600, 1000), (40, 300, 260)])
def test_orthogonalize_cuts(w2v, count, m, n, kind):
    """More tiles than one turn of the card, one matrix's and a stack's, and k cut into pieces of several lengths."""
    g = torch.Generator(device="cuda")
    g.manual_seed(m)
    x = torch.randn(count, m, n, generator=g, device="cuda").to(kind)
    out = w2v.orthogonalize(x)
    for i in range(0, count, 13):
        near(out[i], *orth_bound(x[i], kind))


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (24, 8)])
def test_orthogonalize_stacks(w2v, kind, pad, shift):
    """A stack with gaps between rows and matrices, in place and not; one of zeros, one with a NaN, one with an infinity."""
    count, m, n = 6, 70, 45
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    rows = rows_of(g, count * (m + 2), n, kind, 1.0, pad, shift)
    x = rows.view(count, m + 2, n)[:, :m] if pad == 0 else rows.as_strided((count, m, n), ((m + 2) * (n + pad), n + pad, 1))
    x[1] = 0
    x[3, 5, 7] = float("nan")
    x[4, 69, 44] = float("inf")
    out = w2v.orthogonalize(x)
    for i in (0, 2, 5):
        near(out[i], *orth_bound(x[i], kind))
    assert not out[1].any() and out[3].isnan().all() and not out[4].isfinite().any()
    keep = rows.clone()
    w2v.orthogonalize(x, out=x)
    assert torch.equal(x[[0, 1, 2, 5]], out[[0, 1, 2, 5]]) and untouched(rows)
    between = torch.ones(count, m + 2, dtype=torch.bool, device="cuda")
    between[:, :m] = False
    assert torch.equal(rows[between.flatten()], keep[between.flatten()])


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e30])
def test_orthogonalize_does_not_depend_on_the_size(w2v, scale):
    """Squares of these leave fp32's range; eps 0 leaves the ratio alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = rows_of(g, 60, 90, torch.float32, scale)
    near(w2v.orthogonalize(x, eps=0.0), *orth_bound(x, torch.float32, eps=0.0))


@pytest.mark.parametrize("steps", [1, 2, 10])
def test_orthogonalize_steps(w2v, steps):
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = rows_of(g, 90, 60, torch.float32)
    near(w2v.orthogonalize(x, steps=steps), *orth_bound(x, torch.float32, steps=steps))


def test_orthogonalize_rows_of_very_different_sizes(w2v):
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = rows_of(g, 128, 256, torch.float32)
    x *= 10.0 ** torch.linspace(-6, 0, 128, device="cuda")[:, None]
    near(w2v.orthogonalize(x), *orth_bound(x, torch.float32))


def low_rank(g, m, n, rank):
    """m x n of this rank; entries of 1 and -1 for rank 0, small integers, which 8 bits hold, for rank 1."""
    if rank == 0:
        return torch.sign(torch.randn(m, 1, generator=g, device="cuda")) * torch.sign(torch.randn(1, n, generator=g, device="cuda"))
    a, b = (torch.randn(s, generator=g, device="cuda") for s in ((m, rank), (rank, n)))
    return (3 * a).round().clamp(-11, 11) * (3 * b).round().clamp(-11, 11) if rank == 1 else a @ b


def decaying(g, m, n, power):
    """Singular values 1, 2^-power, 3^-power, ..."""
    r = min(m, n)
    a, b = (torch.linalg.qr(torch.randn(k, r, generator=g, device="cuda"))[0] for k in (m, n))
    return a * torch.arange(1, r + 1, device="cuda") ** -float(power) @ b.T


def steady_bound(want, kind, steps=5):
    """Whatever the singular values. All types: X is stored within 2^-22, and in the directions that it lacks a step multiplies
    what that leaves by 3.4445, in all by their sum over the steps (five: 686, 1.6e-4 of an X of norm 1; ten: 3.3e5, as it would
    be in any arithmetic of that many bits), for a result of 0.68 at least; as much again for the sums' roundings. And the
    result's own. bf16: as much as that again for products of 11 bits: what a step stores is within 2^-12 (3e-4 where all
    roundings have one sign), and its factors of up to 3.9 belong to X's own directions, in which they do not pile up, so that
    some ten such errors add up."""
    own = torch.finfo(kind).eps / 2 * (2 if kind == torch.bfloat16 else 1)
    grown = sum(3.4445**k for k in range(1, steps + 1)) * 2.0**-22 / 0.68
    return (own + 2 * grown) * want.norm()


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("m,n,rank", [(1024, 1024, 0), (1024, 1024, 1), (512, 1024, 8), (1024, 512, 64), (300, 700, 8),
                                      (1400, 300, 8), (1024, 1024, 256)])
def test_orthogonalize_few_directions(w2v, m, n, rank, kind):
    """Gradients of few rows have a low rank: the roundings of the directions that they lack may not grow into the result."""
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n + rank)
    x = low_rank(g, m, n, rank).to(kind)
    want = steps64(x)
    near(w2v.orthogonalize(x), want, steady_bound(want, kind))


@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("power", [1, 2, 4])
def test_orthogonalize_decaying_directions(w2v, power, kind):
    g = torch.Generator(device="cuda")
    g.manual_seed(power)
    for m, n in ((512, 1024), (700, 200)):
        x = decaying(g, m, n, power).to(kind)
        want = steps64(x)
        near(w2v.orthogonalize(x), want, steady_bound(want, kind))


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 10])
@pytest.mark.parametrize("m,n", [(300, 700), (700, 300)])
def test_orthogonalize_few_directions_steps(w2v, m, n, steps):
    g = torch.Generator(device="cuda")
    g.manual_seed(steps)
    x = torch.stack([low_rank(g, m, n, rank) for rank in (1, 8)]).bfloat16()
    out = w2v.orthogonalize(x, steps=steps)
    for a, b in zip(x, out):
        want = steps64(a, steps=steps)
        near(b, want, steady_bound(want, torch.bfloat16, steps))


@pytest.mark.parametrize("gkind", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_muon_gradients_of_few_directions(w2v, gkind):
    """bf16 parameters: the update of a zero matrix is the orthogonalised momentum itself."""
    rng = torch.Generator(device="cuda")
    rng.manual_seed(12)
    shapes = [(512, 1024), (1024, 512), (512, 1024), (300, 100)]
    grads = [(low_rank(rng, *s, r) * 1e-2).to(gkind) for s, r in zip(shapes, (1, 8, 64, 3))]
    params = [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    w2v.Muon(params, grads, momentum=0.9, scale=1.0).step(1.0)
    for p, g in zip(params, grads):
        want = -steps64(g.double() + 0.9 * g.double())
        near(p, want, steady_bound(want, torch.bfloat16))


def test_orthogonalize_nothing(w2v):
    for shape in ((0, 5), (5, 0), (0, 3, 4), (2, 0, 4)):
        x = torch.empty(shape, device="cuda")
        assert w2v.orthogonalize(x).shape == shape


def test_orthogonalize_one_matrix_as_a_stack(w2v):
    """A stack whose matrices lie in the same memory."""
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    x = rows_of(g, 70, 40, torch.float32)
    out = w2v.orthogonalize(x.expand(3, 70, 40))
    for t in out:
        near(t, *orth_bound(x, torch.float32))


def test_orthogonalize_more_matrices_than_a_launch(w2v):
    """5,000 small ones go in two launches."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn(5000, 3, 6, generator=g, device="cuda")
    out = w2v.orthogonalize(x)
    for i in (0, 4095, 4096, 4999):
        near(out[i], *orth_bound(x[i], torch.float32))


# ------------------------------------------------------------------ Muon
def muon64(params, grads, m, momentum, nesterov, lr, decay, scale, grad_scale=1.0):
    """One step in 64 bits from the values at hand: (params, m, bounds in norm)."""
    new, mom, bounds = [], [], []
    for i, (p, g) in enumerate(zip(params, grads)):
        g64 = g.double() * grad_scale
        m64 = momentum * m[i].double() + g64
        u = g64 + momentum * m64 if nesterov else m64
        o, off = orth_bound(u, torch.bfloat16 if p.dtype == torch.bfloat16 else torch.float32)
        s = max(1.0, p.shape[0] / max(1, p.shape[1]))**0.5 if scale is None else scale
        want = p.double() * (1 - lr * decay) - lr * s * o
        new.append(want)
        mom.append((m64, 3 * U * (momentum * m[i].double().abs() + g64.abs())))
        eps = torch.finfo(p.dtype).eps / 2
        bounds.append(abs(lr) * s * off + eps * want.norm() + 4 * U * (p.double().norm() + lr * s * o.norm()))
    return new, mom, bounds


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("gkind", TYPES, ids=IDS)
@pytest.mark.parametrize("kind", TYPES, ids=IDS)
def test_muon_steps(w2v, kind, gkind, nesterov):
    """Matrices of several shapes, one of them empty, one kind twice and apart; three steps, each from what the one before
    left."""
    rng = torch.Generator(device="cuda")
    rng.manual_seed(7)
    shapes = [(40, 70), (70, 40), (40, 70), (1, 9), (0, 4), (33, 33), (40, 70)]
    params = [rows_of(rng, *s, kind, 0.2, i % 3) for i, s in enumerate(shapes)]
    grads = [rows_of(rng, *s, gkind, 1e-2, (i + 1) % 3) for i, s in enumerate(shapes)]
    opt = w2v.Muon(params, grads, momentum=0.9, nesterov=nesterov, weight_decay=0.1)
    for step in range(3):
        for g in grads:
            g.copy_((torch.randn(g.shape, generator=rng, device="cuda") * 1e-2).to(gkind))
        moments = [opt.m[o:o + p.numel()].view(p.shape).clone() for o, p in zip(opt.offsets, params)]
        want, mom, bounds = muon64([p.clone() for p in params], grads, moments, 0.9, nesterov, 0.05, 0.1, None, 0.5)
        opt.step(0.05, grad_scale=0.5)
        for i, p in enumerate(params):
            if p.numel():
                near(p, want[i], bounds[i])
                got = opt.m[opt.offsets[i]:opt.offsets[i] + p.numel()].view(p.shape)
                within(got, mom[i][0], mom[i][1] + 1e-40, "momentum")
    assert all(untouched(t) for t in params + grads)
    gaps = torch.ones_like(opt.m, dtype=torch.bool)
    for o, p in zip(opt.offsets, params):
        gaps[o:o + p.numel()] = False
    assert not opt.m[gaps].any()


def test_muon_scale_decay_and_state(w2v):
    """A factor and a decay for each matrix; an optimizer resumed from another's momentum goes on as that one would."""
    rng = torch.Generator(device="cuda")
    rng.manual_seed(9)
    params = [rows_of(rng, 30, 20, torch.float32, 0.2), rows_of(rng, 20, 30, torch.float32, 0.2)]
    grads = [rows_of(rng, *p.shape, torch.float32) for p in params]
    first = w2v.Muon(params, grads, scale=[0.5, 2.0], weight_decay=[0.0, 0.3])
    first.step(0.1)
    copies = [p.clone() for p in params]
    second = w2v.Muon(copies, grads, scale=[0.5, 2.0], weight_decay=[0.0, 0.3], state=first.m.clone())
    want = []
    for i, (p, s, decay) in enumerate(zip(params, (0.5, 2.0), (0.0, 0.3))):
        m = [first.m[first.offsets[i]:first.offsets[i] + p.numel()].view(p.shape)]
        (w,), _, (b,) = muon64([p], [grads[i]], m, 0.95, True, 0.1, decay, s)
        want.append((w, b))
    first.step(0.1)
    second.step(0.1)
    for p, q, (w, b) in zip(params, copies, want):
        assert torch.equal(p, q)
        near(p, w, b)
    assert torch.equal(first.m, second.m)


def test_muon_of_nothing(w2v):
    """A list of empty matrices: there is no momentum, and a step does nothing."""
    params = [torch.empty(0, 5, device="cuda"), torch.empty(7, 0, device="cuda", dtype=torch.bfloat16)]
    opt = w2v.Muon(params, [torch.empty_like(p) for p in params])
    assert opt.n_moments == 0
    opt.step(0.1)
    torch.cuda.synchronize()


def test_muon_many_kinds_in_one_list(w2v):
    """Matrices that share a shape go through the products together, and come out as they do alone."""
    rng = torch.Generator(device="cuda")
    rng.manual_seed(2)
    shapes = [(64, 96), (200, 130), (64, 96), (130, 200), (64, 96)]
    kinds = [torch.float32, torch.bfloat16, torch.bfloat16, torch.float16, torch.float32]
    params = [rows_of(rng, *s, k, 0.2) for s, k in zip(shapes, kinds)]
    grads = [rows_of(rng, *s, k, 1e-2) for s, k in zip(shapes, kinds)]
    alone = [p.clone() for p in params]
    w2v.Muon(params, grads).step(0.1)
    for p, g, want in zip(alone, grads, params):
        w2v.Muon([p], [g]).step(0.1)
        # the cut of a product may differ with the number of matrices: the sums' order, not more
        scale = 2.0**-7 if p.dtype == torch.bfloat16 else 2.0**-10 if p.dtype == torch.float16 else 1e-5
        assert (p.double() - want.double()).norm() <= scale * want.double().norm()


# ------------------------------------------------------------------ graphs and streams
@pytest.mark.parametrize("kind", TYPES, ids=IDS)
@pytest.mark.parametrize("n", [5, 300])
def test_captured_step_replays(w2v, n, kind):
    """Forward, backward and Muon with a learning rate in memory, captured, and replayed over what was spoilt in between, with
    eager work and synchronizations between the replays."""
    rng, x, wg, wu, wd = inputs(n, 96, 160, kind, 21)
    dy = rows_of(rng, n, 96, kind, 0.1)
    y, gate, up = w2v.gated_ffn(x, wg, wu, wd, save=True)
    grads = [torch.empty_like(t) for t in (wg, wu, wd)]
    dx, lr = torch.empty_like(x), torch.tensor([0.02], device="cuda")
    weights = [t.clone() for t in (wg, wu, wd)]
    opt = w2v.Muon(weights, grads)
    ws = [w2v.gated_ffn_workspace(x, 160), w2v.gated_ffn_workspace(x, 160, grads=True)]

    def step():
        w2v.gated_ffn(x, *weights, save=True, out=y, gate=gate, up=up, workspace=ws[0])
        w2v.gated_ffn_backward(dy, x, *weights, gate, up, dx=dx, dw_gate=grads[0], dw_up=grads[1], dw_down=grads[2],
                               workspace=ws[1])
        opt.step(lr)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    arrays = [y, gate, up, dx, *grads, *weights, opt.m]
    for rate in (0.02, 0.1, 0.005):
        start = [t.clone() for t in weights], opt.m.clone()
        lr.fill_(rate)
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in arrays]
        for t, s in zip(weights, start[0]):
            t.copy_(s)
        opt.m.copy_(start[1])
        for t in (y, gate, up, dx, *grads, *ws, opt._workspace):
            t.fill_(111)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(arrays, want):
            assert torch.equal(a, b)


def test_two_streams_at_once(w2v):
    """Calls that overlap, each with its own workspace, as they come out alone."""
    sets = [inputs(900, 256, 512, torch.float32, s)[1:] for s in (1, 2)]
    want = [(w2v.gated_ffn(*a)[0], w2v.orthogonalize(a[1])) for a in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [None, None]
    for _ in range(3):
        for i, (a, s) in enumerate(zip(sets, streams)):
            with torch.cuda.stream(s):
                got[i] = w2v.gated_ffn(*a)[0], w2v.orthogonalize(a[1])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


# ------------------------------------------------------------------ a step of all of them
def test_block_between_norm_and_softmax(w2v):
    """layer_norm, gated_ffn, hs_loss and back, with Muon for the block's matrices and AdamW for the tables and the norm's
    vectors: every gradient as 64-bit autograd has it, and every update as the formulas do."""
    import numpy as np
    import synth
    d, h, n = 48, 80, 200
    w = synth.Workload("block", 20_000, 300, 1.0, 4, d, 3, 1e-3)
    tok = torch.from_numpy(synth.workload_corpus(w)).cuda()
    voc = w2v.build_vocab(tok, w.vocab, w.min_count)
    tree = w2v.build_huffman(voc.vocab_counts)
    syn0, syn1 = synth.init_weights(voc.V, d)
    syn1 = np.random.RandomState(1).standard_normal(syn1.shape).astype(np.float32) * 0.2
    model = w2v.make_model(syn0, syn1, voc, tree)
    g, _, wg, wu, wd = inputs(1, d, h, torch.float32, 31)
    x = rows_of(g, n, d, torch.float32)
    gain, bias = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
    targets = torch.randint(0, voc.V, (n,), generator=g, device="cuda", dtype=torch.int32)
    weights = torch.full((n,), 1.0 / n, device="cuda")

    z, mean, rstd = w2v.layer_norm(x, gain, bias)
    y, gate, up = w2v.gated_ffn(z, wg, wu, wd, save=True)
    loss, dy, dsyn1 = w2v.hs_loss(model, y, targets, weights)
    dz, *dws = w2v.gated_ffn_backward(dy, z, wg, wu, wd, gate, up)
    dx, dgain, dbias = w2v.layer_norm_backward(dz, x, gain, mean, rstd)

    leaves = [t.detach().double().clone().requires_grad_() for t in (x, gain, bias, wg, wu, wd, model.vectors()[1][:voc.V - 1])]
    zz = torch.nn.functional.layer_norm(leaves[0], (d,), leaves[1], leaves[2], 1e-5)
    gg = zz @ leaves[3].T
    yy = (gg * torch.sigmoid(gg) * (zz @ leaves[4].T)) @ leaves[5].T
    total = 0.0
    off, code, length = tree.point_off.long(), tree.code, tree.codelen.long()
    for j in range(tree.max_len):
        live = length[targets.long()] > j
        word = targets.long()[live]
        node = tree.points[off[word] + j].long()
        sign = 1 - 2 * ((code[word] >> j) & 1).double()
        total = total - (torch.nn.functional.logsigmoid(sign * (yy[live] * leaves[6][node]).sum(1)) * weights[live].double()).sum()
    total.backward()
    assert abs((loss.double() * weights.double()).sum() - total) <= 1e-5 * abs(total)
    for name, got, leaf in zip(("x", "gain", "bias", "gate", "up", "down", "syn1"),
                               (dx, dgain, dbias, *dws, dsyn1[:voc.V - 1, :d]), leaves):
        # a chain of six products of up to 200 terms, each within (k + 70) U = 1.6e-5 of its absolute terms, which cancel to
        # no less than a tenth of their norm
        assert (got.double() - leaf.grad).norm() <= 1e-3 * leaf.grad.norm(), name

    matrices, mgrads = [wg, wu, wd], [t.contiguous() for t in dws]
    tables, tgrads = [model.vectors()[1], gain, bias], [dsyn1[:, :d], dgain, dbias]
    before = [t.clone() for t in matrices + tables]
    want, _, bounds = muon64(matrices, mgrads, [torch.zeros_like(t) for t in matrices], 0.95, True, 0.02, 0.0, None)
    w2v.Muon(matrices, mgrads).step(0.02)
    w2v.AdamW(tables, tgrads, weight_decay=0.0).step(1, 1e-3)
    for t, v, b in zip(matrices, want, bounds):
        near(t, v, b)
    for t, old, grad in zip(tables, before[3:], tgrads):
        moved = grad.abs() > 1e-5              # AdamW's first step is lr along the gradient's sign
        assert ((old - t - 1e-3 * grad.sign()).abs()[moved] <= 2e-5).all()
    again = w2v.gated_ffn(w2v.layer_norm(x, gain, bias)[0], wg, wu, wd)[0]
    assert w2v.hs_loss(model, again, targets, weights, grads=False)[0].mean() < loss.mean()


def test_as_an_autograd_function(w2v):
    """The two calls are the halves of a user's autograd.Function."""
    class Block(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, wg, wu, wd):
            y, gate, up = w2v.gated_ffn(x, wg, wu, wd, "gelu", save=True)
            ctx.save_for_backward(x, wg, wu, wd, gate, up)
            return y

        @staticmethod
        def backward(ctx, dy):
            return w2v.gated_ffn_backward(dy.contiguous(), *ctx.saved_tensors, "gelu")

    _, x, wg, wu, wd = inputs(70, 40, 56, torch.float32, 17)
    leaves = [t.clone().requires_grad_() for t in (x, wg, wu, wd)]
    Block.apply(*leaves).sum().backward()
    _, gate, up = w2v.gated_ffn(x, wg, wu, wd, "gelu", save=True)
    want, bounds = back64(torch.ones_like(x), x, wg, wu, wd, gate, up, "gelu", torch.float32)
    for t, w, b in zip(leaves, want, bounds):
        within(t.grad, w, b, "grad")


# ------------------------------------------------------------------ refusals of the binding
def test_refusals(w2v):
    _, x, wg, wu, wd = inputs(4, 8, 12, torch.float32, 1)
    y, gate, up = w2v.gated_ffn(x, wg, wu, wd, save=True)
    bad = [lambda: w2v.gated_ffn(x, wg, wu, wd, "tanh"), lambda: w2v.gated_ffn(x.cpu(), wg, wu, wd),
           lambda: w2v.gated_ffn(x, wg.bfloat16(), wu, wd), lambda: w2v.gated_ffn(x, wg, wu[:-1], wd),
           lambda: w2v.gated_ffn(x, wg, wu, wd.T), lambda: w2v.gated_ffn(x.double(), wg, wu, wd),
           lambda: w2v.gated_ffn(x[0], wg, wu, wd), lambda: w2v.gated_ffn(x, wg, wu, wd, gate=gate),
           lambda: w2v.gated_ffn(x, wg, wu, wd, out=y[:, :7]), lambda: w2v.gated_ffn(x, wg, wu, wd, workspace=y),
           lambda: w2v.gated_ffn_backward(y[:3], x, wg, wu, wd, gate, up),
           lambda: w2v.gated_ffn_backward(y, x, wg, wu, wd, gate[:, :11], up),
           lambda: w2v.gated_ffn_backward(y, x, wg, wu, wd, gate, up, dw_gate=wd),
           lambda: w2v.orthogonalize(x.double()), lambda: w2v.orthogonalize(x[0]), lambda: w2v.orthogonalize(x.T),
           lambda: w2v.orthogonalize(x, out=wg), lambda: w2v.orthogonalize(x.cpu()),
           lambda: w2v.Muon([], []), lambda: w2v.Muon([wg], [wu, wd]), lambda: w2v.Muon([wg], [wd]),
           lambda: w2v.Muon([wg[0]], [wu[0]]), lambda: w2v.Muon([wg.T], [wu.T]), lambda: w2v.Muon([wg], [wu], scale=[1.0, 2.0]),
           lambda: w2v.Muon([wg], [wu], state=torch.zeros(5, device="cuda")), lambda: w2v.Muon([wg], [wu.double()])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was taken")
    for call in (lambda: w2v.gated_ffn(x, wg, wu, wd, out=wd[:4, :8].as_strided((4, 8), (12, 1))),
                 lambda: w2v.gated_ffn(x, wg, wu, wd, save=True, gate=gate, up=gate),
                 lambda: w2v.gated_ffn_backward(y, x, wg, wu, wd, gate, up, dw_gate=wg),
                 lambda: w2v.orthogonalize(x, steps=0), lambda: w2v.orthogonalize(x, steps=21),
                 lambda: w2v.orthogonalize(x, eps=-1.0), lambda: w2v.Muon([wg, wg], [wu, wu]),
                 lambda: w2v.Muon([wg], [wu], momentum=1.0).step(0.1), lambda: w2v.Muon([wg], [wu]).step(float("nan"))):
        with pytest.raises(w2v.W2VError):
            call()
