"""A learned block between a hidden vector and the softmax, and the optimizer of its matrices, as a list of timed cases.

The block is a gated feed-forward: y = (act(x Wg') * (x Wu')) Wd' for rows x, with its backward pass (gated_ffn,
gated_ffn_backward). Its weights are matrices, which Muon updates: momentum, then an update that Newton-Schulz products
make nearly orthogonal (Muon.step, and orthogonalize for one matrix). Each case is one such call through the package's
public functions.

With own = False run() computes the same in elementary torch operations in 32 bits, rounded once at the end.

Shapes: the repository's widths (50 to 300 columns in rows padded to 32 floats, batches of up to 65,536 centres), widths
that models with 16-bit activations have, and odd sizes between them.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)   # of the odd polynomial that a Newton-Schulz step applies to singular values
STEPS, NORM_EPS = 5, 1e-7
MOMENTUM, DECAY, LR = 0.95, 0.01, 0.02


def listed() -> list[dict]:
    return [
        # one hidden vector of the headline workload's width, as a query is answered: latency is all there is
        dict(name="ffn_1x300_h800", op="ffn", rows=1, dim=300, hidden=800, type="f32", act="silu", save=False),
        # one 16-bit token of a wide model: every weight is read for one row
        dict(name="ffn_1x4096_h10240_bf16", op="ffn", rows=1, dim=4_096, hidden=10_240, type="bf16", act="silu", save=False),
        # a batch of window means at the headline's width, with what the backward pass needs
        dict(name="ffn_65536x300_h800", op="ffn", rows=65_536, dim=300, hidden=800, type="f32", act="silu", save=True),
        # 16-bit activations of a batch of tokens
        dict(name="ffn_16384x4096_h10240_bf16", op="ffn", rows=16_384, dim=4_096, hidden=10_240, type="bf16", act="silu",
             save=True),
        # a small batch at the paper's width
        dict(name="ffn_back_257x100_h400", op="ffn_back", rows=257, dim=100, hidden=400, type="f32", act="gelu"),
        # odd rows and columns: no row but the first starts on a vector's border
        dict(name="ffn_back_4099x1023_h2731_f16", op="ffn_back", rows=4_099, dim=1_023, hidden=2_731, type="f16", act="gelu"),
        # the batch of window means on its way back: 65,536 rows share three weight gradients
        dict(name="ffn_back_65536x300_h800", op="ffn_back", rows=65_536, dim=300, hidden=800, type="f32", act="silu"),
        # a training step's largest products
        dict(name="ffn_back_8192x4096_h10240_bf16", op="ffn_back", rows=8_192, dim=4_096, hidden=10_240, type="bf16",
             act="silu"),
        # the smallest block's matrix: fifteen dependent products of a few microseconds
        dict(name="orth_100x400", op="orth", count=1, rows=100, cols=400, type="f32"),
        # odd sizes, taller than wide, 16-bit
        dict(name="orth_2731x1023_f16", op="orth", count=1, rows=2_731, cols=1_023, type="f16"),
        # the largest matrix
        dict(name="orth_4096x10240", op="orth", count=1, rows=4_096, cols=10_240, type="f32"),
        # a stack of layers: three matrices each, 16-bit weights and gradients, momentum in 32 bits
        dict(name="muon_layers_bf16", op="muon", layers=12, dim=1_024, hidden=2_816, type="bf16"),
    ]


def _log_int(rng, lo: float, hi: float) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng) -> dict:
    op = rng.choice(["ffn", "ffn", "ffn_back", "ffn_back", "orth", "orth", "muon"])
    kind = rng.choice(["f32", "bf16", "f16"])
    if op in ("ffn", "ffn_back"):
        dim = rng.choice([_log_int(rng, 40, 4096), _log_int(rng, 40, 512), 50, 100, 128, 200, 256, 300, 512, 1024, 2048, 4096])
        hidden = rng.choice([_log_int(rng, dim, 4 * dim), 8 * dim // 3, 2 * dim, 4 * dim, (8 * dim // 3 + 127) // 128 * 128])
        most = 5e10 if kind == "f32" else 3e11      # rows x dim x hidden; the largest listed ones have 3.4e11 and 6.9e11
        case = dict(op=op, rows=_log_int(rng, 1, min(65_536, most / (dim * hidden))), dim=dim, hidden=hidden, type=kind,
                    act=rng.choice(["silu", "silu", "gelu"]))
        if op == "ffn":
            case["save"] = rng.random() < 0.5
        return case
    if op == "orth":
        rows, cols = (rng.choice([_log_int(rng, 1, 4096), _log_int(rng, 40, 2048), 50, 100, 256, 300, 1024, 2048])
                      for _ in range(2))
        count = 1 if rows * cols > 2**21 else rng.choice([1, 1, rng.randint(2, 4)])
        return dict(op=op, count=count, rows=rows, cols=cols, type=kind)
    dim = rng.choice([rng.randint(40, 640), 100, 200, 256, 300, 512, 640])
    return dict(op=op, layers=rng.randint(1, 12), dim=dim, hidden=rng.choice([8 * dim // 3, 4 * dim, rng.randint(dim, 4 * dim)]),
                type=kind)


# ------------------------------------------------------------------ inputs
def _rows(g, rows: int, dim: int, kind: torch.dtype, scale: float = 1.0) -> torch.Tensor:
    """[rows, dim] in rows padded to 32 elements where dim is even; packed where it is odd."""
    stride = dim if dim % 2 else (dim + 31) // 32 * 32
    out = torch.zeros(rows, stride, dtype=kind, device="cuda")
    out[:, :dim] = (torch.randn(rows, dim, generator=g, device="cuda") * scale).to(kind)
    return out[:, :dim]


def _matrix(g, rows: int, cols: int, kind: torch.dtype) -> torch.Tensor:
    return (torch.randn(rows, cols, generator=g, device="cuda") / math.sqrt(cols)).to(kind)


def prepare(case: dict, seed: int) -> dict:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"ffn": _prepare_ffn, "ffn_back": _prepare_ffn, "orth": _prepare_orth, "muon": _prepare_muon}[case["op"]](case, g)


def _prepare_ffn(case: dict, g) -> dict:
    n, d, h, kind = case["rows"], case["dim"], case["hidden"], TYPES[case["type"]]
    s = dict(case=case, x=_rows(g, n, d, kind), wg=_matrix(g, h, d, kind), wu=_matrix(g, h, d, kind),
             wd=_matrix(g, d, h, kind))
    back = case["op"] == "ffn_back"
    if back:                           # what the forward pass left, and buffers for the gradients
        s["gate"], s["up"] = ((s["x"].float() @ w.float().t()).to(kind) for w in (s["wg"], s["wu"]))
        s["dy"] = _rows(g, n, d, kind, 0.05)
        s.update({"d" + k: torch.empty_like(s[k]) for k in ("x", "wg", "wu", "wd")})
    else:
        s["y"] = torch.empty_like(s["x"])
        if case["save"]:
            s["gate"], s["up"] = (torch.empty(n, h, dtype=kind, device="cuda") for _ in range(2))
    if own:                            # the workspace that a program keeps from call to call
        import paper_1606_07822_amd as w2v
        s["workspace"] = w2v.gated_ffn_workspace(s["x"], h, grads=back)
    return s


def _prepare_orth(case: dict, g) -> dict:
    """Gradients as training makes them: a few strong directions over noise."""
    b, m, n, kind = case["count"], case["rows"], case["cols"], TYPES[case["type"]]
    r = min(m, n, 16)
    x = torch.randn(b, m, n, generator=g, device="cuda")
    left, right = torch.randn(b, m, r, generator=g, device="cuda"), torch.randn(b, r, n, generator=g, device="cuda")
    x = ((x + torch.bmm(left, right) * 0.3) * 1e-3).to(kind)
    s = dict(case=case, g=x if b > 1 else x[0])
    s["out"] = torch.empty_like(s["g"])
    if own:
        import paper_1606_07822_amd as w2v
        s["workspace"] = w2v.orthogonalize_workspace(s["g"])
    return s


def _prepare_muon(case: dict, g) -> dict:
    """Gate and up matrices and their layer's down matrix, each kind in a stack of its own whose slices are the tensors."""
    k, d, h, kind = case["layers"], case["dim"], case["hidden"], TYPES[case["type"]]
    s = dict(case=case)
    s["stacks"] = [(torch.randn(c, m, n, generator=g, device="cuda") / math.sqrt(n)).to(kind)
                   for c, m, n in ((2 * k, h, d), (k, d, h))]
    s["gstacks"] = [(torch.randn(p.shape, generator=g, device="cuda") * 1e-2).to(kind) for p in s["stacks"]]
    s["places"] = -(-h * d // 256) * 256           # a matrix's share of the momentum, from a multiple of 256 on
    m = torch.randn(3 * k, s["places"], generator=g, device="cuda") * 1e-2
    m[:, h * d:] = 0
    s["m"] = m
    if own:                            # the optimizer, which a program makes once, resumed from this momentum
        import paper_1606_07822_amd as w2v
        s["opt"] = w2v.Muon([p for t in s["stacks"] for p in t], [q for t in s["gstacks"] for q in t], momentum=MOMENTUM,
                            weight_decay=DECAY, state=m.view(-1))
    return s


# ------------------------------------------------------------------ one pass
def run(state: dict):
    op = state["case"]["op"]
    if own:
        return _own(op, state)
    return {"ffn": _plain_ffn, "ffn_back": _plain_ffn_back, "orth": _plain_orth, "muon": _plain_muon}[op](state)


def _own(op: str, s: dict):
    import paper_1606_07822_amd as w2v
    if op == "ffn":
        y, gate, up = w2v.gated_ffn(s["x"], s["wg"], s["wu"], s["wd"], s["case"]["act"], save=s["case"]["save"], out=s["y"],
                                    gate=s.get("gate"), up=s.get("up"), workspace=s["workspace"])
        return (y, gate, up) if s["case"]["save"] else y
    if op == "ffn_back":
        return w2v.gated_ffn_backward(s["dy"], s["x"], s["wg"], s["wu"], s["wd"], s["gate"], s["up"], s["case"]["act"],
                                      dx=s["dx"], dw_gate=s["dwg"], dw_up=s["dwu"], dw_down=s["dwd"],
                                      workspace=s["workspace"])
    if op == "orth":
        return w2v.orthogonalize(s["g"], out=s["out"], workspace=s["workspace"])
    s["opt"].step(LR)
    return s["stacks"], s["m"]


def _act(kind: str, g: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
    """The activation and its slope."""
    if kind == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _plain_ffn(s: dict):
    kind, x = s["x"].dtype, s["x"].float()
    gate, up = x @ s["wg"].float().t(), x @ s["wu"].float().t()
    y = ((_act(s["case"]["act"], gate)[0] * up) @ s["wd"].float().t()).to(kind)
    return (y, gate.to(kind), up.to(kind)) if s["case"]["save"] else y


def _plain_ffn_back(s: dict):
    kind = s["x"].dtype
    x, dy, gate, up = (s[k].float() for k in ("x", "dy", "gate", "up"))
    a, slope = _act(s["case"]["act"], gate)
    dh = dy @ s["wd"].float()
    dwd = dy.t() @ (a * up)
    du = dh * a
    dg = dh * up * slope
    dx = dg @ s["wg"].float() + du @ s["wu"].float()
    return dx.to(kind), (dg.t() @ x).to(kind), (du.t() @ x).to(kind), dwd.to(kind)


def _orthogonal(x: torch.Tensor) -> torch.Tensor:
    """[count, rows, cols] in 32 bits: five Newton-Schulz steps from x over its Frobenius norm."""
    a, b, c = COEFFICIENTS
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    x = x / (x.double().square().sum((1, 2), keepdim=True).sqrt().float() + NORM_EPS)
    for _ in range(STEPS):
        gram = torch.bmm(x, x.transpose(1, 2))
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return x.transpose(1, 2) if tall else x


def _plain_orth(s: dict):
    g = s["g"].float()
    return _orthogonal(g if g.dim() == 3 else g[None]).to(s["g"].dtype).reshape(s["g"].shape)


def _plain_muon(s: dict):
    at, size = 0, s["case"]["dim"] * s["case"]["hidden"]
    for p, g in zip(s["stacks"], s["gstacks"]):
        g = g.float()
        m = s["m"][at:at + p.shape[0], :size].view(p.shape)
        at += p.shape[0]
        m.copy_(m * MOMENTUM + g)
        o = _orthogonal(g + m * MOMENTUM)
        scale = math.sqrt(max(1.0, p.shape[1] / p.shape[2]))
        p.copy_(p.float() * (1 - LR * DECAY) - (LR * scale) * o)
    return s["stacks"], s["m"]


# ------------------------------------------------------------------ in 64 bits
def exact(case: dict, seed: int):
    s = prepare(case, seed)
    return {"ffn": _exact_ffn, "ffn_back": _exact_ffn, "orth": _exact_orth, "muon": _exact_muon}[case["op"]](case, s)


def _exact_act(kind: str, g: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
    if kind == "silu":
        return g / (1 + (-g).exp()), g.sigmoid() + g * g.sigmoid() * (-g).sigmoid()
    return g * 0.5 * torch.special.erfc(-g / 2**0.5), 0.5 * torch.special.erfc(-g / 2**0.5) + g * (-g.pow(2) / 2).exp() / (2 * math.pi)**0.5


def _exact_ffn(case: dict, s: dict):
    """In slices of the rows, so that a few of the largest case's 64-bit arrays live at a time."""
    back = case["op"] == "ffn_back"
    wg, wu, wd = (s[k].double() for k in ("wg", "wu", "wd"))
    sums, parts = [torch.zeros_like(w) for w in (wg, wu, wd)], []
    for lo in range(0, case["rows"], 8192):
        x = s["x"][lo:lo + 8192].double()
        if not back:
            gate, up = torch.mm(x, wg.T), torch.mm(x, wu.T)
            parts.append((torch.mm(_exact_act(case["act"], gate)[0].mul_(up), wd.T), gate, up))
            continue
        dy, gate, up = (s[k][lo:lo + 8192].double() for k in ("dy", "gate", "up"))
        value, slope = _exact_act(case["act"], gate)
        dh = torch.mm(dy, wd)
        dg, du = dh * (slope * up), dh * value
        parts.append((torch.addmm(torch.mm(dg, wg), du, wu),))
        sums[0].addmm_(dg.T, x)
        sums[1].addmm_(du.T, x)
        sums[2].addmm_(dy.T, value * up)
    whole = tuple(torch.cat(p) for p in zip(*parts))
    if back:
        return whole[0], *sums
    return whole if case["save"] else whole[0]


def _exact_polynomial(g: torch.Tensor) -> torch.Tensor:
    """One matrix, as the polynomial in its own (cols x cols or rows x rows) products: x (a + b x'x + c (x'x)^2)."""
    x = g.double()
    x = x / (torch.linalg.vector_norm(x) + NORM_EPS)
    a, b, c = COEFFICIENTS
    eye = torch.eye(min(x.shape), dtype=torch.float64, device="cuda")
    for _ in range(STEPS):
        if x.shape[0] <= x.shape[1]:
            q = torch.mm(x, x.T)
            x = torch.mm(a * eye + torch.mm(q, b * eye + c * q), x)
        else:
            q = torch.mm(x.T, x)
            x = torch.mm(x, a * eye + torch.mm(q, b * eye + c * q))
    return x


def _exact_orth(case: dict, s: dict):
    g = s["g"]
    return _exact_polynomial(g) if g.dim() == 2 else torch.stack([_exact_polynomial(t) for t in g])


def _exact_muon(case: dict, s: dict):
    size = case["dim"] * case["hidden"]
    new = [torch.empty(p.shape, dtype=torch.float64, device="cuda") for p in s["stacks"]]
    m = s["m"].double()
    k = 0
    for stack, grads, outs in zip(s["stacks"], s["gstacks"], new):
        for p, g, out in zip(stack, grads, outs):
            m[k, :size] = MOMENTUM * m[k, :size] + g.double().flatten()
            o = _exact_polynomial(g.double() + MOMENTUM * m[k, :size].view(p.shape))
            out.copy_(p.double() - LR * (DECAY * p.double() + o * max(1.0, p.shape[0] / p.shape[1])**0.5))
            k += 1
    return new, m


# ------------------------------------------------------------------ what a pass cannot do without
def _newton_schulz(rows: int, cols: int) -> float:
    """Operations of the steps: two products with the long side, one of the short side's squares; the first and the last of
    them symmetric, of which half is enough."""
    r, c = min(rows, cols), max(rows, cols)
    return STEPS * (r * (r + 1.0) * c + r * (r + 1.0) * r + 2.0 * r * r * c)


def work(case: dict) -> dict:
    size = torch.empty(0, dtype=TYPES[case["type"]]).element_size()
    if case["op"] in ("ffn", "ffn_back"):
        n, d, h = case["rows"], case["dim"], case["hidden"]
        if case["op"] == "ffn":
            return dict(bytes=size * (2 * n * d + 3 * d * h + (2 * n * h if case["save"] else 0)), flops=6.0 * n * d * h)
        return dict(bytes=size * (3 * n * d + 6 * d * h + 2 * n * h), flops=12.0 * n * d * h)
    if case["op"] == "orth":
        b, m, n = case["count"], case["rows"], case["cols"]
        return dict(bytes=2 * size * b * m * n, flops=b * _newton_schulz(m, n))
    k, d, h = 3 * case["layers"], case["dim"], case["hidden"]
    return dict(bytes=k * d * h * (3 * size + 8), flops=k * _newton_schulz(d, h))
