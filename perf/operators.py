"""The operators of a mini-batch training step as a list of timed cases.

A step on a batch of hidden vectors is: normalise them (layer_norm), score the
target words under the hierarchical softmax and take its gradients (hs_loss),
go back through the normalisation (layer_norm_backward), and update every
table and vector from its gradient (AdamW.step, moments in 32 or in 8 bits).
Each case is one such call through the package's public functions.

With own = False run() computes the same in elementary torch operations: in 32
bits, in 64 where a sum runs over the rows of a batch, rounded once at the end.

Shapes: the repository's workloads (30 K to 1 M words, 50 to 300 columns in
rows padded to 32 floats, batches of up to 65,536 centres), widths that models
with 16-bit activations have, and odd sizes between them.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5              # layer norm
MASKED = 0.05           # share of a batch's rows without a target (a centre whose window is empty)
BLOCK = 256             # elements that share a scale, moments in 8 bits
BETA1, BETA2, ADAM_EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.01
ROUNDING_SEED = 7


def listed() -> list[dict]:
    return [
        # one hidden vector of the headline workload's width, as a query is scored: latency is all there is
        dict(name="norm_1x300", op="norm", rows=1, dim=300, type="f32", affine=True),
        # 16-bit activations of a batch of tokens
        dict(name="norm_16384x4096_bf16", op="norm", rows=16_384, dim=4_096, type="bf16", affine=True),
        # odd rows and columns: no row but the first starts on a vector's border
        dict(name="norm_back_4099x1023_f16", op="norm_back", rows=4_099, dim=1_023, type="f16", affine=True),
        # a batch of window means at the headline's width (rows of 320 floats): 65,536 rows share one weight gradient
        dict(name="norm_back_65536x300", op="norm_back", rows=65_536, dim=300, type="f32", affine=True),
        # one hidden vector scored against its word in the largest tree: a walk of some twenty dependent rows
        dict(name="loss_1_v1m_d300", op="loss", rows=1, words=1_000_000, dim=300, type="f32", zipf=1.05, grads=False),
        # a small batch with its gradients at the paper's width
        dict(name="loss_grad_257_v30k_d100", op="loss", rows=257, words=30_000, dim=100, type="f32", zipf=1.0, grads=True),
        # a batch of centres at 200 columns: more rows than a tree of this size has paths apart
        dict(name="loss_grad_65536_v100k_d200", op="loss", rows=65_536, words=100_000, dim=200, type="f32", zipf=1.0,
             grads=True),
        # the headline's tables: a gradient of 1.2 GB, most of it zero
        dict(name="loss_grad_65536_v1m_d300", op="loss", rows=65_536, words=1_000_000, dim=300, type="f32", zipf=1.05,
             grads=True),
        # 16-bit hidden states of the widest rows the tables have
        dict(name="loss_grad_8191_v50k_d1024_bf16", op="loss", rows=8_191, words=50_021, dim=1_024, type="bf16", zipf=1.0,
             grads=True),
        # the smallest model's two tables and its normalisation's vectors: one launch's latency
        dict(name="adamw_tables_v1k_d50", op="adamw", kind="tables", words=1_000, dim=50, type="f32", bits=32),
        # the headline's tables: 600 M parameters in rows of 320 floats
        dict(name="adamw_tables_v1m_d300", op="adamw", kind="tables", words=1_000_000, dim=300, type="f32", bits=32),
        # 16-bit weights of a stack of layers, 209 tensors from a thousand to four million elements, moments in 8 bits
        dict(name="adamw_layers_bf16_8bit", op="adamw", kind="layers", layers=26, dim=1_024, type="bf16", bits=8),
    ]


def _log_int(rng, lo: float, hi: float) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng) -> dict:
    op = rng.choice(["norm", "norm_back", "norm_back", "loss", "loss", "loss", "adamw", "adamw"])
    if op in ("norm", "norm_back"):
        dim = rng.choice([_log_int(rng, 24, 8192), rng.choice([50, 100, 128, 200, 256, 300, 512, 1024, 2048, 4096])])
        return dict(op=op, rows=_log_int(rng, 1, min(65_536, 2**26 // dim)), dim=dim,
                    type=rng.choice(["f32", "bf16", "f16"]), affine=rng.random() < 0.8)
    if op == "loss":
        dim = rng.choice([rng.randint(40, 512), rng.randint(513, 1024), 50, 64, 100, 128, 200, 256, 300])
        words = _log_int(rng, 1e3, 1e6 if dim <= 300 else 1e5)
        return dict(op=op, rows=_log_int(rng, 1, 65_536 * min(1.0, 300 / dim)), words=words, dim=dim,
                    type=rng.choice(["f32", "f32", "bf16", "f16"]), zipf=rng.choice([1.0, 1.05]),
                    grads=rng.random() < 0.8)
    if rng.random() < 0.5:
        dim = rng.choice([rng.randint(40, 512), 50, 100, 200, 300])
        return dict(op=op, kind="tables", words=_log_int(rng, 1e3, 1e6 * min(1.0, 300 / dim)), dim=dim, type="f32",
                    bits=32)
    return dict(op=op, kind="layers", layers=rng.randint(1, 24), dim=rng.choice([rng.randint(65, 1024), 256, 512, 768]),
                type=rng.choice(["f32", "bf16", "f16"]), bits=rng.choice([8, 8, 32]))


# ------------------------------------------------------------------ the tree
@functools.lru_cache(maxsize=4)
def _tree(words: int, zipf: float) -> dict:
    """The Huffman tree of Zipf counts (100 occurrences a word on average): leaves in ascending count, ties to the
    leaf, merge a makes inner node a, the root is the last. Host arrays, and each inner node's share of the text."""
    p = np.arange(1, words + 1, dtype=np.float64) ** -zipf
    counts = (p / p.sum() * 100 * words).astype(np.int64) + 5
    leaves = counts[::-1].tolist()
    inner, parent = [0] * (words - 1), [0] * (2 * words - 1)   # leaf i: word words-1-i; inner node a: words + a
    bit = np.zeros(2 * words - 1, dtype=np.uint8)
    i = j = 0
    for a in range(words - 1):
        total = 0
        for b in (0, 1):
            if i < words and (j >= a or leaves[i] <= inner[j]):
                total += leaves[i]
                k = i
                i += 1
            else:
                total += inner[j]
                k = words + j
                j += 1
            parent[k] = a
            bit[k] = b
        inner[a] = total
    parent = np.asarray(parent, dtype=np.int32)
    root = words - 2
    at = np.arange(words - 1, -1, -1, dtype=np.int64)          # word v's node in that numbering
    chain, turns = [], []
    done = np.zeros(words, dtype=bool)
    length = np.zeros(words, dtype=np.int32)
    while not done.all():
        up = parent[at]
        chain.append(np.where(done, -1, up))
        turns.append(bit[at])
        length += ~done
        done = done | (up == root)
        at = np.where(done, at, words + up)
    off = np.zeros(words + 1, dtype=np.int32)
    np.cumsum(length, out=off[1:])
    points, code = np.empty(off[-1], dtype=np.int32), np.zeros(words, dtype=np.uint64)
    for step, (c, t) in enumerate(zip(chain, turns)):          # step 0 is the word's own parent, the path's end
        live = c >= 0
        depth = length[live] - 1 - step
        points[off[:-1][live] + depth] = c[live]
        code[live] |= t[live].astype(np.uint64) << depth.astype(np.uint64)
    return dict(counts=counts, codelen=length.astype(np.uint8), code=code.view(np.int64), off=off, points=points,
                longest=int(length.max()), share=np.asarray(inner, dtype=np.float64) / counts.sum())


# ------------------------------------------------------------------ inputs
def _rows(g, rows: int, dim: int, kind: torch.dtype, scale: float = 1.0, shift: float = 0.0) -> torch.Tensor:
    """[rows, dim] in rows padded to 32 elements where dim is even; packed where it is odd."""
    stride = dim if dim % 2 else (dim + 31) // 32 * 32
    out = torch.zeros(rows, stride, dtype=kind, device="cuda")
    out[:, :dim] = (torch.randn(rows, dim, generator=g, device="cuda") * scale + shift).to(kind)
    return out[:, :dim]


def _padded(rows: int, dim: int) -> torch.Tensor:
    return torch.zeros(rows, (dim + 31) // 32 * 32, device="cuda")


def prepare(case: dict, seed: int) -> dict:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"norm": _prepare_norm, "norm_back": _prepare_norm, "loss": _prepare_loss,
            "adamw": _prepare_adamw}[case["op"]](case, g)


def _prepare_norm(case: dict, g) -> dict:
    n, d, kind = case["rows"], case["dim"], TYPES[case["type"]]
    x = _rows(g, n, d, kind, 1.3, 0.4)
    s = dict(case=case, x=x, w=None, b=None)
    if case["affine"]:
        s["w"] = 1 + 0.2 * torch.randn(d, generator=g, device="cuda")
        s["b"] = 0.1 * torch.randn(d, generator=g, device="cuda")
    if case["op"] == "norm_back":
        s["dy"] = _rows(g, n, d, kind, 0.05)
        wide = x.double()                      # what the forward pass left
        mean = wide.mean(1)
        s["mean"] = mean.float()
        s["rstd"] = ((wide - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
    s["y"] = torch.empty_like(x)
    return s


def _prepare_loss(case: dict, g) -> dict:
    n, d, v = case["rows"], case["dim"], case["words"]
    t = _tree(v, case["zipf"])
    dev = lambda a: torch.from_numpy(a).to("cuda")  # noqa: E731
    counts = dev(t["counts"])
    edges = counts.cumsum(0).double()
    targets = torch.searchsorted(edges, torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * edges[-1],
                                 right=True).clamp_(max=v - 1).to(torch.int32)
    if n > 1:
        targets[torch.rand(n, generator=g, device="cuda") < MASKED] = -1
    syn1 = _padded(v - 1, d)
    syn1[:, :d] = torch.randn(v - 1, d, generator=g, device="cuda") * (1.5 / math.sqrt(d))
    s = dict(case=case, x=_rows(g, n, d, TYPES[case["type"]]), targets=targets, syn1=syn1, longest=t["longest"],
             codelen=dev(t["codelen"]), code=dev(t["code"]), off=dev(t["off"]), points=dev(t["points"]),
             weights=(0.5 + torch.rand(n, generator=g, device="cuda")) / n)
    if own:   # the model's handle and the gradient buffers, which a program keeps
        import paper_1606_07822_amd as w2v
        tree = w2v.Tree(s["codelen"], s["code"], s["off"], s["points"], t["longest"])
        s["model"] = w2v.Model(_padded(v, d), syn1, d, counts, int(t["counts"].sum()), tree)
        s["loss"] = torch.empty(n, device="cuda")
        if case["grads"]:
            s["dx"] = torch.empty_like(s["x"])
            s["dsyn1"] = _padded(v - 1, d)
        s["workspace"] = w2v.hs_loss_workspace(s["model"], s["x"], grads=case["grads"])
    return s


def _layer_sizes(case: dict) -> list[int]:
    """A stack of layers: four square matrices, two of 4 dim x dim, two vectors each, and one vector at the end."""
    d = case["dim"]
    return ([d, d * d, d * d, d * d, d * d, d, 4 * d * d, 4 * d * d] * case["layers"]) + [d]


def _prepare_adamw(case: dict, g) -> dict:
    kind, d = TYPES[case["type"]], case["dim"]
    s = dict(case=case, step=100)
    if case["kind"] == "tables":
        v = case["words"]
        params, grads = [], []
        for rows in (v, v - 1):
            for to, scale in ((params, 0.3), (grads, 0.01)):
                to.append(_padded(rows, d)[:, :d])
                to[-1].copy_(torch.randn(rows, d, generator=g, device="cuda").mul_(scale))
        for _ in range(2):
            params.append(torch.randn(d, generator=g, device="cuda"))
            grads.append(torch.randn(d, generator=g, device="cuda") * 0.01)
        sizes, decay = [p.numel() for p in params], [DECAY, DECAY, 0.0, 0.0]
    else:
        sizes = _layer_sizes(case)
        decay = [0.0 if n == d else DECAY for n in sizes]
    blocks = [-(-n // BLOCK) for n in sizes]
    at = np.concatenate([[0], np.cumsum(blocks)]) * BLOCK     # each tensor starts on a block's border
    total = int(at[-1])
    inside = torch.ones(total, dtype=torch.bool, device="cuda")
    for n, lo, hi in zip(sizes, at, at[1:]):
        inside[int(lo) + n:int(hi)] = False
    if case["kind"] == "layers":
        flat = (torch.randn(total, generator=g, device="cuda") * 0.05).mul_(inside).to(kind)
        gflat = (torch.randn(total, generator=g, device="cuda") * 0.01).mul_(inside).to(kind)
        params = [flat[int(lo):int(lo) + n] for n, lo in zip(sizes, at)]
        grads = [gflat[int(lo):int(lo) + n] for n, lo in zip(sizes, at)]
        s.update(flat=flat, gflat=gflat)
    m = torch.randn(total, generator=g, device="cuda").mul_(inside)
    r = (torch.rand(total, generator=g, device="cuda") + 0.05).mul_(inside)
    if case["bits"] == 8:
        m = (m * 100).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        r = (r * 240).to(torch.uint8)
        scales = torch.rand(2, total // BLOCK, generator=g, device="cuda") + 0.5
        s.update(ms=scales[0] * 2e-5, vs=scales[1] * 6e-3)
        s.update(m=m, v=r)
    else:
        s.update(m=m * 3e-3, v=(r * 1e-2).square_())
    s.update(params=params, grads=grads, sizes=sizes, at=[int(a) for a in at], decay=decay)
    if own:   # the optimizer, which a program makes once, resumed from these moments
        import paper_1606_07822_amd as w2v
        state = (s["m"], s["v"], s["ms"], s["vs"]) if case["bits"] == 8 else (s["m"], s["v"])
        s["opt"] = w2v.AdamW(params, grads, bits=case["bits"], betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=decay,
                             seed=ROUNDING_SEED, state=state)
        s["wide"] = (torch.empty(total, device="cuda"), torch.empty(total, device="cuda")) if case["bits"] == 8 else None
    return s


# ------------------------------------------------------------------ one pass
def run(state: dict):
    op = state["case"]["op"]
    if own:
        return _own(op, state)
    return {"norm": _plain_norm, "norm_back": _plain_norm_back, "loss": _plain_loss, "adamw": _plain_adamw}[op](state)


def _own(op: str, s: dict):
    import paper_1606_07822_amd as w2v
    if op == "norm":
        return w2v.layer_norm(s["x"], s["w"], s["b"], EPS, out=s["y"])
    if op == "norm_back":
        return w2v.layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], dx=s["y"])
    if op == "loss":
        grads = s["case"]["grads"]
        loss, dx, dsyn1 = w2v.hs_loss(s["model"], s["x"], s["targets"], s["weights"], grads=grads, loss=s["loss"],
                                      dx=s.get("dx"), dsyn1=s.get("dsyn1"), workspace=s["workspace"])
        return (loss, dx, dsyn1[:, :s["case"]["dim"]]) if grads else loss
    s["opt"].step(s["step"], LR)
    s["step"] += 1
    m, v = s["opt"].moments(*s["wide"]) if s["wide"] else (s["m"], s["v"])
    return ([s["flat"]] if "flat" in s else s["params"]), m, v


def _plain_norm(s: dict):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    y = c * rstd
    if s["w"] is not None:
        y = y * s["w"] + s["b"]
    return y.to(s["x"].dtype), mean[:, 0], rstd[:, 0]


def _plain_norm_back(s: dict):
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    h = (s["x"].float() - s["mean"][:, None]) * rstd
    a = dy if s["w"] is None else dy * s["w"]
    dx = rstd * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
    dw = db = None
    if s["w"] is not None:
        dw, db = (dy * h).sum(0, dtype=torch.float64).float(), dy.sum(0, dtype=torch.float64).float()
    return dx.to(s["x"].dtype), dw, db


def _plain_loss(s: dict):
    d, targets, longest = s["case"]["dim"], s["targets"].long(), s["longest"]
    x = s["x"].float()
    word = targets.clamp(min=0)
    level = torch.arange(longest, device="cuda")
    on = (level < s["codelen"][word].long()[:, None]) & (targets >= 0)[:, None]           # [rows, levels]
    node = torch.where(on, s["points"][(s["off"][word].long()[:, None] + level).clamp(max=s["points"].numel() - 1)].long(), 0)
    sign = 1 - 2 * ((s["code"][word][:, None] >> level) & 1).float()
    y = s["syn1"][:, :d][node]                                                             # [rows, levels, d]
    z = sign * (y * x[:, None, :]).sum(2)
    loss = torch.where(on, torch.log1p(torch.exp(-z.abs())) + (-z).clamp(min=0), 0).sum(1)
    if not s["case"]["grads"]:
        return loss
    g = torch.where(on, -sign / (1 + torch.exp(z)), 0) * s["weights"][:, None]
    dx = (g[:, :, None] * y).sum(1)
    del y
    dsyn1 = torch.zeros(s["syn1"].shape[0], d, dtype=torch.float64, device="cuda")
    dsyn1.index_add_(0, node.flatten(), (g.double()[:, :, None] * x.double()[:, None, :]).flatten(0, 1))
    return loss, dx.to(s["x"].dtype), dsyn1.float()


def _moments_of(s: dict, m: torch.Tensor, v: torch.Tensor):
    """The moments that 8-bit codes stand for: m in e4m3, sqrt(v) in four bits of exponent and four of fraction."""
    m = (m.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * s["ms"][:, None]).flatten()
    c = v.to(torch.int32)
    r = torch.where(c < 16, c.float() * 2.0**-18, ((c + 112 * 16) << 19).view(torch.float32))
    r = (r.view(-1, BLOCK) * s["vs"][:, None]).flatten()
    return m, r * r


def _mix(h: torch.Tensor) -> torch.Tensor:
    """Murmur3's 32-bit finaliser, on values below 2^32 held in 64 bits."""
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & 0xFFFFFFFF
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & 0xFFFFFFFF
    return h ^ (h >> 16)


def _plain_codes(s: dict, m: torch.Tensor, v: torch.Tensor) -> None:
    """Moments to 8 bits: m to the nearest code, sqrt(v) up or down at random in proportion to its place between two."""
    blocks = m.view(-1, BLOCK)
    scale = blocks.abs().amax(1) * (1 / 448)
    scale = torch.where(scale < 2.0**-126, 0, scale)
    inverse = torch.where(scale > 0, 1 / scale, 0)
    s["m"].copy_((blocks * inverse[:, None]).flatten().to(torch.float8_e4m3fn).view(torch.uint8))
    s["ms"].copy_(scale)
    r = torch.sqrt(v)
    blocks = r.view(-1, BLOCK)
    scale = blocks.amax(1) * (16 / 31)
    inverse = torch.where(scale > 0, 1 / scale, 0)
    t = (blocks * inverse[:, None]).flatten()
    key = _mix(torch.full((1,), (ROUNDING_SEED ^ (s["step"] * 0x9E3779B9)) & 0xFFFFFFFF, device="cuda"))
    i = torch.arange(m.numel(), device="cuda")
    h = _mix(((i >> 1) & 0xFFFFFFFF) ^ key)
    h = torch.where((i & 1) == 1, h >> 16, h & 0xFFFF).to(torch.int32)
    normal = ((t.view(torch.int32) + h * 8 + 4) >> 19) - 112 * 16
    small = torch.floor(t * 2.0**18 + (h.float() + 0.5) * 2.0**-16).to(torch.int32)
    code = torch.where(t < 2.0**-14, small, normal).clamp(max=255)
    s["v"].copy_(torch.where((r > 0) & (code == 0), 1, code).to(torch.uint8))
    s["vs"].copy_(scale)


def _plain_adamw(s: dict):
    case, t = s["case"], s["step"]
    size = LR / (1 - BETA1**t)
    root = 1 / math.sqrt(1 - BETA2**t)
    m, v = (s["m"], s["v"]) if case["bits"] == 32 else _moments_of(s, s["m"], s["v"])
    if case["kind"] == "layers":     # one pass over the tensors' common storage, each with its decay
        keep = torch.tensor([1 - LR * w for w in s["decay"]], device="cuda")
        spans = torch.tensor([hi - lo for lo, hi in zip(s["at"], s["at"][1:])], device="cuda")
        parts = [(s["flat"], s["gflat"], m, v, torch.repeat_interleave(keep, spans, output_size=s["at"][-1]))]
    else:
        parts = [(p, g, m[lo:lo + n].view(p.shape), v[lo:lo + n].view(p.shape), 1 - LR * w)
                 for p, g, n, lo, w in zip(s["params"], s["grads"], s["sizes"], s["at"], s["decay"])]
    for p, grad, m1, v1, keep in parts:
        g = grad.float()
        m1.copy_(m1 * BETA1 + g * (1 - BETA1))
        v1.copy_(v1 * BETA2 + (g * g) * (1 - BETA2))
        p.copy_(p.float() * keep - (m1 * size) / (torch.sqrt(v1) * root + ADAM_EPS))
    if case["bits"] == 8:
        _plain_codes(s, m, v)
        m, v = _moments_of(s, s["m"], s["v"])
    s["step"] = t + 1
    return ([s["flat"]] if "flat" in s else s["params"]), m, v


# ------------------------------------------------------------------ in 64 bits
def exact(case: dict, seed: int):
    s = prepare(case, seed)
    if case["op"] in ("norm", "norm_back"):
        return _exact_norm(case, s)
    return _exact_loss(case, s) if case["op"] == "loss" else _exact_adamw(case, s)


def _exact_norm(case: dict, s: dict):
    x, d = s["x"].double(), case["dim"]
    w = None if s["w"] is None else s["w"].double()
    if case["op"] == "norm":
        mean = x.sum(1) / d
        var = (x - mean[:, None]).pow(2).sum(1) / d
        rstd = (var + EPS).pow(-0.5)
        y = (x - mean[:, None]) * rstd[:, None]
        return (y if w is None else torch.addcmul(s["b"].double(), y, w)), mean, rstd
    rstd = s["rstd"].double()[:, None]
    h, dy = (x - s["mean"].double()[:, None]) * rstd, s["dy"].double()
    a = dy if w is None else dy * w
    dx = rstd / d * (d * a - a.sum(1, keepdim=True) - h * (a * h).sum(1, keepdim=True))
    return (dx, None, None) if w is None else (dx, (dy * h).sum(0), dy.sum(0))


def _exact_loss(case: dict, s: dict):
    """Level by level from the root down."""
    n, d, grads = case["rows"], case["dim"], case["grads"]
    x = s["x"].double()
    loss = torch.zeros(n, dtype=torch.float64, device="cuda")
    dx = torch.zeros_like(x) if grads else None
    dsyn1 = torch.zeros(s["syn1"].shape[0], d, dtype=torch.float64, device="cuda") if grads else None
    row = torch.nonzero(s["targets"] >= 0)[:, 0]
    word = s["targets"].long()[row]
    for j in range(s["longest"]):
        live = s["codelen"][word].long() > j
        row, word = row[live], word[live]
        node = s["points"][s["off"][word].long() + j].long()
        label = 1 - ((s["code"][word] >> j) & 1).double()
        y = s["syn1"][node, :d].double()
        p = (y * x[row]).sum(1).sigmoid()
        loss[row] -= torch.where(label > 0, p, 1 - p).log()
        if grads:
            g = ((p - label) * s["weights"].double()[row])[:, None]
            dx[row] += g * y
            dsyn1.index_add_(0, node, g * x[row])
    return (loss, dx, dsyn1) if grads else loss


def _exact_adamw(case: dict, s: dict):
    """Parameters in 64 bits. Moments held in 8 bits have no such value: where a moment lies within a 32-bit rounding of
    the border between two codes, 64 bits put it on the border's other side, a whole code away."""
    t = s["step"]
    narrow = case["bits"] == 8
    m, v = _moments_of(s, s["m"], s["v"]) if narrow else (s["m"], s["v"])
    new, first, second = [], torch.zeros(0 if narrow else m.numel(), dtype=torch.float64, device="cuda"), None
    second = torch.zeros_like(first)
    flat = torch.zeros(s["at"][-1], dtype=torch.float64, device="cuda") if "flat" in s else None
    for p, g, n, lo, w in zip(s["params"], s["grads"], s["sizes"], s["at"], s["decay"]):
        g = g.double().flatten()
        m1 = BETA1 * m[lo:lo + n].double() + (1 - BETA1) * g
        v1 = BETA2 * v[lo:lo + n].double() + (1 - BETA2) * g.pow(2)
        step = LR * (m1 / (1 - BETA1**t)) / ((v1 / (1 - BETA2**t)).sqrt() + ADAM_EPS)
        out = (p.double().flatten() * (1 - LR * w) - step).view(p.shape)
        if flat is None:
            new.append(out)
        else:
            flat[lo:lo + n] = out
        if not narrow:
            first[lo:lo + n], second[lo:lo + n] = m1, v1
    return ([flat] if flat is not None else new), (None if narrow else first), (None if narrow else second)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case: dict) -> dict:
    size = torch.empty(0, dtype=TYPES[case["type"]]).element_size()
    d = case["dim"]
    if case["op"] in ("norm", "norm_back"):
        n, back = case["rows"], case["op"] == "norm_back"
        vectors = (8 + 4 * back) * d if case["affine"] else 0       # weight and bias; weight and two gradients
        return dict(bytes=(3 if back else 2) * n * d * size + 8 * n + vectors, flops=(14 if back else 8) * n * d)
    if case["op"] == "loss":
        t = _tree(case["words"], case["zipf"])
        rows = case["rows"] * (1 - MASKED if case["rows"] > 1 else 1)
        steps = rows * float(t["share"].sum())                      # nodes on the batch's paths
        nodes = float((1 - (1 - t["share"]) ** rows).sum())         # different ones among them
        b = rows * d * size + nodes * d * 4 + case["rows"] * 8
        if case["grads"]:
            b += case["rows"] * (d * size + 4) + (case["words"] - 1) * d * 4
        return dict(bytes=b, flops=(6 if case["grads"] else 2) * steps * d)
    if case["kind"] == "tables":
        n = (2 * case["words"] + 1) * d
    else:
        n = sum(_layer_sizes(case))
    # parameter in and out, gradient in; moments in and out, and as 32-bit values where they are held in 8 bits
    moments = 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 8
    return dict(bytes=n * (3 * size + moments), flops=16 * n)
