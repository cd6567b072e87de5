"""Argument checks of the feed-forward block's, orthogonalize's and Muon's C ABI: reported before anything is launched (no GPU
needed)."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def w2v():
    import paper_1606_07822_amd as w2v
    if not os.path.exists(w2v.LIB_PATH):
        pytest.skip("libw2v.so not built")
    return w2v


X, WG, WU, WD, Y, GATE, UP, WS, DY, DX, DG, DU, DD = (0x100000 * k for k in range(1, 14))   # addresses that are never read
INF, NAN = float("inf"), float("nan")


def forward_args(w2v, **kw):
    a = dict(x=(X, 8), w_gate=(WG, 8), w_up=(WU, 8), w_down=(WD, 12), rows=4, dim=8, hidden=12, type=0, act=0, y=(Y, 8),
             gate=(GATE, 12), up=(UP, 12), ws=WS, ws_bytes=1 << 20, stream=None)
    a.update(kw)
    return [w2v.CRows(*v) if isinstance(v, tuple) else v for v in a.values()]


@pytest.mark.parametrize("kw,code,msg", [
    (dict(rows=-1), -1, "rows"), (dict(rows=2**31), -1, "rows"), (dict(dim=0), -1, "dim"), (dict(dim=2**20 + 1), -1, "dim"),
    (dict(hidden=0), -1, "hidden"), (dict(hidden=2**20 + 1), -1, "hidden"), (dict(type=3), -1, "type"), (dict(type=-1), -1, "type"),
    (dict(act=2), -1, "act"), (dict(act=-1), -1, "act"), (dict(x=(None, 8)), -1, "x is NULL"), (dict(x=(X, 7)), -1, "x's stride"),
    (dict(x=(X + 2, 8)), -1, "aligned"), (dict(w_gate=(None, 8)), -1, "w_gate is NULL"), (dict(w_gate=(WG, 7)), -1, "w_gate's"),
    (dict(w_up=(WU, 3)), -1, "w_up's"), (dict(w_down=(WD, 11)), -1, "w_down's"), (dict(w_down=(None, 12)), -1, "w_down is NULL"),
    (dict(y=(None, 8)), -1, "y is NULL"), (dict(y=(Y, 7)), -1, "y's"), (dict(y=(X, 9)), -1, "same stride"),
    (dict(y=(WG, 8)), -1, "y"), (dict(y=(GATE, 12)), -1, "y"), (dict(gate=(GATE, 11)), -1, "gate's"), (dict(gate=(UP, 12)), -1, "gate may not"),
    (dict(up=(X, 12)), -1, "up may not"), (dict(gate=(WD, 12)), -1, "gate may not"), (dict(type=1, x=(X + 1, 8)), -1, "aligned"),
    (dict(x=(X, 2**61)), -1, "too large"), (dict(ws=None), -1, "workspace is NULL"), (dict(ws=WS + 16), -1, "workspace must be"),
    (dict(ws_bytes=100), -3, "workspace"),
])
def test_gated_ffn_argument_errors(w2v, kw, code, msg):
    assert w2v.lib().w2v_gated_ffn(*forward_args(w2v, **kw)) == code
    assert msg in w2v.last_error()


def backward_args(w2v, **kw):
    a = dict(dy=(DY, 8), x=(X, 8), w_gate=(WG, 8), w_up=(WU, 8), w_down=(WD, 12), gate=(GATE, 12), up=(UP, 12), rows=4, dim=8,
             hidden=12, type=0, act=0, dx=(DX, 8), dw_gate=(DG, 8), dw_up=(DU, 8), dw_down=(DD, 12), ws=WS, ws_bytes=1 << 20,
             stream=None)
    a.update(kw)
    return [w2v.CRows(*v) if isinstance(v, tuple) else v for v in a.values()]


@pytest.mark.parametrize("kw,code,msg", [
    (dict(dy=(None, 8)), -1, "dy is NULL"), (dict(x=(None, 8)), -1, "x is NULL"), (dict(gate=(None, 12)), -1, "gate is NULL"),
    (dict(up=(None, 12)), -1, "up is NULL"), (dict(dy=(DY, 7)), -1, "dy's"), (dict(dx=(DX, 7)), -1, "dx's"),
    (dict(dw_gate=(DG, 7)), -1, "dw_gate's"), (dict(dw_down=(DD, 11)), -1, "dw_down's"), (dict(dx=(DY, 9)), -1, "same stride"),
    (dict(dx=(X, 9)), -1, "same stride"), (dict(dx=(WG, 8)), -1, "dx may be"), (dict(dx=(GATE, 12)), -1, "dx may be"),
    (dict(dx=(DG, 8)), -1, "dw_gate may not"), (dict(dw_gate=(WG, 8)), -1, "dw_gate may not"), (dict(dw_up=(DG, 8)), -1, "may not"),
    (dict(dw_down=(WD, 12)), -1, "dw_down may not"), (dict(dw_gate=(X, 8)), -1, "dw_gate may not"), (dict(dw_up=(DU + 2, 8)), -1, "aligned"),
    (dict(rows=-1), -1, "rows"), (dict(dim=0), -1, "dim"), (dict(type=7), -1, "type"), (dict(act=5), -1, "act"),
    (dict(ws=None), -1, "workspace is NULL"), (dict(ws_bytes=64), -3, "workspace"),
])
def test_gated_ffn_backward_argument_errors(w2v, kw, code, msg):
    assert w2v.lib().w2v_gated_ffn_backward(*backward_args(w2v, **kw)) == code
    assert msg in w2v.last_error()


def test_arrays_of_no_rows_may_lie_anywhere(w2v):
    """Where they end at another array, too: nothing is read or written there."""
    for kw in (dict(gate=(UP, 12)), dict(up=(WD, 12)), dict(y=(GATE, 8)), dict(y=(X, 9)), dict(gate=(X, 12), up=(X, 12), y=(X, 8))):
        assert w2v.lib().w2v_gated_ffn(*forward_args(w2v, rows=0, **kw)) == 0, kw
    none = (None, 0)
    for dx in ((WG, 8), (GATE, 12), (X, 8)):
        assert w2v.lib().w2v_gated_ffn_backward(*backward_args(w2v, rows=0, dx=dx, dw_gate=none, dw_up=none, dw_down=none)) == 0


def test_gated_ffn_workspace_sizes(w2v):
    """Nothing for no rows or for sizes out of range; never less for more rows."""
    for name in ("w2v_gated_ffn_workspace_bytes", "w2v_gated_ffn_backward_workspace_bytes"):
        size = getattr(w2v.lib(), name)
        assert size(0, 8, 8, 0) == 0 and size(-1, 8, 8, 0) == 0 and size(4, 0, 8, 0) == 0 and size(4, 8, 2**21, 0) == 0
        assert size(4, 8, 8, 9) == 0 and size(2**31, 8, 8, 0) == 0
        for kind in (0, 1, 2):
            for n in (1, 16, 17, 64, 65, 300, 70_000):
                # at least h, as the second product reads it
                assert size(n, 100, 400, kind) >= n * 400 * 2
    assert w2v.lib().w2v_gated_ffn_backward_workspace_bytes(2**31 - 1, 4096, 2**20, 0) > 2**50   # 64 bits throughout


def orth_args(**kw):
    a = dict(g=X, g_stride=8, g_step=64, batch=3, rows=6, cols=8, type=0, steps=5, eps=1e-7, out=Y, out_stride=8, out_step=64,
             ws=WS, ws_bytes=1 << 22, stream=None)
    a.update(kw)
    return list(a.values())


def test_orthogonalize_workspace_sizes(w2v):
    """Nothing for sizes out of range, the largest counts of matrices among them (a count that wrapped divided by zero)."""
    size = w2v.lib().w2v_orthogonalize_workspace_bytes
    assert size(1, 6, 8, 0) > 0 and size(2**31 - 1, 1, 1, 0) > 0 and size(0, 6, 8, 0) == 0
    for bad in ((2**31, 1, 1, 0), (2**63 - 1, 1, 1, 0), (2**63 - 4000, 6, 8, 1), (-1, 1, 1, 0), (1, 2**20 + 1, 1, 0), (1, 1, 1, 3)):
        assert size(*bad) == 0


@pytest.mark.parametrize("kw,code,msg", [
    (dict(batch=2**31), -1, "batch"), (dict(batch=2**63 - 1, g_step=0, out_step=48), -1, "batch"),
    (dict(g=None), -1, "g is NULL"), (dict(out=None), -1, "out is NULL"), (dict(g_stride=7), -1, "g's"), (dict(out_stride=7), -1, "out's"),
    (dict(batch=-1), -1, "batch"), (dict(rows=-1), -1, "rows"), (dict(cols=2**20 + 1), -1, "cols"), (dict(type=3), -1, "type"),
    (dict(steps=0), -1, "steps"), (dict(steps=21), -1, "steps"), (dict(eps=-1.0), -1, "eps"), (dict(eps=NAN), -1, "eps"),
    (dict(eps=INF), -1, "eps"), (dict(out_step=47), -1, "overlap"), (dict(g_step=-8), -1, "g_step"), (dict(out=X, out_step=72), -1, "same strides"),
    (dict(out=X, out_stride=9), -1, "same strides"), (dict(g=X + 2), -1, "aligned"), (dict(g_step=2**62), -1, "too large"),
    (dict(ws=None), -1, "workspace is NULL"), (dict(ws_bytes=64), -3, "workspace"),
])
def test_orthogonalize_argument_errors(w2v, kw, code, msg):
    assert w2v.lib().w2v_orthogonalize(*orth_args(**kw)) == code
    assert msg in w2v.last_error()


def matrices(w2v, *changes):
    """Three matrices with distinct memory."""
    t = (w2v.CMuonMatrix * 3)()
    for i in range(3):
        t[i] = w2v.CMuonMatrix(X + 0x10000 * i, Y + 0x10000 * i, 6, 8, 8, 8, 256 * i, 0, 0, 0.0, 1.0)
    for i, name, value in changes:
        setattr(t[i], name, value)
    return t


@pytest.mark.parametrize("change,msg", [
    ((1, "rows", -1), "matrix 1"), ((1, "cols", 2**20 + 1), "matrix 1"), ((2, "param_type", 3), "type"), ((0, "grad_type", -1), "type"),
    ((1, "param", None), "NULL"), ((1, "grad", None), "NULL"), ((1, "param_stride", 7), "stride"), ((1, "grad_stride", 7), "stride"),
    ((1, "moment_offset", 100), "moment_offset"), ((1, "moment_offset", -256), "moment_offset"), ((1, "moment_offset", 768), "moment_offset"),
    ((1, "moment_offset", 0), "overlap"), ((1, "param", X), "overlap"), ((1, "weight_decay", NAN), "weight_decay"), ((1, "scale", INF), "scale"),
    ((1, "param", X + 2), "aligned"),
])
def test_muon_plan_errors(w2v, change, msg):
    assert w2v.lib().w2v_muon_build_plan(matrices(w2v, change), 3, 768, WS, 1 << 16, None) == w2v.W2V_E_ARG
    assert msg in w2v.last_error()


def test_muon_plan_arguments(w2v):
    build, t = w2v.lib().w2v_muon_build_plan, matrices(w2v)
    for args, code, msg in [((t, -1, 768, WS, 1 << 16), -1, "matrices_host"), ((None, 1, 768, WS, 1 << 16), -1, "matrices_host"),
                            ((t, 3, 700, WS, 1 << 16), -1, "n_moments"), ((t, 3, 512, WS, 1 << 16), -1, "moment_offset"),
                            ((t, 3, 768, None, 1 << 16), -1, "workspace"), ((t, 3, 768, WS, 8), -3, "workspace"),
                            ((t, 3, 768, WS + 8, 1 << 16), -1, "workspace")]:
        assert build(*args, None) == code
        assert msg in w2v.last_error()
    assert w2v.lib().w2v_muon_plan_bytes(t, 3) > 0 and w2v.lib().w2v_muon_workspace_bytes(t, 3) > 0
    assert w2v.lib().w2v_muon_plan_bytes(None, 3) == w2v.lib().w2v_muon_workspace_bytes(None, 3) == 0
    assert w2v.lib().w2v_muon_workspace_bytes(matrices(w2v, (0, "rows", 2**21)), 3) == 0
    empty = matrices(w2v, *((i, "rows", 0) for i in range(3)))
    assert w2v.lib().w2v_muon_workspace_bytes(empty, 3) == 0


@pytest.mark.parametrize("kw,code,msg", [
    (dict(lr=NAN), -1, "lr"), (dict(lr=INF), -1, "lr"), (dict(momentum=1.0), -1, "momentum"), (dict(momentum=-0.1), -1, "momentum"),
    (dict(momentum=NAN), -1, "momentum"), (dict(eps=-1.0), -1, "eps"), (dict(eps=NAN), -1, "eps"), (dict(steps=0), -1, "steps"),
    (dict(steps=21), -1, "steps"), (dict(lr_device=X + 2), -1, "lr_device"), (dict(plan=None), -1, "plan is NULL"),
    (dict(plan=WS + 16), -1, "plan must be"), (dict(m=None), -1, "m is NULL"), (dict(m=DG + 2), -1, "aligned"),
    (dict(p=None), -1, "params"), (dict(ws=None), -1, "workspace is NULL"), (dict(ws_bytes=64), -3, "workspace"), (dict(n=-1), -1, "matrices"),
])
def test_muon_step_argument_errors(w2v, kw, code, msg):
    p = w2v.CMuonParams(0.1, 0.9, 1e-7, None, 1.0, 1, 5, 0)
    for k in ("lr", "momentum", "eps", "steps", "lr_device"):
        if k in kw:
            setattr(p, k, kw[k])
    a = dict(n=3, plan=WS, m=DG, p=ctypes.byref(p), ws=DU, ws_bytes=1 << 24)
    a.update({k: v for k, v in kw.items() if k in a})
    assert w2v.lib().w2v_muon_step(matrices(w2v), a["n"], a["plan"], a["m"], a["p"], a["ws"], a["ws_bytes"], None) == code
    assert msg in w2v.last_error()
