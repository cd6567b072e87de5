"""Argument checks of the mini-batch operators' C ABI: reported before anything is launched (no GPU needed)."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def w2v():
    import paper_1606_07822_amd as w2v
    if not os.path.exists(w2v.LIB_PATH):
        pytest.skip("libw2v.so not built")
    return w2v


A, B, C, D, E, F = (0x10000 * k for k in range(1, 7))   # addresses that are never read


def norm_args(**kw):
    a = dict(x=A, type=0, rows=4, dim=8, x_stride=8, weight=B, bias=C, w_type=0, eps=1e-5, y=D, y_stride=8, mean=E,
             rstd=F, stream=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("kw,msg", [
    (dict(rows=-1), "rows"), (dict(dim=0), "dim"), (dict(dim=16385, x_stride=16385, y_stride=16385), "dim"),
    (dict(type=3), "type"), (dict(type=-1), "type"), (dict(type=1, w_type=2), "w_type"), (dict(x_stride=7), "x's stride"),
    (dict(y_stride=7), "y's stride"), (dict(x=None), "x is NULL"), (dict(y=None), "y is NULL"), (dict(x=A + 2), "aligned"),
    (dict(weight=B + 1), "aligned"), (dict(mean=E + 2), "aligned"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps"), (dict(y=A, y_stride=9), "same stride"), (dict(x_stride=2**60), "too large"),
])
def test_layer_norm_argument_errors(w2v, kw, msg):
    assert w2v.lib().w2v_layer_norm(*norm_args(**kw)) == w2v.W2V_E_ARG
    assert msg in w2v.last_error()


def back_args(**kw):
    a = dict(dy=A, dy_stride=8, x=B, type=0, rows=4, dim=8, x_stride=8, weight=C, w_type=0, mean=D, rstd=E, dx=F, dx_stride=8,
             dw=0x80000, db=0x90000, ws=0xA0000, ws_bytes=1 << 20, stream=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("kw,code,msg", [
    (dict(dy=None), -1, "dy is NULL"), (dict(x=None), -1, "x is NULL"), (dict(dx=None), -1, "dx is NULL"),
    (dict(mean=None), -1, "mean is NULL"), (dict(rstd=None), -1, "rstd is NULL"), (dict(dy_stride=3), -1, "dy's stride"),
    (dict(dx_stride=3), -1, "dx's stride"), (dict(dx=A, dx_stride=9), -1, "same stride"), (dict(dx=B, dx_stride=9), -1, "same stride"),
    (dict(ws=None), -1, "workspace is NULL"), (dict(ws=0xA0010), -1, "workspace must be"), (dict(ws_bytes=8), -3, "workspace"),
    (dict(dim=0), -1, "dim"), (dict(dw=0x80002), -1, "aligned"),
])
def test_layer_norm_backward_argument_errors(w2v, kw, code, msg):
    assert w2v.lib().w2v_layer_norm_backward(*back_args(**kw)) == code
    assert msg in w2v.last_error()


def hs_args(w2v, model=None, **kw):
    m = w2v.CModel(None, 0x20000, 100, 50, 64, 0, None, 0, 0x40000, 0x50000, 0x60000, 0x70000)
    for k, v in (model or {}).items():
        setattr(m, k, v)
    a = dict(m=ctypes.byref(m), longest=20, x=A, type=0, rows=4, x_stride=50, targets=C, weights=D, loss=E, dx=F, dx_stride=50,
             dsyn1=0x80000, ds_stride=64, ws=0xA0000, ws_bytes=1 << 30, stream=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("model,kw,code,msg", [
    (dict(V=1), {}, -1, "V must"), (dict(dim=0), {}, -1, "dim"), (dict(dim=1025, row_stride=1028), {}, -1, "dim"),
    (dict(row_stride=49), {}, -1, "row_stride"), (dict(row_stride=66), {}, -1, "row_stride"), (dict(syn1=None), {}, -1, "syn1"),
    (dict(syn1=0x20004), {}, -1, "aligned"), (dict(codelen=None), {}, -1, "Huffman"), (dict(code=None), {}, -1, "Huffman"),
    (dict(point_off=None), {}, -1, "Huffman"), (dict(points=None), {}, -1, "Huffman"), ({}, dict(longest=0), -1, "max_code_len"),
    ({}, dict(longest=65), -1, "max_code_len"), ({}, dict(m=None), -1, "model"), ({}, dict(x=None), -1, "x is NULL"),
    ({}, dict(type=5), -1, "type"), ({}, dict(rows=-1), -1, "rows"), ({}, dict(x_stride=49), -1, "x's stride"),
    ({}, dict(targets=None), -1, "targets"), ({}, dict(targets=C + 1), -1, "aligned"), ({}, dict(dx=A), -1, "dx may not"),
    ({}, dict(dx_stride=3), -1, "dx's stride"), ({}, dict(dsyn1=0x20000), -1, "dsyn1 may not"),
    ({}, dict(ds_stride=49), -1, "dsyn1's stride"), ({}, dict(ws_bytes=100), -3, "workspace"), ({}, dict(ws=None), -1, "workspace"),
])
def test_hs_loss_argument_errors(w2v, model, kw, code, msg):
    assert w2v.lib().w2v_hs_loss(*hs_args(w2v, model, **kw)) == code
    assert msg in w2v.last_error()


def tensor(w2v, **kw):
    t = dict(param=A, grad=B, rows=4, cols=100, param_stride=100, grad_stride=100, moment_offset=0, param_type=0, grad_type=0,
             weight_decay=0.01, reserved0=0)
    t.update(kw)
    return w2v.CAdamWTensor(*t.values())


def build(w2v, tensors, n_moments=1024, plan=0xA0000, plan_bytes=1 << 20):
    table = (w2v.CAdamWTensor * max(len(tensors), 1))(*tensors)
    n = ctypes.c_int64(0)
    return w2v.lib().w2v_adamw_build_plan(table, len(tensors), n_moments, plan, plan_bytes, ctypes.byref(n), None)


@pytest.mark.parametrize("kw,msg", [
    (dict(param=None), "param is NULL"), (dict(grad=None), "grad is NULL"), (dict(rows=-1), "rows and cols"),
    (dict(cols=-1), "rows and cols"), (dict(rows=1 << 30, cols=1 << 20), "2^40"), (dict(param_stride=99), "stride"),
    (dict(grad_stride=99), "stride"), (dict(moment_offset=-256), "moment_offset"), (dict(moment_offset=100), "moment_offset"),
    (dict(moment_offset=768), "moment_offset"), (dict(param_type=7), "type"), (dict(grad_type=-1), "type"),
    (dict(weight_decay=float("nan")), "weight_decay"), (dict(param=A + 2), "aligned"), (dict(grad=B + 1, grad_type=1), "aligned"),
])
def test_adamw_plan_tensor_errors(w2v, kw, msg):
    assert build(w2v, [tensor(w2v, **kw)]) == w2v.W2V_E_ARG
    assert msg in w2v.last_error()


def test_adamw_plan_list_errors(w2v):
    a, b = tensor(w2v), tensor(w2v, param=C, moment_offset=256)
    assert build(w2v, [a, b]) == w2v.W2V_E_ARG and "moments overlap" in w2v.last_error()
    b = tensor(w2v, param=A + 400, moment_offset=512)
    assert build(w2v, [a, b]) == w2v.W2V_E_ARG and "parameters overlap" in w2v.last_error()
    assert build(w2v, [a], n_moments=1000) == w2v.W2V_E_ARG and "multiple of 256" in w2v.last_error()
    assert build(w2v, [a], plan_bytes=300) == w2v.W2V_E_WORKSPACE
    assert build(w2v, [a], plan=None) == w2v.W2V_E_ARG
    assert build(w2v, [a], plan=0xA0010) == w2v.W2V_E_ARG
    assert w2v.lib().w2v_adamw_plan_bytes((w2v.CAdamWTensor * 1)(tensor(w2v, rows=-1)), 1) == 0
    assert w2v.lib().w2v_adamw_plan_bytes((w2v.CAdamWTensor * 1)(a), 1) > 0


@pytest.mark.parametrize("kw,msg", [
    (dict(bits=16), "bits"), (dict(n=-1), "n_chunks"), (dict(plan=None), "plan"), (dict(m=None), "m or v"), (dict(v=None), "m or v"),
    (dict(m=A + 1), "aligned"), (dict(bits=8, ms=None), "m_scale"), (dict(bits=8, vs=None), "v_scale"),
    (dict(lr=float("inf")), "lr"), (dict(beta1=1.0), "beta"), (dict(beta2=-0.1), "beta"), (dict(beta2=float("nan")), "beta"),
    (dict(eps=-1.0), "eps"), (dict(step=0), "step"), (dict(lr_device=0x10002), "aligned"), (dict(step_device=0x10004), "aligned"),
    (dict(p=None), "params"),
])
def test_adamw_step_argument_errors(w2v, kw, msg):
    h = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, lr_device=None, step_device=None, grad_scale=1.0, seed=0)
    h.update({k: v for k, v in kw.items() if k in h})
    p = w2v.CAdamWParams(*h.values())
    a = dict(plan=0xA0000, n=1, bits=32, m=A, v=B, ms=C, vs=D, p=ctypes.byref(p), stream=None)
    a.update({k: v for k, v in kw.items() if k in a})
    assert w2v.lib().w2v_adamw_step(*a.values()) == w2v.W2V_E_ARG
    assert msg in w2v.last_error()


def test_adamw_moments_argument_errors(w2v):
    L = w2v.lib()
    assert L.w2v_adamw_moments(A, B, C, D, 100, E, F, None) == w2v.W2V_E_ARG
    assert L.w2v_adamw_moments(A, None, C, D, 256, E, F, None) == w2v.W2V_E_ARG
    assert L.w2v_adamw_moments(A + 2, B, C, D, 256, E, F, None) == w2v.W2V_E_ARG


def test_workspace_queries(w2v):
    L = w2v.lib()
    assert L.w2v_layer_norm_backward_workspace_bytes(-1, 8) == 0 and L.w2v_layer_norm_backward_workspace_bytes(4, 16385) == 0
    assert L.w2v_layer_norm_backward_workspace_bytes(100000, 300) >= L.w2v_layer_norm_backward_workspace_bytes(1, 300) > 0
    m = w2v.CModel(None, None, 100, 50, 64, 0, None, 0, None, None, None, None)
    q = L.w2v_hs_loss_workspace_bytes
    assert q(ctypes.byref(m), 65, 10) == 0 and q(ctypes.byref(m), 20, -1) == 0 and q(None, 20, 10) == 0
    assert q(ctypes.byref(m), 20, 67584) == q(ctypes.byref(m), 20, 10**7) > q(ctypes.byref(m), 20, 100) > 0


def batch_call(w2v, train=True, model=None, params=None, **kw):
    m = w2v.CModel(0x10000, 0x20000, 100, 50, 64, 0, 0x30000, 1000, 0x40000, 0x50000, 0x60000, 0x70000)
    for k, v in (model or {}).items():
        setattr(m, k, v)
    p = w2v.Params(window=5, corpus_tokens=1000, arch=1, sync_batch=64).c()
    for k, v in (params or {}).items():
        setattr(p, k, v)
    b = dict(gain=A, bias=B, m=C, v=D, m_scale=None, v_scale=None, beta1=0.9, beta2=0.999, eps=1e-8, step0=0, norm_eps=1e-5,
             weight_decay=0.0, bits=32, max_code_len=20, seed=0, reserved0=0)
    a = dict(tokens=0x80000, n=1000, steps=True, total=True, ws=0x900000, ws_bytes=1 << 40)
    b.update({k: v for k, v in kw.items() if k in b})
    a.update({k: v for k, v in kw.items() if k in a})
    cb, steps, terms, total = w2v.CBatchParams(*b.values()), ctypes.c_int64(0), ctypes.c_int64(0), ctypes.c_double(0)
    L = w2v.lib()
    first = (ctypes.byref(m), a["tokens"], a["n"], ctypes.byref(p), ctypes.byref(cb))
    if train:
        return L.w2v_train_batch_epoch(*first, None, ctypes.byref(steps) if a["steps"] else None, None, None, a["ws"],
                                       a["ws_bytes"], None)
    return L.w2v_batch_loglik(*first, ctypes.byref(total) if a["total"] else None, ctypes.byref(terms), a["ws"],
                              a["ws_bytes"], None)


@pytest.mark.parametrize("kw,code,msg", [
    (dict(model=dict(V=1)), -1, "V must"), (dict(model=dict(dim=0)), -1, "dim"), (dict(model=dict(syn0=None)), -1, "syn0"),
    (dict(model=dict(points=None)), -1, "Huffman"), (dict(params=dict(arch=0)), -1, "arch 1"),
    (dict(params=dict(window=11)), -1, "window"), (dict(params=dict(sync_batch=0)), -1, "sync_batch"),
    (dict(params=dict(sync_batch=(1 << 20) + 1)), -1, "sync_batch"), (dict(n=-1), -1, "tokens"), (dict(tokens=None), -1, "tokens"),
    (dict(max_code_len=0), -1, "max_code_len"), (dict(max_code_len=65), -1, "max_code_len"), (dict(gain=None), -1, "together"),
    (dict(bias=None), -1, "together"), (dict(gain=A + 2), -1, "aligned"), (dict(norm_eps=-1.0), -1, "norm_eps"),
    (dict(ws=None), -1, "workspace"), (dict(ws=0x900010), -1, "workspace"), (dict(ws_bytes=100), -3, "workspace"),
])
@pytest.mark.parametrize("train", [True, False])
def test_batch_argument_errors(w2v, train, kw, code, msg):
    assert batch_call(w2v, train, **kw) == code
    assert msg in w2v.last_error()


@pytest.mark.parametrize("kw,msg", [
    (dict(bits=16), "bits"), (dict(m=None), "moment"), (dict(v=None), "moment"), (dict(bits=8), "moment"), (dict(m=C + 2), "moments"),
    (dict(beta1=1.0), "beta"), (dict(beta2=-1.0), "beta"), (dict(eps=-1.0), "eps"), (dict(weight_decay=float("inf")), "weight_decay"),
    (dict(step0=-1), "step0"), (dict(bias=A), "differ"), (dict(steps=None), "steps_host"),
])
def test_batch_training_argument_errors(w2v, kw, msg):
    assert batch_call(w2v, True, **kw) == w2v.W2V_E_ARG
    assert msg in w2v.last_error()


def test_batch_queries(w2v):
    L = w2v.lib()
    m = w2v.CModel(None, None, 100, 50, 64, 0, None, 0, None, None, None, None)
    p = w2v.Params(window=5, arch=1, sync_batch=64).c()
    b = w2v.CBatchParams()
    b.max_code_len = 20
    M, Q, B_ = ctypes.byref(m), ctypes.byref(p), ctypes.byref(b)
    assert L.w2v_batch_n_moments(M, B_) == 5120 + 5120   # 5,000 and 4,950 in blocks of 256
    b.gain = A
    assert L.w2v_batch_n_moments(M, B_) == 5120 + 5120 + 2 * 256
    assert 0 < L.w2v_batch_loglik_workspace_bytes(M, 1000, Q, B_) < L.w2v_train_batch_workspace_bytes(M, 1000, Q, B_)
    p.sync_batch = 0
    assert L.w2v_train_batch_workspace_bytes(M, 1000, Q, B_) == 0 and L.w2v_batch_loglik_workspace_bytes(None, 1, Q, B_) == 0


def test_adamw_plan_finds_packed_parameters_that_overlap_whatever_their_gradients(w2v):
    """A packed parameter whose gradient's rows have gaps is one span as well: a second tensor in its middle would be
    updated twice."""
    a = tensor(w2v, grad_stride=128)                                        # 4 rows of 100 floats, one after the other
    b = tensor(w2v, param=A + 1200, rows=1, cols=10, param_stride=10, grad_stride=10, moment_offset=512)
    for pair in ([a, b], [b, a]):
        assert build(w2v, pair) == w2v.W2V_E_ARG and "parameters overlap" in w2v.last_error()
    beside = tensor(w2v, param=A + 1600, rows=1, cols=10, param_stride=10, grad_stride=10, moment_offset=512)
    assert build(w2v, [a, beside], plan=None) == w2v.W2V_E_ARG and "workspace" in w2v.last_error()
    gaps = tensor(w2v, param_stride=128)                                    # rows with gaps, another's row in one of them
    inside = tensor(w2v, param=A + 400, rows=1, cols=28, param_stride=28, grad_stride=28, moment_offset=512)
    assert build(w2v, [gaps, inside], plan=None) == w2v.W2V_E_ARG and "workspace" in w2v.last_error()


def test_batch_training_refused_has_taken_no_step(w2v):
    """steps_host is the call's own, whatever it held before and whichever check refuses."""
    m = w2v.CModel(0x10000, 0x20000, 100, 50, 64, 0, 0x30000, 1000, 0x40000, 0x50000, 0x60000, 0x70000)
    b = w2v.CBatchParams(A, B, C, D, None, None, 0.9, 0.999, 1e-8, 0, 1e-5, 0.0, 32, 20, 0, 0)
    for arch, n, ws_bytes, code in ((0, 1000, 1 << 40, w2v.W2V_E_ARG), (1, -1, 1 << 40, w2v.W2V_E_ARG),
                                    (1, 1000, 100, w2v.W2V_E_WORKSPACE)):
        p = w2v.Params(window=5, corpus_tokens=1000, arch=arch, sync_batch=64).c()
        steps = ctypes.c_int64(77)
        assert w2v.lib().w2v_train_batch_epoch(ctypes.byref(m), 0x80000, n, ctypes.byref(p), ctypes.byref(b), None,
                                               ctypes.byref(steps), None, None, 0x900000, ws_bytes, None) == code
        assert steps.value == 0
