"""MI355X hierarchical-softmax word2vec: Python binding of libw2v.so.

Argument marshalling only: every step runs in the library's HIP kernels.
PyTorch provides device memory and the current stream. The library never
allocates device memory; workspaces are torch uint8 tensors made here.

Entry points mirror the C ABI in include/w2v.h:
    build_vocab, build_huffman, train_hs_epoch, hs_loglik
    build_noise_table, train_ns_epoch, ns_objective (negative sampling)
    layer_norm, layer_norm_backward, hs_loss, AdamW (a mini-batch step on hidden vectors)
    gated_ffn, gated_ffn_backward, orthogonalize, Muon (a learned block of such a step, and its matrices' optimizer)
    train_batch_epoch, batch_loglik (CBOW in mini-batches with them)
plus the test hooks sample_pairs, keep_thresholds and sample_negatives.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass, field

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libw2v.so")

W2V_OK, W2V_E_ARG, W2V_E_RANGE, W2V_E_WORKSPACE, W2V_E_DEVICE = 0, -1, -2, -3, -4
N_STATS = 5
STAT_NAMES = ("raw_tokens", "in_vocab_tokens", "kept_centres", "pairs", "node_updates")

P = ctypes.c_void_p
I32, I64, U64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64


class W2VError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"w2v error {code}: {msg}")
        self.code = code


class CModel(ctypes.Structure):
    _fields_ = [("syn0", P), ("syn1", P), ("V", I32), ("dim", I32), ("row_stride", I32), ("reserved0", I32),
                ("vocab_counts", P), ("train_words", I64), ("codelen", P), ("code", P), ("point_off", P),
                ("points", P)]


class CParams(ctypes.Structure):
    _fields_ = [("arch", I32), ("mode", I32), ("window", I32), ("doc_len", I32), ("sample", ctypes.c_double),
                ("alpha0", ctypes.c_float), ("epoch", I32), ("n_epochs", I32), ("reserved1", I32),
                ("corpus_tokens", I64), ("first_raw_index", I64), ("seed", U64), ("cache_k", I32),
                ("flush_every", I32), ("sync_batch", I32), ("workers", I32), ("write_policy", I32),
                ("flush_policy", I32), ("hot_k", I32), ("negative", I32), ("cache_mode", I32),
                ("span_refresh", I32), ("span_stash", I32), ("stash_from", I32)]


class CAdamWTensor(ctypes.Structure):
    _fields_ = [("param", P), ("grad", P), ("rows", I64), ("cols", I64), ("param_stride", I64), ("grad_stride", I64),
                ("moment_offset", I64), ("param_type", I32), ("grad_type", I32), ("weight_decay", ctypes.c_float),
                ("reserved0", I32)]


class CAdamWParams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", I64), ("lr_device", P), ("step_device", P),
                ("grad_scale", ctypes.c_float), ("seed", ctypes.c_uint32)]


class CBatchParams(ctypes.Structure):
    _fields_ = [("gain", P), ("bias", P), ("m", P), ("v", P), ("m_scale", P), ("v_scale", P),
                ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double), ("step0", I64),
                ("norm_eps", ctypes.c_float), ("weight_decay", ctypes.c_float), ("bits", I32), ("max_code_len", I32),
                ("seed", ctypes.c_uint32), ("reserved0", I32)]


class CRows(ctypes.Structure):
    _fields_ = [("p", P), ("stride", I64)]


class CMuonMatrix(ctypes.Structure):
    _fields_ = [("param", P), ("grad", P), ("rows", I64), ("cols", I64), ("param_stride", I64), ("grad_stride", I64),
                ("moment_offset", I64), ("param_type", I32), ("grad_type", I32), ("weight_decay", ctypes.c_float),
                ("scale", ctypes.c_float)]


class CMuonParams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("momentum", ctypes.c_double), ("eps", ctypes.c_double), ("lr_device", P),
                ("grad_scale", ctypes.c_float), ("nesterov", I32), ("steps", I32), ("reserved0", I32)]


assert ctypes.sizeof(CRows) == 16 and ctypes.sizeof(CMuonMatrix) == 72 and ctypes.sizeof(CMuonParams) == 48
assert ctypes.sizeof(CBatchParams) == 104
assert ctypes.sizeof(CModel) == 80 and ctypes.sizeof(CParams) == 112
assert ctypes.sizeof(CAdamWTensor) == 72 and ctypes.sizeof(CAdamWParams) == 64

_LIB = None


def lib() -> ctypes.CDLL:
    """The loaded libw2v.so; raises if it has not been built."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "(there is no fallback implementation)")
        L = ctypes.CDLL(LIB_PATH)
        L.w2v_last_error.restype = ctypes.c_char_p
        L.w2v_last_error.argtypes = []
        L.w2v_build_vocab_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_build_vocab_workspace_bytes.argtypes = [I32]
        L.w2v_build_vocab.restype = ctypes.c_int
        L.w2v_build_vocab.argtypes = [P, I64, I32, I64, P, P, P, P, P, P, P, P, ctypes.c_size_t, P]
        L.w2v_build_huffman_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_build_huffman_workspace_bytes.argtypes = [I32]
        L.w2v_build_huffman.restype = ctypes.c_int
        L.w2v_build_huffman.argtypes = [P, I32, P, P, P, P, I64, P, P, P, ctypes.c_size_t, P]
        L.w2v_train_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_train_workspace_bytes.argtypes = [ctypes.POINTER(CModel), I64, ctypes.POINTER(CParams)]
        L.w2v_train_hs_epoch.restype = ctypes.c_int
        L.w2v_train_hs_epoch.argtypes = [ctypes.POINTER(CModel), P, I64, ctypes.POINTER(CParams), P, P,
                                         ctypes.c_size_t, P]
        L.w2v_last_train_kernel_ms.restype = ctypes.c_int
        L.w2v_last_train_kernel_ms.argtypes = [ctypes.POINTER(ctypes.c_float)]
        L.w2v_train_word_span.restype = I32
        L.w2v_train_word_span.argtypes = [ctypes.POINTER(CModel), ctypes.POINTER(CParams)]
        L.w2v_last_train_launch.restype = ctypes.c_int
        L.w2v_last_train_launch.argtypes = [ctypes.POINTER(I32), ctypes.POINTER(I32)]
        L.w2v_hs_loglik_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_hs_loglik_workspace_bytes.argtypes = [ctypes.POINTER(CModel), I64, ctypes.POINTER(CParams)]
        L.w2v_hs_loglik.restype = ctypes.c_int
        L.w2v_hs_loglik.argtypes = [ctypes.POINTER(CModel), P, I64, ctypes.POINTER(CParams), P, P, P, P,
                                    ctypes.c_size_t, P]
        L.w2v_sample_pairs_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_sample_pairs_workspace_bytes.argtypes = [I32, I64, ctypes.POINTER(CParams)]
        L.w2v_sample_pairs.restype = ctypes.c_int
        L.w2v_sample_pairs.argtypes = [P, I64, I32, P, I64, ctypes.POINTER(CParams), P, P, I64, P, P, P, P, P,
                                       ctypes.c_size_t, P]
        L.w2v_keep_thresholds.restype = ctypes.c_int
        L.w2v_keep_thresholds.argtypes = [P, I32, ctypes.c_double, I64, P, P]
        L.w2v_noise_table_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_noise_table_workspace_bytes.argtypes = [I32]
        L.w2v_build_noise_table.restype = ctypes.c_int
        L.w2v_build_noise_table.argtypes = [P, I32, I32, P, P, P, ctypes.c_size_t, P]
        L.w2v_train_ns_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_train_ns_workspace_bytes.argtypes = [ctypes.POINTER(CModel), I64, ctypes.POINTER(CParams)]
        L.w2v_train_ns_epoch.restype = ctypes.c_int
        L.w2v_train_ns_epoch.argtypes = [ctypes.POINTER(CModel), P, I32, P, I64, ctypes.POINTER(CParams), P, P,
                                         ctypes.c_size_t, P]
        L.w2v_ns_objective_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_ns_objective_workspace_bytes.argtypes = [ctypes.POINTER(CModel), I64, ctypes.POINTER(CParams)]
        L.w2v_ns_objective.restype = ctypes.c_int
        L.w2v_ns_objective.argtypes = [ctypes.POINTER(CModel), P, I32, P, I64, ctypes.POINTER(CParams), P, P, P, P,
                                       ctypes.c_size_t, P]
        L.w2v_noalloc_scratch_bytes.restype = ctypes.c_size_t
        L.w2v_noalloc_scratch_bytes.argtypes = []
        L.w2v_hs_loglik_noalloc.restype = ctypes.c_int
        L.w2v_hs_loglik_noalloc.argtypes = [ctypes.POINTER(CModel), P, I64, ctypes.POINTER(CParams), P, P, P, P]
        L.w2v_sample_negatives_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_sample_negatives_workspace_bytes.argtypes = [I32, I64, ctypes.POINTER(CParams)]
        L.w2v_sample_negatives.restype = ctypes.c_int
        L.w2v_sample_negatives.argtypes = [P, I64, I32, P, I64, ctypes.POINTER(CParams), P, I32, P, I64, P, P, P,
                                           ctypes.c_size_t, P]
        L.w2v_layer_norm.restype = ctypes.c_int
        L.w2v_layer_norm.argtypes = [P, I32, I64, I32, I64, P, P, I32, ctypes.c_float, P, I64, P, P, P]
        L.w2v_layer_norm_backward_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_layer_norm_backward_workspace_bytes.argtypes = [I64, I32]
        L.w2v_layer_norm_backward.restype = ctypes.c_int
        L.w2v_layer_norm_backward.argtypes = [P, I64, P, I32, I64, I32, I64, P, I32, P, P, P, I64, P, P, P,
                                              ctypes.c_size_t, P]
        L.w2v_hs_loss_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_hs_loss_workspace_bytes.argtypes = [ctypes.POINTER(CModel), I32, I64]
        L.w2v_hs_loss.restype = ctypes.c_int
        L.w2v_hs_loss.argtypes = [ctypes.POINTER(CModel), I32, P, I32, I64, I64, P, P, P, P, I64, P, I64, P,
                                  ctypes.c_size_t, P]
        L.w2v_adamw_plan_bytes.restype = ctypes.c_size_t
        L.w2v_adamw_plan_bytes.argtypes = [ctypes.POINTER(CAdamWTensor), I32]
        L.w2v_adamw_build_plan.restype = ctypes.c_int
        L.w2v_adamw_build_plan.argtypes = [ctypes.POINTER(CAdamWTensor), I32, I64, P, ctypes.c_size_t, P, P]
        L.w2v_adamw_step.restype = ctypes.c_int
        L.w2v_adamw_step.argtypes = [P, I64, I32, P, P, P, P, ctypes.POINTER(CAdamWParams), P]
        L.w2v_adamw_moments.restype = ctypes.c_int
        L.w2v_adamw_moments.argtypes = [P, P, P, P, I64, P, P, P]
        batch = [ctypes.POINTER(CModel), I64, ctypes.POINTER(CParams), ctypes.POINTER(CBatchParams)]
        L.w2v_batch_n_moments.restype = I64
        L.w2v_batch_n_moments.argtypes = [ctypes.POINTER(CModel), ctypes.POINTER(CBatchParams)]
        L.w2v_train_batch_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_train_batch_workspace_bytes.argtypes = batch
        L.w2v_train_batch_epoch.restype = ctypes.c_int
        L.w2v_train_batch_epoch.argtypes = [ctypes.POINTER(CModel), P, I64, ctypes.POINTER(CParams),
                                            ctypes.POINTER(CBatchParams), P, P, P, P, P, ctypes.c_size_t, P]
        L.w2v_batch_loglik_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_batch_loglik_workspace_bytes.argtypes = batch
        L.w2v_batch_loglik.restype = ctypes.c_int
        L.w2v_batch_loglik.argtypes = [ctypes.POINTER(CModel), P, I64, ctypes.POINTER(CParams),
                                       ctypes.POINTER(CBatchParams), P, P, P, ctypes.c_size_t, P]
        for name in ("w2v_gated_ffn", "w2v_gated_ffn_backward"):
            size = getattr(L, name + "_workspace_bytes")
            size.restype, size.argtypes = ctypes.c_size_t, [I64, I32, I32, I32]
        L.w2v_gated_ffn.restype = ctypes.c_int
        L.w2v_gated_ffn.argtypes = [CRows] * 4 + [I64, I32, I32, I32, I32] + [CRows] * 3 + [P, ctypes.c_size_t, P]
        L.w2v_gated_ffn_backward.restype = ctypes.c_int
        L.w2v_gated_ffn_backward.argtypes = [CRows] * 7 + [I64, I32, I32, I32, I32] + [CRows] * 4 + [P, ctypes.c_size_t, P]
        L.w2v_orthogonalize_workspace_bytes.restype = ctypes.c_size_t
        L.w2v_orthogonalize_workspace_bytes.argtypes = [I64, I32, I32, I32]
        L.w2v_orthogonalize.restype = ctypes.c_int
        L.w2v_orthogonalize.argtypes = [P, I64, I64, I64, I32, I32, I32, I32, ctypes.c_double, P, I64, I64, P,
                                        ctypes.c_size_t, P]
        for name in ("w2v_muon_plan_bytes", "w2v_muon_workspace_bytes"):
            getattr(L, name).restype, getattr(L, name).argtypes = ctypes.c_size_t, [ctypes.POINTER(CMuonMatrix), I32]
        L.w2v_muon_build_plan.restype = ctypes.c_int
        L.w2v_muon_build_plan.argtypes = [ctypes.POINTER(CMuonMatrix), I32, I64, P, ctypes.c_size_t, P]
        L.w2v_muon_step.restype = ctypes.c_int
        L.w2v_muon_step.argtypes = [ctypes.POINTER(CMuonMatrix), I32, P, P, ctypes.POINTER(CMuonParams), P,
                                    ctypes.c_size_t, P]
        _LIB = L
    return _LIB


def last_error() -> str:
    return lib().w2v_last_error().decode()


def _check(rc: int):
    if rc != W2V_OK:
        raise W2VError(rc, last_error())


def _dev_ptr(t: torch.Tensor | None, dtype: torch.dtype, name: str):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream(device: torch.device | None = None) -> int:
    if device is None or device.index is None:
        return torch.cuda.current_stream(device).cuda_stream
    return torch._C._cuda_getCurrentRawStream(device.index)   # the same without a Stream object: 0.1 us, not 1.7


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


# ---------------------------------------------------------------- vocabulary
@dataclass
class Vocab:
    counts_by_id: torch.Tensor   # int64[id_space]
    vocab_ids: torch.Tensor      # int32[V]
    vocab_counts: torch.Tensor   # int64[V]
    id_to_vocab: torch.Tensor    # int32[id_space]
    V: int
    train_words: int
    tokens: torch.Tensor | None  # int32[n] vocabulary indices (-1 = dropped)


def build_vocab(tokens: torch.Tensor, id_space: int, min_count: int = 5, remap: bool = True) -> Vocab:
    """Count ids, keep count >= min_count, order by (count desc, id asc); optionally remap tokens."""
    dev = tokens.device
    n = tokens.numel()
    counts = torch.empty(id_space, dtype=torch.int64, device=dev)
    ids = torch.empty(id_space, dtype=torch.int32, device=dev)
    vc = torch.empty(id_space, dtype=torch.int64, device=dev)
    i2v = torch.empty(id_space, dtype=torch.int32, device=dev)
    out = torch.empty(n, dtype=torch.int32, device=dev) if remap else None
    ws = _workspace(lib().w2v_build_vocab_workspace_bytes(id_space), dev)
    V = ctypes.c_int32(0)
    tw = ctypes.c_int64(0)
    _check(lib().w2v_build_vocab(_dev_ptr(tokens, torch.int32, "tokens"), n, id_space, min_count,
                                 counts.data_ptr(), ids.data_ptr(), vc.data_ptr(), i2v.data_ptr(),
                                 out.data_ptr() if out is not None else None, ctypes.byref(V), ctypes.byref(tw),
                                 ws.data_ptr(), ws.numel(), _stream(dev)))
    v = V.value
    return Vocab(counts, ids[:v], vc[:v], i2v, v, tw.value, out)


# ---------------------------------------------------------------- Huffman
@dataclass
class Tree:
    codelen: torch.Tensor    # uint8[V]
    code: torch.Tensor       # int64[V] (bit patterns of uint64)
    point_off: torch.Tensor  # int32[V+1]
    points: torch.Tensor     # int32[sum len]
    max_len: int


def build_huffman(vocab_counts: torch.Tensor) -> Tree:
    dev = vocab_counts.device
    V = vocab_counts.numel()
    vc = vocab_counts.contiguous()
    codelen = torch.empty(V, dtype=torch.uint8, device=dev)
    code = torch.empty(V, dtype=torch.int64, device=dev)
    off = torch.empty(V + 1, dtype=torch.int32, device=dev)
    ws = _workspace(lib().w2v_build_huffman_workspace_bytes(V), dev)
    plen = ctypes.c_int64(0)
    mlen = ctypes.c_int32(0)
    # codes are at most 64 long: one call with a buffer of that bound builds the tree once
    points = torch.empty(max(V * min(64, V - 1), 1), dtype=torch.int32, device=dev)
    _check(lib().w2v_build_huffman(_dev_ptr(vc, torch.int64, "vocab_counts"), V, codelen.data_ptr(),
                                   code.data_ptr(), off.data_ptr(), points.data_ptr(), points.numel(),
                                   ctypes.byref(plen), ctypes.byref(mlen), ws.data_ptr(), ws.numel(), _stream(dev)))
    return Tree(codelen, code, off, points[:plen.value], mlen.value)


# ---------------------------------------------------------------- model
def padded_stride(dim: int) -> int:
    """Row stride in floats: dim rounded up to 32 (128-byte rows)."""
    return (dim + 31) // 32 * 32


@dataclass
class Model:
    syn0: torch.Tensor          # float32[V, stride]
    syn1: torch.Tensor          # float32[V-1, stride]
    dim: int
    vocab_counts: torch.Tensor  # int64[V]
    train_words: int
    tree: Tree

    @property
    def V(self) -> int:
        return self.syn0.shape[0]

    @property
    def stride(self) -> int:
        return self.syn0.shape[1]

    def c(self) -> CModel:
        for name, t in (("syn0", self.syn0), ("syn1", self.syn1)):
            _dev_ptr(t, torch.float32, name)
        tr = self.tree
        return CModel(self.syn0.data_ptr(), self.syn1.data_ptr(), self.V, self.dim, self.stride, 0,
                      _dev_ptr(self.vocab_counts, torch.int64, "vocab_counts"), self.train_words,
                      tr.codelen.data_ptr() if tr else None, tr.code.data_ptr() if tr else None,
                      tr.point_off.data_ptr() if tr else None, tr.points.data_ptr() if tr else None)

    def vectors(self) -> tuple[torch.Tensor, torch.Tensor]:
        """(syn0[:, :dim], syn1[:, :dim]) views."""
        return self.syn0[:, :self.dim], self.syn1[:, :self.dim]


def make_model(syn0_init, syn1_init, vocab: Vocab, tree: Tree, device="cuda", stride: int | None = None,
               pad_value: float = 0.0) -> Model:
    """Copy [V, dim] initial weights (numpy or torch) into device rows of `stride` floats (default
    padded_stride(dim)); the padding columns hold pad_value."""
    s0 = torch.as_tensor(syn0_init, dtype=torch.float32)
    s1 = torch.as_tensor(syn1_init, dtype=torch.float32)
    V, dim = s0.shape
    stride = padded_stride(dim) if stride is None else stride
    syn0 = torch.full((V, stride), pad_value, dtype=torch.float32, device=device)
    syn1 = torch.full((max(V - 1, 1), stride), pad_value, dtype=torch.float32, device=device)
    syn0[:, :dim].copy_(s0)
    syn1[:V - 1, :dim].copy_(s1)
    return Model(syn0, syn1, dim, vocab.vocab_counts.contiguous(), vocab.train_words, tree)


# CBOW applies one update per node and centre, so its row stores lose more of
# the contended upper nodes' changes than skip-gram's; by default those rows
# take atomic adds there -- except with the word-row span (write_policy bit 3),
# where the stored rows measured both faster and no worse (1e8 tokens, d = 300:
# 254 instead of 488 ms, held-out CBOW objective -10.066 instead of -10.096).
HOT_K_CBOW = 1024


@dataclass
class Params:
    """Fields of w2v_params (include/w2v.h). hot_k=None picks 0 for skip-gram
    and HOT_K_CBOW for CBOW (0 for CBOW with the word-row span, write_policy bit 3)."""
    window: int
    sample: float = 0.0
    alpha0: float = 0.025
    arch: int = 0
    mode: int = 0
    doc_len: int = 1000
    epoch: int = 0
    n_epochs: int = 1
    corpus_tokens: int = 0
    first_raw_index: int = 0
    seed: int = 3
    cache_k: int = 31
    flush_every: int = 1000
    sync_batch: int = 4096
    workers: int = 0
    write_policy: int = 5
    flush_policy: int = 1
    hot_k: int | None = None
    negative: int = 5
    cache_mode: int = 0
    span_refresh: int = 0
    span_stash: int = 0
    stash_from: int = 0
    extra: dict = field(default_factory=dict)

    def c(self) -> CParams:
        return CParams(self.arch, self.mode, self.window, self.doc_len, float(self.sample), float(self.alpha0),
                       self.epoch, self.n_epochs, 0, self.corpus_tokens, self.first_raw_index, self.seed,
                       self.cache_k, self.flush_every, self.sync_batch, self.workers, self.write_policy,
                       self.flush_policy, self.resolved_hot_k(), self.negative, self.cache_mode, self.span_refresh,
                       self.span_stash, self.stash_from)

    def resolved_hot_k(self) -> int:
        if self.hot_k is not None:
            return self.hot_k
        return HOT_K_CBOW if self.arch == 1 and not (self.write_policy & 8) else 0


# ---------------------------------------------------------------- training
def train_hs_epoch(model: Model, tokens: torch.Tensor, p: Params, stats: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None) -> torch.Tensor:
    """One pass over tokens (vocabulary indices). Returns the device stats tensor int64[5]; does not sync."""
    dev = tokens.device
    cm, cp = model.c(), p.c()
    if cp.corpus_tokens <= 0:
        cp.corpus_tokens = tokens.numel()
    need = lib().w2v_train_workspace_bytes(ctypes.byref(cm), tokens.numel(), ctypes.byref(cp))
    if workspace is None or workspace.numel() < need:
        workspace = _workspace(need, dev)
    if stats is None:
        stats = torch.zeros(N_STATS, dtype=torch.int64, device=dev)
    _check(lib().w2v_train_hs_epoch(ctypes.byref(cm), _dev_ptr(tokens, torch.int32, "tokens"), tokens.numel(),
                                    ctypes.byref(cp), _dev_ptr(stats, torch.int64, "stats"), workspace.data_ptr(),
                                    workspace.numel(), _stream(dev)))
    return stats


def train_workspace_bytes(model: Model, n_tokens: int, p: Params) -> int:
    cm, cp = model.c(), p.c()
    if cp.corpus_tokens <= 0:
        cp.corpus_tokens = n_tokens
    return int(lib().w2v_train_workspace_bytes(ctypes.byref(cm), n_tokens, ctypes.byref(cp)))


def train_word_span(model: Model, p: Params) -> int:
    """Half-width of the word-row span kept in registers across centres for these settings (0: none)."""
    cm, cp = model.c(), p.c()
    if cp.corpus_tokens <= 0:
        cp.corpus_tokens = 1
    h = int(lib().w2v_train_word_span(ctypes.byref(cm), ctypes.byref(cp)))
    if h < 0:
        raise W2VError(W2V_E_ARG, last_error())
    return h


def last_train_kernel_ms() -> float:
    ms = ctypes.c_float(0)
    _check(lib().w2v_last_train_kernel_ms(ctypes.byref(ms)))
    return float(ms.value)


def last_train_launch() -> tuple[int, int]:
    """(workgroups, wavefronts) of the last asynchronous training launch."""
    g = ctypes.c_int32(0)
    wv = ctypes.c_int32(0)
    _check(lib().w2v_last_train_launch(ctypes.byref(g), ctypes.byref(wv)))
    return g.value, wv.value


def last_train_resources() -> dict:
    """LDS bytes per workgroup, VGPRs per lane and wavefronts per SIMD of the last asynchronous training
    launch."""
    lds, vg, occ = ctypes.c_int32(0), ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().w2v_last_train_resources(ctypes.byref(lds), ctypes.byref(vg), ctypes.byref(occ)))
    return {"lds_bytes_per_workgroup": lds.value, "vgprs": vg.value, "waves_per_simd": occ.value}


def hs_loglik(model: Model, tokens: torch.Tensor, p: Params):
    """(sum of the held-out objective, n_terms, n_nodes). Synchronises.

    p.arch 0/2: log P(v|w) summed over the sampler's pairs; p.arch 1 (CBOW):
    log P(v|h) summed over the sampled centres with a window, h = the mean of
    the window words' vectors.
    """
    dev = tokens.device
    cm, cp = model.c(), p.c()
    ws = _workspace(lib().w2v_hs_loglik_workspace_bytes(ctypes.byref(cm), tokens.numel(), ctypes.byref(cp)), dev)
    s = ctypes.c_double(0)
    npairs = ctypes.c_int64(0)
    nn = ctypes.c_int64(0)
    _check(lib().w2v_hs_loglik(ctypes.byref(cm), _dev_ptr(tokens, torch.int32, "tokens"), tokens.numel(),
                               ctypes.byref(cp), ctypes.byref(s), ctypes.byref(npairs), ctypes.byref(nn),
                               ws.data_ptr(), ws.numel(), _stream(dev)))
    return s.value, npairs.value, nn.value


def hs_loglik_noalloc(model: Model, tokens: torch.Tensor, p: Params):
    """hs_loglik on the library's static scratch (no workspace is allocated). Synchronises."""
    dev = tokens.device
    cm, cp = model.c(), p.c()
    s = ctypes.c_double(0)
    npairs = ctypes.c_int64(0)
    nn = ctypes.c_int64(0)
    _check(lib().w2v_hs_loglik_noalloc(ctypes.byref(cm), _dev_ptr(tokens, torch.int32, "tokens"), tokens.numel(),
                                       ctypes.byref(cp), ctypes.byref(s), ctypes.byref(npairs), ctypes.byref(nn),
                                       _stream(dev)))
    return s.value, npairs.value, nn.value


# ---------------------------------------------------------------- test hooks
@dataclass
class Pairs:
    centre: torch.Tensor | None
    context: torch.Tensor | None
    total: int
    n_kept: int
    checksum: int
    keep_mask: torch.Tensor | None


def sample_pairs(tokens: torch.Tensor, V: int, vocab_counts: torch.Tensor, train_words: int, p: Params,
                 cap: int = 0, want_mask: bool = False) -> Pairs:
    dev = tokens.device
    cp = p.c()
    n = tokens.numel()
    ws = _workspace(lib().w2v_sample_pairs_workspace_bytes(V, n, ctypes.byref(cp)), dev)
    c = torch.empty(max(cap, 1), dtype=torch.int64, device=dev)
    x = torch.empty(max(cap, 1), dtype=torch.int64, device=dev)
    mask = torch.empty(max(n, 1), dtype=torch.uint8, device=dev) if want_mask else None
    npairs = ctypes.c_int64(0)
    nk = ctypes.c_int64(0)
    cs = ctypes.c_uint64(0)
    _check(lib().w2v_sample_pairs(_dev_ptr(tokens, torch.int32, "tokens"), n, V,
                                  _dev_ptr(vocab_counts, torch.int64, "vocab_counts"), train_words, ctypes.byref(cp),
                                  c.data_ptr() if cap else None, x.data_ptr() if cap else None, cap,
                                  mask.data_ptr() if mask is not None else None, ctypes.byref(npairs),
                                  ctypes.byref(nk), ctypes.byref(cs), ws.data_ptr(), ws.numel(), _stream(dev)))
    m = min(cap, npairs.value)
    return Pairs(c[:m] if cap else None, x[:m] if cap else None, npairs.value, nk.value, cs.value,
                 mask[:n] if mask is not None else None)


def keep_thresholds(vocab_counts: torch.Tensor, sample: float, train_words: int) -> torch.Tensor:
    V = vocab_counts.numel()
    thr = torch.empty(V, dtype=torch.int64, device=vocab_counts.device)
    _check(lib().w2v_keep_thresholds(_dev_ptr(vocab_counts, torch.int64, "vocab_counts"), V, float(sample),
                                     train_words, thr.data_ptr(), _stream(vocab_counts.device)))
    return thr


def kernel_source_hash() -> str:
    """First 16 hex digits of sha256 over the training kernel's sources (ties stored counter data to a build)."""
    import hashlib
    h = hashlib.sha256()
    for f in ("train.hip", "w2v_internal.h"):
        with open(os.path.join(os.path.dirname(os.path.abspath(__file__)), "csrc", f), "rb") as fh:
            h.update(fh.read())
    return h.hexdigest()[:16]


# ---------------------------------------------------------- negative sampling
@dataclass
class Noise:
    table: torch.Tensor   # int32[2^log2_size] vocabulary indices
    log2_size: int
    total_weight: int


def noise_log2_size(V: int) -> int:
    """A table of about 64 entries per word: 2^ceil(log2(64 V)), between 2^10 and 2^27."""
    return max(10, min(27, (64 * max(V, 1) - 1).bit_length()))


def build_noise_table(vocab_counts: torch.Tensor, log2_size: int | None = None) -> Noise:
    V = vocab_counts.numel()
    L = noise_log2_size(V) if log2_size is None else log2_size
    dev = vocab_counts.device
    table = torch.empty(1 << L, dtype=torch.int32, device=dev)
    ws = _workspace(lib().w2v_noise_table_workspace_bytes(V), dev)
    tot = ctypes.c_int64(0)
    _check(lib().w2v_build_noise_table(_dev_ptr(vocab_counts, torch.int64, "vocab_counts"), V, L, table.data_ptr(),
                                       ctypes.byref(tot), ws.data_ptr(), ws.numel(), _stream(dev)))
    return Noise(table, L, tot.value)


def make_ns_model(syn0_init, syn1_init, vocab: Vocab, device="cuda", stride: int | None = None,
                  pad_value: float = 0.0) -> Model:
    """[V, dim] input and output vectors in device rows of `stride` floats (default padded_stride(dim);
    padding columns hold pad_value), no tree."""
    s0 = torch.as_tensor(syn0_init, dtype=torch.float32)
    s1 = torch.as_tensor(syn1_init, dtype=torch.float32)
    V, dim = s0.shape
    if tuple(s1.shape) != (V, dim):
        raise ValueError("output vectors must be [V, dim]")
    stride = padded_stride(dim) if stride is None else stride
    syn0 = torch.full((V, stride), pad_value, dtype=torch.float32, device=device)
    syn1 = torch.full((V, stride), pad_value, dtype=torch.float32, device=device)
    syn0[:, :dim].copy_(s0)
    syn1[:, :dim].copy_(s1)
    return Model(syn0, syn1, dim, vocab.vocab_counts.contiguous(), vocab.train_words, None)


def train_ns_epoch(model: Model, noise: Noise, tokens: torch.Tensor, p: Params,
                   stats: torch.Tensor | None = None) -> torch.Tensor:
    """One pass of skip-gram with shared negatives. Returns the device stats int64[5]; does not sync."""
    dev = tokens.device
    cm, cp = model.c(), p.c()
    if cp.corpus_tokens <= 0:
        cp.corpus_tokens = tokens.numel()
    ws = _workspace(lib().w2v_train_ns_workspace_bytes(ctypes.byref(cm), tokens.numel(), ctypes.byref(cp)), dev)
    if stats is None:
        stats = torch.zeros(N_STATS, dtype=torch.int64, device=dev)
    _check(lib().w2v_train_ns_epoch(ctypes.byref(cm), _dev_ptr(noise.table, torch.int32, "noise table"),
                                    noise.log2_size, _dev_ptr(tokens, torch.int32, "tokens"), tokens.numel(),
                                    ctypes.byref(cp), _dev_ptr(stats, torch.int64, "stats"), ws.data_ptr(),
                                    ws.numel(), _stream(dev)))
    return stats


def ns_objective(model: Model, noise: Noise, tokens: torch.Tensor, p: Params):
    """(sum of the negative-sampling objective over the sampler's pairs, n_pairs, n_terms). Synchronises."""
    dev = tokens.device
    cm, cp = model.c(), p.c()
    ws = _workspace(lib().w2v_ns_objective_workspace_bytes(ctypes.byref(cm), tokens.numel(), ctypes.byref(cp)), dev)
    s = ctypes.c_double(0)
    npairs = ctypes.c_int64(0)
    nt = ctypes.c_int64(0)
    _check(lib().w2v_ns_objective(ctypes.byref(cm), _dev_ptr(noise.table, torch.int32, "noise table"),
                                  noise.log2_size, _dev_ptr(tokens, torch.int32, "tokens"), tokens.numel(),
                                  ctypes.byref(cp), ctypes.byref(s), ctypes.byref(npairs), ctypes.byref(nt),
                                  ws.data_ptr(), ws.numel(), _stream(dev)))
    return s.value, npairs.value, nt.value


@dataclass
class Negatives:
    negatives: torch.Tensor | None   # int32[min(cap, kept), K], -1 = dropped
    n_kept: int
    checksum: int


def sample_negatives(tokens: torch.Tensor, V: int, vocab_counts: torch.Tensor, train_words: int, p: Params,
                     noise: Noise, cap: int = 0) -> Negatives:
    dev = tokens.device
    cp = p.c()
    n = tokens.numel()
    ws = _workspace(lib().w2v_sample_negatives_workspace_bytes(V, n, ctypes.byref(cp)), dev)
    out = torch.empty(max(cap, 1) * p.negative, dtype=torch.int32, device=dev)
    nk = ctypes.c_int64(0)
    cs = ctypes.c_uint64(0)
    _check(lib().w2v_sample_negatives(_dev_ptr(tokens, torch.int32, "tokens"), n, V,
                                      _dev_ptr(vocab_counts, torch.int64, "vocab_counts"), train_words,
                                      ctypes.byref(cp), _dev_ptr(noise.table, torch.int32, "noise table"),
                                      noise.log2_size, out.data_ptr() if cap else None, cap, ctypes.byref(nk),
                                      ctypes.byref(cs), ws.data_ptr(), ws.numel(), _stream(dev)))
    m = min(cap, nk.value)
    return Negatives(out[:m * p.negative].view(m, p.negative) if cap else None, nk.value, cs.value)


# ---------------------------------------------------- a mini-batch step on hidden vectors
# These calls work on the tensors' memory and know nothing of autograd: a tensor that requires gradients is taken as its
# values, results carry no graph, and what is written in place (out, dx, parameters, moments) does not move autograd's
# version counters. A forward and its backward call are a user's autograd.Function's two halves.
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _type_of(t: torch.Tensor, name: str) -> int:
    if t.dtype not in _TYPES:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return _TYPES[t.dtype]


def _rows_ptr(t: torch.Tensor, name: str, like: torch.Tensor, dtype: torch.dtype | None = None) -> tuple[int, int]:
    """(pointer, row stride) of a [rows, dim] tensor of like's shape, device and (or dtype's) type."""
    if t.device != like.device or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor on the rows' device")
    if t.dtype != (dtype or like.dtype):
        raise ValueError(f"{name} must be {dtype or like.dtype}, got {t.dtype}")
    if t.dim() != 2 or t.shape != like.shape:
        raise ValueError(f"{name} must have the shape {tuple(like.shape)}, got {tuple(t.shape)}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return t.data_ptr(), t.stride(0)


def _vector_ptr(t: torch.Tensor | None, dtype: torch.dtype, n: int, dev: torch.device, name: str):
    if t is None:
        return None
    ptr = _dev_ptr(t, dtype, name)
    if t.device != dev or t.numel() != n:
        raise ValueError(f"{name} must hold {n} elements on {dev}, got {tuple(t.shape)} on {t.device}")
    return ptr


def _affine_ptr(t: torch.Tensor | None, x: torch.Tensor, name: str):
    if t is None:
        return None
    return _vector_ptr(t, torch.float32 if t.dtype == torch.float32 else x.dtype, x.shape[1], x.device, name)


class _On:
    """The current device for the time of a call (streams belong to a device, and launches go to the current one)."""

    def __init__(self, dev: torch.device):
        self.other = None if torch.cuda.current_device() == dev.index else torch.cuda.device(dev)

    def __enter__(self):
        if self.other:
            self.other.__enter__()

    def __exit__(self, *exc):
        if self.other:
            self.other.__exit__(*exc)


def _kept(workspace: torch.Tensor | None, need: int, dev: torch.device) -> torch.Tensor | None:
    """The caller's workspace, or a new one where there is none or it is too small."""
    if need == 0:
        return None
    if workspace is not None:
        _dev_ptr(workspace, torch.uint8, "workspace")
        if workspace.device != dev:
            raise ValueError(f"workspace must be on {dev}")
        if workspace.numel() >= need:
            return workspace
    return _workspace(need, dev)


def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None,
               eps: float = 1e-5, out: torch.Tensor | None = None
               ) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Rows of x [rows, dim] normalised: (y, mean, rstd), y in x's type (in out, which may be x), mean and rstd float32.
    weight and bias: float32 or x's type. y carries no autograd graph: layer_norm_backward takes the gradients. Does not
    sync."""
    xp, xs = _rows_ptr(x, "x", x)
    kind = _type_of(x, "x")
    y = torch.empty_like(x, memory_format=torch.contiguous_format) if out is None else out
    yp, ys = _rows_ptr(y, "out", x)
    wp, bp = _affine_ptr(weight, x, "weight"), _affine_ptr(bias, x, "bias")
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias must have the same type")
    w = weight if weight is not None else bias
    n, dim = x.shape
    stats = torch.empty(2, n, dtype=torch.float32, device=x.device)
    with _On(x.device):
        _check(lib().w2v_layer_norm(xp, kind, n, dim, xs, wp, bp, 0 if w is None else _TYPES[w.dtype], eps, yp, ys,
                                    stats.data_ptr(), stats.data_ptr() + 4 * n, _stream(x.device)))
    return y, *stats.unbind()


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor | None, mean: torch.Tensor,
                        rstd: torch.Tensor, dx: torch.Tensor | None = None, dweight: torch.Tensor | None = None,
                        dbias: torch.Tensor | None = None, workspace: torch.Tensor | None = None
                        ) -> tuple[torch.Tensor, torch.Tensor | None, torch.Tensor | None]:
    """Gradients (dx, dweight, dbias) of layer_norm for the upstream gradient dy, from its x, mean and rstd. dx in x's
    type (may be dy or x); dweight and dbias float32: new ones with a weight where neither is given, otherwise those that
    are given (None for the other). Does not sync."""
    xp, xs = _rows_ptr(x, "x", x)
    kind = _type_of(x, "x")
    dyp, dys = _rows_ptr(dy, "dy", x)
    n, dim = x.shape
    dev = x.device
    dx = torch.empty_like(x, memory_format=torch.contiguous_format) if dx is None else dx
    dxp, dxs = _rows_ptr(dx, "dx", x)
    if weight is not None and dweight is None and dbias is None:
        both = torch.empty(2, dim, dtype=torch.float32, device=dev)
        dweight, dbias = both.unbind()
    dwp = _vector_ptr(dweight, torch.float32, dim, dev, "dweight")
    dbp = _vector_ptr(dbias, torch.float32, dim, dev, "dbias")
    wp = _affine_ptr(weight, x, "weight")
    mp, rp = _vector_ptr(mean, torch.float32, n, dev, "mean"), _vector_ptr(rstd, torch.float32, n, dev, "rstd")
    need = lib().w2v_layer_norm_backward_workspace_bytes(n, dim) if dwp or dbp else 0
    with _On(dev):
        ws = _kept(workspace, need, dev)
        _check(lib().w2v_layer_norm_backward(dyp, dys, xp, kind, n, dim, xs, wp,
                                             0 if weight is None else _TYPES[weight.dtype], mp, rp, dxp, dxs, dwp, dbp,
                                             None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(),
                                             _stream(dev)))
    return dx, dweight, dbias


def _tree_of(model: Model) -> Tree:
    if model.tree is None:
        raise ValueError("the model has no Huffman tree")
    return model.tree


def hs_loss_workspace(model: Model, x: torch.Tensor, grads: bool = True) -> torch.Tensor | None:
    """A workspace for hs_loss on x's rows, to be kept from call to call (calls that overlap need one each)."""
    if not grads:
        return None
    cm = model.c()
    return _workspace(lib().w2v_hs_loss_workspace_bytes(ctypes.byref(cm), _tree_of(model).max_len, x.shape[0]), x.device)


def _own_gradient(model: Model) -> torch.Tensor:
    """Memory of syn1's shape for hs_loss, zeros where that writes none: in padding of 32 floats or more (shorter padding
    gets the kernels' zeros), and in rows that belong to no inner node."""
    d = torch.empty_like(model.syn1)
    if d.shape[1] != model.stride or model.stride - model.dim >= 32:
        d[:, model.dim:].zero_()
    if d.shape[0] != model.V - 1:
        d[model.V - 1:].zero_()
    return d


def hs_loss(model: Model, x: torch.Tensor, targets: torch.Tensor, weights: torch.Tensor | None = None,
            grads: bool = True, loss: torch.Tensor | None = None, dx: torch.Tensor | None = None,
            dsyn1: torch.Tensor | None = None, workspace: torch.Tensor | None = None
            ) -> tuple[torch.Tensor, torch.Tensor | None, torch.Tensor | None]:
    """(loss, dx, dsyn1): -log P(targets[i] | x[i]) under the model's hierarchical softmax (float32) and, with grads,
    the gradients of sum(weights * loss) for x [rows, dim] and for model.syn1 (dsyn1 float32 of syn1's shape, all rows
    written: their first dim columns, and zeros in padding of less than 32; a new dsyn1 has zeros in all its padding).
    targets int32, negative: none. The loss carries no autograd graph, whatever x requires: dx and dsyn1 are the gradients.
    Does not sync."""
    xp, xs = _rows_ptr(x, "x", x)
    kind, longest = _type_of(x, "x"), _tree_of(model).max_len
    n, dev = x.shape[0], x.device
    if x.shape[1] != model.dim:
        raise ValueError(f"x must have {model.dim} columns, got {x.shape[1]}")
    if model.syn1.device != dev:
        raise ValueError(f"the model must be on {dev}")
    tp = _vector_ptr(targets, torch.int32, n, dev, "targets")
    wp = _vector_ptr(weights, torch.float32, n, dev, "weights")
    if loss is None:
        loss = torch.empty(n, dtype=torch.float32, device=dev)
    dxp = dxs = dsp = None
    if grads:
        dx = torch.empty_like(x, memory_format=torch.contiguous_format) if dx is None else dx
        dxp, dxs = _rows_ptr(dx, "dx", x)
        dsyn1 = _own_gradient(model) if dsyn1 is None else dsyn1
        dsp, _ = _rows_ptr(dsyn1, "dsyn1", model.syn1)
    else:
        dx = dsyn1 = None
    cm = model.c()
    with _On(dev):
        ws = None
        if grads:
            ws = _kept(workspace, lib().w2v_hs_loss_workspace_bytes(ctypes.byref(cm), longest, n), dev)
        _check(lib().w2v_hs_loss(ctypes.byref(cm), longest, xp, kind, n, xs, tp, wp,
                                 _vector_ptr(loss, torch.float32, n, dev, "loss"), dxp, dxs or 0, dsp,
                                 dsyn1.stride(0) if grads else 0, None if ws is None else ws.data_ptr(),
                                 0 if ws is None else ws.numel(), _stream(dev)))
    return loss, dx, dsyn1


class AdamW:
    """AdamW over a list of tensors and their gradient buffers, updated in place by one launch a step.

    params, grads: float32, bfloat16 or float16 tensors of equal shapes, contiguous or 2-D with contiguous rows (views
    such as Model.vectors()). The buffers are fixed: write each step's gradients into `grads`. bits: of the moments, 32
    or 8. weight_decay: one number, or one for each tensor. A tensor's .grad is not looked at, and autograd does not see a
    step's writes.

    m and v hold all tensors' moments, tensor i's from offsets[i] on (multiples of 256): float32, or uint8 codes with the
    scales m_scale and v_scale (see include/w2v.h). state: those arrays of an earlier optimizer, (m, v) or
    (m, v, m_scale, v_scale), which are then used as they are; zeros otherwise."""

    BLOCK = 256

    def __init__(self, params, grads, bits: int = 32, betas: tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay=0.01, seed: int = 0, state=None):
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        if not params or len(params) != len(grads):
            raise ValueError("params and grads must be lists of the same length, at least 1")
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * len(params)
        if len(decay) != len(params):
            raise ValueError("weight_decay must be a number or hold one for each tensor")
        self.params, self.grads, self.bits, self.betas, self.eps, self.seed = (list(params), list(grads), bits, betas,
                                                                              eps, seed)
        self.device = dev = params[0].device
        self.offsets, at = [], 0
        table = (CAdamWTensor * len(params))()
        for i, (p, g) in enumerate(zip(params, grads)):
            for t, name in ((p, f"params[{i}]"), (g, f"grads[{i}]")):
                if not t.is_cuda or t.device != dev:
                    raise ValueError(f"{name} must be a GPU tensor on {dev}")
                if t.shape != p.shape:
                    raise ValueError(f"{name} must have the shape {tuple(p.shape)}, got {tuple(t.shape)}")
                if not (t.is_contiguous() or (t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1))):
                    raise ValueError(f"{name} must be contiguous, or 2-D with contiguous rows")
            rows, cols = (1, p.numel()) if p.is_contiguous() and g.is_contiguous() else p.shape
            table[i] = CAdamWTensor(p.data_ptr(), g.data_ptr(), rows, cols, p.stride(0) if rows > 1 else cols,
                                    g.stride(0) if rows > 1 else cols, at, _type_of(p, f"params[{i}]"),
                                    _type_of(g, f"grads[{i}]"), decay[i], 0)
            self.offsets.append(at)
            at += -(-p.numel() // self.BLOCK) * self.BLOCK
        self.n_moments = at
        kind = torch.float32 if bits == 32 else torch.uint8
        shapes = [(at, kind), (at, kind)] + [(at // self.BLOCK, torch.float32)] * (2 if bits == 8 else 0)
        if state is None:
            state = [torch.zeros(n, dtype=d, device=dev) for n, d in shapes]
        if len(state) != len(shapes):
            raise ValueError(f"state must hold {len(shapes)} arrays")
        for k, (t, (n, d)) in enumerate(zip(state, shapes)):
            _vector_ptr(t, d, n, dev, f"state[{k}]")
        self._state = (*state, None, None)[:4]
        self._buffers = [t.detach() for t in (*params, *grads)]   # the plan's memory stays, whatever becomes of the tensors
        self._plan = _workspace(lib().w2v_adamw_plan_bytes(table, len(params)), dev)
        chunks = ctypes.c_int64(0)
        with _On(dev):
            _check(lib().w2v_adamw_build_plan(table, len(params), at, self._plan.data_ptr(), self._plan.numel(),
                                              ctypes.byref(chunks), _stream(dev)))
        self._chunks = chunks.value

    m, v, m_scale, v_scale = (property(lambda self, k=k: self._state[k]) for k in range(4))

    def step(self, step, lr, grad_scale: float = 1.0) -> None:
        """Step number `step` (1, 2, ...) with the learning rate lr. Either may be a one-element tensor on the device
        (int64, float32) that is read when the step runs, so that a captured step can be replayed with new values. Does
        not sync."""
        p = CAdamWParams(0.0, self.betas[0], self.betas[1], self.eps, 1, None, None, grad_scale, self.seed & 0xFFFFFFFF)
        if isinstance(lr, torch.Tensor):
            p.lr_device = _vector_ptr(lr, torch.float32, 1, self.device, "lr")
        else:
            p.lr = lr
        if isinstance(step, torch.Tensor):
            p.step_device = _vector_ptr(step, torch.int64, 1, self.device, "step")
        else:
            p.step = step
        narrow = self.bits == 8
        with _On(self.device):
            _check(lib().w2v_adamw_step(self._plan.data_ptr(), self._chunks, self.bits, self.m.data_ptr(),
                                        self.v.data_ptr(), self.m_scale.data_ptr() if narrow else None,
                                        self.v_scale.data_ptr() if narrow else None, ctypes.byref(p),
                                        _stream(self.device)))

    def moments(self, m_out: torch.Tensor | None = None, v_out: torch.Tensor | None = None
                ) -> tuple[torch.Tensor, torch.Tensor]:
        """The moments' values, float32[n_moments] each: m and v themselves, or what the 8-bit codes stand for (in m_out
        and v_out). Does not sync."""
        if self.bits == 32:
            return self.m, self.v
        outs = [torch.empty(self.n_moments, dtype=torch.float32, device=self.device) if t is None else t
                for t in (m_out, v_out)]
        mp, vp = (_vector_ptr(t, torch.float32, self.n_moments, self.device, "m_out or v_out") for t in outs)
        with _On(self.device):
            _check(lib().w2v_adamw_moments(self.m.data_ptr(), self.v.data_ptr(), self.m_scale.data_ptr(),
                                           self.v_scale.data_ptr(), self.n_moments, mp, vp, _stream(self.device)))
        return outs[0], outs[1]


# ------------------------------------------------- a learned block of such a step, and its matrices' optimizer
def _with_workspace(workspace: torch.Tensor | None, size, dev: torch.device, call) -> None:
    """call(pointer, bytes) with the caller's workspace, or with a new one of size() bytes where there is none or it is too
    small (which the call says before it launches anything)."""
    with _On(dev):
        if workspace is not None:
            ptr = _dev_ptr(workspace, torch.uint8, "workspace")
            if workspace.device != dev:
                raise ValueError(f"workspace must be on {dev}")
            rc = call(ptr, workspace.numel())
            if rc != W2V_E_WORKSPACE:
                return _check(rc)
        ws = _workspace(size(), dev)
        _check(call(ws.data_ptr(), ws.numel()))


_ACTS = {"silu": 0, "gelu": 1}


def _matrix(t: torch.Tensor | None, shape: tuple[int, int], like: torch.Tensor, name: str) -> CRows:
    """A [rows, columns] tensor of like's type and device with contiguous rows; None: no array."""
    if t is None:
        return CRows(None, 0)
    if t.device != like.device or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor on x's device")
    if t.dtype != like.dtype:
        raise ValueError(f"{name} must be {like.dtype}, got {t.dtype}")
    if t.dim() != 2 or tuple(t.shape) != shape:
        raise ValueError(f"{name} must have the shape {shape}, got {tuple(t.shape)}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return CRows(t.data_ptr(), t.stride(0))


def _block_of(x: torch.Tensor, w_gate, w_up, w_down, act: str):
    """(rows, dim, hidden, type, act) and the arrays x and weights of a gated feed-forward block."""
    if x.dim() != 2 or w_gate.dim() != 2:
        raise ValueError("x and w_gate must have two dimensions")
    if act not in _ACTS:
        raise ValueError(f"act must be one of {', '.join(_ACTS)}")
    n, d, h = x.shape[0], x.shape[1], w_gate.shape[0]
    kind = _type_of(x, "x")
    return (n, d, h, kind, _ACTS[act]), (_matrix(x, (n, d), x, "x"), _matrix(w_gate, (h, d), x, "w_gate"),
                                         _matrix(w_up, (h, d), x, "w_up"), _matrix(w_down, (d, h), x, "w_down"))


def gated_ffn_workspace(x: torch.Tensor, hidden: int, grads: bool = False) -> torch.Tensor:
    """A workspace for gated_ffn (with grads: for gated_ffn_backward) on x's rows, to be kept from call to call (calls that
    overlap need one each)."""
    size = lib().w2v_gated_ffn_backward_workspace_bytes if grads else lib().w2v_gated_ffn_workspace_bytes
    return _workspace(size(x.shape[0], x.shape[1], hidden, _type_of(x, "x")), x.device)


def gated_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, act: str = "silu",
              save: bool = False, out: torch.Tensor | None = None, gate: torch.Tensor | None = None,
              up: torch.Tensor | None = None, workspace: torch.Tensor | None = None
              ) -> tuple[torch.Tensor, torch.Tensor | None, torch.Tensor | None]:
    """(y, gate, up) of y = (act(x w_gate') * (x w_up')) w_down' for rows x [rows, dim], weights [hidden, dim] twice and
    [dim, hidden], all of one type; act "silu" or "gelu". With save, gate and up [rows, hidden] hold the two products for
    gated_ffn_backward (None otherwise). y goes into out, which may be x; gate and up into those that are given. 16-bit
    tensors' act() * () is rounded to their type before it meets w_down, except in calls of few rows. y carries no autograd
    graph. Does not sync."""
    sizes, arrays = _block_of(x, w_gate, w_up, w_down, act)
    n, d, h = sizes[:3]
    y = torch.empty(n, d, dtype=x.dtype, device=x.device) if out is None else out
    if save:
        gate, up = (torch.empty(n, h, dtype=x.dtype, device=x.device) if t is None else t for t in (gate, up))
    elif gate is not None or up is not None:
        raise ValueError("gate and up are written with save only")
    outs = _matrix(y, (n, d), x, "out"), _matrix(gate, (n, h), x, "gate"), _matrix(up, (n, h), x, "up")
    _with_workspace(workspace, lambda: lib().w2v_gated_ffn_workspace_bytes(*sizes[:4]), x.device,
                    lambda ws, size: lib().w2v_gated_ffn(*arrays, *sizes, *outs, ws, size, _stream(x.device)))
    return y, gate, up


def gated_ffn_backward(dy: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                       gate: torch.Tensor, up: torch.Tensor, act: str = "silu", dx: torch.Tensor | None = None,
                       dw_gate: torch.Tensor | None = None, dw_up: torch.Tensor | None = None,
                       dw_down: torch.Tensor | None = None, workspace: torch.Tensor | None = None
                       ) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gradients (dx, dw_gate, dw_up, dw_down) of gated_ffn for the upstream gradient dy, from its x, its weights, and gate
    and up as it saved them; all of x's type. dx may be dy or x. Does not sync."""
    sizes, arrays = _block_of(x, w_gate, w_up, w_down, act)
    n, d, h = sizes[:3]
    ins = _matrix(dy, (n, d), x, "dy"), *arrays, _matrix(gate, (n, h), x, "gate"), _matrix(up, (n, h), x, "up")
    shapes = (n, d), (h, d), (h, d), (d, h)
    grads = [torch.empty(s, dtype=x.dtype, device=x.device) if t is None else t
             for t, s in zip((dx, dw_gate, dw_up, dw_down), shapes)]
    outs = [_matrix(t, s, x, name) for t, s, name in zip(grads, shapes, ("dx", "dw_gate", "dw_up", "dw_down"))]
    _with_workspace(workspace, lambda: lib().w2v_gated_ffn_backward_workspace_bytes(*sizes[:4]), x.device,
                    lambda ws, size: lib().w2v_gated_ffn_backward(*ins, *sizes, *outs, ws, size, _stream(x.device)))
    return tuple(grads)


def _stack_of(t: torch.Tensor, name: str, like: torch.Tensor) -> tuple[int, int, int]:
    """(pointer, row stride, matrix stride) of a matrix, or a stack of them, of like's shape, type and device."""
    if t.device != like.device or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor on g's device")
    if t.dtype != like.dtype or t.shape != like.shape or t.dim() not in (2, 3):
        raise ValueError(f"{name} must be {like.dtype} of the shape {tuple(like.shape)}, of two or three dimensions")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return t.data_ptr(), t.stride(-2), t.stride(0) if t.dim() == 3 else 0


def orthogonalize_workspace(g: torch.Tensor) -> torch.Tensor:
    """A workspace for orthogonalize on matrices of g's shape, to be kept from call to call (calls that overlap need one
    each)."""
    return _workspace(lib().w2v_orthogonalize_workspace_bytes(g.shape[0] if g.dim() == 3 else 1, *g.shape[-2:],
                                                              _type_of(g, "g")), g.device)


def orthogonalize(g: torch.Tensor, steps: int = 5, eps: float = 1e-7, out: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None) -> torch.Tensor:
    """The matrix g [rows, cols], or each of a stack [count, rows, cols], with its singular values brought near one by
    `steps` Newton-Schulz steps from g over its Frobenius norm plus eps; in g's type, in out, which may be g. Does not
    sync."""
    gp = _stack_of(g, "g", g)
    kind = _type_of(g, "g")
    out = torch.empty_like(g, memory_format=torch.contiguous_format) if out is None else out
    op = _stack_of(out, "out", g)
    sizes = g.shape[0] if g.dim() == 3 else 1, *g.shape[-2:], kind
    _with_workspace(workspace, lambda: lib().w2v_orthogonalize_workspace_bytes(*sizes), g.device,
                    lambda ws, size: lib().w2v_orthogonalize(*gp, *sizes, steps, eps, *op, ws, size, _stream(g.device)))
    return out


class Muon:
    """Muon over a list of matrices and their gradient buffers, updated in place: momentum, then an update orthogonalised by
    Newton-Schulz products. AdamW is for the other tensors.

    params, grads: 2-D float32, bfloat16 or float16 tensors of equal shapes with contiguous rows. The buffers are fixed:
    write each step's gradients into `grads`. weight_decay: one number, or one for each matrix. scale: what an
    orthogonalised update is multiplied with beside the learning rate, one number or one for each matrix; None takes
    sqrt(max(1, rows / cols)). A tensor's .grad is not looked at, and autograd does not see a step's writes. One step at a
    time: the workspace belongs to the optimizer.

    m holds all matrices' momenta, matrix i's from offsets[i] on (multiples of 256), float32. state: that array of an
    earlier optimizer, which is then used as it is; zeros otherwise."""

    BLOCK = 256

    def __init__(self, params, grads, momentum: float = 0.95, nesterov: bool = True, steps: int = 5, eps: float = 1e-7,
                 weight_decay=0.0, scale=None, state: torch.Tensor | None = None):
        if not params or len(params) != len(grads):
            raise ValueError("params and grads must be lists of the same length, at least 1")
        lists = []
        for name, v in (("weight_decay", weight_decay), ("scale", scale)):
            lists.append(list(v) if isinstance(v, (list, tuple)) else [v] * len(params))
            if len(lists[-1]) != len(params):
                raise ValueError(f"{name} must be a number or hold one for each matrix")
        self.params, self.grads, self.momentum, self.nesterov, self.steps, self.eps = (list(params), list(grads), momentum,
                                                                                       nesterov, steps, eps)
        self.device = dev = params[0].device
        self.offsets, at = [], 0
        self._table = table = (CMuonMatrix * len(params))()
        for i, (p, g, decay, factor) in enumerate(zip(params, grads, *lists)):
            for t, name in ((p, f"params[{i}]"), (g, f"grads[{i}]")):
                if not t.is_cuda or t.device != dev:
                    raise ValueError(f"{name} must be a GPU tensor on {dev}")
                if t.dim() != 2 or t.shape != p.shape:
                    raise ValueError(f"{name} must have two dimensions and the shape {tuple(p.shape)}, got {tuple(t.shape)}")
                if t.shape[1] > 1 and t.stride(1) != 1:
                    raise ValueError(f"{name}'s rows must be contiguous")
            rows, cols = p.shape
            if factor is None:
                factor = max(1.0, rows / max(1, cols)) ** 0.5
            table[i] = CMuonMatrix(p.data_ptr(), g.data_ptr(), rows, cols, p.stride(0), g.stride(0), at,
                                   _type_of(p, f"params[{i}]"), _type_of(g, f"grads[{i}]"), decay, factor)
            self.offsets.append(at)
            at += -(-p.numel() // self.BLOCK) * self.BLOCK
        self.n_moments = at
        self.m = torch.zeros(at, dtype=torch.float32, device=dev) if state is None else state
        self._m_ptr = _vector_ptr(self.m, torch.float32, at, dev, "state")
        self._buffers = [t.detach() for t in (*params, *grads, self.m)]   # their memory stays, whatever becomes of the tensors
        n = len(params)
        self._plan = _workspace(lib().w2v_muon_plan_bytes(table, n), dev)
        self._workspace = _workspace(lib().w2v_muon_workspace_bytes(table, n), dev)
        with _On(dev):
            _check(lib().w2v_muon_build_plan(table, n, at, self._plan.data_ptr(), self._plan.numel(), _stream(dev)))

    def step(self, lr, grad_scale: float = 1.0) -> None:
        """One step with the learning rate lr, which may be a one-element float32 tensor on the device that is read when the
        step runs, so that a captured step can be replayed with new values. Does not sync."""
        p = CMuonParams(0.0, self.momentum, self.eps, None, grad_scale, int(self.nesterov), self.steps, 0)
        if isinstance(lr, torch.Tensor):
            p.lr_device = _vector_ptr(lr, torch.float32, 1, self.device, "lr")
        else:
            p.lr = lr
        with _On(self.device):
            _check(lib().w2v_muon_step(self._table, len(self._table), self._plan.data_ptr(), self._m_ptr, ctypes.byref(p),
                                       self._workspace.data_ptr(), self._workspace.numel(), _stream(self.device)))


# ------------------------------------------------------------- training in mini-batches
class BatchState:
    """What train_batch_epoch keeps beside the model: the layer norm's gain and bias (norm=True; the hidden vector is the
    window's mean itself otherwise), AdamW's moments (bits 32 or 8) and the number of steps taken."""

    def __init__(self, model: Model, norm: bool = True, bits: int = 32, betas: tuple[float, float] = (0.9, 0.999),
                 eps: float = 1e-8, weight_decay: float = 0.0, norm_eps: float = 1e-5, seed: int = 0):
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        dev = model.syn0.device
        self.device, self.bits, self.betas, self.eps = dev, bits, betas, eps
        self.weight_decay, self.norm_eps, self.seed, self.steps = weight_decay, norm_eps, seed, 0
        self.gain = torch.ones(model.dim, dtype=torch.float32, device=dev) if norm else None
        self.bias = torch.zeros(model.dim, dtype=torch.float32, device=dev) if norm else None
        self._sizes = (model.V, model.dim)
        cm, cb = model.c(), self._c(model)
        self.n_moments = n = lib().w2v_batch_n_moments(ctypes.byref(cm), ctypes.byref(cb))
        kind = torch.float32 if bits == 32 else torch.uint8
        self.m, self.v = (torch.zeros(n, dtype=kind, device=dev) for _ in range(2))
        self.m_scale, self.v_scale = (torch.zeros(n // AdamW.BLOCK, dtype=torch.float32, device=dev) if bits == 8 else None
                                      for _ in range(2))

    def _c(self, model: Model, m=None, v=None, m_scale=None, v_scale=None) -> CBatchParams:
        if model.syn0.device != self.device:
            raise ValueError(f"the model must be on {self.device}")
        gain, bias = (_vector_ptr(t, torch.float32, model.dim, self.device, name)
                      for t, name in ((self.gain, "gain"), (self.bias, "bias")))
        return CBatchParams(gain, bias, m, v, m_scale, v_scale, self.betas[0], self.betas[1], self.eps, self.steps,
                            self.norm_eps, self.weight_decay, self.bits, _tree_of(model).max_len, self.seed & 0xFFFFFFFF, 0)

    def c(self, model: Model) -> CBatchParams:
        n, kind = self.n_moments, torch.float32 if self.bits == 32 else torch.uint8
        m, v = (_vector_ptr(t, kind, n, self.device, name) for t, name in ((self.m, "m"), (self.v, "v")))
        scales = [None, None] if self.bits == 32 else [
            _vector_ptr(t, torch.float32, n // AdamW.BLOCK, self.device, name)
            for t, name in ((self.m_scale, "m_scale"), (self.v_scale, "v_scale"))]
        cm, cb = model.c(), self._c(model, m, v, *scales)
        if (model.V, model.dim) != self._sizes or lib().w2v_batch_n_moments(ctypes.byref(cm), ctypes.byref(cb)) != n:
            raise ValueError(f"the state belongs to a model of other sizes, {self._sizes[0]} words of {self._sizes[1]} columns")
        return cb


def train_batch_epoch(model: Model, tokens: torch.Tensor, p: Params, state: BatchState,
                      stats: torch.Tensor | None = None, workspace: torch.Tensor | None = None
                      ) -> tuple[torch.Tensor, float, int]:
    """One pass of CBOW (p.arch 1) over tokens (vocabulary indices) in batches of p.sync_batch kept centres, with AdamW.
    (device stats int64[5], sum of log P over the centres as they were trained on, their number). Synchronises."""
    dev = tokens.device
    cm, cp, cb = model.c(), p.c(), state.c(model)
    if cp.corpus_tokens <= 0:
        cp.corpus_tokens = max(1, tokens.numel())
    if stats is None:
        stats = torch.zeros(N_STATS, dtype=torch.int64, device=dev)
    sp, tp = _vector_ptr(stats, torch.int64, N_STATS, dev, "stats"), _dev_ptr(tokens, torch.int32, "tokens")
    if dev != state.device:
        raise ValueError(f"tokens must be on {state.device}")
    steps, terms, s = ctypes.c_int64(0), ctypes.c_int64(0), ctypes.c_double(0)
    with _On(dev):
        ws = _kept(workspace, max(1, lib().w2v_train_batch_workspace_bytes(ctypes.byref(cm), tokens.numel(), ctypes.byref(cp),
                                                                          ctypes.byref(cb))), dev)
        rc = lib().w2v_train_batch_epoch(ctypes.byref(cm), tp, tokens.numel(), ctypes.byref(cp), ctypes.byref(cb), sp,
                                         ctypes.byref(steps), ctypes.byref(s), ctypes.byref(terms), ws.data_ptr(),
                                         ws.numel(), _stream(dev))
    state.steps += steps.value   # after an error, too: the moments hold the steps before it
    _check(rc)
    return stats, s.value, terms.value


def batch_loglik(model: Model, tokens: torch.Tensor, p: Params, state: BatchState) -> tuple[float, int]:
    """Held-out score of a model trained by train_batch_epoch: (sum of log P(centre | hidden vector), number of centres
    with a window) over the sampler's centres, through the state's layer norm. Synchronises."""
    dev = tokens.device
    cm, cp, cb = model.c(), p.c(), state.c(model)
    if cp.corpus_tokens <= 0:
        cp.corpus_tokens = max(1, tokens.numel())
    if dev != state.device:
        raise ValueError(f"tokens must be on {state.device}")
    s, terms = ctypes.c_double(0), ctypes.c_int64(0)
    with _On(dev):
        ws = _workspace(lib().w2v_batch_loglik_workspace_bytes(ctypes.byref(cm), tokens.numel(), ctypes.byref(cp),
                                                               ctypes.byref(cb)), dev)
        _check(lib().w2v_batch_loglik(ctypes.byref(cm), _dev_ptr(tokens, torch.int32, "tokens"), tokens.numel(),
                                      ctypes.byref(cp), ctypes.byref(cb), ctypes.byref(s), ctypes.byref(terms),
                                      ws.data_ptr(), ws.numel(), _stream(dev)))
    return s.value, terms.value
