"""ctypes binding of libtrajspec (include/traj_spec.h).

Argument marshalling only: every step of the verification path runs in the HIP
kernels of the library.  PyTorch supplies device memory and the current stream.
If the library is not built the calls raise -- there is no fallback.
"""

import ctypes
import functools
import os

import torch

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libtrajspec.so")

TRAJ_OK = 0
STATUS_NAMES = {0: "TRAJ_OK", 1: "TRAJ_E_NULL", 2: "TRAJ_E_SHAPE", 3: "TRAJ_E_DTYPE",
                4: "TRAJ_E_UNSUPPORTED", 5: "TRAJ_E_WORKSPACE", 6: "TRAJ_E_HIP", 7: "TRAJ_E_ARG"}
TRAJ_BF16, TRAJ_F32 = 0, 1
MODES = {"exact": 0, "top1": 1, "topk": 2}
TRAVERSALS = {"greedy": 0, "longest": 1}
DEV_BAD_PARENT = 0x1
DEV_BAD_LEAF = 0x2
DEV_BAD_BLOCK = 0x4
DEV_BAD_ROOT = 0x8
DEV_BAD_LENGTH = 0x10
DEV_BAD_PAGE = 0x20
DEV_BAD_MASK = 0x40
DEV_BAD_HISTORY = 0x80


class TrajSpecError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = _lib().traj_status_string(status).decode()
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} ({msg})")


class AttnShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("L", ctypes.c_int32), ("Hq", ctypes.c_int32),
                ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32), ("S", ctypes.c_int32), ("scale", ctypes.c_float)]


class LogitsShape(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("vocab", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("dtype", ctypes.c_int32)]


class Drafts(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("N", ctypes.c_int32), ("L", ctypes.c_int32), ("k", ctypes.c_int32),
                ("tokens", ctypes.c_void_p), ("parent", ctypes.c_void_p), ("committed", ctypes.c_void_p),
                ("conf0", ctypes.c_void_p), ("idx0", ctypes.c_void_p), ("mode", ctypes.c_int32),
                ("traversal", ctypes.c_int32)]


class Accepted(ctypes.Structure):
    _fields_ = [("leaf", ctypes.c_void_p), ("on_path", ctypes.c_void_p), ("n_accepted", ctypes.c_void_p),
                ("out_tokens", ctypes.c_void_p), ("hi", ctypes.c_void_p)]


class TreeShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("L", ctypes.c_int32), ("k", ctypes.c_int32), ("n_prev", ctypes.c_int32),
                ("width", ctypes.c_int32), ("depth", ctypes.c_int32), ("branch", ctypes.c_int32),
                ("full", ctypes.c_int32), ("n_max", ctypes.c_int32), ("branch_deep", ctypes.c_int32)]


class LayerDims(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("inter", ctypes.c_int32), ("rms_eps", ctypes.c_float),
                ("rope_theta", ctypes.c_float)]


class RefreshShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("S", ctypes.c_int32), ("L", ctypes.c_int32), ("Hq", ctypes.c_int32),
                ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32), ("scale", ctypes.c_float)]


class LayerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down")]


class PagedShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "Hq", "Hkv", "D", "num_pages", "page_size", "max_pages")] + \
               [(n, ctypes.c_int64) for n in ("table_stride", "page_stride", "token_stride", "head_stride")]


class LogitAdjust(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows_per_seq", "history_size", "bias_size", "n_masks")] + \
               [(n, ctypes.c_void_p) for n in ("history", "history_len", "repetition", "frequency", "presence", "bias_ids",
                                               "bias", "mask", "mask_index")] + [("mask_stride", ctypes.c_int64)]


_LIB = None

EXPORTS = {
    "traj_verify_attn_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(AttnShape)]),
    "traj_verify_attn": (ctypes.c_int32, [ctypes.c_void_p] * 7 + [ctypes.POINTER(AttnShape), ctypes.c_void_p,
                                                                   ctypes.c_size_t, ctypes.c_void_p]),
    "traj_confidence_topk_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(LogitsShape), ctypes.c_int32]),
    "traj_confidence_topk": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                              ctypes.POINTER(LogitsShape), ctypes.c_void_p, ctypes.c_size_t,
                                              ctypes.c_void_p]),
    "traj_confidence_topk_noalloc": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p,
                                                      ctypes.c_void_p, ctypes.POINTER(LogitsShape), ctypes.c_void_p]),
    "traj_accept": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(Drafts), ctypes.c_float,
                                     ctypes.POINTER(Accepted), ctypes.c_void_p]),
    "traj_verify_attn_peers": (ctypes.c_int32, [ctypes.c_void_p] * 8 + [ctypes.POINTER(AttnShape), ctypes.c_void_p,
                                                                         ctypes.c_size_t, ctypes.c_void_p]),
    "traj_joint_peers": (ctypes.c_int32, [ctypes.c_int32] * 3 + [ctypes.c_void_p] * 4),
    "traj_interblock_trigger": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32,
                                                 ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p,
                                                 ctypes.c_void_p, ctypes.c_void_p]),
    "traj_tree_max_nodes": (ctypes.c_int32, [ctypes.POINTER(TreeShape)]),
    "traj_verify_layer_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(AttnShape), ctypes.POINTER(LayerDims)]),
    "traj_refresh_layer_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(RefreshShape), ctypes.POINTER(LayerDims)]),
    "traj_refresh_layer": (ctypes.c_int32, [ctypes.c_void_p, ctypes.POINTER(LayerWeights), ctypes.POINTER(LayerDims),
                                            ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                            ctypes.POINTER(RefreshShape), ctypes.c_void_p, ctypes.c_size_t,
                                            ctypes.c_void_p]),
    "traj_verify_layer": (ctypes.c_int32, [ctypes.c_void_p, ctypes.POINTER(LayerWeights), ctypes.POINTER(LayerDims),
                                           ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                           ctypes.POINTER(AttnShape), ctypes.c_void_p, ctypes.c_size_t,
                                           ctypes.c_void_p]),
    "traj_linear_workspace_size": (ctypes.c_size_t, [ctypes.c_int64] * 3),
    "traj_linear": (ctypes.c_int32, [ctypes.c_void_p] * 3 + [ctypes.c_int64] * 3 +
                    [ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "traj_build_tree": (ctypes.c_int32, [ctypes.c_void_p] * 6 + [ctypes.POINTER(TreeShape), ctypes.c_float]
                        + [ctypes.c_void_p] * 7),
    "traj_paged_append": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_int64] * 3 + [ctypes.c_void_p] * 7 +
                          [ctypes.POINTER(PagedShape), ctypes.c_float, ctypes.c_void_p]),
    "traj_paged_attn_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(PagedShape)]),
    "traj_paged_attn": (ctypes.c_int32, [ctypes.c_void_p] * 7 + [ctypes.POINTER(PagedShape), ctypes.c_float, ctypes.c_int32,
                                                                 ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "traj_confidence_topk_adjusted_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(LogitsShape), ctypes.c_int32,
                                                                       ctypes.POINTER(LogitAdjust)]),
    "traj_confidence_topk_adjusted": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                                       ctypes.POINTER(LogitsShape), ctypes.POINTER(LogitAdjust),
                                                       ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "traj_paged_append_eight": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_int64] * 3 + [ctypes.c_void_p] * 9 +
                           [ctypes.POINTER(PagedShape), ctypes.c_int32, ctypes.c_float, ctypes.c_void_p]),
    "traj_paged_append_eight_within": (ctypes.c_int32, [ctypes.c_void_p, ctypes.c_int64] * 3 + [ctypes.c_void_p] * 10 +
                                       [ctypes.POINTER(PagedShape), ctypes.c_int32, ctypes.c_float, ctypes.c_void_p]),
    "traj_paged_attn_eight_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(PagedShape), ctypes.c_int32]),
    "traj_paged_attn_eight": (ctypes.c_int32, [ctypes.c_void_p] * 9 + [ctypes.POINTER(PagedShape), ctypes.c_int32, ctypes.c_float,
                                                                  ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t,
                                                                  ctypes.c_void_p]),
    "traj_quantize_eight": (ctypes.c_int32, [ctypes.c_void_p] * 3 + [ctypes.c_int64] * 2 + [ctypes.c_void_p]),
    "traj_linear_eight_workspace_size": (ctypes.c_size_t, [ctypes.c_int64] * 3),
    "traj_linear_eight": (ctypes.c_int32, [ctypes.c_void_p] * 4 + [ctypes.c_int64] * 3 +
                     [ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "traj_status_string": (ctypes.c_char_p, [ctypes.c_int32]),
    "traj_version": (ctypes.c_char_p, []),
    "traj_get_device_status": (ctypes.c_int32, [ctypes.POINTER(ctypes.c_int32), ctypes.c_int32, ctypes.c_void_p]),
}


def _lib():
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2608_27514_amd.build`")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = lib
    return _LIB


def load():
    """Load the library (raises if it is missing) and return its ctypes handle."""
    return _lib()


def version():
    return _lib().traj_version().decode()


def built_digest():
    """Source digest the loaded library was built from (stamped into traj_version())."""
    return version().rsplit(" ", 1)[-1]


def check_build():
    """Raise unless the loaded library was built from the sources checked out next to it."""
    from .build import source_digest
    want = source_digest()
    got = built_digest()
    if got != want:
        raise RuntimeError(f"{LIB_PATH} was built from other sources (digest {got[:16]}, sources {want[:16]}); "
                           "rebuild with `python -m paper_2608_27514_amd.build`")
    return got


def _check(status, where):
    if status != TRAJ_OK:
        raise TrajSpecError(status, where)


def _stream(stream):
    """The stream's handle.  The current one is asked for by handle: building a Stream object for it
    takes 2.7 us, as long as the smallest kernels run."""
    if stream is not None:
        return stream.cuda_stream
    if not torch.cuda.is_initialized():
        torch.cuda.init()
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _dev(t, name, dtype=None):
    """Checks a device tensor argument; returns its address (None when it is empty)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr() if t.numel() > 0 else None


def _ptr(t):
    return t.data_ptr() if t is not None and t.numel() > 0 else None


# ---------------------------------------------------------------- attention

def attn_shape(q, k_cache, scale=0.0):
    B, N, L, Hq, D = q.shape
    S, Hkv = k_cache.shape[1], k_cache.shape[2]
    return AttnShape(B, N, L, Hq, Hkv, D, S, float(scale))


def verify_attn_workspace_size(shape):
    return int(_lib().traj_verify_attn_workspace_size(ctypes.byref(shape)))


def verify_attn(q, k_cache, v_cache, k_draft, v_draft, draft_parent, out=None, scale=0.0, workspace=None,
                stream=None, peers=None):
    """Trajectory-masked attention; returns ``out`` [B,N,L,Hq,D] bf16.  ``peers`` ([B,N]
    int64 holding uint64 bit masks) adds visible drafts per draft (traj_verify_attn_peers)."""
    bf16 = torch.bfloat16
    qp, kcp, vcp = _dev(q, "q", bf16), _dev(k_cache, "k_cache", bf16), _dev(v_cache, "v_cache", bf16)
    kdp, vdp = _dev(k_draft, "k_draft", bf16), _dev(v_draft, "v_draft", bf16)
    parent = _dev(draft_parent, "draft_parent", torch.int32)
    if peers is not None:
        peers_p = _dev(peers, "peers", torch.int64)
        if tuple(peers.shape) != tuple(draft_parent.shape):
            raise ValueError("peers must be [B,N] like draft_parent")
    if out is None:
        out = torch.empty_like(q)
    outp = _dev(out, "out", bf16)
    shape = attn_shape(q, k_cache, scale)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if peers is None:
        st = _lib().traj_verify_attn(qp, kcp, vcp, kdp, vdp, parent, outp, ctypes.byref(shape), _ptr(workspace),
                                     ws_bytes, _stream(stream))
        _check(st, "traj_verify_attn")
    else:
        st = _lib().traj_verify_attn_peers(qp, kcp, vcp, kdp, vdp, parent, peers_p, outp, ctypes.byref(shape),
                                           _ptr(workspace), ws_bytes, _stream(stream))
        _check(st, "traj_verify_attn_peers")
    return out


def joint_peers(B, n_cur, n_next, root_cur=None, root_next=None, out=None, device=None, stream=None):
    """Peer masks of a joint packing (traj_joint_peers): drafts [0, n_cur) hold block t's
    tree, [n_cur, n_cur + n_next) block t+1's; root_cur / root_next are [B] int32 device
    tensors (None = root 0).  Returns a [B, n_cur + n_next] int64 device tensor holding the
    uint64 bit masks traj_verify_attn_peers takes."""
    for name, t in (("root_cur", root_cur), ("root_next", root_next)):
        if t is not None:
            _dev(t, name, torch.int32)
            if t.numel() != B:
                raise ValueError(f"{name} must hold B entries")
    if out is None:
        dev = device or (root_cur.device if root_cur is not None else
                         root_next.device if root_next is not None else torch.device("cuda"))
        out = torch.empty((B, n_cur + n_next), dtype=torch.int64, device=dev)
    _dev(out, "out", torch.int64)
    _check(_lib().traj_joint_peers(B, n_cur, n_next, _ptr(root_cur), _ptr(root_next), _ptr(out), _stream(stream)),
           "traj_joint_peers")
    return out


def interblock_trigger(state, conf, threshold, out=None, stream=None):
    """Inter-block trigger per sequence from state [B,2L] int32 and conf [B,2L,k] (or
    [B*2L,k]) float32; returns dict trigger [B] uint8, c_cur [B], c_next [B] float32."""
    B, L2 = state.shape
    if L2 % 2:
        raise ValueError("state must hold two blocks (2L positions) per sequence")
    k = conf.numel() // (B * L2)
    if conf.numel() != B * L2 * k:
        raise ValueError("conf must hold B*2L*k entries")
    _dev(state, "state", torch.int32)
    _dev(conf, "conf", torch.float32)
    dev = state.device
    if out is None:
        out = {"trigger": torch.empty(B, dtype=torch.uint8, device=dev),
               "c_cur": torch.empty(B, dtype=torch.float32, device=dev),
               "c_next": torch.empty(B, dtype=torch.float32, device=dev)}
    st = _lib().traj_interblock_trigger(_ptr(state), _ptr(conf), B, L2 // 2, k, float(threshold),
                                        _ptr(out["trigger"]), _ptr(out.get("c_cur")), _ptr(out.get("c_next")),
                                        _stream(stream))
    _check(st, "traj_interblock_trigger")
    return out


# ---------------------------------------------------------------- confidence / top-k

def logits_shape(logits):
    rows, vocab = logits.shape
    dt = {torch.bfloat16: TRAJ_BF16, torch.float32: TRAJ_F32}.get(logits.dtype)
    if dt is None:
        raise TypeError("logits must be bfloat16 or float32")
    return LogitsShape(rows, vocab, logits.stride(0), dt)


def confidence_topk_workspace_size(logits, k):
    return int(_lib().traj_confidence_topk_workspace_size(ctypes.byref(logits_shape(logits)), int(k)))


def confidence_topk(logits, k, conf=None, idx=None, workspace=None, stream=None):
    """Returns (conf [R,k] float32, idx [R,k] int32).  ``logits`` [R,V] may have a row
    stride larger than V (its last dimension must be contiguous)."""
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
        raise TypeError("logits must be a CUDA (HIP) tensor")
    if logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits must be 2-D with a contiguous last dimension")
    shape = logits_shape(logits)
    R = logits.shape[0]
    if conf is None:
        conf = torch.empty((R, k), dtype=torch.float32, device=logits.device)
    if idx is None:
        idx = torch.empty((R, k), dtype=torch.int32, device=logits.device)
    _dev(conf, "conf", torch.float32)
    _dev(idx, "idx", torch.int32)
    if workspace is None:
        need = int(_lib().traj_confidence_topk_workspace_size(ctypes.byref(shape), int(k)))
        if need > 0:
            workspace = torch.empty(need, dtype=torch.uint8, device=logits.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _lib().traj_confidence_topk(logits.data_ptr(), int(k), _ptr(conf), _ptr(idx),
                                     ctypes.byref(shape), _ptr(workspace), ws_bytes, _stream(stream))
    _check(st, "traj_confidence_topk")
    return conf, idx


def confidence_topk_noalloc(logits, k, conf=None, idx=None, stream=None):
    """traj_confidence_topk_noalloc: the same results as :func:`confidence_topk` without a
    workspace (the library's fixed per-device scratch holds the split records)."""
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
        raise TypeError("logits must be a CUDA (HIP) tensor")
    if logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits must be 2-D with a contiguous last dimension")
    shape = logits_shape(logits)
    R = logits.shape[0]
    if conf is None:
        conf = torch.empty((R, k), dtype=torch.float32, device=logits.device)
    if idx is None:
        idx = torch.empty((R, k), dtype=torch.int32, device=logits.device)
    _dev(conf, "conf", torch.float32)
    _dev(idx, "idx", torch.int32)
    st = _lib().traj_confidence_topk_noalloc(logits.data_ptr(), int(k), _ptr(conf), _ptr(idx),
                                             ctypes.byref(shape), _stream(stream))
    _check(st, "traj_confidence_topk_noalloc")
    return conf, idx


# ---------------------------------------------------------------- acceptance

def accept(conf, idx, tokens, parent, committed, conf0, idx0, threshold, mode="exact", traversal="greedy",
           out=None, stream=None):
    """Acceptance; returns a dict of device tensors (leaf, on_path, n_accepted,
    out_tokens, hi).  conf/idx may be [B*N*L, k] or [B,N,L,k]; a position whose first idx is
    negative has no candidate and is left masked."""
    B, N, L = tokens.shape
    k = conf0.shape[-1]
    if conf.numel() != B * N * L * k or idx.numel() != B * N * L * k:
        raise ValueError("conf/idx must hold B*N*L*k entries")
    f32, i32 = torch.float32, torch.int32
    confp, idxp = _dev(conf, "conf", f32), _dev(idx, "idx", i32)
    _dev(tokens, "tokens", i32)
    _dev(parent, "parent", i32)
    _dev(committed, "committed", i32)
    _dev(conf0, "conf0", f32)
    _dev(idx0, "idx0", i32)
    if out is None:
        dev, empty = tokens.device, torch.empty
        out = {
            "leaf": empty(B, dtype=i32, device=dev),
            "on_path": empty((B, N), dtype=torch.uint8, device=dev),
            "n_accepted": empty(B, dtype=i32, device=dev),
            "out_tokens": empty((B, L), dtype=i32, device=dev),
            "hi": empty((B, N, L), dtype=torch.uint8, device=dev),
        }
    dr = Drafts(B, N, L, k, tokens.data_ptr(), parent.data_ptr(), committed.data_ptr(), conf0.data_ptr(),
                idx0.data_ptr(), MODES[mode], TRAVERSALS[traversal])
    ac = Accepted(out["leaf"].data_ptr(), out["on_path"].data_ptr(), out["n_accepted"].data_ptr(),
                  out["out_tokens"].data_ptr(), out["hi"].data_ptr())
    st = _lib().traj_accept(confp, idxp, ctypes.byref(dr), float(threshold), ctypes.byref(ac),
                            _stream(stream))
    _check(st, "traj_accept")
    return out


# ---------------------------------------------------------------- tree construction
def tree_shape(B, L, k, width, depth, branch, full=False, n_prev=0, n_max=None, branch_deep=1):
    sh = TreeShape(B, L, k, n_prev, width, depth, branch, 1 if full else 0, 0, branch_deep)
    if n_max is None:
        n_max = int(_lib().traj_tree_max_nodes(ctypes.byref(sh)))
        if n_max < 0:
            raise ValueError("invalid tree shape")
    sh.n_max = n_max
    return sh


def tree_max_nodes(B, L, k, width, depth, branch, full=False, branch_deep=1):
    return int(_lib().traj_tree_max_nodes(ctypes.byref(tree_shape(B, L, k, width, depth, branch, full, n_max=0,
                                                                  branch_deep=branch_deep))))


def build_tree(state, conf0, idx0, threshold, width, depth, branch, full=False, leaf=None, conf=None, idx=None,
               n_max=None, out=None, stream=None, branch_deep=1):
    """Next step's draft tree (Alg. 1) from the accepted state; returns a dict of device
    tensors tokens [B,n_max,L], parent [B,n_max], n_nodes [B], score [B,n_max],
    conf_next / idx_next [B,L,k].  With ``leaf`` (traj_accept's leaf) the candidates come
    from conf/idx [B,N,L,k] (or [B*N*L,k]) of the verified tree, else from conf0/idx0.  A slot with a
    negative idx is no candidate (:func:`confidence_topk_adjusted`)."""
    B, L = state.shape
    k = conf0.shape[-1]
    for name, t, dt in (("state", state, torch.int32), ("conf0", conf0, torch.float32), ("idx0", idx0, torch.int32)):
        _dev(t, name, dt)
    n_prev = 0
    if leaf is not None:
        _dev(leaf, "leaf", torch.int32)
        _dev(conf, "conf", torch.float32)
        _dev(idx, "idx", torch.int32)
        n_prev = conf.numel() // (B * L * k)
        if conf.numel() != B * n_prev * L * k or idx.numel() != conf.numel():
            raise ValueError("conf/idx must hold B*N*L*k entries")
    sh = tree_shape(B, L, k, width, depth, branch, full, n_prev, n_max, branch_deep)
    dev = state.device
    if out is None:
        out = {
            "tokens": torch.empty((B, sh.n_max, L), dtype=torch.int32, device=dev),
            "parent": torch.empty((B, sh.n_max), dtype=torch.int32, device=dev),
            "n_nodes": torch.empty(B, dtype=torch.int32, device=dev),
            "score": torch.empty((B, sh.n_max), dtype=torch.float32, device=dev),
            "conf_next": torch.empty((B, L, k), dtype=torch.float32, device=dev),
            "idx_next": torch.empty((B, L, k), dtype=torch.int32, device=dev),
        }
    st = _lib().traj_build_tree(_ptr(state), _ptr(leaf), _ptr(conf), _ptr(idx), _ptr(conf0), _ptr(idx0),
                                ctypes.byref(sh), float(threshold), _ptr(out["tokens"]), _ptr(out["parent"]),
                                _ptr(out["n_nodes"]), _ptr(out.get("score")), _ptr(out.get("conf_next")),
                                _ptr(out.get("idx_next")), _stream(stream))
    _check(st, "traj_build_tree")
    return out


# ---------------------------------------------------------------- verification layer
LAYER_WEIGHTS = ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down")


def layer_workspace_size(B, N, L, Hq, Hkv, D, S, hidden, inter, rms_eps=1e-5, rope_theta=500000.0):
    sh = AttnShape(B, N, L, Hq, Hkv, D, S, 0.0)
    return int(_lib().traj_verify_layer_workspace_size(ctypes.byref(sh),
                                                       ctypes.byref(LayerDims(hidden, inter, rms_eps, rope_theta))))


def _expect_shape(t, name, shape):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def verify_layer(x, weights, k_cache, v_cache, draft_parent, Hq, pos0=None, inter=None, rms_eps=1e-5,
                 rope_theta=500000.0, scale=0.0, workspace=None, stream=None):
    """One verification decoder layer over the packed draft tokens; updates x [B,N,L,hidden]
    (bf16) in place and returns it.  ``weights`` maps LAYER_WEIGHTS names to bf16 tensors."""
    B, N, L, hidden = x.shape
    D = hidden // Hq
    S, Hkv = k_cache.shape[1], k_cache.shape[2]
    if inter is None:
        inter = weights["w_down"].shape[0]
    _dev(x, "x", torch.bfloat16)
    for n in LAYER_WEIGHTS:
        _dev(weights[n], n, torch.bfloat16)
    for n, shape in (("attn_norm", (hidden,)), ("w_qkv", (hidden, (Hq + 2 * Hkv) * D)), ("w_o", (Hq * D, hidden)),
                     ("mlp_norm", (hidden,)), ("w_gate_up", (hidden, 2 * inter)), ("w_down", (inter, hidden))):
        _expect_shape(weights[n], n, shape)
    for t, n in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        _dev(t, n, torch.bfloat16)
        _expect_shape(t, n, (B, S, Hkv, D))
    _dev(draft_parent, "draft_parent", torch.int32)
    _expect_shape(draft_parent, "draft_parent", (B, N))
    if pos0 is not None:
        _dev(pos0, "pos0", torch.int32)
        _expect_shape(pos0, "pos0", (B,))
    sh = AttnShape(B, N, L, Hq, Hkv, D, S, float(scale))
    dims = LayerDims(hidden, inter, rms_eps, rope_theta)
    need = int(_lib().traj_verify_layer_workspace_size(ctypes.byref(sh), ctypes.byref(dims)))
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    lw = LayerWeights(*[weights[n].data_ptr() for n in LAYER_WEIGHTS])
    st = _lib().traj_verify_layer(_ptr(x), ctypes.byref(lw), ctypes.byref(dims), _ptr(k_cache), _ptr(v_cache),
                                  _ptr(draft_parent), _ptr(pos0), ctypes.byref(sh), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "traj_verify_layer")
    return x


def refresh_layer_workspace_size(B, S, L, Hq, Hkv, D, hidden, inter, rms_eps=1e-5, rope_theta=500000.0):
    sh = RefreshShape(B, S, L, Hq, Hkv, D, 0.0)
    return int(_lib().traj_refresh_layer_workspace_size(ctypes.byref(sh),
                                                        ctypes.byref(LayerDims(hidden, inter, rms_eps, rope_theta))))


def refresh_layer(x, weights, block_start, Hq, Hkv, L, k_cache=None, v_cache=None, inter=None, rms_eps=1e-5,
                  rope_theta=500000.0, scale=0.0, workspace=None, stream=None):
    """Dual-cache refresh: one decoder layer over whole sequences x [B, S + L, hidden] (bf16,
    updated in place) with bidirectional attention; the rotated K and the V of every position
    outside each sequence's block [block_start[b], block_start[b] + L) go to k_cache / v_cache
    [B, S, Hkv, D] (allocated when None).  Returns (x, k_cache, v_cache)."""
    B, T, hidden = x.shape
    S = T - L
    D = hidden // Hq
    if inter is None:
        inter = weights["w_down"].shape[0]
    _dev(x, "x", torch.bfloat16)
    for n in LAYER_WEIGHTS:
        _dev(weights[n], n, torch.bfloat16)
    for n, shape in (("attn_norm", (hidden,)), ("w_qkv", (hidden, (Hq + 2 * Hkv) * D)), ("w_o", (Hq * D, hidden)),
                     ("mlp_norm", (hidden,)), ("w_gate_up", (hidden, 2 * inter)), ("w_down", (inter, hidden))):
        _expect_shape(weights[n], n, shape)
    _dev(block_start, "block_start", torch.int32)
    _expect_shape(block_start, "block_start", (B,))
    if k_cache is None:
        k_cache = torch.empty(B, S, Hkv, D, dtype=torch.bfloat16, device=x.device)
    if v_cache is None:
        v_cache = torch.empty(B, S, Hkv, D, dtype=torch.bfloat16, device=x.device)
    for t, n in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        _dev(t, n, torch.bfloat16)
        _expect_shape(t, n, (B, S, Hkv, D))
    sh = RefreshShape(B, S, L, Hq, Hkv, D, float(scale))
    dims = LayerDims(hidden, inter, rms_eps, rope_theta)
    need = int(_lib().traj_refresh_layer_workspace_size(ctypes.byref(sh), ctypes.byref(dims)))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)
    lw = LayerWeights(*[weights[n].data_ptr() for n in LAYER_WEIGHTS])
    st = _lib().traj_refresh_layer(_ptr(x), ctypes.byref(lw), ctypes.byref(dims), _ptr(block_start), _ptr(k_cache),
                                   _ptr(v_cache), ctypes.byref(sh), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "traj_refresh_layer")
    return x, k_cache, v_cache


def linear_workspace_size(M, K, N):
    return int(_lib().traj_linear_workspace_size(M, K, N))


def linear(x, w, y=None, accumulate=False, workspace=None, stream=None):
    """y = x @ w (+ y when accumulate) for bf16 x [..., K] and w [K, N]; returns y [..., N].
    Few-row shapes split K when given a workspace (allocated here when None)."""
    _dev(x, "x", torch.bfloat16)
    _dev(w, "w", torch.bfloat16)
    K, N = w.shape
    if x.shape[-1] != K:
        raise ValueError(f"x has {x.shape[-1]} columns, w has {K} rows")
    M = x.numel() // K
    if y is None:
        if accumulate:
            raise ValueError("accumulate needs y")
        y = torch.empty(x.shape[:-1] + (N,), dtype=torch.bfloat16, device=x.device)
    _dev(y, "y", torch.bfloat16)
    _expect_shape(y, "y", x.shape[:-1] + (N,))
    if workspace is None:
        need = linear_workspace_size(M, K, N)
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device) if need > 0 else None
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib().traj_linear(_ptr(x), _ptr(w), _ptr(y), M, K, N, 1 if accumulate else 0, _ptr(workspace), ws_bytes,
                              _stream(stream)), "traj_linear")
    return y


# ---------------------------------------------------------------- paged cache
def _current():
    """Index of the current device, on which the library launches."""
    return torch._C._cuda_getDevice() if torch.cuda.is_initialized() else -2


def _here(t, name, dev):
    """A tensor of another device than the current one is refused."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{dev}")


def _empty(shape, dtype, device, stream):
    """Memory for a call on ``stream``: taken from that stream's pool, so that nothing frees or reuses it early."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _arg(t, name, dtype, shape, dev):
    """Checks a contiguous tensor of this type and shape on device `dev`; returns its address.  One condition for what
    is right (a decoding step makes such checks some thirty times), the reasons for what is not."""
    if type(t) is torch.Tensor and t.dtype is dtype and t.get_device() == dev and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    p = _dev(t, name, dtype)
    _expect_shape(t, name, shape)
    _here(t, name, dev)
    return p


def _int32(**sizes):
    """A size past 31 bits would be another one in the C structures."""
    for name, n in sizes.items():
        if n >= 1 << 31:
            raise ValueError(f"{name} must be below 2^31, got {n}")


def _room(workspace, dev):
    """A caller's workspace as (address, bytes)."""
    _here(workspace, "workspace", dev)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return _ptr(workspace), workspace.numel() * workspace.element_size()


@functools.lru_cache(maxsize=1024)
def _paged_struct(B, T, Hq, pages, strides, table, table_strides):
    """The C shape of a paged call, by sizes and strides alone: (structure, reference to it)."""
    if len(pages) != 4 or strides[3] != 1:
        raise ValueError("k_pages and v_pages must be [pages, page_size, Hkv, D] with a contiguous last dimension")
    if len(table) != 2 or table[0] != B or table_strides[1] != 1 and table[1] > 1:
        raise ValueError("page_table must be [B, max_pages] with contiguous rows")
    _int32(B=B, T=T, heads=Hq, pages=pages[0], page_size=pages[1], kv_heads=pages[2], head_size=pages[3], max_pages=table[1])
    # a dimension of one entry has no stride that matters
    sh = PagedShape(B, T, Hq, pages[2], pages[3], pages[0], pages[1], table[1], max(table_strides[0], table[1]) if B <= 1 else table_strides[0],
                    strides[0] if pages[0] > 1 else 16, strides[1] if pages[1] > 1 else 16, strides[2] if pages[2] > 1 else 16)
    return sh, ctypes.byref(sh)


@functools.lru_cache(maxsize=1024)
def _paged_workspace(*sizes):
    return int(_lib().traj_paged_attn_workspace_size(_paged_struct(*sizes)[1]))


def _paged_sizes(B, T, Hq, k_pages, v_pages, page_table, dev, element=torch.bfloat16):
    """Checks the pools and the table; returns what :func:`_paged_struct` takes."""
    tensor = torch.Tensor
    if not (isinstance(k_pages, tensor) and k_pages.dtype is element and k_pages.get_device() == dev and isinstance(v_pages, tensor)
            and v_pages.dtype is element and v_pages.get_device() == dev and isinstance(page_table, tensor)
            and page_table.dtype is torch.int32 and page_table.get_device() == dev):
        for t, n, dt in ((k_pages, "k_pages", element), (v_pages, "v_pages", element), (page_table, "page_table", torch.int32)):
            _here(t, n, dev)
            if t.dtype is not dt:
                raise TypeError(f"{n} must be {dt}, got {t.dtype}")
    pages, strides = k_pages.shape, k_pages.stride()
    if v_pages.shape != pages or v_pages.stride() != strides:
        raise ValueError("k_pages and v_pages must have the same shape and strides")
    return B, T, Hq, pages, strides, page_table.shape, page_table.stride()


def _token_rows(t, name, shape, dev):
    """Checks a [B, T, heads, D] tensor whose token rows hold their heads side by side; returns (address, row stride)."""
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.bfloat16 and t.get_device() == dev and t.shape == shape):
        _here(t, name, dev)
        if t.dtype is not torch.bfloat16:
            raise TypeError(f"{name} must be {torch.bfloat16}, got {t.dtype}")
        _expect_shape(t, name, shape)
    B, T, heads, D = shape
    sb, st, sh, sd = t.stride()
    row = st if T > 1 else sb if B > 1 else heads * D
    if sd != 1 or (heads > 1 and sh != D) or (B > 1 and T > 1 and sb != T * st):
        raise ValueError(f"{name} must have evenly spaced token rows of contiguous heads")
    return t.data_ptr(), row


def _append_rows(B, T, Hq, Hkv, D, k, v, q, q_out, n_new, dev, stream):
    """Checks the new tokens' rows of an append call; returns their addresses and strides, and q_out (allocated when None).
    Shapes are plain tuples: putting one together from pieces of torch.Size costs some 0.8 us, 5% of a call."""
    shape = (B, T, Hkv, D)
    kp, ks = _token_rows(k, "k", shape, dev)
    vp, vs = _token_rows(v, "v", shape, dev)
    qp, qs, qop = None, 0, None
    if q is not None:
        shape = (B, T, Hq, D)
        qp, qs = _token_rows(q, "q", shape, dev)
        if q_out is None:
            if n_new is None:
                q_out = _empty(shape, torch.bfloat16, q.device, stream)
            else:
                with torch.cuda.stream(stream):  # None: the current one
                    q_out = torch.zeros(shape, dtype=torch.bfloat16, device=q.device)
        qop = _arg(q_out, "q_out", torch.bfloat16, shape, dev)
    elif q_out is not None:
        raise ValueError("q_out needs q")
    return kp, ks, vp, vs, qp, qs, qop, q_out


def paged_append(k, v, k_pages, v_pages, page_table, start, q=None, q_out=None, n_new=None, pos0=None,
                 rope_theta=500000.0, stream=None):
    """Rotates the new tokens' keys (and queries) by position and writes keys and values into the pages.

    k, v [B,T,Hkv,D] and q [B,T,Hq,D] (bf16) may be views into a projection's rows; k_pages / v_pages
    [pages, page_size, Hkv, D] with any strides but the last dimension's; page_table [B, max_pages] int32; start,
    n_new (None: T each) and pos0 (None: start) [B] int32.  Token t of sequence b gets cache index start[b] + t and
    position pos0[b] + t; rows t >= n_new[b] are padding and left alone.  Returns q_out [B,T,Hq,D] (allocated when
    None; its padding rows are then zero), or None without q."""
    B, T, Hkv, D = k.shape
    Hq = q.shape[2] if q is not None else Hkv
    dev = _current()
    sh, ref = _paged_struct(*_paged_sizes(B, T, Hq, k_pages, v_pages, page_table, dev))
    if sh.Hkv != Hkv or sh.D != D:
        raise ValueError(f"k has {Hkv} heads of {D}, the pages {sh.Hkv} of {sh.D}")
    kp, ks, vp, vs, qp, qs, qop, q_out = _append_rows(B, T, Hq, Hkv, D, k, v, q, q_out, n_new, dev, stream)
    i32, per_seq = torch.int32, (B,)
    st = _lib().traj_paged_append(qp, qs, kp, ks, vp, vs, qop, k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(),
                                  _arg(start, "start", i32, per_seq, dev),
                                  None if n_new is None else _arg(n_new, "n_new", i32, per_seq, dev),
                                  None if pos0 is None else _arg(pos0, "pos0", i32, per_seq, dev), ref, rope_theta, _stream(stream))
    if st != TRAJ_OK:
        _check(st, "traj_paged_append")
    return q_out


def paged_attn_workspace_size(q, k_pages, v_pages, page_table):
    return _paged_workspace(*_paged_sizes(*q.shape[:3], k_pages, v_pages, page_table, _current()))


def paged_attn(q, k_pages, v_pages, page_table, lens, out=None, scale=0.0, causal=False, n_new=None, workspace=None, stream=None):
    """Attention of T new tokens per sequence, q [B,T,Hq,D] (bf16), over the first lens[b] cached keys of each
    (causal: the new tokens are the last n_new[b] of them and see those up to themselves).  Pages and table as
    :func:`paged_append`; lens and n_new (None: T each) [B] int32.  Returns ``out`` [B,T,Hq,D]; a row that sees no key
    and the padding rows t >= n_new[b] are zero."""
    shape = B, T, Hq, D = q.shape
    bf16 = torch.bfloat16
    dev = _current()
    qp = _arg(q, "q", bf16, shape, dev)
    sizes = _paged_sizes(B, T, Hq, k_pages, v_pages, page_table, dev)
    sh, ref = _paged_struct(*sizes)
    if sh.D != D:
        raise ValueError(f"q has heads of {D}, the pages of {sh.D}")
    if out is None:
        out = _empty(shape, bf16, q.device, stream)
    ws, ws_bytes = None, 0
    if workspace is None:
        ws_bytes = _paged_workspace(*sizes)
        if ws_bytes > 0:
            workspace = _empty((ws_bytes,), torch.uint8, q.device, stream)
            ws = workspace.data_ptr()
    else:
        ws, ws_bytes = _room(workspace, dev)
    st = _lib().traj_paged_attn(qp, k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr(), _arg(lens, "lens", torch.int32, (B,), dev),
                                None if n_new is None else _arg(n_new, "n_new", torch.int32, (B,), dev), _arg(out, "out", bf16, shape, dev), ref, scale, 1 if causal else 0, ws, ws_bytes, _stream(stream))
    if st != TRAJ_OK:
        _check(st, "traj_paged_attn")
    return out


# ---------------------------------------------------------------- 8 bits
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _scale_block(pages, k_scale, v_scale, dev):
    """Checks the scales of pools of this shape; returns (address, address, tokens of a scale)."""
    blocks = k_scale.shape[1] if k_scale.dim() == 3 else 0
    if blocks < 1 or pages[1] % blocks:
        raise ValueError(f"k_scale must be [pages, blocks, Hkv] with blocks dividing the page's {pages[1]} tokens")
    shape = (pages[0], blocks, pages[2])
    return _arg(k_scale, "k_scale", E8M0, shape, dev), _arg(v_scale, "v_scale", E8M0, shape, dev), pages[1] // blocks


def paged_append8(k, v, k_pages, v_pages, k_scale, v_scale, page_table, start, q=None, q_out=None, n_new=None, pos0=None,
                  rope_theta=500000.0, stream=None, lens=None):
    """:func:`paged_append` to a cache in 8 bits: k_pages / v_pages [pages, page_size, Hkv, D] float8_e4m3fn, and k_scale /
    v_scale [pages, blocks, Hkv] float8_e8m0fnu, a scale for each block of page_size / blocks tokens (at most 64) and head.
    A block's scale is the smallest power of two that brings its rows to 448 at most.  Rows of a block before start[b] keep
    their values (rounded again where the scale grows).  So do rows behind the call's last token up to lens[b], the
    sequence's tokens, where lens (int32 [B]) is given: a block denoised in front of a cached suffix needs it.  Other rows behind the
    call's keep their bits under the new scale, so their values are lost."""
    B, T, Hkv, D = k.shape
    Hq = q.shape[2] if q is not None else Hkv
    dev = _current()
    sh, ref = _paged_struct(*_paged_sizes(B, T, Hq, k_pages, v_pages, page_table, dev, E4M3))
    ksp, vsp, sb = _scale_block(k_pages.shape, k_scale, v_scale, dev)
    if sh.Hkv != Hkv or sh.D != D:
        raise ValueError(f"k has {Hkv} heads of {D}, the pages {sh.Hkv} of {sh.D}")
    kp, ks, vp, vs, qp, qs, qop, q_out = _append_rows(B, T, Hq, Hkv, D, k, v, q, q_out, n_new, dev, stream)
    i32, per_seq = torch.int32, (B,)
    st = _lib().traj_paged_append_eight_within(qp, qs, kp, ks, vp, vs, qop, k_pages.data_ptr(), v_pages.data_ptr(), ksp, vsp,
                                               page_table.data_ptr(), _arg(start, "start", i32, per_seq, dev),
                                               None if n_new is None else _arg(n_new, "n_new", i32, per_seq, dev),
                                               None if pos0 is None else _arg(pos0, "pos0", i32, per_seq, dev),
                                               None if lens is None else _arg(lens, "lens", i32, per_seq, dev), ref, sb, rope_theta,
                                               _stream(stream))
    if st != TRAJ_OK:
        _check(st, "traj_paged_append_eight")
    return q_out


@functools.lru_cache(maxsize=1024)
def _paged8_workspace(sb, *sizes):
    return int(_lib().traj_paged_attn_eight_workspace_size(_paged_struct(*sizes)[1], sb))


def paged_attn8_workspace_size(q, k_pages, v_pages, k_scale, v_scale, page_table):
    dev = _current()
    sizes = _paged_sizes(*q.shape[:3], k_pages, v_pages, page_table, dev, E4M3)
    return _paged8_workspace(_scale_block(k_pages.shape, k_scale, v_scale, dev)[2], *sizes)


def paged_attn8(q, k_pages, v_pages, k_scale, v_scale, page_table, lens, out=None, scale=0.0, causal=False, n_new=None,
                workspace=None, stream=None):
    """:func:`paged_attn` over a cache in 8 bits (pools and scales as :func:`paged_append8`)."""
    shape = B, T, Hq, D = q.shape
    bf16 = torch.bfloat16
    dev = _current()
    qp = _arg(q, "q", bf16, shape, dev)
    sizes = _paged_sizes(B, T, Hq, k_pages, v_pages, page_table, dev, E4M3)
    sh, ref = _paged_struct(*sizes)
    ksp, vsp, sb = _scale_block(k_pages.shape, k_scale, v_scale, dev)
    if sh.D != D:
        raise ValueError(f"q has heads of {D}, the pages of {sh.D}")
    if out is None:
        out = _empty(shape, bf16, q.device, stream)
    ws, ws_bytes = None, 0
    if workspace is None:
        ws_bytes = _paged8_workspace(sb, *sizes)
        if ws_bytes > 0:
            workspace = _empty((ws_bytes,), torch.uint8, q.device, stream)
            ws = workspace.data_ptr()
    else:
        ws, ws_bytes = _room(workspace, dev)
    st = _lib().traj_paged_attn_eight(qp, k_pages.data_ptr(), v_pages.data_ptr(), ksp, vsp, page_table.data_ptr(),
                                      _arg(lens, "lens", torch.int32, (B,), dev), None if n_new is None else _arg(n_new, "n_new", torch.int32, (B,), dev),
                                      _arg(out, "out", bf16, shape, dev), ref, sb, scale, 1 if causal else 0, ws, ws_bytes, _stream(stream))
    if st != TRAJ_OK:
        _check(st, "traj_paged_attn_eight")
    return out


def _weight8_shapes(K, N):
    KP = -(-K // 128) * 128
    return (KP // 64, N, 64), (-(-N // 128), KP // 128)


def quantize8(w, w8=None, w_scale=None, stream=None):
    """A weight matrix w [K, N] (bf16) in 8 bits for :func:`linear8`: returns (w8, w_scale), w8 [KP / 64, N, 64]
    float8_e4m3fn holding value (k, n) at [k // 64, n, k % 64] (KP: K rounded up to a multiple of 128), w_scale
    [ceil(N / 128), KP / 128] float8_e8m0fnu a power of two per block of 128 x 128."""
    dev = _current()
    if not isinstance(w, torch.Tensor) or w.dim() != 2:
        raise ValueError("w must be [K, N]")
    K, N = w.shape
    wp = _arg(w, "w", torch.bfloat16, w.shape, dev)
    values, scales = _weight8_shapes(K, N)
    if w8 is None:
        w8 = _empty(values, E4M3, w.device, stream)
    if w_scale is None:
        w_scale = _empty(scales, E8M0, w.device, stream)
    _check(_lib().traj_quantize_eight(wp, _arg(w8, "w8", E4M3, values, dev), _arg(w_scale, "w_scale", E8M0, scales, dev), K, N, _stream(stream)),
           "traj_quantize_eight")
    return w8, w_scale


@functools.lru_cache(maxsize=1024)
def linear8_workspace_size(M, K, N):
    return int(_lib().traj_linear_eight_workspace_size(M, K, N))


def linear8(x, w8, w_scale, y=None, accumulate=False, workspace=None, stream=None):
    """:func:`linear` with weights in 8 bits, as :func:`quantize8` makes them: y = x @ w (+ y when accumulate) for bf16 x
    [..., K], each row's blocks of 128 of k taken to 8 bits with a power of two; returns y [..., N] bf16."""
    dev = _current()
    xp = _arg(x, "x", torch.bfloat16, x.shape, dev)
    if x.dim() < 1 or w8.dim() != 3:
        raise ValueError("x must be [..., K] and w8 [KP / 64, N, 64]")
    K, N = x.shape[-1], w8.shape[1]
    values, scales = _weight8_shapes(K, N)
    wp, sp = _arg(w8, "w8", E4M3, values, dev), _arg(w_scale, "w_scale", E8M0, scales, dev)
    M = x.numel() // max(K, 1)
    shape = x.shape[:-1] + (N,)
    if y is None:
        if accumulate:
            raise ValueError("accumulate needs y")
        y = _empty(shape, torch.bfloat16, x.device, stream)
    yp = _arg(y, "y", torch.bfloat16, shape, dev)
    if workspace is None:
        ws, ws_bytes = None, linear8_workspace_size(M, K, N)
        if ws_bytes > 0:
            workspace = _empty((ws_bytes,), torch.uint8, x.device, stream)
            ws = workspace.data_ptr()
    else:
        ws, ws_bytes = _room(workspace, dev)
    st = _lib().traj_linear_eight(xp, wp, sp, yp, M, K, N, 1 if accumulate else 0, ws, ws_bytes, _stream(stream))
    if st != TRAJ_OK:
        _check(st, "traj_linear_eight")
    return y


# ---------------------------------------------------------------- adjusted logits
def _logit_adjust(dev, R, V, per, history, history_len, repetition, frequency, presence, bias_ids, bias, mask, mask_index):
    if per < 1:
        raise ValueError("rows_per_seq must be at least 1")
    f32, i32 = torch.float32, torch.int32
    n = -(-R // per)
    H = NB = masks = mask_stride = 0
    hp = lp = rp = fp = pp = ip = bp = mp = xp = None
    if history is not None:
        H = history.shape[-1]
        hp = _arg(history, "history", i32, (n, H), dev)
    elif not (history_len is None and repetition is None and frequency is None and presence is None):
        raise ValueError("history_len, repetition, frequency and presence need history")
    if history_len is not None:
        lp = _arg(history_len, "history_len", i32, (n,), dev)
    if repetition is not None:
        rp = _arg(repetition, "repetition", f32, (n,), dev)
    if frequency is not None:
        fp = _arg(frequency, "frequency", f32, (n,), dev)
    if presence is not None:
        pp = _arg(presence, "presence", f32, (n,), dev)
    if (bias_ids is None) != (bias is None):
        raise ValueError("bias_ids and bias go together")
    if bias is not None:
        NB = bias.shape[-1]
        ip, bp = _arg(bias_ids, "bias_ids", i32, (n, NB), dev), _arg(bias, "bias", f32, (n, NB), dev)
    if mask is not None:
        mp = _arg(mask, "mask", i32, mask.shape, dev)
        if mask.dim() != 2 or mask.shape[0] < 1 or mask.shape[1] < -(-V // 32):
            raise ValueError(f"mask must be [n_masks, at least {-(-V // 32)}] words")
        masks, mask_stride = mask.shape
        if mask_index is None and masks < R:
            raise ValueError("mask must have a row for every row of logits, or mask_index one entry")
    if mask_index is not None:
        if mask is None:
            raise ValueError("mask_index needs mask")
        xp = _arg(mask_index, "mask_index", i32, (R,), dev)
    if max(per, H, NB, masks) >= 1 << 31:
        _int32(rows_per_seq=per, history=H, biases=NB, masks=masks)
    return LogitAdjust(per, H, NB, masks, hp, lp, rp, fp, pp, ip, bp, mp, xp, mask_stride)


def _logit_rows(logits):
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
        raise TypeError("logits must be a CUDA (HIP) tensor")
    if logits.dim() != 2 or logits.stride(1) != 1 and logits.shape[1] > 1:
        raise ValueError("logits must be 2-D with a contiguous last dimension")
    sh = logits_shape(logits)
    if sh.rows <= 1:
        sh.row_stride = max(sh.row_stride, sh.vocab)
    return sh


@functools.lru_cache(maxsize=1024)
def _adjust_workspace(rows, vocab, row_stride, dtype, k, per, H, NB):
    _int32(k=k, rows_per_seq=per, history=H, biases=NB)
    return int(_lib().traj_confidence_topk_adjusted_workspace_size(ctypes.byref(LogitsShape(rows, vocab, row_stride, dtype)), k,
                                                                   ctypes.byref(LogitAdjust(per, H, NB))))


def confidence_topk_adjusted_workspace_size(logits, k, rows_per_seq, history=None, bias=None):
    """Bytes for a call with these logits and lists (their sizes count)."""
    sh = _logit_rows(logits)
    return _adjust_workspace(sh.rows, sh.vocab, sh.row_stride, sh.dtype, int(k), int(rows_per_seq),
                             0 if history is None else history.shape[-1], 0 if bias is None else bias.shape[-1])


def confidence_topk_adjusted(logits, k, rows_per_seq, history=None, history_len=None, repetition=None, frequency=None,
                             presence=None, bias_ids=None, bias=None, mask=None, mask_index=None, conf=None, idx=None,
                             workspace=None, stream=None):
    """:func:`confidence_topk` of the logits under each request's penalties, biases and grammar (the adjusted logits
    are written nowhere).  Row r belongs to sequence r // rows_per_seq.  Per sequence: history [n, H] int32 with
    history_len [n] (ids outside the vocabulary are padding, a masked position's -1 among them), repetition, frequency
    and presence penalties [n] float32, bias_ids / bias [n, NB]; mask [n_masks, words] int32 holds a bit per token
    (bit v % 32 of word v // 32; 0 forbids) and mask_index [R] int32 each row's mask (-1: none; without it row r takes
    mask r).  Slots without an allowed token hold confidence 0 and index -1."""
    sh = _logit_rows(logits)
    dev = _current()
    _here(logits, "logits", dev)
    k, per = int(k), int(rows_per_seq)
    if k >= 1 << 31:
        _int32(k=k)
    R = sh.rows
    a = _logit_adjust(dev, R, sh.vocab, per, history, history_len, repetition, frequency, presence, bias_ids, bias, mask, mask_index)
    shape = (R, k)
    if conf is None:
        conf = _empty(shape, torch.float32, logits.device, stream)
    if idx is None:
        idx = _empty(shape, torch.int32, logits.device, stream)
    ws, ws_bytes = None, 0
    if workspace is None:
        ws_bytes = _adjust_workspace(R, sh.vocab, sh.row_stride, sh.dtype, k, per, a.history_size, a.bias_size)
        if ws_bytes > 0:
            workspace = _empty((ws_bytes,), torch.uint8, logits.device, stream)
            ws = workspace.data_ptr()
    else:
        ws, ws_bytes = _room(workspace, dev)
    st = _lib().traj_confidence_topk_adjusted(logits.data_ptr(), k, _arg(conf, "conf", torch.float32, shape, dev),
                                              _arg(idx, "idx", torch.int32, shape, dev), ctypes.byref(sh), ctypes.byref(a), ws, ws_bytes,
                                              _stream(stream))
    if st != TRAJ_OK:
        _check(st, "traj_confidence_topk_adjusted")
    return conf, idx


def device_status(reset=True, stream=None):
    """Synchronises the stream and returns the device status bits (TRAJ_DEV_*)."""
    flags = ctypes.c_int32(0)
    _check(_lib().traj_get_device_status(ctypes.byref(flags), 1 if reset else 0, _stream(stream)),
           "traj_get_device_status")
    return flags.value
