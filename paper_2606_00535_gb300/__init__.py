"""GB300 (sm_103a) tree verification for DREAM-S speculative decoding.

A thin binding over the C ABI of ``libdreams.so`` (declared in
``include/dreams.h``): each function checks the dtype, device and layout of
its torch tensors, passes their ``data_ptr()`` and the current CUDA stream to
the C entry point of the same name, and raises on a non-OK status. Every
step of the computation runs in the library's CUDA kernels; there is no CPU
or PyTorch fallback, and importing this package on a machine without the
built library raises.

The step it implements (paper Sec. 2, "Speculative decoding"): the target
model scores all draft tokens in one pass, then accepts drafts while they
equal its own greedy prediction; here the drafts form a tree.

    out, lse = tree_verify_attn(q, kv, tree, scale)          # per layer
    res = verify_step(logits, tree, kv, max_path)            # argmax + walk + compaction
"""
from __future__ import annotations

import ctypes
import os
import re
import threading
from dataclasses import dataclass
from typing import Dict, List, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdreams.so")
HEADER = os.path.join(os.path.dirname(_HERE), "include", "dreams.h")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_SCRATCH_LIMIT = 0, 1, 2, 3, 4, 5
NOALLOC_ARGMAX_MAX_ROWS = 16384
F32, BF16 = 0, 1
DATA_BAD_PARENT, DATA_BAD_TREE_LEN, DATA_BAD_KV_LEN, DATA_BAD_PAGE, DATA_BAD_PATH = 1, 2, 4, 8, 16
DATA_TIMEOUT = 0x20  # a kernel gave up waiting on its own pipeline
DATA_NO_PAGES, DATA_SHARED_PAGE, DATA_BAD_INDEX = 0x40, 0x80, 0x100
TEST_ATTENTION, TEST_LM_HEAD = 1, 2  # kernel families of test_set_stall


class DreamsError(RuntimeError):
    def __init__(self, fn: str, status: int):
        msg = _lib().dreams_status_string(status).decode()
        if status == ERR_CUDA:
            msg += f" (cudaError {_lib().dreams_last_cuda_error()})"
        super().__init__(f"{fn}: {msg}")
        self.status = status


class _KVCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("n_layers", ctypes.c_int32),
                ("layer_stride", ctypes.c_int64), ("Hkv", ctypes.c_int32), ("D", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("page_table", ctypes.c_void_p),
                ("page_size", ctypes.c_int32), ("pages_per_seq", ctypes.c_int32),
                ("num_pages", ctypes.c_int32)]


class _Tree(ctypes.Structure):
    _fields_ = [("parent", ctypes.c_void_p), ("tokens", ctypes.c_void_p), ("tree_len", ctypes.c_void_p),
                ("kv_len", ctypes.c_void_p), ("B", ctypes.c_int32), ("T_max", ctypes.c_int32)]


class _PagePool(ctypes.Structure):
    _fields_ = [("page_table", ctypes.c_void_p), ("refcount", ctypes.c_void_p), ("B", ctypes.c_int32),
                ("pages_per_seq", ctypes.c_int32), ("num_pages", ctypes.c_int32)]


_LIB: Optional[ctypes.CDLL] = None
_LOCK = threading.Lock()


def _lib() -> ctypes.CDLL:
    global _LIB
    if _LIB is None:
        with _LOCK:
            if _LIB is None:
                if not os.path.exists(LIB_PATH):
                    raise ImportError(f"libdreams.so is not built ({LIB_PATH}); run "
                                      "`python -c 'import __graft_entry__ as g; g.build()'`")
                lib = ctypes.CDLL(LIB_PATH)
                p, i32, i64, sz, f32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t,
                                        ctypes.c_float)
                pkv, ptr, ppl = ctypes.POINTER(_KVCache), ctypes.POINTER(_Tree), ctypes.POINTER(_PagePool)
                sig = {
                    "dreams_tree_verify_attn_workspace_size": (sz, [pkv, ptr, i32]),
                    "dreams_tree_verify_attn_launches": (i32, [pkv, ptr, i32]),
                    "dreams_tree_verify_attn": (ctypes.c_int, [p, i64, i64, pkv, i32, ptr, i32, f32, p, p, p, sz, p,
                                                               p]),
                    "dreams_vocab_argmax_workspace_size": (sz, [i64, i64]),
                    "dreams_vocab_argmax": (ctypes.c_int, [p, ctypes.c_int, i64, i64, i64, p, p, sz, p]),
                    "dreams_accept_path": (ctypes.c_int, [p, ptr, i32, p, p, p, p, p, p]),
                    "dreams_kv_compact": (ctypes.c_int, [pkv, i32, p, p, p, i32, p, p]),
                    "dreams_verify_step_workspace_size": (sz, [ptr, i64]),
                    "dreams_verify_step": (ctypes.c_int, [p, ctypes.c_int, i64, i64, ptr, pkv, i32, p, p, p, p,
                                                          p, p, sz, p, p]),
                    "dreams_vocab_argmax_noalloc": (ctypes.c_int, [p, ctypes.c_int, i64, i64, i64, p, p]),
                    "dreams_attention_workspace_size": (sz, [pkv, i32, i32, i32, i32, i32]),
                    "dreams_attention": (ctypes.c_int, [p, i64, i64, pkv, i32, p, p, i32, i32, i32, f32, i32, p, p,
                                                        p, p, sz, p, p]),
                    "dreams_lm_head_argmax_workspace_size": (sz, [i64]),
                    "dreams_lm_head_argmax": (ctypes.c_int, [p, i64, i64, i64, p, i64, i64, p, p, p, sz, p, p]),
                    "dreams_visual_importance_workspace_size": (sz, [i64, i64, i64, i64]),
                    "dreams_visual_importance": (ctypes.c_int, [p, ctypes.c_int, i64, i64, i64, i64, i64, i64, i32,
                                                                p, p, p, sz, p]),
                    "dreams_vocab_sample_workspace_size": (sz, [i64, i64]),
                    "dreams_vocab_sample": (ctypes.c_int, [p, ctypes.c_int, i64, i64, i64, f32, p, p, p, sz, p]),
                    "dreams_verify_step_sampled_workspace_size": (sz, [ptr, i64]),
                    "dreams_verify_step_sampled": (ctypes.c_int, [p, ctypes.c_int, i64, i64, ptr, pkv, i32, f32, p,
                                                                  p, p, p, p, p, p, sz, p, p]),
                    "dreams_verify_step_speculative": (ctypes.c_int, [p, p, ctypes.c_int, i64, i64, ptr, pkv, i32,
                                                                      f32, p, p, p, p, p, p, p, p]),
                    "dreams_window_attention": (ctypes.c_int, [p, i64, i64, pkv, i32, p, p, p, i32, i32, i32, f32,
                                                               i32, i32, p, p, p, p]),
                    "dreams_kv_reserve_workspace_size": (sz, [ppl]),
                    "dreams_kv_reserve": (ctypes.c_int, [ppl, p, p, p, sz, p, p]),
                    "dreams_kv_release": (ctypes.c_int, [ppl, p, p, p, p]),
                    "dreams_kv_fork_workspace_size": (sz, [ppl]),
                    "dreams_kv_fork": (ctypes.c_int, [pkv, ppl, p, p, p, p, sz, p, p]),
                    "dreams_kv_append": (ctypes.c_int, [pkv, i32, p, p, i64, i64, p, p, i32, i32, p, p]),
                    "dreams_kv_prune": (ctypes.c_int, [pkv, i32, p, i32, i32, i32, p, p, p, p, p]),
                    "dreams_test_set_stall": (ctypes.c_int, [i32, i32, i64]),
                    "dreams_status_string": (ctypes.c_char_p, [ctypes.c_int]),
                    "dreams_version": (i32, []),
                    "dreams_last_cuda_error": (i32, []),
                }
                for name, (res, args) in sig.items():
                    fn = getattr(lib, name)
                    fn.restype = res
                    fn.argtypes = args
                _LIB = lib
    return _LIB


def declared_functions() -> list:
    """Names of the functions ``include/dreams.h`` declares."""
    text = open(HEADER).read()
    return sorted(set(re.findall(r"^\s*(?:const\s+)?[\w\s\*]*?\b(dreams_\w+)\s*\(", text, re.M)))


def version() -> int:
    return int(_lib().dreams_version())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream, dev: torch.device) -> ctypes.c_void_p:
    """The given stream, or the current stream of the tensors' device ``dev``."""
    s = torch.cuda.current_stream(dev) if stream is None else stream
    if s.device != dev:
        raise ValueError(f"stream is on {s.device}, the tensors on {dev}")
    return ctypes.c_void_p(s.cuda_stream)


def _new(shape, dtype, dev: torch.device, stream) -> torch.Tensor:
    """A result of a call on ``stream``. Made with that stream current, so that
    the memory is that stream's: what used it before is done when the call runs.
    It is not given out again before what the current stream does with it is done."""
    if stream is None or dev.type != "cuda":
        return torch.empty(shape, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=dev)
    t.record_stream(torch.cuda.current_stream(dev))
    return t


def _check(name: str, st: int):
    if st != OK:
        raise DreamsError(name, st)


def _call(name: str, dev: torch.device, *args) -> None:
    """Calls the C entry point with the tensors' device current (the library
    runs on the current CUDA device) and raises on a non-OK status."""
    if dev.type != "cuda":
        raise ValueError(f"{name}: tensors must be on a CUDA device, got {dev}")
    with torch.cuda.device(dev):
        st = getattr(_lib(), name)(*args)
    _check(name, st)


def _rows_view(logits: torch.Tensor) -> torch.Tensor:
    """[rows, V] view of ``logits`` (no copy) with contiguous rows."""
    if logits.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("logits must be float32 or bfloat16")
    V = int(logits.shape[-1])
    try:
        x = logits if logits.dim() == 2 else logits.view(-1, V)
    except RuntimeError as e:
        raise ValueError("logits' leading dimensions must flatten without a copy") from e
    if x.stride(-1) != 1:
        raise ValueError("logits rows must be contiguous")
    return x


def _need_out(out: torch.Tensor, name: str, dtype, dev, numel: int) -> torch.Tensor:
    _need(out, name, dtype, dev)
    if out.numel() < numel:
        raise ValueError(f"{name} holds {out.numel()} elements, the call uses {numel}")
    return out


def _ws(workspace: Optional[torch.Tensor], dev):
    """Pointer and byte size of a caller's workspace (contiguous, on dev), or
    (None, 0)."""
    if workspace is None:
        return None, 0
    if not isinstance(workspace, torch.Tensor) or workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {dev}")
    return _ptr(workspace), workspace.numel() * workspace.element_size()


def _status(status: Optional[torch.Tensor], dev):
    """Pointer to the caller's device status word (int32, on dev), or None."""
    return None if status is None else _ptr(_need_out(status, "status", torch.int32, dev, 1))


def _outputs(outputs: Optional[tuple], B: int, max_path: int, dev, stream) -> tuple:
    """(accept_len [B], path [B, max_path], out_tokens [B, max_path],
    new_kv_len [B]): the caller's, checked, or new."""
    if outputs is None:
        return _walk_outputs(B, max_path, dev, stream)
    if len(outputs) != 4:
        raise ValueError("outputs must be (accept_len, path, out_tokens, new_kv_len)")
    acc, path, toks, nkl = outputs
    return (_need_out(acc, "accept_len", torch.int32, dev, B),
            _need_out(path, "path", torch.int32, dev, B * max_path),
            _need_out(toks, "out_tokens", torch.int32, dev, B * max_path),
            _need_out(nkl, "new_kv_len", torch.int32, dev, B))


def _need(t: torch.Tensor, name: str, dtype, dev) -> torch.Tensor:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != dev:
        raise ValueError(f"{name} must be on {dev}, got {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


@dataclass
class KVCache:
    """K/V cache of one or more layers (bf16).

    Contiguous: ``k, v`` of shape ``[B, capacity, Hkv, D]`` (one layer) or
    ``[n_layers, B, capacity, Hkv, D]``. Paged: ``[num_pages, 64, Hkv, D]``
    (or with a leading layer dim) plus ``page_table`` int32 ``[B, pages_per_seq]``.
    """
    k: torch.Tensor
    v: torch.Tensor
    page_table: Optional[torch.Tensor] = None

    def __post_init__(self):
        if self.k.shape != self.v.shape:
            raise ValueError("k and v shapes differ")
        dev = self.k.device
        _need(self.k, "k", torch.bfloat16, dev)
        _need(self.v, "v", torch.bfloat16, dev)
        nd = self.k.dim()
        if nd not in (4, 5):
            raise ValueError("k must be 4-D or 5-D")
        self.n_layers = self.k.shape[0] if nd == 5 else 1
        shp = self.k.shape[1:] if nd == 5 else self.k.shape
        self.layer_stride = int(shp.numel()) if nd == 5 else 0
        self.Hkv, self.D = int(shp[2]), int(shp[3])
        if self.page_table is None:
            self.B = int(shp[0])
            self.capacity = int(shp[1])
            self.page_size = self.pages_per_seq = self.num_pages = 0
        else:
            _need(self.page_table, "page_table", torch.int32, dev)
            self.B = int(self.page_table.shape[0])
            self.page_size = int(shp[1])
            self.pages_per_seq = int(self.page_table.shape[1])
            self.num_pages = int(shp[0])
            self.capacity = self.pages_per_seq * self.page_size
        self._c = _KVCache(self.k.data_ptr(), self.v.data_ptr(), self.n_layers, self.layer_stride, self.Hkv,
                           self.D, self.capacity,
                           None if self.page_table is None else self.page_table.data_ptr(),
                           self.page_size, self.pages_per_seq, self.num_pages)


@dataclass
class Tree:
    """Draft trees of a batch: int32 ``parent``, ``tokens`` [B, T_max];
    ``tree_len``, ``kv_len`` [B] (all on the same CUDA device)."""
    parent: torch.Tensor
    tokens: torch.Tensor
    tree_len: torch.Tensor
    kv_len: torch.Tensor

    def __post_init__(self):
        dev = self.parent.device
        for n in ("parent", "tokens", "tree_len", "kv_len"):
            _need(getattr(self, n), n, torch.int32, dev)
        self.B, self.T_max = (int(x) for x in self.parent.shape)
        if tuple(self.tokens.shape) != (self.B, self.T_max) or self.tree_len.numel() != self.B or \
                self.kv_len.numel() != self.B:
            raise ValueError("tree tensor shapes disagree")
        self._c = _Tree(self.parent.data_ptr(), self.tokens.data_ptr(), self.tree_len.data_ptr(),
                        self.kv_len.data_ptr(), self.B, self.T_max)


# Zero-filled workspaces, one per (function, device, stream); the kernels
# leave them zero-filled after each call. One that has become too small is kept
# (a captured graph may have its address); each new one is at least twice as
# large, so that all of them together are less than twice the last.
_WS: Dict[Tuple[str, int, int], torch.Tensor] = {}
_WS_OUTGROWN: List[torch.Tensor] = []


def _workspace(kind: str, nbytes: int, device: torch.device, stream) -> Optional[torch.Tensor]:
    if nbytes == 0:
        return None
    key = (kind, device.index if device.index is not None else torch.cuda.current_device(),
           (torch.cuda.current_stream(device) if stream is None else stream).cuda_stream)
    ws = _WS.get(key)
    if ws is None or ws.numel() < nbytes:
        if ws is not None:
            _WS_OUTGROWN.append(ws)
            nbytes = max(nbytes, 2 * ws.numel())
        with torch.cuda.stream(stream):  # filled on the stream that uses it
            ws = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        _WS[key] = ws
    return ws


def tree_verify_attn_workspace_size(kv: KVCache, tree: Tree, Hq: int) -> int:
    return int(_lib().dreams_tree_verify_attn_workspace_size(ctypes.byref(kv._c), ctypes.byref(tree._c), Hq))


def tree_verify_attn_launches(kv: KVCache, tree: Tree, Hq: int) -> int:
    """Kernel launches one tree_verify_attn call with these shapes makes."""
    return int(_lib().dreams_tree_verify_attn_launches(ctypes.byref(kv._c), ctypes.byref(tree._c), Hq))


VERIFY_STEP_LAUNCHES = 2  # dreams_verify_step: the argmax, then the walk and compaction
VERIFY_STEP_SAMPLED_LAUNCHES = 3  # draw statistics, draw selection, walk + compaction


def _cache_covers(kv: "KVCache", B: int, D: Optional[int] = None) -> None:
    """The cache holds (at least) the B sequences a call reads or writes, with
    head dim D when given."""
    if kv.B < B:
        raise ValueError(f"the KV cache holds {kv.B} sequences, the call addresses {B}")
    if D is not None and kv.D != D:
        raise ValueError(f"q's head dim {D} differs from the cache's {kv.D}")


def _q_strides(q: torch.Tensor, name: str = "q", heads: str = "Hq") -> Tuple[int, int]:
    """(sequence stride, token stride) in elements of a bf16 [B, T, Hq, D]
    query tensor whose head rows are dense (a view into a fused QKV output
    qualifies). The strides of dimensions of one token, head or column say
    nothing, and are not looked at."""
    if not isinstance(q, torch.Tensor) or q.dtype != torch.bfloat16 or q.dim() != 4:
        raise TypeError(f"{name} must be a 4-D bfloat16 tensor [B, T, {heads}, D]")
    sb, st, sh, sd = q.stride()
    _, T, H, D = q.shape
    if (sd != 1 and D > 1) or (sh != D and H > 1):
        raise ValueError(f"{name}'s head rows must be dense (strides [.., .., D, 1])")
    return sb, st if T > 1 else H * D


def tree_verify_attn(q: torch.Tensor, kv: KVCache, tree: Tree, scale: float, layer: int = 0,
                     out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                     want_lse: bool = False, workspace: Optional[torch.Tensor] = None,
                     status: Optional[torch.Tensor] = None, stream=None):
    """Tree-masked attention of the tree tokens' queries ``q`` (bf16
    [B, T_max, Hq, D], head rows dense, tokens and sequences may be strided)
    over the cache. Returns (out, lse or None); out is dense."""
    dev = q.device
    sb, stt = _q_strides(q)
    Hq = int(q.shape[2])
    if tuple(q.shape[:2]) != (tree.B, tree.T_max):
        raise ValueError(f"q must be [B, T_max, Hq, D] with the tree's B = {tree.B}, T_max = {tree.T_max}")
    _cache_covers(kv, tree.B, int(q.shape[3]))
    if out is None:
        out = _new(tuple(q.shape), torch.bfloat16, dev, stream)
    _need(out, "out", torch.bfloat16, dev)
    if tuple(out.shape) != tuple(q.shape):
        raise ValueError("out must have q's shape")
    if lse is None and want_lse:
        lse = _new(q.shape[:3], torch.float32, dev, stream)
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
        if tuple(lse.shape) != tuple(q.shape[:3]):
            raise ValueError("lse must be [B, T_max, Hq]")
    need = tree_verify_attn_workspace_size(kv, tree, Hq)
    if workspace is None:
        workspace = _workspace("attn", need, dev, stream)
    _call("dreams_tree_verify_attn", dev,
          _ptr(q), sb, stt, ctypes.byref(kv._c), layer, ctypes.byref(tree._c), Hq, float(scale), _ptr(out),
          _ptr(lse), *_ws(workspace, dev),
          _status(status, dev), _stream(stream, dev))
    return out, lse


def vocab_argmax(logits: torch.Tensor, out: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Row-wise argmax of a 2-D (or flattened leading dims) f32 / bf16 tensor."""
    x = _rows_view(logits)
    rows, V = int(x.shape[0]), int(x.shape[1])
    dev = logits.device
    if out is None:
        out = _new(logits.shape[:-1], torch.int32, dev, stream)
    _need_out(out, "out", torch.int32, dev, rows)
    need = int(_lib().dreams_vocab_argmax_workspace_size(rows, V))
    if workspace is None:
        workspace = _workspace("argmax", need, dev, stream)
    _call("dreams_vocab_argmax", dev,
          _ptr(x), F32 if x.dtype == torch.float32 else BF16, rows, V, int(x.stride(0)), _ptr(out),
          *_ws(workspace, dev), _stream(stream, dev))
    return out


def vocab_argmax_noalloc(logits: torch.Tensor, out: torch.Tensor, stream=None) -> torch.Tensor:
    """Row-wise argmax into a caller-provided ``out`` without any device
    allocation, for callers that must not allocate while it runs (see
    ``dreams_vocab_argmax_noalloc`` in include/dreams.h): the library's fixed
    scratch serves at most NOALLOC_ARGMAX_MAX_ROWS rows, and calls that overlap
    on the GPU race. Nothing here allocates: ``logits`` must flatten to
    [rows, V] as a view, and ``out`` must hold at least ``rows`` int32."""
    x = _rows_view(logits)
    rows, V = int(x.shape[0]), int(x.shape[1])
    if rows > NOALLOC_ARGMAX_MAX_ROWS:
        raise ValueError(f"{rows} rows exceed the fixed scratch of {NOALLOC_ARGMAX_MAX_ROWS} rows")
    dev = logits.device
    _need_out(out, "out", torch.int32, dev, rows)
    _call("dreams_vocab_argmax_noalloc", dev, _ptr(x), F32 if x.dtype == torch.float32 else BF16, rows, V,
          int(x.stride(0)), _ptr(out), _stream(stream, dev))
    return out


def vocab_sample(logits: torch.Tensor, temperature: float, uniforms: torch.Tensor,
                 out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
    """One draw per row of a 2-D (or flattened leading dims) f32 / bf16 tensor
    from softmax(row / temperature), by inverse transform with the row's
    uniform (``uniforms``: f32, one per row, on the same device)."""
    x = _rows_view(logits)
    rows, V = int(x.shape[0]), int(x.shape[1])
    dev = logits.device
    _need(uniforms, "uniforms", torch.float32, dev)
    if uniforms.numel() != rows:
        raise ValueError("uniforms must hold one value per row")
    if out is None:
        out = _new(logits.shape[:-1], torch.int32, dev, stream)
    _need_out(out, "out", torch.int32, dev, rows)
    need = int(_lib().dreams_vocab_sample_workspace_size(rows, V))
    if workspace is None:
        workspace = _workspace("sample", need, dev, stream)
    _call("dreams_vocab_sample", dev,
          _ptr(x), F32 if x.dtype == torch.float32 else BF16, rows, V, int(x.stride(0)), float(temperature),
          _ptr(uniforms), _ptr(out), *_ws(workspace, dev),
          _stream(stream, dev))
    return out


ATTN_FULL = 1    # query t attends slots 0 .. kv_len - 1 (cross-attention)
ATTN_CAUSAL = 2  # query t attends slots 0 .. kv_len + t (prefill self-attention)


def attention(q: torch.Tensor, kv: KVCache, q_len: torch.Tensor, kv_len: torch.Tensor, scale: float, mode: int,
              layer: int = 0, out: Optional[torch.Tensor] = None, want_lse: bool = False,
              want_entropy: bool = False, workspace: Optional[torch.Tensor] = None,
              status: Optional[torch.Tensor] = None, stream=None):
    """Attention without a tree (ATTN_FULL: the draft's cross-attention to
    target features; ATTN_CAUSAL: a layer's prefill). q: bf16 [B, T_max, Hq,
    D], head rows dense, tokens and sequences may be strided. Returns (out,
    lse, entropy); out is dense; lse and entropy are None unless asked."""
    dev = q.device
    sb, stt = _q_strides(q)
    B, T_max, Hq = int(q.shape[0]), int(q.shape[1]), int(q.shape[2])
    for n, t in (("q_len", q_len), ("kv_len", kv_len)):
        _need(t, n, torch.int32, dev)
        if t.numel() < B:
            raise ValueError(f"{n} holds {t.numel()} entries, q has {B} sequences")
    _cache_covers(kv, B, int(q.shape[3]))
    if out is None:
        out = _new(tuple(q.shape), torch.bfloat16, dev, stream)
    _need(out, "out", torch.bfloat16, dev)
    if tuple(out.shape) != tuple(q.shape):
        raise ValueError("out must have q's shape")
    lse = _new((B, T_max, Hq), torch.float32, dev, stream) if want_lse else None
    ent = _new((B, T_max, Hq), torch.float32, dev, stream) if want_entropy else None
    need = int(_lib().dreams_attention_workspace_size(ctypes.byref(kv._c), B, T_max, Hq, mode, int(want_entropy)))
    if workspace is None:
        workspace = _workspace("attention", need, dev, stream)
    _call("dreams_attention", dev, _ptr(q), sb, stt, ctypes.byref(kv._c), layer, _ptr(q_len), _ptr(kv_len), B,
          T_max, Hq, float(scale), mode, _ptr(out), _ptr(lse), _ptr(ent), *_ws(workspace, dev),
          _status(status, dev), _stream(stream, dev))
    return out, lse, ent


def lm_head_argmax(hidden: torch.Tensor, weight: torch.Tensor, out: Optional[torch.Tensor] = None,
                   out_max: Optional[torch.Tensor] = None, want_max: bool = False,
                   workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                   stream=None):
    """argmax over the vocabulary of hidden @ weight.T (bf16 [rows, K] and
    [V, K], f32 accumulation) without writing the logits. Returns the indices
    (int32 [rows]) and, with ``want_max``, the maximum logits (f32 [rows])."""
    for n, t in (("hidden", hidden), ("weight", weight)):
        if t.dtype != torch.bfloat16 or t.dim() != 2 or t.stride(1) != 1:
            raise TypeError(f"{n} must be a 2-D bf16 tensor with contiguous rows")
    if weight.device != hidden.device or weight.shape[1] != hidden.shape[1]:
        raise ValueError("hidden and weight must share the device and the hidden size")
    rows, K = int(hidden.shape[0]), int(hidden.shape[1])
    V = int(weight.shape[0])
    dev = hidden.device
    if out is None:
        out = _new(rows, torch.int32, dev, stream)
    _need_out(out, "out", torch.int32, dev, rows)
    if out_max is None and want_max:
        out_max = _new(rows, torch.float32, dev, stream)
    if out_max is not None:
        _need_out(out_max, "out_max", torch.float32, dev, rows)
    need = int(_lib().dreams_lm_head_argmax_workspace_size(rows))
    if workspace is None:
        workspace = _workspace("lm_head", need, dev, stream)
    _call("dreams_lm_head_argmax", dev, _ptr(hidden), rows, K, int(hidden.stride(0)), _ptr(weight), V,
          int(weight.stride(0)), _ptr(out), _ptr(out_max), *_ws(workspace, dev), _status(status, dev),
          _stream(stream, dev))
    return (out, out_max) if want_max or out_max is not None else out


def visual_importance(attn: torch.Tensor, v0: int, n_vis: int, r: int, workspace: Optional[torch.Tensor] = None,
                      stream=None):
    """Eq. 2 importance of the visual tokens (key positions v0 .. v0+n_vis-1)
    from attention weights [B, H, Q, K] (f32 / bf16, contiguous), and the r
    kept positions in increasing order. Returns (importance f32 [B, n_vis],
    keep int32 [B, r])."""
    if attn.dtype not in (torch.float32, torch.bfloat16) or attn.dim() != 4 or not attn.is_contiguous():
        raise TypeError("attn must be a contiguous [B, H, Q, K] float32/bfloat16 tensor")
    B, H, Q, K = (int(x) for x in attn.shape)
    dev = attn.device
    imp = _new((B, n_vis), torch.float32, dev, stream)
    keep = _new((B, r), torch.int32, dev, stream)
    need = int(_lib().dreams_visual_importance_workspace_size(B, H, Q, n_vis))
    if workspace is None:
        workspace = _workspace("importance", need, dev, stream)
    _call("dreams_visual_importance", dev, _ptr(attn), F32 if attn.dtype == torch.float32 else BF16, B, H, Q, K, v0,
          n_vis, r, _ptr(imp), _ptr(keep), *_ws(workspace, dev),
          _stream(stream, dev))
    return imp, keep


def _walk_outputs(B: int, max_path: int, dev, stream):
    return (_new(B, torch.int32, dev, stream),
            _new((B, max_path), torch.int32, dev, stream),
            _new((B, max_path), torch.int32, dev, stream),
            _new(B, torch.int32, dev, stream))


def accept_path(argmax: torch.Tensor, tree: Tree, max_path: int, status: Optional[torch.Tensor] = None,
                stream=None) -> dict:
    """Greedy acceptance over the trees. Returns a dict of device tensors."""
    dev = tree.parent.device
    _need_out(argmax, "argmax", torch.int32, dev, tree.B * tree.T_max)
    acc, path, toks, nkl = _walk_outputs(tree.B, max_path, dev, stream)
    _call("dreams_accept_path", dev, _ptr(argmax), ctypes.byref(tree._c), max_path, _ptr(acc), _ptr(path),
          _ptr(toks), _ptr(nkl), _status(status, dev), _stream(stream, dev))
    return {"accept_len": acc, "path": path, "out_tokens": toks, "new_kv_len": nkl}


def kv_compact(kv: KVCache, kv_len: torch.Tensor, accept_len: torch.Tensor, path: torch.Tensor,
               status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Moves the accepted slots into place, in all layers of ``kv``."""
    dev = kv.k.device
    for n, t in (("kv_len", kv_len), ("accept_len", accept_len), ("path", path)):
        _need(t, n, torch.int32, dev)
    if path.dim() != 2:
        raise ValueError("path must be [B, max_path]")
    B, max_path = (int(x) for x in path.shape)
    for n, t in (("kv_len", kv_len), ("accept_len", accept_len)):
        if t.numel() < B:
            raise ValueError(f"{n} holds {t.numel()} entries, path has {B} rows")
    _cache_covers(kv, B)
    _call("dreams_kv_compact", dev, ctypes.byref(kv._c), B, _ptr(kv_len), _ptr(accept_len), _ptr(path), max_path,
          _status(status, dev), _stream(stream, dev))


def verify_step_sampled_workspace_size(tree: Tree, V: int) -> int:
    return int(_lib().dreams_verify_step_sampled_workspace_size(ctypes.byref(tree._c), V))


def verify_step_workspace_size(tree: Tree, V: int) -> int:
    return int(_lib().dreams_verify_step_workspace_size(ctypes.byref(tree._c), V))


def verify_step(logits: torch.Tensor, tree: Tree, kv: KVCache, max_path: int,
                argmax_out: Optional[torch.Tensor] = None, outputs: Optional[tuple] = None,
                workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                stream=None) -> dict:
    """Argmax of the tree rows of ``logits`` ([B, T_max, V] f32/bf16), greedy
    acceptance and KV compaction, in one call (two kernel launches)."""
    dev = tree.parent.device
    if logits.dtype not in (torch.float32, torch.bfloat16) or logits.device != dev:
        raise TypeError("logits must be float32/bfloat16 on the tree's device")
    if logits.dim() != 3 or tuple(logits.shape[:2]) != (tree.B, tree.T_max) or logits.stride(-1) != 1 or \
            logits.stride(0) != logits.shape[1] * logits.stride(1):
        raise ValueError("logits must be [B, T_max, V] with uniformly strided contiguous rows")
    V = int(logits.shape[2])
    if argmax_out is not None:
        _need_out(argmax_out, "argmax_out", torch.int32, dev, tree.B * tree.T_max)
    acc, path, toks, nkl = _outputs(outputs, tree.B, max_path, dev, stream)
    st = _status(status, dev)
    _cache_covers(kv, tree.B)
    need = verify_step_workspace_size(tree, V)
    if workspace is None:
        workspace = _workspace("step", need, dev, stream)
    _call("dreams_verify_step", dev,
          _ptr(logits), F32 if logits.dtype == torch.float32 else BF16, V, int(logits.stride(1)),
          ctypes.byref(tree._c), ctypes.byref(kv._c), max_path, _ptr(argmax_out), _ptr(acc), _ptr(path),
          _ptr(toks), _ptr(nkl), *_ws(workspace, dev), st,
          _stream(stream, dev))
    return {"accept_len": acc, "path": path, "out_tokens": toks, "new_kv_len": nkl}


def verify_step_sampled(logits: torch.Tensor, tree: Tree, kv: KVCache, max_path: int, temperature: float,
                        uniforms: torch.Tensor, sample_out: Optional[torch.Tensor] = None,
                        outputs: Optional[tuple] = None, workspace: Optional[torch.Tensor] = None,
                        status: Optional[torch.Tensor] = None, stream=None) -> dict:
    """The verification tail at temperature > 0: the target's draw per tree
    node (``uniforms``: f32 [B, T_max]) takes the place of the argmax, then
    acceptance and KV compaction, in one call (three kernel launches)."""
    dev = tree.parent.device
    if logits.dtype not in (torch.float32, torch.bfloat16) or logits.device != dev:
        raise TypeError("logits must be float32/bfloat16 on the tree's device")
    if logits.dim() != 3 or tuple(logits.shape[:2]) != (tree.B, tree.T_max) or logits.stride(-1) != 1 or \
            logits.stride(0) != logits.shape[1] * logits.stride(1):
        raise ValueError("logits must be [B, T_max, V] with uniformly strided contiguous rows")
    _need(uniforms, "uniforms", torch.float32, dev)
    if tuple(uniforms.shape) != (tree.B, tree.T_max):
        raise ValueError("uniforms must be [B, T_max]")
    V = int(logits.shape[2])
    if sample_out is not None:
        _need_out(sample_out, "sample_out", torch.int32, dev, tree.B * tree.T_max)
    acc, path, toks, nkl = _outputs(outputs, tree.B, max_path, dev, stream)
    st = _status(status, dev)
    _cache_covers(kv, tree.B)
    need = verify_step_sampled_workspace_size(tree, V)
    if workspace is None:
        workspace = _workspace("step_sampled", need, dev, stream)
    _call("dreams_verify_step_sampled", dev,
          _ptr(logits), F32 if logits.dtype == torch.float32 else BF16, V, int(logits.stride(1)),
          ctypes.byref(tree._c), ctypes.byref(kv._c), max_path, float(temperature), _ptr(uniforms),
          _ptr(sample_out), _ptr(acc), _ptr(path), _ptr(toks), _ptr(nkl), *_ws(workspace, dev),
          st, _stream(stream, dev))
    return {"accept_len": acc, "path": path, "out_tokens": toks, "new_kv_len": nkl}


def verify_step_speculative(target_logits: torch.Tensor, draft_logits: torch.Tensor, tree: Tree, kv: KVCache,
                            max_path: int, temperature: float, u_accept: torch.Tensor, u_resample: torch.Tensor,
                            outputs: Optional[tuple] = None, status: Optional[torch.Tensor] = None,
                            stream=None) -> dict:
    """The verification tail at temperature > 0 by speculative sampling over
    the tree: a draft is accepted with probability min(1, r/q) against the
    current residual r, a rejection renormalises max(0, r - q), and the bonus is
    drawn from what is left (``dreams_verify_step_speculative``). target_logits
    and draft_logits: [B, T_max, V] f32/bf16 with the same strides; u_accept,
    u_resample: f32 [B, T_max]. Then acceptance outputs and KV compaction."""
    dev = tree.parent.device
    for n, t in (("target_logits", target_logits), ("draft_logits", draft_logits)):
        if t.dtype not in (torch.float32, torch.bfloat16) or t.device != dev:
            raise TypeError(f"{n} must be float32/bfloat16 on the tree's device")
        if t.dim() != 3 or tuple(t.shape[:2]) != (tree.B, tree.T_max) or t.stride(-1) != 1 or \
                t.stride(0) != t.shape[1] * t.stride(1):
            raise ValueError(f"{n} must be [B, T_max, V] with uniformly strided contiguous rows")
    if draft_logits.dtype != target_logits.dtype or draft_logits.shape != target_logits.shape or \
            draft_logits.stride() != target_logits.stride():
        raise ValueError("target and draft logits must share dtype, shape and strides")
    for n, t in (("u_accept", u_accept), ("u_resample", u_resample)):
        _need(t, n, torch.float32, dev)
        if tuple(t.shape) != (tree.B, tree.T_max):
            raise ValueError(f"{n} must be [B, T_max]")
    V = int(target_logits.shape[2])
    acc, path, toks, nkl = _outputs(outputs, tree.B, max_path, dev, stream)
    st = _status(status, dev)
    _cache_covers(kv, tree.B)
    _call("dreams_verify_step_speculative", dev,
          _ptr(target_logits), _ptr(draft_logits), F32 if target_logits.dtype == torch.float32 else BF16, V,
          int(target_logits.stride(1)), ctypes.byref(tree._c), ctypes.byref(kv._c), max_path, float(temperature),
          _ptr(u_accept), _ptr(u_resample), _ptr(acc), _ptr(path), _ptr(toks), _ptr(nkl), st,
          _stream(stream, dev))
    return {"accept_len": acc, "path": path, "out_tokens": toks, "new_kv_len": nkl}


def _launch(name: str, dev: torch.device, stream, *args) -> None:
    """_call for the calls a decode step makes many times: the device is
    switched only when another one is current, and the raw handle of the
    current stream is read without wrapping it. The stream comes last."""
    if dev.type != "cuda":
        raise ValueError(f"{name}: tensors must be on a CUDA device, got {dev}")
    if stream is None:
        s = torch._C._cuda_getCurrentRawStream(dev.index)
    elif stream.device != dev:
        raise ValueError(f"stream is on {stream.device}, the tensors on {dev}")
    else:
        s = stream.cuda_stream
    fn = getattr(_LIB or _lib(), name)
    if torch._C._cuda_getDevice() == dev.index:
        st = fn(*args, s)
    else:
        with torch.cuda.device(dev):
            st = fn(*args, s)
    if st != OK:
        raise DreamsError(name, st)


def _scratch(pool: "PagePool", workspace: Optional[torch.Tensor], dev: torch.device, stream):
    """(address, bytes) of the caller's workspace, or of the pool's own for this
    stream; nothing off the GPU, where the launch refuses."""
    if workspace is not None:
        return _ws(workspace, dev)
    if dev.type != "cuda":
        return None, 0
    s = torch._C._cuda_getCurrentRawStream(dev.index) if stream is None else stream.cuda_stream
    ws = pool._by_stream.get(s)
    if ws is None:
        if stream is not None and stream.device != dev:
            raise ValueError(f"stream is on {stream.device}, the tensors on {dev}")
        # made with the stream current: its memory is then that stream's, so what used it before is done
        # when the call runs, and what uses it after the pool is gone comes after the call
        with torch.cuda.stream(stream):
            ws = torch.empty(max(pool._reserve_bytes, pool._fork_bytes), dtype=torch.uint8, device=dev)
        ws = pool._by_stream.setdefault(s, ws)
    return ws.data_ptr(), ws.numel()


@dataclass
class PagePool:
    """The pages of a paged cache: its page table and ``refcount`` (int32
    [num_pages]: how many table entries hold each page; 0 = free). The calls
    below change both, so calls on one pool from several streams have to be ordered
    like all uses of its tensors. ``PagePool.empty(kv)`` starts with every page
    free. The pool owns the workspaces of its calls, one per stream; a captured call
    uses them at every replay, so the pool has to live as long as the graph."""
    kv: KVCache
    refcount: torch.Tensor

    def __post_init__(self):
        if self.kv.page_table is None:
            raise ValueError("a page pool needs a paged cache")
        _need(self.refcount, "refcount", torch.int32, self.kv.k.device)
        if self.refcount.numel() != self.kv.num_pages:
            raise ValueError(f"refcount must hold one entry per page ({self.kv.num_pages})")
        self.B = self.kv.B
        self._c = _PagePool(self.kv.page_table.data_ptr(), self.refcount.data_ptr(), self.kv.B,
                            self.kv.pages_per_seq, self.kv.num_pages)
        self._reserve_bytes = int(_lib().dreams_kv_reserve_workspace_size(ctypes.byref(self._c)))
        self._fork_bytes = int(_lib().dreams_kv_fork_workspace_size(ctypes.byref(self._c)))
        self._by_stream: Dict[int, torch.Tensor] = {}  # workspaces; they hold no state between calls

    @classmethod
    def empty(cls, kv: KVCache) -> "PagePool":
        if kv.page_table is None:
            raise ValueError("a page pool needs a paged cache")
        kv.page_table.fill_(-1)
        return cls(kv, torch.zeros(kv.num_pages, dtype=torch.int32, device=kv.k.device))


def _per_seq(t: torch.Tensor, name: str, B: int, dev) -> int:
    """Address of an int32 array with an entry for each of B sequences."""
    _need(t, name, torch.int32, dev)
    if t.numel() < B:
        raise ValueError(f"{name} holds {t.numel()} entries, the call addresses {B} sequences")
    return t.data_ptr()


def window_attention(q: torch.Tensor, kv: KVCache, q_len: torch.Tensor, kv_len: torch.Tensor, scale: float,
                     window: int, sinks: int = 0, parent: Optional[torch.Tensor] = None, layer: int = 0,
                     out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, want_lse: bool = False,
                     status: Optional[torch.Tensor] = None, stream=None):
    """Attention in which a query at position p sees the slots of the last
    ``window`` positions (its own among them) and of the first ``sinks`` ones.
    q: bf16 [B, T_max, Hq, D] (head rows dense, tokens and sequences may be
    strided), the queries of slots kv_len .. kv_len + q_len - 1 (q_len 0: idle);
    with ``parent`` (int32 [B, T_max]) they are the nodes of a draft tree.
    Returns (out, lse or None); rows past q_len are left untouched."""
    dev = q.device
    sb, stt = _q_strides(q)
    B, T_max, Hq, D = q.shape
    ql, kl = _per_seq(q_len, "q_len", B, dev), _per_seq(kv_len, "kv_len", B, dev)
    _cache_covers(kv, B, D)
    if kv.k.device != dev:
        raise ValueError(f"the KV cache is on {kv.k.device}, q on {dev}")
    par = None
    if parent is not None:
        _need(parent, "parent", torch.int32, dev)
        if tuple(parent.shape) != (B, T_max):
            raise ValueError("parent must be [B, T_max]")
        par = parent.data_ptr()
    if out is None:
        out = _new((B, T_max, Hq, D), torch.bfloat16, dev, stream)
    else:
        _need(out, "out", torch.bfloat16, dev)
        if out.shape != q.shape:
            raise ValueError("out must have q's shape")
    if lse is None:
        if want_lse:
            lse = _new((B, T_max, Hq), torch.float32, dev, stream)
    else:
        _need(lse, "lse", torch.float32, dev)
        if lse.shape != q.shape[:3]:
            raise ValueError("lse must be [B, T_max, Hq]")
    _launch("dreams_window_attention", dev, stream, q.data_ptr(), sb, stt, ctypes.byref(kv._c), layer, par, ql, kl, B,
            T_max, Hq, float(scale), window, sinks, out.data_ptr(), None if lse is None else lse.data_ptr(),
            None if status is None else _status(status, dev))
    return out, lse


def kv_reserve(pool: PagePool, kv_len: torch.Tensor, n_new: torch.Tensor, workspace: Optional[torch.Tensor] = None,
               status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Pages for slots kv_len .. kv_len + n_new - 1 of every sequence, where
    they have none: free pages, lowest ids first."""
    dev = pool.refcount.device
    kl, nn = _per_seq(kv_len, "kv_len", pool.B, dev), _per_seq(n_new, "n_new", pool.B, dev)
    ws, ws_bytes = _scratch(pool, workspace, dev, stream)
    _launch("dreams_kv_reserve", dev, stream, ctypes.byref(pool._c), kl, nn, ws, ws_bytes, _status(status, dev))


def kv_release(pool: PagePool, begin: torch.Tensor, end: torch.Tensor, status: Optional[torch.Tensor] = None,
               stream=None) -> None:
    """Gives back the pages wholly inside slots begin .. end - 1 of every
    sequence (eviction behind a window, an unused tail, a finished sequence)."""
    dev = pool.refcount.device
    _launch("dreams_kv_release", dev, stream, ctypes.byref(pool._c), _per_seq(begin, "begin", pool.B, dev),
            _per_seq(end, "end", pool.B, dev), _status(status, dev))


def kv_fork(pool: PagePool, parent: torch.Tensor, kv_len: torch.Tensor, new_kv_len: Optional[torch.Tensor] = None,
            workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
            stream=None) -> torch.Tensor:
    """Sequence i becomes a copy of what sequence parent[i] was (-1: empty),
    for all at once: full pages are shared, the partly filled last page is copied
    in all layers. Returns the new lengths."""
    dev = pool.refcount.device
    par, kl = _per_seq(parent, "parent", pool.B, dev), _per_seq(kv_len, "kv_len", pool.B, dev)
    if new_kv_len is None:
        new_kv_len = _new(pool.B, torch.int32, dev, stream)
    ws, ws_bytes = _scratch(pool, workspace, dev, stream)
    _launch("dreams_kv_fork", dev, stream, ctypes.byref(pool.kv._c), ctypes.byref(pool._c), par, kl,
            _per_seq(new_kv_len, "new_kv_len", pool.B, dev), ws, ws_bytes, _status(status, dev))
    return new_kv_len


KV_FORK_LAUNCHES = 2  # the table and counts, then the copies of partly filled pages


def kv_append(kv: KVCache, k_new: torch.Tensor, v_new: torch.Tensor, kv_len: torch.Tensor, n_new: torch.Tensor,
              layer: int = 0, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Writes rows k_new, v_new (bf16 [B, T_max, Hkv, D], head rows dense, the
    same strides; views of a fused projection qualify) to slots kv_len ..
    kv_len + n_new - 1 of one layer."""
    dev = kv.k.device
    sb, stt = _q_strides(k_new, "k_new", "Hkv")
    B, T_max, Hkv, D = k_new.shape
    if k_new.shape != v_new.shape or v_new.dtype != torch.bfloat16 or k_new.device != dev or v_new.device != dev:
        raise ValueError("k_new and v_new must share shape, bfloat16 and the cache's device")
    if k_new.stride() != v_new.stride():
        vb, vt = _q_strides(v_new, "v_new", "Hkv")
        if vt != stt or (vb != sb and B > 1):
            raise ValueError("k_new and v_new must share their strides")
    if Hkv != kv.Hkv:
        raise ValueError(f"k_new has {Hkv} heads, the cache {kv.Hkv}")
    _cache_covers(kv, B, D)
    _launch("dreams_kv_append", dev, stream, ctypes.byref(kv._c), layer, k_new.data_ptr(), v_new.data_ptr(), sb, stt,
            _per_seq(kv_len, "kv_len", B, dev), _per_seq(n_new, "n_new", B, dev), B, T_max, _status(status, dev))


def kv_prune(kv: KVCache, keep: torch.Tensor, v0: int, n_vis: int, kv_len: torch.Tensor,
             refcount: Optional[torch.Tensor] = None, new_kv_len: Optional[torch.Tensor] = None,
             status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Keeps the slots ``keep`` (int32 [B, r], strictly increasing, as
    visual_importance returns them) of the n_vis visual slots from v0 on and
    closes the gap, in all layers. ``refcount`` (of a page pool): refuse to
    write shared pages. Returns the new lengths, kv_len - (n_vis - r)."""
    dev = kv.k.device
    _need(keep, "keep", torch.int32, dev)
    if keep.dim() != 2:
        raise ValueError("keep must be [B, r]")
    B, r = keep.shape
    _cache_covers(kv, B)
    kl = _per_seq(kv_len, "kv_len", B, dev)
    if refcount is not None:
        if kv.page_table is None:
            raise ValueError("refcount goes with a paged cache")
        _need_out(refcount, "refcount", torch.int32, dev, kv.num_pages)
    if new_kv_len is None:
        new_kv_len = _new(B, torch.int32, dev, stream)
    _launch("dreams_kv_prune", dev, stream, ctypes.byref(kv._c), B, keep.data_ptr() if r else None, v0, n_vis, r, kl,
            None if refcount is None else refcount.data_ptr(), _per_seq(new_kv_len, "new_kv_len", B, dev),
            _status(status, dev))
    return new_kv_len


VERIFY_STEP_SPECULATIVE_LAUNCHES = 1  # one cluster per sequence: walk, residual sums, bonus, compaction


def test_set_stall(kernels: int, stall_at: int, wait_limit_ns: int = 20_000_000) -> None:
    """Test hook for the bounded pipeline waits (``dreams_test_set_stall``):
    later launches of the selected kernel families withhold their copies from
    the ``stall_at``-th tile on and give up waiting after ``wait_limit_ns``.
    ``stall_at < 0`` restores normal operation."""
    _check("dreams_test_set_stall", _lib().dreams_test_set_stall(int(kernels), int(stall_at), int(wait_limit_ns)))
