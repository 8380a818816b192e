"""Thin ctypes binding of libpbd (include/pbd.h): argument marshalling only.

Every computation of the speculative step runs in the HIP library; PyTorch
provides device memory and the stream.  The functions below carry the C names
and take torch tensors (device int32 / float32) or raw pointers.  If the built
library is missing, loading fails loudly: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "lib", "libpbd.so")

PBD_OK = 0
PBD_ERR_INVALID_ARG = -1
PBD_ERR_SHAPE = -2
PBD_ERR_CAPACITY = -3
PBD_ERR_STATE = -4
PBD_ERR_HIP = -5
PBD_ERR_UNSUPPORTED = -6

PBD_DTYPE_F32 = 0
PBD_DTYPE_BF16 = 1

PBD_PASS_DEFAULT = 0
PBD_PASS_ADAPTER_ON = 1
PBD_PASS_ADAPTER_OFF = 2
PBD_PASS_MASK_BLOCK = 4
PBD_PASS_MASK_CAUSAL = 8

PBD_OPERANDS_BF16 = 0
PBD_OPERANDS_BF16X2 = 1

KCLASSES = ("gemm", "lmhead", "attn", "combine", "norm", "other", "fused")

PBD_STATUS_CAPACITY = 1
PBD_STATUS_TOKEN = 2
PBD_STATUS_FORCED_N = 4
PBD_STATUS_TIMEOUT = 8
PBD_STATUS_PAGE = 16

EXPORTED = (
    "pbd_packed_weight_bytes", "pbd_kv_bytes", "pbd_workspace_bytes", "pbd_init_weights",
    "pbd_prefill", "pbd_draft_block", "pbd_draft_block_layers", "pbd_draft_block_denoise",
    "pbd_verify_block", "pbd_verify_block_noalloc", "pbd_draft_block_unanchored", "pbd_verify_block_unanchored", "pbd_accept_commit",
    "pbd_sync_status", "pbd_set_attn_keys_per_split", "pbd_set_attn_query_split", "pbd_set_operand_precision",
    "pbd_set_pass_mode", "pbd_set_wait_limit", "pbd_profile_enable", "pbd_profile_read", "pbd_profile_stage_times", "pbd_last_error", "pbd_destroy",
    "pbd_paged_append", "pbd_paged_attention", "pbd_paged_attention_workspace_bytes", "pbd_paged_evict",
    "pbd_paged_evict_workspace_bytes", "pbd_token_logprobs", "pbd_token_logprobs_workspace_bytes",
    "pbd_context_pages", "pbd_decode_paged", "pbd_decode_paged_workspace_bytes",
)


class PbdConfig(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32), ("hidden", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("ffn", ctypes.c_int32),
        ("vocab", ctypes.c_int32), ("lora_rank", ctypes.c_int32), ("lora_alpha", ctypes.c_float),
        ("block", ctypes.c_int32), ("mask_id", ctypes.c_int32), ("rms_eps", ctypes.c_float),
        ("rope_theta", ctypes.c_float), ("qk_norm", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("max_batch", ctypes.c_int32), ("max_seq", ctypes.c_int32), ("prefill_chunk", ctypes.c_int32),
    ]


class PbdLayerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "attn_norm", "q", "k", "v", "o", "q_norm", "k_norm", "mlp_norm", "gate", "up", "down")] + [
        ("lora_a", ctypes.c_void_p * 7), ("lora_b", ctypes.c_void_p * 7)]


class PbdWeights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("final_norm", ctypes.c_void_p),
                ("layers", ctypes.POINTER(PbdLayerWeights))]


class PbdPages(ctypes.Structure):
    """pbd_pages; made by make_pages or Engine.pbd_context_pages, which keep the tensors alive."""
    _fields_ = [
        ("dtype", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32),
        ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("layer_stride", ctypes.c_int64),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("table", ctypes.c_void_p),
        ("table_width", ctypes.c_int32), ("score", ctypes.c_void_p), ("slot_pos", ctypes.c_void_p),
        ("slot_stride", ctypes.c_int64), ("state_layer_stride", ctypes.c_int64), ("status", ctypes.c_void_p),
    ]


_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load libpbd.so (built by paper_2607_12422_amd.build); raises if absent."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"PEFT-BD HIP library not built: {p} is missing "
                           "(run paper_2607_12422_amd.build.build())")
    lib = ctypes.CDLL(p)
    vp, i32, u32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_size_t
    i64, f32 = ctypes.c_int64, ctypes.c_float
    cfgp = ctypes.POINTER(PbdConfig)
    sig = {
        "pbd_packed_weight_bytes": (sz, [cfgp]),
        "pbd_kv_bytes": (sz, [cfgp]),
        "pbd_workspace_bytes": (sz, [cfgp]),
        "pbd_init_weights": (ctypes.c_int, [cfgp, ctypes.POINTER(PbdWeights), vp, sz, vp, sz, vp, sz, vp,
                                            ctypes.POINTER(vp)]),
        "pbd_prefill": (ctypes.c_int, [vp, i32, vp, vp, i32, vp, vp, vp]),
        "pbd_draft_block": (ctypes.c_int, [vp, i32, vp, vp, u32, vp, vp, vp]),
        "pbd_draft_block_layers": (ctypes.c_int, [vp, i32, vp, vp, u32, i32, vp, vp, vp]),
        "pbd_draft_block_denoise": (ctypes.c_int, [vp, i32, vp, vp, u32, i32, vp, vp, vp, vp, vp]),
        "pbd_draft_block_unanchored": (ctypes.c_int, [vp, i32, vp, vp, u32, vp, vp, vp, vp]),
        "pbd_verify_block_unanchored": (ctypes.c_int, [vp, i32, vp, vp, u32, vp, vp, vp]),
        "pbd_verify_block": (ctypes.c_int, [vp, i32, vp, vp, vp, u32, vp, vp, vp]),
        "pbd_verify_block_noalloc": (ctypes.c_int, [vp, i32, vp, vp, vp, u32, vp, vp, vp]),
        "pbd_accept_commit": (ctypes.c_int, [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]),
        "pbd_sync_status": (ctypes.c_int, [vp, vp, ctypes.POINTER(i32)]),
        "pbd_set_attn_keys_per_split": (ctypes.c_int, [vp, i32]),
        "pbd_set_attn_query_split": (ctypes.c_int, [vp, i32]),
        "pbd_set_operand_precision": (ctypes.c_int, [vp, i32]),
        "pbd_set_pass_mode": (ctypes.c_int, [vp, i32]),
        "pbd_set_wait_limit": (ctypes.c_int, [vp, i32]),
        "pbd_profile_enable": (ctypes.c_int, [vp, i32]),
        "pbd_profile_read": (ctypes.c_int, [vp, i32, ctypes.POINTER(ctypes.c_double),
                                            ctypes.POINTER(ctypes.c_int64)]),
        "pbd_profile_stage_times": (ctypes.c_int, [vp, ctypes.POINTER(ctypes.c_uint64), i32,
                                                    ctypes.POINTER(i32)]),
        "pbd_paged_append": (ctypes.c_int, [vp, i32, i32, vp, vp, vp, i64, vp, vp, vp, vp, vp, f32, vp, i32, vp, vp, vp]),
        "pbd_paged_attention_workspace_bytes": (sz, [vp, i32, i32]),
        "pbd_paged_attention": (ctypes.c_int, [vp, i32, vp, i64, vp, i32, f32, vp, vp, vp, sz, vp]),
        "pbd_paged_evict_workspace_bytes": (sz, [vp, i32, i32]),
        "pbd_paged_evict": (ctypes.c_int, [vp, i32, vp, i32, vp, vp, i32, i32, vp, vp, vp, vp, sz, vp]),
        "pbd_token_logprobs_workspace_bytes": (sz, [i32, i32, i32]),
        "pbd_token_logprobs": (ctypes.c_int, [i32, i32, i32, vp, i64, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]),
        "pbd_context_pages": (ctypes.c_int, [vp, vp]),
        "pbd_decode_paged_workspace_bytes": (sz, [vp, vp, i32, i32]),
        "pbd_decode_paged": (ctypes.c_int, [vp, vp, i32, vp, vp, vp, i32, u32, vp, vp, sz, vp]),
        "pbd_last_error": (ctypes.c_char_p, [vp]),
        "pbd_destroy": (None, [vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if path is None:
        _lib = lib
    return lib


class PbdError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{msg} (status {code})")
        self.code = code


def make_config(cfg, max_batch: int, max_seq: int, prefill_chunk: int = 0) -> PbdConfig:
    """pbd_config from a model description with the attribute names of pbd_config."""
    return PbdConfig(
        n_layers=cfg.n_layers, hidden=cfg.hidden, n_q_heads=cfg.n_q_heads, n_kv_heads=cfg.n_kv_heads,
        head_dim=cfg.head_dim, ffn=cfg.ffn, vocab=cfg.vocab, lora_rank=cfg.lora_rank,
        lora_alpha=cfg.lora_alpha, block=cfg.block, mask_id=cfg.mask_id, rms_eps=cfg.rms_eps,
        rope_theta=cfg.rope_theta, qk_norm=1 if cfg.qk_norm else 0,
        dtype=PBD_DTYPE_BF16 if cfg.dtype == "bf16" else PBD_DTYPE_F32,
        max_batch=max_batch, max_seq=max_seq, prefill_chunk=prefill_chunk)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def pbd_packed_weight_bytes(cfg: PbdConfig) -> int:
    return load_library().pbd_packed_weight_bytes(ctypes.byref(cfg))


def pbd_kv_bytes(cfg: PbdConfig) -> int:
    return load_library().pbd_kv_bytes(ctypes.byref(cfg))


def pbd_workspace_bytes(cfg: PbdConfig) -> int:
    return load_library().pbd_workspace_bytes(ctypes.byref(cfg))


def pbd_last_error(ctx=None) -> str:
    s = load_library().pbd_last_error(ctx)
    return s.decode() if s else ""


def _check(rc: int, ctx=None):
    if rc != PBD_OK:
        raise PbdError(rc, pbd_last_error(ctx))


# -- operators over a paged KV cache, and log probabilities ----------------------------
# The tensors of a call lie on one device; the stream is that device's current
# one unless another is given.  Shapes and types are checked here, because the
# library sees pointers only; the values are the library's to check.  A decode
# step makes these calls one after another with little work on the device, so
# their own time counts: messages are made where a check fails only.


def _need(ok: bool, what: str):
    if not ok:
        raise PbdError(PBD_ERR_INVALID_ARG, what)


def _dtype_id(t, what: str) -> int:
    d = str(t.dtype)
    _need(d in ("torch.float32", "torch.bfloat16"), f"{what} must be float32 or bfloat16")
    return PBD_DTYPE_BF16 if d == "torch.bfloat16" else PBD_DTYPE_F32


def _i32(t, n: int, what: str, device: int):
    """Pointer of a contiguous int32 tensor of n elements on a device (-1: the host; None: NULL)."""
    if t is None:
        return None
    if t.dtype is not _torch.int32 or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
        raise PbdError(PBD_ERR_INVALID_ARG, f"{what} must be a contiguous int32 tensor of {n} elements, with the others")
    return t.data_ptr()


def _f32(t, n: int, what: str, device: int):
    if t is None:
        return None
    if t.dtype is not _torch.float32 or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
        raise PbdError(PBD_ERR_INVALID_ARG, f"{what} must be a contiguous float32 tensor of {n} elements, with the others")
    return t.data_ptr()


def _space(ws, device: int):
    """(pointer, bytes) of a workspace tensor."""
    if ws is None or not ws.is_contiguous() or ws.get_device() != device:
        raise PbdError(PBD_ERR_INVALID_ARG, "ws must be a contiguous tensor, with the others")
    return ws.data_ptr(), ws.nbytes


def _call(device: int, stream, fn, *args, ctx=None):
    """fn(*args, stream) with the device current."""
    if device < 0:
        raise PbdError(PBD_ERR_INVALID_ARG, "the tensors must be on a GPU")
    if stream is None:
        st = _raw_stream(device)
    else:
        st = stream.cuda_stream if hasattr(stream, "cuda_stream") else stream
    if device == _torch.cuda.current_device():
        rc = fn(*args, st)
    else:
        with _torch.cuda.device(device):
            rc = fn(*args, st)
    if rc != PBD_OK:
        _check(rc, ctx)


def _raw_stream(device: int) -> int:
    """The device's current stream: torch's own short way to the handle, where it has one (0.1 us against 1.1)."""
    short = getattr(_torch._C, "_cuda_getCurrentRawStream", None)
    return short(device) if short else _torch.cuda.current_stream(device).cuda_stream


class _LazyTorch:
    """torch, imported when an operator first needs it (the module's other users may not)."""

    def __getattr__(self, name):
        import torch
        global _torch
        _torch = torch
        return getattr(torch, name)


_torch = _LazyTorch()


def make_pages(k, v, table, n_q_heads: int, head_dim: int, score=None, slot_pos=None, status=None) -> PbdPages:
    """pbd_pages of a cache of one layer, k and v [n_pages][n_kv_heads][page_size * head_dim], or of several,
    [layers][n_pages][...]; table int32 [batch][pages]; score float32 and slot_pos int32 [batch][n_kv_heads][slots]
    (layers first where k has them).  Pages and heads may have any strides, a page of a head is contiguous.  status
    int32 [1]: without it a sequence with a bad length or page is skipped silently."""
    _need(k.dim() in (3, 4) and v.shape == k.shape and v.dtype == k.dtype and v.stride() == k.stride(),
          "k and v must be alike, [n_pages][n_kv_heads][page_size * head_dim], layers first")
    _need(k.stride(-1) == 1, "a page of a head must be contiguous")
    _need(head_dim > 0 and k.shape[-1] % head_dim == 0, "a page does not hold whole positions")
    dev = k.get_device()
    p = PbdPages(dtype=_dtype_id(k, "k"), n_q_heads=n_q_heads, n_kv_heads=k.shape[-2], head_dim=head_dim,
                 page_size=k.shape[-1] // head_dim, n_pages=k.shape[-3], page_stride=k.stride(-3),
                 head_stride=k.stride(-2), layer_stride=k.stride(0) if k.dim() == 4 else 0, k=k.data_ptr(),
                 v=v.data_ptr())
    _need(v.get_device() == dev, "k and v must be on one device")
    return _attach(p, dev, k.shape[0] if k.dim() == 4 else None, table, score, slot_pos, status, (k, v))


def _attach(p: PbdPages, device: int, layers, table, score, slot_pos, status, keep) -> PbdPages:
    _need(table.dim() == 2 and table.dtype == _torch.int32 and table.is_contiguous() and table.get_device() == device,
          "table must be a contiguous int32 tensor [batch][pages] with the cache")
    p.table, p.table_width = table.data_ptr(), table.shape[1]
    B, H, slots = table.shape[0], p.n_kv_heads, None
    for t, dt, what in ((score, _torch.float32, "score"), (slot_pos, _torch.int32, "slot_pos")):
        if t is None:
            continue
        slots = t.shape[-1] if slots is None else slots
        want = (B, H, slots) if layers is None else (layers, B, H, slots)
        _need(t.dtype == dt and tuple(t.shape) == want and t.is_contiguous() and t.get_device() == device,
              f"{what} must be a contiguous {dt} tensor {list(want)} with the cache")
        setattr(p, what, t.data_ptr())
    if slots is not None:
        p.slot_stride = slots
        p.state_layer_stride = B * H * slots if layers is not None else 0
    if status is not None:
        p.status = _i32(status, 1, "status", device)
    p.keep = keep + (table, score, slot_pos, status)
    p.device, p.rows, p.layers, p.ref = device, B, layers, ctypes.byref(p)
    return p


def layer_pages(pages: PbdPages, layer: int) -> PbdPages:
    """One layer of a cache of several."""
    _need(pages.layers is not None and 0 <= layer < pages.layers, f"the cache has no layer {layer}")
    esz = 2 if pages.dtype == PBD_DTYPE_BF16 else 4
    p = PbdPages.from_buffer_copy(pages)
    p.k = pages.k + layer * pages.layer_stride * esz
    p.v = pages.v + layer * pages.layer_stride * esz
    for name in ("score", "slot_pos"):
        if getattr(pages, name):
            setattr(p, name, getattr(pages, name) + layer * pages.state_layer_stride * 4)
    p.keep, p.device, p.rows, p.layers, p.ref = pages.keep, pages.device, pages.rows, None, ctypes.byref(p)
    return p


def pbd_paged_attention_workspace_bytes(pages: PbdPages, batch: int, max_len: int) -> int:
    return load_library().pbd_paged_attention_workspace_bytes(ctypes.byref(pages), batch, max_len)


def pbd_paged_attention(pages: PbdPages, q, lens, max_len: int, out, ws, lse=None, scale: Optional[float] = None,
                        stream=None):
    """q float32 [batch][n_q_heads][head_dim] (any stride from a sequence to the next), lens int32 [batch]; out
    float32 like q, lse float32 [batch][n_q_heads].  scale: 1 / sqrt(head_dim) if None."""
    dev, HQ, D = pages.device, pages.n_q_heads, pages.head_dim
    B = lens.numel()
    if (q.dtype is not _torch.float32 or q.shape != (B, HQ, D) or q.stride(2) != 1 or (q.stride(1) != D and HQ > 1) or
            q.get_device() != dev):
        raise PbdError(PBD_ERR_INVALID_ARG,
                       "q must be float32 [batch][n_q_heads][head_dim], the heads of a sequence contiguous")
    if B > pages.rows:
        raise PbdError(PBD_ERR_INVALID_ARG, "the table has fewer rows than lens")
    w, wb = _space(ws, dev)
    _call(dev, stream, load_library().pbd_paged_attention, pages.ref, B, q.data_ptr(),
          q.stride(0) if B > 1 else HQ * D, _i32(lens, B, "lens", dev), max_len,
          D ** -0.5 if scale is None else scale, _f32(out, B * HQ * D, "out", dev), _f32(lse, B * HQ, "lse", dev), w, wb)


def _rows_at(t, strides) -> bool:
    """Whether the dimensions of more than one element have these strides."""
    return all(n == 1 or a == b for n, a, b in zip(t.shape, t.stride(), strides))


def pbd_paged_append(pages: PbdPages, k, v, lens, pos, rope, q=None, q_out=None, n_new=None, q_norm=None, k_norm=None,
                     eps: float = 1e-6, len_out=None, stream=None):
    """k, v float32 [batch][rows][n_kv_heads * head_dim] and q [batch][rows][n_q_heads * head_dim], all with the same
    stride from a row to the next (columns of one projection); lens, pos, n_new, len_out int32 [batch]; rope float32
    [positions][head_dim / 2][2]; q_norm, k_norm [head_dim] in the cache's type; q_out float32 like q, contiguous."""
    dev, H, HQ, D = pages.device, pages.n_kv_heads, pages.n_q_heads, pages.head_dim
    B, R, _ = k.shape
    # rows lie at one stride: that of the rows, or of the sequences where each has one
    stride = k.stride(1) if R > 1 else k.stride(0) if B > 1 else max(HQ, H) * D
    whole = (R * stride, stride, 1)
    for t, width, what in ((k, H * D, "k"), (v, H * D, "v"), (q, HQ * D, "q")):
        if t is not None and (t.dtype is not _torch.float32 or t.shape != (B, R, width) or t.get_device() != dev or
                              (t.stride() != whole and not _rows_at(t, whole))):
            raise PbdError(PBD_ERR_INVALID_ARG,
                           f"{what} must be float32 [batch][rows][{width}] with the row stride of k")
    if B > pages.rows:
        raise PbdError(PBD_ERR_INVALID_ARG, "the table has fewer rows than k")
    if (rope.dtype is not _torch.float32 or not rope.is_contiguous() or rope.get_device() != dev or
            rope.shape != (rope.size(0), D // 2, 2)):
        raise PbdError(PBD_ERR_INVALID_ARG, "rope must be contiguous float32 [positions][head_dim / 2][2]")
    for t, what in ((q_norm, "q_norm"), (k_norm, "k_norm")):
        if t is not None and (t.numel() != D or not t.is_contiguous() or t.get_device() != dev or
                              t.dtype is not (_torch.bfloat16 if pages.dtype == PBD_DTYPE_BF16 else _torch.float32)):
            raise PbdError(PBD_ERR_INVALID_ARG, f"{what} must be a contiguous [head_dim] tensor of the cache's type")
    _call(dev, stream, load_library().pbd_paged_append, pages.ref, B, R, _ptr(q), k.data_ptr(), v.data_ptr(),
          stride, _i32(lens, B, "lens", dev), _i32(n_new, B, "n_new", dev), _i32(pos, B, "pos", dev), _ptr(q_norm),
          _ptr(k_norm), eps, rope.data_ptr(), rope.size(0), _f32(q_out, B * R * HQ * D, "q_out", dev),
          _i32(len_out, B, "len_out", dev))


def pbd_paged_evict_workspace_bytes(pages: PbdPages, batch: int, max_len: int) -> int:
    return load_library().pbd_paged_evict_workspace_bytes(ctypes.byref(pages), batch, max_len)


def pbd_paged_evict(pages: PbdPages, lens, max_len: int, keep, new_lens, ws, pos=None, recent: int = 0, sink: int = 0,
                    score_out=None, slot_pos_out=None, stream=None):
    """lens, keep, pos, new_lens int32 [batch]; score_out, slot_pos_out like the cache's score and slot_pos, which
    they are if None."""
    dev = pages.device
    B = lens.numel()
    if B > pages.rows:
        raise PbdError(PBD_ERR_INVALID_ARG, "the table has fewer rows than lens")
    n = pages.rows * pages.n_kv_heads * pages.slot_stride
    so = pages.score if score_out is None else _f32(score_out, n, "score_out", dev)
    po = pages.slot_pos if slot_pos_out is None else _i32(slot_pos_out, n, "slot_pos_out", dev)
    w, wb = _space(ws, dev)
    _call(dev, stream, load_library().pbd_paged_evict, pages.ref, B, _i32(lens, B, "lens", dev), max_len,
          _i32(keep, B, "keep", dev), _i32(pos, B, "pos", dev), recent, sink, so, po,
          _i32(new_lens, B, "new_lens", dev), w, wb)


def pbd_token_logprobs_workspace_bytes(rows: int, vocab: int, top_n: int) -> int:
    return load_library().pbd_token_logprobs_workspace_bytes(rows, vocab, top_n)


def pbd_token_logprobs(logits, tokens, logprob, ws, entropy=None, top_ids=None, top_logprobs=None, status=None,
                       stream=None):
    """logits float32 or bfloat16 [..., vocab] (rows at one stride), tokens int32 [rows] (-1: padding) and logprob
    float32 [rows], or both None; entropy float32 [rows]; top_ids int32 and top_logprobs float32 [rows, n]; status
    int32 [1]: without it a row with a bad token is skipped silently."""
    dev = logits.get_device()
    x = logits if logits.dim() == 2 else logits.view(-1, logits.shape[-1])
    R, V = x.shape
    dt = PBD_DTYPE_F32 if x.dtype is _torch.float32 else _dtype_id(x, "logits")
    if x.stride(1) != 1 and V > 1:
        raise PbdError(PBD_ERR_INVALID_ARG, "the logits of a row must be contiguous")
    n = 0 if top_ids is None else top_ids.shape[-1]
    w, wb = _space(ws, dev)
    _call(dev, stream, load_library().pbd_token_logprobs, R, V, dt, x.data_ptr(),
          x.stride(0) if R > 1 else V, _i32(tokens, R, "tokens", dev), n, _f32(logprob, R, "logprob", dev),
          _f32(entropy, R, "entropy", dev), _i32(top_ids, R * n, "top_ids", dev),
          _f32(top_logprobs, R * n, "top_logprobs", dev), _i32(status, 1, "status", dev), w, wb)


class Engine:
    """Owns the device buffers (torch tensors) of one pbd context.

    ``weights`` is a mapping/object with the canonical weights already on the
    device (see ``upload_weights``).  Buffers are allocated with torch, so the
    library itself never allocates device memory.
    """

    def __init__(self, cfg, dev_weights, max_batch: int, max_seq: int, device="cuda:0", stream=None,
                 prefill_chunk: int = 0):
        import torch
        self.lib = load_library()
        self.cfg = cfg
        self.pcfg = make_config(cfg, max_batch, max_seq, prefill_chunk)
        self.device = torch.device(device)
        nb = self.lib.pbd_packed_weight_bytes(ctypes.byref(self.pcfg))
        if nb == 0:
            raise PbdError(PBD_ERR_SHAPE, "configuration rejected by pbd_packed_weight_bytes")
        nkv = self.lib.pbd_kv_bytes(ctypes.byref(self.pcfg))
        nws = self.lib.pbd_workspace_bytes(ctypes.byref(self.pcfg))
        self.packed = torch.empty(nb, dtype=torch.uint8, device=self.device)
        self.kv = torch.empty(nkv, dtype=torch.uint8, device=self.device)
        self.ws = torch.empty(nws, dtype=torch.uint8, device=self.device)
        self._w = dev_weights
        layers = (PbdLayerWeights * cfg.n_layers)()
        for i, lw in enumerate(dev_weights["layers"]):
            L = layers[i]
            for n in ("attn_norm", "q", "k", "v", "o", "q_norm", "k_norm", "mlp_norm", "gate", "up", "down"):
                setattr(L, n, _ptr(lw[n]))
            for j, n in enumerate(("q", "k", "v", "o", "gate", "up", "down")):
                A, B = lw["lora"][n] if cfg.lora_rank > 0 else (None, None)
                L.lora_a[j] = _ptr(A)
                L.lora_b[j] = _ptr(B)
        self._layers = layers
        pw = PbdWeights(embed=_ptr(dev_weights["embed"]), final_norm=_ptr(dev_weights["final_norm"]),
                        layers=ctypes.cast(layers, ctypes.POINTER(PbdLayerWeights)))
        ctx = ctypes.c_void_p()
        rc = self.lib.pbd_init_weights(ctypes.byref(self.pcfg), ctypes.byref(pw), _ptr(self.packed), nb,
                                       _ptr(self.kv), nkv, _ptr(self.ws), nws, _stream(stream),
                                       ctypes.byref(ctx))
        _check(rc, None)
        self.ctx = ctx.value

    # -- the C calls, same names ------------------------------------------------
    def pbd_prefill(self, tokens, lengths, max_len: int, seq_len, anchor, stream=None):
        rc = self.lib.pbd_prefill(self.ctx, int(lengths.shape[0]), _ptr(tokens), _ptr(lengths), int(max_len),
                                  _ptr(seq_len), _ptr(anchor), _stream(stream))
        _check(rc, self.ctx)

    def pbd_draft_block(self, seq_len, anchor, draft, logits=None, flags: int = PBD_PASS_DEFAULT,
                        batch: Optional[int] = None, stream=None):
        B = int(seq_len.shape[0]) if batch is None else batch
        rc = self.lib.pbd_draft_block(self.ctx, B, _ptr(seq_len), _ptr(anchor), flags, _ptr(draft),
                                      _ptr(logits), _stream(stream))
        _check(rc, self.ctx)

    def pbd_draft_block_layers(self, seq_len, anchor, draft, n_layers: int, logits=None,
                               flags: int = PBD_PASS_DEFAULT, batch: Optional[int] = None, stream=None):
        B = int(seq_len.shape[0]) if batch is None else batch
        rc = self.lib.pbd_draft_block_layers(self.ctx, B, _ptr(seq_len), _ptr(anchor), flags, int(n_layers),
                                             _ptr(draft), _ptr(logits), _stream(stream))
        _check(rc, self.ctx)

    def pbd_draft_block_denoise(self, seq_len, anchor, draft, n_steps: int, conf=None, fixed_at=None,
                                logits=None, flags: int = PBD_PASS_DEFAULT, batch: Optional[int] = None,
                                stream=None):
        B = int(seq_len.shape[0]) if batch is None else batch
        rc = self.lib.pbd_draft_block_denoise(self.ctx, B, _ptr(seq_len), _ptr(anchor), flags, int(n_steps),
                                              _ptr(draft), _ptr(conf), _ptr(fixed_at), _ptr(logits),
                                              _stream(stream))
        _check(rc, self.ctx)

    def pbd_verify_block(self, seq_len, anchor, draft, verify, logits=None, flags: int = PBD_PASS_DEFAULT,
                         batch: Optional[int] = None, stream=None):
        B = int(seq_len.shape[0]) if batch is None else batch
        rc = self.lib.pbd_verify_block(self.ctx, B, _ptr(seq_len), _ptr(anchor), _ptr(draft), flags,
                                       _ptr(verify), _ptr(logits), _stream(stream))
        _check(rc, self.ctx)

    def pbd_verify_block_noalloc(self, seq_len, anchor, draft, verify, logits=None,
                                 flags: int = PBD_PASS_DEFAULT, batch: Optional[int] = None, stream=None):
        B = int(seq_len.shape[0]) if batch is None else batch
        rc = self.lib.pbd_verify_block_noalloc(self.ctx, B, _ptr(seq_len), _ptr(anchor), _ptr(draft), flags,
                                               _ptr(verify), _ptr(logits), _stream(stream))
        _check(rc, self.ctx)

    def pbd_draft_block_unanchored(self, seq_len, anchor, draft, verify, logits=None,
                                   flags: int = PBD_PASS_DEFAULT, batch: Optional[int] = None, stream=None):
        B = int(seq_len.shape[0]) if batch is None else batch
        rc = self.lib.pbd_draft_block_unanchored(self.ctx, B, _ptr(seq_len), _ptr(anchor), flags, _ptr(draft),
                                                 _ptr(verify), _ptr(logits), _stream(stream))
        _check(rc, self.ctx)

    def pbd_verify_block_unanchored(self, seq_len, draft, verify, logits=None, flags: int = PBD_PASS_DEFAULT,
                                    batch: Optional[int] = None, stream=None):
        B = int(seq_len.shape[0]) if batch is None else batch
        rc = self.lib.pbd_verify_block_unanchored(self.ctx, B, _ptr(seq_len), _ptr(draft), flags, _ptr(verify),
                                                  _ptr(logits), _stream(stream))
        _check(rc, self.ctx)

    def pbd_accept_commit(self, draft, verify, seq_len, anchor, n_accepted, out_tokens, forced_n=None,
                          batch: Optional[int] = None, stream=None):
        B = int(seq_len.shape[0]) if batch is None else batch
        rc = self.lib.pbd_accept_commit(self.ctx, B, _ptr(draft), _ptr(verify), _ptr(forced_n), _ptr(seq_len),
                                        _ptr(anchor), _ptr(n_accepted), _ptr(out_tokens), _stream(stream))
        _check(rc, self.ctx)

    def pbd_context_pages(self, table=None, score=None, slot_pos=None) -> PbdPages:
        """The context's own cache as pages; table: every position of every sequence slot if None."""
        import torch
        p = PbdPages()
        _check(self.lib.pbd_context_pages(self.ctx, ctypes.byref(p)), self.ctx)
        if table is None:
            nblk = -(-self.pcfg.max_seq // 16)
            slots = torch.arange(self.pcfg.max_batch, dtype=torch.int32, device=self.device)[:, None]
            table = slots * (p.n_kv_heads * nblk) + torch.arange(nblk, dtype=torch.int32, device=self.device)
        return _attach(p, self.kv.get_device(), self.cfg.n_layers, table, score, slot_pos, None, (self.kv,))

    def pbd_decode_paged_workspace_bytes(self, pages: PbdPages, batch: int, max_len: int) -> int:
        return self.lib.pbd_decode_paged_workspace_bytes(self.ctx, ctypes.byref(pages), batch, max_len)

    def pbd_decode_paged(self, pages: PbdPages, token, pos, cache_len, max_len: int, ws, logits=None,
                         flags: int = PBD_PASS_DEFAULT, stream=None):
        """token, pos, cache_len int32 [batch], advanced by the call; logits float32 [batch, vocab]."""
        B, dev = token.numel(), pages.device
        _need(dev == self.kv.get_device(), "the cache must be on the context's device")
        _need(B <= pages.rows, "the table has fewer rows than token")
        _need(pages.layers in (None, self.cfg.n_layers), "the cache has not the model's layers")
        w, wb = _space(ws, dev)
        _call(dev, stream, self.lib.pbd_decode_paged, self.ctx, pages.ref, B, _i32(token, B, "token", dev),
              _i32(pos, B, "pos", dev), _i32(cache_len, B, "cache_len", dev), int(max_len), flags,
              _f32(logits, B * self.cfg.vocab, "logits", dev), w, wb, ctx=self.ctx)

    def pbd_sync_status(self, stream=None) -> int:
        st = ctypes.c_int32(0)
        rc = self.lib.pbd_sync_status(self.ctx, _stream(stream), ctypes.byref(st))
        _check(rc, self.ctx)
        return st.value

    def pbd_set_attn_keys_per_split(self, keys: int):
        _check(self.lib.pbd_set_attn_keys_per_split(self.ctx, int(keys)), self.ctx)

    def pbd_set_attn_query_split(self, mode: int):
        _check(self.lib.pbd_set_attn_query_split(self.ctx, int(mode)), self.ctx)

    def pbd_set_operand_precision(self, mode: int):
        _check(self.lib.pbd_set_operand_precision(self.ctx, int(mode)), self.ctx)

    def pbd_set_pass_mode(self, mode: int):
        _check(self.lib.pbd_set_pass_mode(self.ctx, int(mode)), self.ctx)

    def pbd_set_wait_limit(self, polls: int):
        _check(self.lib.pbd_set_wait_limit(self.ctx, int(polls)), self.ctx)

    def pbd_profile_enable(self, on: bool = True):
        _check(self.lib.pbd_profile_enable(self.ctx, 1 if on else 0), self.ctx)

    def pbd_profile_read(self, kclass: int):
        ms = ctypes.c_double(0.0)
        n = ctypes.c_int64(0)
        _check(self.lib.pbd_profile_read(self.ctx, int(kclass), ctypes.byref(ms), ctypes.byref(n)), self.ctx)
        return ms.value, n.value

    def pbd_profile_stage_times(self):
        """Stage timestamps of the last persistent pass: uint64 array [8][32][64][8][4]."""
        import numpy as np
        n = 8 * 32 * 64 * 8 * 4
        buf = (ctypes.c_uint64 * n)()
        got = ctypes.c_int32(0)
        _check(self.lib.pbd_profile_stage_times(self.ctx, buf, n, ctypes.byref(got)), self.ctx)
        return np.frombuffer(buf, dtype=np.uint64, count=got.value).reshape(8, 32, 64, 8, 4).copy()

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.pbd_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def upload_weights(w, dtype: str, device="cuda:0"):
    """Copy host weights (objects with the canonical attribute names, float32
    NumPy arrays) to device tensors of the model dtype; returns the mapping the
    Engine reads.  Values are copied unchanged (bf16 inputs must already be
    bf16-representable)."""
    import torch
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def dev(a):
        return torch.from_numpy(a).to(device=device).to(tdt).contiguous()

    layers = []
    for lw in w.layers:
        d = {n: dev(getattr(lw, n)) for n in
             ("attn_norm", "q", "k", "v", "o", "q_norm", "k_norm", "mlp_norm", "gate", "up", "down")}
        d["lora"] = {n: (dev(A), dev(B)) for n, (A, B) in lw.lora.items()}
        layers.append(d)
    return {"embed": dev(w.embed), "final_norm": dev(w.final_norm), "layers": layers}
