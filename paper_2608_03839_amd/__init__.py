"""Oilbird semantic draft source on AMD Instinct MI355X (gfx950).

Thin Python binding over the C ABI declared in ``include/oilbird.h``
(``liboilbird.so``, built by ``python -m paper_2608_03839_amd.build``).  Every
step of the retrieval path runs in the library's HIP kernels; this module only
marshals torch tensors (device memory) and the current torch stream into the
C calls.  There is no fallback: if the library is missing, importing the
binding's entry points raises.

Entry points carry the names of the C calls without their ``oil_`` prefix:
``pool_create``, ``pool_append``, ``pool_size``, ``query_workspace_bytes``,
``pool_query_topk``, ``gather_continuations``, ``tree_merge``; ``Pool`` bundles
a pool's buffers and handle, ``RecyclePool`` those of the rejected-branch ring
and ``KvCache`` those of the verifier's 4-bit key/value cache.  ``prompt_attend`` and
``prompt_weigh`` take whole prompts before they enter a cache, ``token_logprobs``
what the verifier answers.
"""
from __future__ import annotations

import ctypes
import math
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liboilbird.so")

OIL_F32, OIL_BF16 = 0, 1
MAX_K, MAX_B, MAX_NODES, MAX_BANDS = 64, 512, 256, 4
MAX_B_FP8 = 512
LEX_MAX_CTX, LEX_MAX_N, LEX_MAX_LEN, LEX_MAX_CAND = 32, 16, 64, 4096
LEX_MAX_HIST = 1 << 20
SCORE_ROOM_MAX = 2 << 30
REC_DEPTH, REC_MAX_OUT = 6, 8
KV_MAX_DIM, KV_MAX_HEADS, KV_MAX_GROUP = 128, 256, 64
PROMPT_MAX_ROWS, PROMPT_MAX_LD, LOGITS_MAX_ROWS = 1 << 28, 1 << 24, 1 << 23

_lib = None


class OilError(RuntimeError):
    def __init__(self, call, status):
        self.status = status
        msg = lib().oil_status_string(status).decode()
        super().__init__(f"{call} failed: {msg} (status {status})")


class DepthRule(ctypes.Structure):
    """Copy-depth rule of Eq. 3 (see oil_depth_rule)."""
    _fields_ = [("theta", ctypes.c_float), ("n_bands", ctypes.c_int32),
                ("band_min", ctypes.c_float * MAX_BANDS), ("band_depth", ctypes.c_int32 * MAX_BANDS)]

    @classmethod
    def make(cls, theta, band_min, band_depth):
        r = cls()
        r.theta = float(theta)
        r.n_bands = len(band_min)
        if len(band_min) != len(band_depth) or len(band_min) > MAX_BANDS:
            raise ValueError("band_min and band_depth must have equal length <= 4")
        for j, (m, dd) in enumerate(zip(band_min, band_depth)):
            r.band_min[j] = float(m)
            r.band_depth[j] = int(dd)
        return r

    @classmethod
    def paper(cls, theta=0.8):
        """D(s) = 48 if s >= 0.90, 8 if s >= 0.82, else 0 (Eq. 3)."""
        return cls.make(theta, [0.90, 0.82], [48, 8])

    @classmethod
    def fixed(cls, L, theta=0.8):
        """A fixed span of L tokens for every entry of a fired query."""
        return cls.make(theta, [-math.inf], [L])


def lib():
    """Load liboilbird.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2608_03839_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        P, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        sig = {
            "oil_key_stride": (i32, [i32]),
            "oil_pool_key_bytes": (sz, [i32, i64]),
            "oil_pool_create": (i32, [i32, i64, P, P, P, P, ctypes.POINTER(P)]),
            "oil_pool_key_bytes_fp8": (sz, [i32, i64]),
            "oil_pool_create_fp8": (i32, [i32, i64, P, P, P, P, P, ctypes.POINTER(P)]),
            "oil_pool_destroy": (i32, [P]),
            "oil_pool_size": (i32, [P, ctypes.POINTER(i64)]),
            "oil_pool_append": (i32, [P, P, i32, P, P, P, i64, P]),
            "oil_query_workspace_bytes": (sz, [P, i32, i32]),
            "oil_query_workspace_least_bytes": (sz, [P, i32, i32]),
            "oil_pool_query_topk": (i32, [P, P, i32, i32, i32, P, P, sz, P, P, P]),
            "oil_pool_query_topk_noalloc": (i32, [P, P, i32, i32, i32, P, P, P, P]),
            "oil_gather_continuations": (i32, [P, P, P, i32, i32, ctypes.POINTER(DepthRule), i32,
                                               P, P, P]),
            "oil_tree_merge": (i32, [i32, P, P, P, i32, i32, i32, i32, i32, P, P, i32, i32, P, P, i32,
                                     i32, i32, i32, P, P, P, P, P]),
            "oil_status_string": (ctypes.c_char_p, [i32]),
            "oil_tree_mask": (i32, [i32, i32, P, P, P, P]),
            "oil_lexical_workspace_bytes": (sz, [P, i32, i32, i32]),
            "oil_recycle_key_bytes": (sz, [i32, i64]),
            "oil_recycle_create": (i32, [i32, i64, P, P, P, P, P, ctypes.POINTER(P)]),
            "oil_recycle_destroy": (i32, [P]),
            "oil_recycle_insert_workspace_bytes": (sz, [i32, i32]),
            "oil_recycle_insert": (i32, [P, i32, i32, P, P, P, P, P, P, P, i32, P, sz, P]),
            "oil_recycle_query_workspace_bytes": (sz, [P, i32]),
            "oil_recycle_query": (i32, [P, P, i32, P, i32, ctypes.c_float, i32, i32, P, sz, P, P, P, P]),
            "oil_lexical_drafts": (i32, [P, P, P, i32, i32, P, P, P, i32, i32, i32, i32, i32, P, sz, P, P, P,
                                         P]),
            "oil_accept_walk": (i32, [i32, i32, P, P, P, P, P, P, P, P]),
            "oil_kv_bytes": (sz, [i32, i32, i32, i64]),
            "oil_kv_create": (i32, [i32, i32, i32, i64, P, P, P, P, P, ctypes.POINTER(P)]),
            "oil_kv_destroy": (i32, [P]),
            "oil_kv_reset": (i32, [P, P, i32, P]),
            "oil_kv_append": (i32, [P, P, i32, P, P, i32, i64, i32, P, P, P, P]),
            "oil_kv_append_packed": (i32, [P, P, i32, P, i64, P, P, i32, i64, P, P]),
            "oil_prompt_attend_workspace_bytes": (sz, [i32, i64, i32, i32]),
            "oil_prompt_weigh_workspace_bytes": (sz, [i32, i64, i32, i32, i64]),
            "oil_prompt_attend": (i32, [P, i32, i64, P, i64, i32, P, P, i64, i32, i32, ctypes.c_float, P, sz, P, P, P]),
            "oil_prompt_weigh": (i32, [P, i32, i64, P, i64, i32, P, P, i64, i32, i32, i64, ctypes.c_float, P, sz, P,
                                       P]),
            "oil_token_logprobs_workspace_bytes": (sz, [i32, i64, i32, i32, i32]),
            "oil_token_logprobs": (i32, [i32, i64, P, P, i32, i32, i64, P, i32, i32, P, sz, P, P, P, P, P]),
            "oil_kv_read": (i32, [P, P, i32, i64, i64, P, P, i32, P]),
            "oil_kv_attend_workspace_bytes": (sz, [P, i32, i32, i32]),
            "oil_kv_attend": (i32, [P, P, i32, P, i64, i32, P, P, i64, P, P, i32, ctypes.c_float, P, sz, P, P,
                                    P]),
            "oil_kv_weigh": (i32, [P, P, i32, P, i64, i32, P, i32, P, P, ctypes.c_float, P]),
            "oil_kv_evict_workspace_bytes": (sz, [P, i32, i64]),
            "oil_kv_evict": (i32, [P, P, i32, i64, i64, P, sz, P]),
            "oil_read_stream": (i32, [P, sz, P, P]),
            "oil_scan_timer_start": (i32, [i32, i32]),
            "oil_scan_timer_stop": (i32, [ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_double)]),
        }
        for name, (res, args) in sig.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


# ---------------------------------------------------------------- marshalling
def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if not t.is_contiguous():
        raise ValueError("contiguous tensor expected")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _dtype_code(t):
    if t.dtype == torch.float32:
        return OIL_F32
    if t.dtype == torch.bfloat16:
        return OIL_BF16
    raise ValueError(f"rows must be float32 or bfloat16, got {t.dtype}")


def _check(call, status):
    if status != 0:
        raise OilError(call, status)


def _i32(t, name):
    if t.dtype != torch.int32:
        raise ValueError(f"{name} must be int32")
    return t


def _empty(shape, dtype, device, stream=None):
    """Memory for work on ``stream``: what torch's allocator gives on another stream may
    still be in use there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _new(shape, dtype, like, stream):
    """Memory on the device of ``like`` for work on ``stream``."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _elsewhere(t, name, index):
    raise ValueError(f"{name} must be on cuda:{index}, got {t.device}")


def _shaped(t, name, shape, dtype, index):
    """Address of a dense tensor of exactly this shape and type on device ``index``, or None."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} of shape {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    if t.get_device() != index:
        _elsewhere(t, name, index)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _row_stride(t, name, index):
    """Elements between consecutive rows of a (B, N, heads, dim) tensor on device ``index``
    whose rows are dense (a slice of a fused projection's output, say)."""
    if t.get_device() != index:
        _elsewhere(t, name, index)
    B, N, H, D = t.shape
    if t.is_contiguous():
        return H * D
    if (D > 1 and t.stride(3) != 1) or (H > 1 and t.stride(2) != D):
        raise ValueError(f"{name}: the heads of a row must be dense")
    ld = t.stride(1) if N > 1 else t.stride(0) if B > 1 else H * D
    if B > 1 and t.stride(0) != N * ld:
        raise ValueError(f"{name}: requests must be as far apart as their rows")
    return ld


def _packed_stride(t, name, index):
    """Elements between consecutive rows of a (rows, heads, dim) tensor on device ``index``
    whose rows are dense."""
    shape = t.shape
    if len(shape) != 3:
        raise ValueError(f"{name} must be (rows, heads, dim), got {tuple(shape)}")
    if t.get_device() != index:
        _elsewhere(t, name, index)
    T, H, D = shape
    row, head, value = t.stride()
    if (D > 1 and value != 1) or (H > 1 and head != D):
        raise ValueError(f"{name}: the heads of a row must be dense")
    return row if T > 1 else H * D


def _stream_on(stream, index):
    """The stream's handle: torch's current one of device ``index`` by default."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(index)
    if stream.device.index != index:
        raise ValueError(f"the stream must be on cuda:{index}, got {stream.device}")
    return stream.cuda_stream


def _call_on(index, name, *args):
    """The C call with device ``index`` current, which launches go to."""
    call = getattr(lib(), name)
    if torch._C._cuda_getDevice() == index:
        status = call(*args)
    else:
        with torch.cuda.device(index):
            status = call(*args)
    _check(name, status)


def _device_of(t, name):
    index = t.get_device()
    if index < 0:
        raise ValueError(f"{name} must be on a device, got {t.device}")
    return index


# ---------------------------------------------------------------- C calls
def key_stride(dim: int) -> int:
    return lib().oil_key_stride(dim)


def pool_key_bytes(dim: int, capacity: int) -> int:
    return lib().oil_pool_key_bytes(dim, capacity)


def pool_create(dim, capacity, key_buf, token_buf, trace_buf, prompt_buf=None):
    h = ctypes.c_void_p()
    _check("oil_pool_create", lib().oil_pool_create(dim, capacity, _ptr(key_buf), _ptr(token_buf),
                                                    _ptr(trace_buf), _ptr(prompt_buf),
                                                    ctypes.byref(h)))
    return h


def pool_destroy(handle):
    _check("oil_pool_destroy", lib().oil_pool_destroy(handle))


def pool_size(handle) -> int:
    n = ctypes.c_int64()
    _check("oil_pool_size", lib().oil_pool_size(handle, ctypes.byref(n)))
    return n.value


def pool_append(handle, keys, tokens, trace_ids, prompt_ids=None, stream=None):
    n = keys.shape[0] if keys.dim() == 2 else 0
    _check("oil_pool_append", lib().oil_pool_append(
        handle, _ptr(keys), _dtype_code(keys), _ptr(_i32(tokens, "tokens")),
        _ptr(_i32(trace_ids, "trace_ids")),
        _ptr(None if prompt_ids is None else _i32(prompt_ids, "prompt_ids")), n, _stream(stream)))


def query_workspace_bytes(handle, B, k) -> int:
    return lib().oil_query_workspace_bytes(handle, B, k)


def query_workspace_least_bytes(handle, B, k) -> int:
    return lib().oil_query_workspace_least_bytes(handle, B, k)


def pool_query_topk(handle, queries, k, workspace, scores, idx, exclude_prompt=None, stream=None):
    B = queries.shape[0]
    _check("oil_pool_query_topk", lib().oil_pool_query_topk(
        handle, _ptr(queries), _dtype_code(queries), B, k,
        _ptr(None if exclude_prompt is None else _i32(exclude_prompt, "exclude_prompt")),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(scores),
        _ptr(_i32(idx, "idx")), _stream(stream)))


def pool_query_topk_noalloc(handle, queries, k, scores, idx, exclude_prompt=None, stream=None):
    """oil_pool_query_topk on the library's static scratch (no workspace)."""
    B = queries.shape[0]
    _check("oil_pool_query_topk_noalloc", lib().oil_pool_query_topk_noalloc(
        handle, _ptr(queries), _dtype_code(queries), B, k,
        _ptr(None if exclude_prompt is None else _i32(exclude_prompt, "exclude_prompt")),
        _ptr(scores), _ptr(_i32(idx, "idx")), _stream(stream)))


QUERY_SCRATCH_BYTES = 32 << 20


def lexical_workspace_bytes(handle, B, max_cand, H=0) -> int:
    return lib().oil_lexical_workspace_bytes(handle, B, max_cand, H)


def lexical_drafts(handle, ctx, ctx_len, n_lex, L_lex, workspace, lex_tokens, lex_len,
                   exclude_prompt=None, min_match=2, max_cand=LEX_MAX_CAND, stream=None, lex_capped=None,
                   hist=None, hist_len=None):
    """``hist`` (B, H) int32 device tensor or None: request b's own committed
    tokens in its first ``hist_len[b]`` entries, indexed beside the pool."""
    B, C = ctx.shape
    H = 0 if hist is None else hist.shape[1]
    _check("oil_lexical_drafts", lib().oil_lexical_drafts(
        handle, _ptr(_i32(ctx, "ctx")), _ptr(_i32(ctx_len, "ctx_len")), C, B,
        _ptr(None if exclude_prompt is None else _i32(exclude_prompt, "exclude_prompt")),
        _ptr(None if hist is None else _i32(hist, "hist")),
        _ptr(None if hist_len is None else _i32(hist_len, "hist_len")), H, n_lex,
        L_lex, min_match, max_cand, _ptr(workspace), workspace.numel() * workspace.element_size(),
        _ptr(_i32(lex_tokens, "lex_tokens")), _ptr(_i32(lex_len, "lex_len")),
        _ptr(None if lex_capped is None else _i32(lex_capped, "lex_capped")), _stream(stream)))


def gather_continuations(handle, idx, scores, rule: DepthRule, L, chain_tokens, chain_len,
                         stream=None):
    B, k = idx.shape
    _check("oil_gather_continuations", lib().oil_gather_continuations(
        handle, _ptr(_i32(idx, "idx")), _ptr(scores), B, k, ctypes.byref(rule), L,
        _ptr(chain_tokens), _ptr(chain_len), _stream(stream)))


LEX_RET, LEX_RET_LEN = 3, 32   # Algorithm 1: top-3 automaton branches, <= 32 tokens, join C


def tree_merge(anchor, lex_tokens, lex_len, lex_budget, sem_tokens, sem_len, sem_budget,
               max_nodes, node_token, node_parent, node_source, n_nodes, stream=None,
               rec_tokens=None, rec_len=None, lex_ret=None, lex_ret_len=LEX_RET_LEN):
    """Root-first merge.  ``lex_tokens`` (B, n_lex, L_lex) or None; ``sem_tokens`` (B, k, L);
    ``rec_tokens`` (B, n_rec, L_rec) recycled-pool rollouts or None.  The first
    ``lex_ret`` lexical drafts (default min(3, n_lex)), cut to ``lex_ret_len``
    tokens, re-walk the tree inside sem_budget after the retrieved chains."""
    B = anchor.shape[0]
    if lex_tokens is None or lex_tokens.shape[1] == 0:
        n_lex, L_lex, lt, ll = 0, 1, None, None
    else:
        n_lex, L_lex, lt, ll = lex_tokens.shape[1], lex_tokens.shape[2], lex_tokens, lex_len
    if rec_tokens is None or rec_tokens.shape[1] == 0:
        n_rec, L_rec, rt, rl = 0, 1, None, None
    else:
        n_rec, L_rec, rt, rl = rec_tokens.shape[1], rec_tokens.shape[2], rec_tokens, rec_len
    k, L = sem_tokens.shape[1], sem_tokens.shape[2]
    lex_ret = min(LEX_RET, n_lex) if lex_ret is None else lex_ret
    _check("oil_tree_merge", lib().oil_tree_merge(
        B, _ptr(_i32(anchor, "anchor")), _ptr(lt), _ptr(ll), n_lex, L_lex, lex_budget, lex_ret,
        lex_ret_len, _ptr(sem_tokens), _ptr(sem_len), k, L, _ptr(rt), _ptr(rl), n_rec, L_rec, sem_budget,
        max_nodes, _ptr(node_token), _ptr(node_parent), _ptr(node_source), _ptr(n_nodes),
        _stream(stream)))


def tree_mask(node_parent, n_nodes, mask=None, stream=None):
    """Ancestor mask of merged trees: (B, max_nodes, ceil(max_nodes/32)) int32 bit rows."""
    B, mx = node_parent.shape
    if mask is None:
        mask = torch.empty((B, mx, (mx + 31) // 32), dtype=torch.int32, device=node_parent.device)
    _check("oil_tree_mask", lib().oil_tree_mask(B, mx, _ptr(_i32(node_parent, "node_parent")),
                                                _ptr(_i32(n_nodes, "n_nodes")), _ptr(mask),
                                                _stream(stream)))
    return mask


def accept_walk(node_token, node_parent, n_nodes, target, out=None, stream=None):
    """Greedy acceptance: (accept_len (B,), accept_nodes (B, max_nodes), bonus (B,))."""
    B, mx = node_token.shape
    dev = node_token.device
    if out is None:
        out = (torch.empty((B,), dtype=torch.int32, device=dev),
               torch.empty((B, mx), dtype=torch.int32, device=dev),
               torch.empty((B,), dtype=torch.int32, device=dev))
    al, an, bo = out
    _check("oil_accept_walk", lib().oil_accept_walk(
        B, mx, _ptr(_i32(node_token, "node_token")), _ptr(_i32(node_parent, "node_parent")),
        _ptr(_i32(n_nodes, "n_nodes")), _ptr(_i32(target, "target")), _ptr(al), _ptr(an), _ptr(bo),
        _stream(stream)))
    return al, an, bo


def _prompt(q, k, v, starts):
    """(device, T, Hq, D, q's stride, H, k's stride, B) of packed rows of queries, keys and values."""
    index = _device_of(q, "q")
    q_ld, ld = _packed_stride(q, "q", index), _packed_stride(k, "k", index)
    T, Hq, D = q.shape
    if k.shape[0] != T or k.shape[2] != D:
        raise ValueError(f"k must be ({T}, heads, {D}), got {tuple(k.shape)}")
    if v is not None and (v.shape != k.shape or _packed_stride(v, "v", index) != ld):
        raise ValueError("k and v must have the same shape and strides")
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        if t is not None and t.dtype != torch.bfloat16:
            raise ValueError(f"{name} must be bfloat16, got {t.dtype}")
    return index, T, Hq, D, q_ld, k.shape[1], ld, starts.numel() - 1


def _room(workspace, nbytes, index, like, stream):
    """(address, bytes, tensor) of a call's workspace: the one given, torch's memory on the
    call's stream, or none where the call uses none."""
    if workspace is None:
        if nbytes <= 256:
            return None, 0, None
        workspace = _new((nbytes,), torch.uint8, like, stream)
        return workspace.data_ptr(), nbytes, workspace
    if workspace.get_device() != index:
        _elsewhere(workspace, "workspace", index)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be dense")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def prompt_attend(q, k, v, starts, scale=None, stream=None, out=None, workspace=None):
    """Causal attention of packed prompts.  ``q`` (T, Hq, D), ``k`` and ``v`` (T, H, D)
    bfloat16, whose rows may be slices of a fused projection's; ``starts`` (B + 1,) int32:
    sequence b has rows starts[b] .. starts[b + 1] - 1, and query head a reads head
    a / (Hq / H).  Returns (out (T, Hq, D) bfloat16, lse (T, Hq) float32); rows of no
    sequence are left as they were."""
    index, T, Hq, D, q_ld, H, ld, B = _prompt(q, k, v, starts)
    on = _stream_on(stream, index)
    if out is None:
        o, lse = _new((T, Hq, D), torch.bfloat16, q, stream), _new((T, Hq), torch.float32, q, stream)
        o_at, lse_at = o.data_ptr(), lse.data_ptr()
    else:
        o, lse = out
        o_at = _shaped(o, "out", (T, Hq, D), torch.bfloat16, index)
        lse_at = _shaped(lse, "lse", (T, Hq), torch.float32, index)
    at, nbytes, ws = _room(workspace, lib().oil_prompt_attend_workspace_bytes(B, T, Hq, H), index, q, stream)
    _call_on(index, "oil_prompt_attend", _shaped(starts, "starts", (B + 1,), torch.int32, index), B, T, q.data_ptr(),
             q_ld, Hq, k.data_ptr(), v.data_ptr(), ld, H, D, 1.0 / math.sqrt(D) if scale is None else scale,
             at, nbytes, o_at, lse_at, on)
    return o, lse


def prompt_weigh(q, k, lse, starts, last=None, scale=None, stream=None, out=None, workspace=None):
    """The attention weight that each position of packed prompts received from the last
    ``last`` rows (None: all) of its sequence: (H, T) float32, what append's ``weight``
    takes.  ``lse`` as prompt_attend returned it, the others as it took them."""
    index, T, Hq, D, q_ld, H, ld, B = _prompt(q, k, None, starts)
    on = _stream_on(stream, index)
    if out is None:
        out = _new((H, T), torch.float32, q, stream)
        out_at = out.data_ptr()
    else:
        out_at = _shaped(out, "out", (H, T), torch.float32, index)
    last = T if last is None else last
    at, nbytes, ws = _room(workspace, lib().oil_prompt_weigh_workspace_bytes(B, T, Hq, H, last), index, q, stream)
    _call_on(index, "oil_prompt_weigh", _shaped(starts, "starts", (B + 1,), torch.int32, index), B, T, q.data_ptr(),
             q_ld, Hq, _shaped(lse, "lse", (T, Hq), torch.float32, index), k.data_ptr(), ld, H, D, last,
             1.0 / math.sqrt(D) if scale is None else scale, at, nbytes, out_at, on)
    return out


def token_logprobs(logits, tokens=None, top=0, n_rows=None, stream=None, out=None, workspace=None):
    """Log probabilities from rows of logits (B, N, V), float32 or bfloat16: (logprob
    (B, N, M) of the given ``tokens`` (B, N, M) int32, or None without; entropy (B, N);
    the ``top`` most likely tokens (B, N, top) int32, ties to the lower one; their log
    probabilities).  ``n_rows`` (B,) int32: the rows that count; the others give -inf,
    0, -1 and -inf.  A token outside the vocabulary has -inf."""
    index, shape = _device_of(logits, "logits"), logits.shape
    if len(shape) != 3:
        raise ValueError(f"logits must be (requests, rows, vocabulary), got {tuple(shape)}")
    B, N, V = shape
    request, row, value = logits.stride()
    if V > 1 and value != 1:
        raise ValueError("logits: a row must be dense")
    ld = row if N > 1 else request if B > 1 else V
    if B > 1 and request != N * ld:
        raise ValueError("logits: requests must be as far apart as their rows")
    on, f32, i32 = _stream_on(stream, index), torch.float32, torch.int32
    M = 0
    if tokens is not None:
        if tokens.dim() != 3:
            raise ValueError(f"tokens must be (requests, rows, tokens), got {tuple(tokens.shape)}")
        M = tokens.shape[2]
    code = _dtype_code(logits)
    nbytes = lib().oil_token_logprobs_workspace_bytes(B, N, V, code, top)
    if nbytes == 0:
        raise ValueError(f"unsupported logits: {tuple(shape)} top={top}")
    if out is None:
        logprob = None if tokens is None else _new((B, N, M), f32, logits, stream)
        entropy = _new((B, N), f32, logits, stream)
        top_tokens = _new((B, N, top), i32, logits, stream)
        top_logprobs = _new((B, N, top), f32, logits, stream)
        out = logprob, entropy, top_tokens, top_logprobs
        to = [None if t is None else t.data_ptr() for t in out]
    else:
        logprob, entropy, top_tokens, top_logprobs = out
        to = (_shaped(logprob, "logprob", (B, N, M), f32, index), _shaped(entropy, "entropy", (B, N), f32, index),
              _shaped(top_tokens, "top_tokens", (B, N, top), i32, index),
              _shaped(top_logprobs, "top_logprobs", (B, N, top), f32, index))
    at, nbytes, ws = _room(workspace, nbytes, index, logits, stream)
    _call_on(index, "oil_token_logprobs", B, N, _shaped(n_rows, "n_rows", (B,), i32, index), logits.data_ptr(), code, V,
             ld, _shaped(tokens, "tokens", (B, N, M), i32, index), M, top, at, nbytes, *to, on)
    return out


def read_stream(buf, sink, stream=None):
    """Plain streaming read of a device tensor's bytes (measurement aid): the
    XOR of its 64-bit words is XOR-ed into ``sink`` (one int64 on the device)."""
    if not buf.is_cuda or not buf.is_contiguous():
        raise ValueError("read_stream: buf must be a contiguous device tensor")
    if sink.dtype != torch.int64 or sink.numel() != 1 or not sink.is_cuda:
        raise ValueError("read_stream: sink must be one int64 on the device")
    nbytes = buf.numel() * buf.element_size()
    _check("oil_read_stream", lib().oil_read_stream(_ptr(buf), nbytes, _ptr(sink), _stream(stream)))


def scan_timer_start(max_launches: int, every: int = 1):
    """Time pool scans 0, every, 2 * every, ... of the following queries (at
    most max_launches of them)."""
    _check("oil_scan_timer_start", lib().oil_scan_timer_start(max_launches, every))


def scan_timer_stop():
    """-> (number of timed scan launches, summed milliseconds)."""
    n, ms = ctypes.c_int32(), ctypes.c_double()
    _check("oil_scan_timer_stop", lib().oil_scan_timer_stop(ctypes.byref(n), ctypes.byref(ms)))
    return n.value, ms.value


# ---------------------------------------------------------------- convenience
class Pool:
    """A pool and the device buffers it lives in (torch tensors, caller-owned).

    ``key_format`` is "bf16" (the paper's half-precision store) or "fp8" (OCP
    E4M3 keys with a power-of-two scale per row)."""

    def __init__(self, dim: int, capacity: int, device="cuda", with_prompts: bool = True,
                 key_format: str = "bf16"):
        self.dim, self.capacity, self.key_format = dim, capacity, key_format
        self.device = torch.device(device)
        self.tokens = torch.empty((capacity,), dtype=torch.int32, device=self.device)
        self.traces = torch.empty((capacity,), dtype=torch.int32, device=self.device)
        self.prompts = (torch.empty((capacity,), dtype=torch.int32, device=self.device)
                        if with_prompts else None)
        if key_format == "bf16":
            self.stride = key_stride(dim)
            # tiled bf16 storage (see oil_pool_key_bytes); torch's caching allocator
            # aligns blocks to >= 512 bytes
            nbytes = pool_key_bytes(dim, capacity)
            self.keys = torch.empty((nbytes // 2,), dtype=torch.bfloat16, device=self.device)
            self.scales = None
            self.handle = pool_create(dim, capacity, self.keys, self.tokens, self.traces, self.prompts)
        elif key_format == "fp8":
            nbytes = lib().oil_pool_key_bytes_fp8(dim, capacity)
            self.stride = (dim + 127) // 128 * 128
            self.keys = torch.empty((nbytes,), dtype=torch.uint8, device=self.device)
            self.scales = torch.empty((capacity,), dtype=torch.float32, device=self.device)
            h = ctypes.c_void_p()
            _check("oil_pool_create_fp8", lib().oil_pool_create_fp8(
                dim, capacity, _ptr(self.keys), _ptr(self.scales), _ptr(self.tokens), _ptr(self.traces),
                _ptr(self.prompts), ctypes.byref(h)))
            self.handle = h
        else:
            raise ValueError(f"key_format must be 'bf16' or 'fp8', got {key_format!r}")
        self._ws = {}
        self._score_room = 0

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and _lib is not None:
            _lib.oil_pool_destroy(h)
            self.handle = None

    def __len__(self):
        return pool_size(self.handle)

    def append(self, keys, tokens, trace_ids, prompt_ids=None, stream=None):
        pool_append(self.handle, keys, tokens, trace_ids, prompt_ids, stream)

    def workspace(self, B, k):
        key = (B, k)
        if key not in self._ws:
            nb = query_workspace_bytes(self.handle, B, k)
            if nb == 0:
                raise ValueError(f"unsupported query batch/k: B={B} k={k}")
            # workspaces are kept (captured graphs hold their addresses); what they
            # hold beyond the least, room for every score, is bounded over all sizes
            least = query_workspace_least_bytes(self.handle, B, k)
            if self._score_room + nb - least > SCORE_ROOM_MAX:
                nb = least
            self._score_room += nb - least
            self._ws[key] = torch.empty((nb,), dtype=torch.uint8, device=self.device)
        return self._ws[key]

    def query_topk(self, queries, k, exclude_prompt=None, stream=None, out=None):
        B = queries.shape[0]
        if out is None:
            scores = torch.empty((B, k), dtype=torch.float32, device=self.device)
            idx = torch.empty((B, k), dtype=torch.int32, device=self.device)
        else:
            scores, idx = out
        pool_query_topk(self.handle, queries, k, self.workspace(B, k), scores, idx,
                        exclude_prompt, stream)
        return scores, idx

    def lexical(self, ctx, ctx_len, n_lex, L_lex, exclude_prompt=None, min_match=2,
                max_cand=None, stream=None, out=None, capped=None, hist=None, hist_len=None):
        """Exact-suffix lexical drafts: (tokens (B, n_lex, L_lex), lengths (B, n_lex)).
        ``capped``, a (B,) int32 device tensor or None, receives the capacity flags;
        ``hist`` (B, H) / ``hist_len`` (B,), device int32 or None, the requests'
        own committed tokens."""
        B = ctx.shape[0]
        max_cand = LEX_MAX_CAND if max_cand is None else max_cand
        H = 0 if hist is None else hist.shape[1]
        key = ("lex", B, max_cand, H)
        if key not in self._ws:
            nb = lexical_workspace_bytes(self.handle, B, max_cand, H)
            if nb == 0:
                raise ValueError(f"unsupported lexical batch/capacity/history: B={B} max_cand={max_cand} H={H}")
            self._ws[key] = torch.empty((nb,), dtype=torch.uint8, device=self.device)
        if out is None:
            lt = torch.empty((B, n_lex, L_lex), dtype=torch.int32, device=self.device)
            ll = torch.empty((B, n_lex), dtype=torch.int32, device=self.device)
        else:
            lt, ll = out
        lexical_drafts(self.handle, ctx, ctx_len, n_lex, L_lex, self._ws[key], lt, ll,
                       exclude_prompt, min_match, max_cand, stream, lex_capped=capped, hist=hist,
                       hist_len=hist_len)
        return lt, ll

    def gather(self, idx, scores, rule: DepthRule, L, stream=None, out=None):
        B, k = idx.shape
        if out is None:
            ct = torch.empty((B, k, L), dtype=torch.int32, device=self.device)
            cl = torch.empty((B, k), dtype=torch.int32, device=self.device)
        else:
            ct, cl = out
        gather_continuations(self.handle, idx, scores, rule, L, ct, cl, stream)
        return ct, cl


class RecyclePool:
    """The rejected-branch recycled pool: a ring of records over device buffers
    (torch tensors, caller-owned)."""

    def __init__(self, dim: int, capacity: int, device="cuda", stream=None):
        self.dim, self.capacity = dim, capacity
        self.device = torch.device(device)
        nbytes = lib().oil_recycle_key_bytes(dim, capacity)
        if nbytes == 0:
            raise ValueError(f"unsupported recycled pool: dim={dim} capacity={capacity}")
        self.stride = key_stride(dim)
        self.keys = torch.empty((capacity, self.stride), dtype=torch.bfloat16, device=self.device)
        self.tokens = torch.empty((capacity,), dtype=torch.int32, device=self.device)
        self.rollouts = torch.empty((capacity, 8), dtype=torch.int32, device=self.device)
        self.head = torch.empty((1,), dtype=torch.int64, device=self.device)
        h = ctypes.c_void_p()
        _check("oil_recycle_create", lib().oil_recycle_create(
            dim, capacity, _ptr(self.keys), _ptr(self.tokens), _ptr(self.rollouts), _ptr(self.head),
            _stream(stream), ctypes.byref(h)))
        self.handle = h
        self._ws = {}

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and _lib is not None:
            _lib.oil_recycle_destroy(h)
            self.handle = None

    def _workspace(self, key, nbytes):
        if nbytes == 0:
            raise ValueError(f"unsupported recycled pool call {key}")
        if key not in self._ws or self._ws[key].numel() < nbytes:
            self._ws[key] = torch.empty((nbytes,), dtype=torch.uint8, device=self.device)
        return self._ws[key]

    def insert(self, node_token, node_parent, n_nodes, target, accept_len, accept_nodes, states,
               stream=None):
        """Records of the rejected nodes of B verified trees; ``states`` is
        (B, max_nodes, dim) float32 or bfloat16."""
        B, mx = node_token.shape
        ws = self._workspace(("ins", B, mx), lib().oil_recycle_insert_workspace_bytes(B, mx))
        _check("oil_recycle_insert", lib().oil_recycle_insert(
            self.handle, B, mx, _ptr(_i32(node_token, "node_token")), _ptr(_i32(node_parent, "node_parent")),
            _ptr(_i32(n_nodes, "n_nodes")), _ptr(_i32(target, "target")), _ptr(_i32(accept_len, "accept_len")),
            _ptr(_i32(accept_nodes, "accept_nodes")), _ptr(states), _dtype_code(states), _ptr(ws),
            ws.numel(), _stream(stream)))

    def query(self, queries, anchor, theta=0.8, n_out=4, L_out=REC_DEPTH, stream=None, out=None):
        """Rollouts of the best records per request: (scores (B, n_out), tokens
        (B, n_out, L_out), lengths (B, n_out))."""
        B = queries.shape[0]
        ws = self._workspace(("q", B), lib().oil_recycle_query_workspace_bytes(self.handle, B))
        if out is None:
            sc = torch.empty((B, n_out), dtype=torch.float32, device=self.device)
            tk = torch.empty((B, n_out, L_out), dtype=torch.int32, device=self.device)
            ln = torch.empty((B, n_out), dtype=torch.int32, device=self.device)
        else:
            sc, tk, ln = out
        _check("oil_recycle_query", lib().oil_recycle_query(
            self.handle, _ptr(queries), _dtype_code(queries), _ptr(_i32(anchor, "anchor")), B,
            ctypes.c_float(theta), n_out, L_out, _ptr(ws), ws.numel(), _ptr(sc), _ptr(tk), _ptr(ln),
            _stream(stream)))
        return sc, tk, ln


class _Workspaces:
    """A stream's workspaces: beginnings of one buffer, whose size at least doubles when
    it grows.  Outgrown buffers are kept, as captured graphs may hold their addresses;
    all together stay below four times the largest need."""

    SIZES = 4096  # calls' sizes remembered

    def __init__(self):
        self.buffers, self.by_sizes = [], {}

    def get(self, key, nbytes, device, stream=None):
        if not self.buffers or self.buffers[-1].numel() < nbytes:
            least = 2 * self.buffers[-1].numel() if self.buffers else 0
            self.buffers.append(_empty((max(nbytes, least),), torch.uint8, device, stream))
        if len(self.by_sizes) >= self.SIZES:
            self.by_sizes.clear()
        ws = self.by_sizes[key] = self.buffers[-1][:nbytes]
        return ws


class KvCache:
    """One layer's committed keys and values of up to ``n_slots`` requests, held in
    4 bits, and the device buffers they live in (torch tensors, caller-owned).

    ``state`` (n_slots, 4) int32: length and next position first.  ``positions``
    and ``weights`` (n_slots, n_heads, capacity): each row's position and the
    attention weight it has accumulated (-1 and 0 past a slot's length).
    ``slots`` (B,) int32 names the slots of a call's requests (None: 0 .. B - 1).
    Every tensor and stream of a call is on the cache's device, whichever is current;
    what a call makes itself is the memory of the stream that it is given.
    Calls on one cache are ordered by the caller, as on a pool, but for ``attend``
    and ``read``, which change nothing: several may run on streams of their own.

    A stream's calls share one kept workspace, and so do the graphs captured on it:
    their replays are ordered like the calls.  ``workspace``, a dense device tensor
    of at least ``attend_workspace_bytes`` (``evict_workspace_bytes``) bytes, is
    taken in its place, so that the caches of many layers can share one."""

    def __init__(self, n_slots: int, n_heads: int, head_dim: int, capacity: int, device="cuda", stream=None):
        self.n_slots, self.n_heads, self.head_dim, self.capacity = n_slots, n_heads, head_dim, capacity
        device = torch.device(device)
        self._index = device.index if device.index is not None else torch.cuda.current_device()
        self.device = torch.device(device.type, self._index)
        nbytes = lib().oil_kv_bytes(n_slots, n_heads, head_dim, capacity)
        if nbytes == 0:
            raise ValueError(f"unsupported cache: n_slots={n_slots} n_heads={n_heads} head_dim={head_dim} "
                             f"capacity={capacity}")
        on = self._on(stream)
        self.codes = _empty((nbytes,), torch.uint8, self.device, stream)
        self.positions = _empty((n_slots, n_heads, capacity), torch.int32, self.device, stream)
        self.weights = _empty((n_slots, n_heads, capacity), torch.float32, self.device, stream)
        self.state = _empty((n_slots, 4), torch.int32, self.device, stream)
        h = ctypes.c_void_p()
        self._call("oil_kv_create", n_slots, n_heads, head_dim, capacity, _ptr(self.codes), _ptr(self.positions),
                   _ptr(self.weights), _ptr(self.state), on, ctypes.byref(h))
        self.handle = h
        self._kept = {}

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and _lib is not None:
            _lib.oil_kv_destroy(h)
            self.handle = None

    @property
    def lengths(self):
        return self.state[:, 0]

    def attend_workspace_bytes(self, B, N, n_q_heads):
        return lib().oil_kv_attend_workspace_bytes(self.handle, B, N, n_q_heads)

    def evict_workspace_bytes(self, B, keep):
        return lib().oil_kv_evict_workspace_bytes(self.handle, B, keep)

    @property
    def _ws(self):
        """Workspaces of the calls on torch's current stream, by call and sizes."""
        return self._kept_on(self._on(None)).by_sizes

    def _kept_on(self, on):
        kept = self._kept.get(on)
        if kept is None:
            kept = self._kept[on] = _Workspaces()
        return kept

    def _call(self, name, *args):
        """The C call with the cache's device current, which launches go to."""
        call = getattr(lib(), name)
        if torch._C._cuda_getDevice() == self._index:
            status = call(*args)
        else:
            with torch.cuda.device(self._index):
                status = call(*args)
        _check(name, status)

    def _workspace(self, stream, on, given, call, *sizes):
        """Address and bytes of the workspace of a call of these sizes on the stream ``on``:
        the given one, or the beginning of the stream's kept buffer."""
        if given is not None:
            if given.get_device() != self._index:
                _elsewhere(given, "workspace", self._index)
            if not given.is_contiguous():
                raise ValueError("workspace must be dense")
            return given.data_ptr(), given.numel() * given.element_size()
        kept = self._kept.get(on)
        ws = kept.by_sizes.get((call, sizes)) if kept is not None else None
        if ws is None:
            kept = self._kept_on(on)
            nbytes = getattr(self, f"{call}_workspace_bytes")(*sizes)
            if nbytes == 0:
                raise ValueError(f"unsupported cache call: {call} {sizes}")
            ws = kept.get((call, sizes), nbytes, self.device, stream)
        return ws.data_ptr(), ws.numel()

    def _on(self, stream):
        """The stream's handle: torch's current one of the cache's device by default."""
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self._index)
        if stream.device.index != self._index:
            raise ValueError(f"the stream must be on cuda:{self._index}, got {stream.device}")
        return stream.cuda_stream

    def _heads(self, t, name):
        if t.dim() != 4 or t.shape[3] != self.head_dim:
            raise ValueError(f"{name} must be (requests, rows, heads, {self.head_dim}), got {tuple(t.shape)}")
        return _row_stride(t, name, self._index)

    def _own_rows(self, k, v, what):
        """Stride of the rows k and v (B, N, n_heads, head_dim)."""
        if k.shape != v.shape or k.dtype != v.dtype or k.dim() != 4 or k.shape[2] != self.n_heads:
            raise ValueError(f"{what}: k and v must be alike, (requests, rows, {self.n_heads}, {self.head_dim})")
        ld = self._heads(k, "k")
        if self._heads(v, "v") != ld:
            raise ValueError(f"{what}: k and v must have the same strides")
        return ld

    def reset(self, slots=None, B=None, stream=None):
        """Empty the named slots (all of them when neither slots nor B is given)."""
        B = slots.shape[0] if slots is not None else self.n_slots if B is None else B
        self._call("oil_kv_reset", self.handle, _shaped(slots, "slots", (B,), torch.int32, self._index), B,
                   self._on(stream))

    def append(self, k, v, nodes=None, count=None, weight=None, slots=None, stream=None, starts=None):
        """Append rows of k, v (B, N, n_heads, head_dim), float32 or bfloat16: all
        of them, the first ``count`` (B,), or with ``nodes`` (B, N) the root and the
        accepted nodes as accept_walk returns them; ``weight`` (B, n_heads, N).

        With ``starts`` (B + 1,) int32, packed sequences: k, v (T, n_heads, head_dim),
        request b's rows starts[b] .. starts[b + 1] - 1 of them; ``weight`` (n_heads, T)
        as prompt_weigh returns it."""
        if starts is not None:
            return self._append_packed(k, v, nodes, count, weight, slots, stream, starts)
        ld = self._own_rows(k, v, "append")
        B, N = k.shape[:2]
        on, i, i32 = self._on(stream), self._index, torch.int32
        self._call("oil_kv_append", self.handle, _shaped(slots, "slots", (B,), i32, i), B, k.data_ptr(), v.data_ptr(),
                   _dtype_code(k), ld, N, _shaped(nodes, "nodes", (B, N), i32, i),
                   _shaped(count, "count", (B,), i32, i),
                   _shaped(weight, "weight", (B, self.n_heads, N), torch.float32, i), on)

    def _append_packed(self, k, v, nodes, count, weight, slots, stream, starts):
        if nodes is not None or count is not None:
            raise ValueError("append: packed sequences take neither nodes nor count")
        i, i32 = self._index, torch.int32
        if k.shape != v.shape or k.dtype != v.dtype or tuple(k.shape[1:]) != (self.n_heads, self.head_dim):
            raise ValueError(f"append: packed k and v must be alike, (rows, {self.n_heads}, {self.head_dim})")
        ld = _packed_stride(k, "k", i)
        if _packed_stride(v, "v", i) != ld:
            raise ValueError("append: k and v must have the same strides")
        T, B = k.shape[0], starts.numel() - 1
        on = self._on(stream)
        self._call("oil_kv_append_packed", self.handle, _shaped(slots, "slots", (B,), i32, i), B,
                   _shaped(starts, "starts", (B + 1,), i32, i), T, k.data_ptr(), v.data_ptr(), _dtype_code(k), ld,
                   _shaped(weight, "weight", (self.n_heads, T), torch.float32, i), on)

    def read(self, first, n, B=None, slots=None, dtype=torch.bfloat16, stream=None, out=None):
        """Rows first .. first + n - 1 as the values they stand for: (k, v), each
        (B, n_heads, n, head_dim); zeros past a slot's length."""
        B = slots.shape[0] if slots is not None else self.n_slots if B is None else B
        shape = (B, self.n_heads, n, self.head_dim)
        on, i = self._on(stream), self._index
        if out is None:
            out = tuple(_empty(shape, dtype, self.device, stream) for _ in range(2))
        k, v = out
        self._call("oil_kv_read", self.handle, _shaped(slots, "slots", (B,), torch.int32, i), B, first, n,
                   _shaped(k, "k", shape, k.dtype, i), _shaped(v, "v", shape, k.dtype, i), _dtype_code(k), on)
        return k, v

    def attend(self, q, k=None, v=None, n_nodes=None, mask=None, scale=None, slots=None, stream=None, out=None,
               workspace=None):
        """Attention of nodes q (B, N, n_q_heads, head_dim) bfloat16 over the cached
        rows and, with k and v (B, N, n_heads, head_dim), over each other: where
        ``mask`` (tree_mask's) says so, or causally.  Returns (out like q, dense,
        lse (B, N, n_q_heads) float32)."""
        q_ld = self._heads(q, "q")
        B, N, Hq, D = q.shape
        ld = 0
        if (k is None) != (v is None):
            raise ValueError("attend: k and v come together")
        if k is not None:
            ld = self._own_rows(k, v, "attend")
            if tuple(k.shape[:2]) != (B, N):
                raise ValueError("attend: k and v must have the rows of q")
        for t, name in ((q, "q"), (k, "k")):
            if t is not None and t.dtype != torch.bfloat16:
                raise ValueError(f"attend: {name} must be bfloat16, got {t.dtype}")
        scale = 1.0 / math.sqrt(D) if scale is None else scale
        on, i, i32 = self._on(stream), self._index, torch.int32
        if out is None:
            out = (_empty((B, N, Hq, D), torch.bfloat16, self.device, stream),
                   _empty((B, N, Hq), torch.float32, self.device, stream))
        o, lse = out
        ws, ws_bytes = self._workspace(stream, on, workspace, "attend", B, N, Hq)
        self._call("oil_kv_attend", self.handle, _shaped(slots, "slots", (B,), i32, i), B, q.data_ptr(), q_ld, Hq,
                   None if k is None else k.data_ptr(), None if v is None else v.data_ptr(), ld,
                   _shaped(n_nodes, "n_nodes", (B,), i32, i), _shaped(mask, "mask", (B, N, (N + 31) // 32), i32, i), N,
                   scale, ws, ws_bytes, _shaped(o, "out", (B, N, Hq, D), torch.bfloat16, i),
                   _shaped(lse, "lse", (B, N, Hq), torch.float32, i), on)
        return o, lse

    def weigh(self, q, lse, nodes=None, count=None, scale=None, slots=None, stream=None):
        """Add the attention weight of the committed rows (named as in append) of
        q, lse, as attend took and returned them, to ``weights``."""
        q_ld = self._heads(q, "q")
        B, N, Hq, D = q.shape
        if q.dtype != torch.bfloat16:
            raise ValueError(f"weigh: q must be bfloat16, got {q.dtype}")
        scale = 1.0 / math.sqrt(D) if scale is None else scale
        on, i, i32 = self._on(stream), self._index, torch.int32
        self._call("oil_kv_weigh", self.handle, _shaped(slots, "slots", (B,), i32, i), B, q.data_ptr(), q_ld, Hq,
                   _shaped(lse, "lse", (B, N, Hq), torch.float32, i), N, _shaped(nodes, "nodes", (B, N), i32, i),
                   _shaped(count, "count", (B,), i32, i), scale, on)

    def evict(self, keep, recent=0, B=None, slots=None, stream=None, workspace=None):
        """Evict every head of the named slots down to ``keep`` rows: the last
        ``recent`` positions and the heaviest others stay."""
        B = slots.shape[0] if slots is not None else self.n_slots if B is None else B
        on, i = self._on(stream), self._index
        ws, ws_bytes = self._workspace(stream, on, workspace, "evict", B, keep)
        self._call("oil_kv_evict", self.handle, _shaped(slots, "slots", (B,), torch.int32, i), B, keep, recent, ws,
                   ws_bytes, on)


def merge_trees(anchor, lex_tokens, lex_len, lex_budget, sem_tokens, sem_len, sem_budget,
                max_nodes, stream=None, out=None, rec_tokens=None, rec_len=None, lex_ret=None,
                lex_ret_len=LEX_RET_LEN):
    """Allocate outputs and run tree_merge; returns (node_token, node_parent, node_source, n_nodes)."""
    B = anchor.shape[0]
    dev = anchor.device
    if out is None:
        nt = torch.empty((B, max_nodes), dtype=torch.int32, device=dev)
        npar = torch.empty((B, max_nodes), dtype=torch.int32, device=dev)
        ns = torch.empty((B, max_nodes), dtype=torch.int8, device=dev)
        nn = torch.empty((B,), dtype=torch.int32, device=dev)
    else:
        nt, npar, ns, nn = out
    tree_merge(anchor, lex_tokens, lex_len, lex_budget, sem_tokens, sem_len, sem_budget, max_nodes,
               nt, npar, ns, nn, stream, rec_tokens, rec_len, lex_ret, lex_ret_len)
    return nt, npar, ns, nn
