"""ctypes binding with the same names as the C ABI in include/ddtree.h (argument marshalling
only).  Tensors are torch tensors on the GPU; the calls enqueue on torch's current stream."""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

DTYPE_BF16 = 0
DTYPE_FP32 = 1

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.environ.get("DDTREE_LIB", os.path.join(_HERE, "libddtree.so"))
_lib = None

_vp, _sz, _i = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
_SIGNATURES = {
    "ddtree_version": (ctypes.c_int, []),
    "ddtree_error_string": (ctypes.c_char_p, [_i]),
    "ddtree_workspace_bytes": (_sz, [_i] * 8),
    "ddtree_verify_attn_workspace_bytes": (_sz, [_i] * 6 + [ctypes.c_longlong]),
    "ddtree_topk": (_i, [_vp, _i, _i, _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "ddtree_build": (_i, [_vp, _vp, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                          _sz, _vp]),
    "ddtree_verify_attn": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i,
                                ctypes.c_float, _i, _vp, _vp, _sz, _vp]),
    "ddtree_accept": (_i, [_vp, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _vp, _sz,
                           _vp]),
    "ddtree_accept_noalloc": (_i, [_vp, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _vp]),
    "ddtree_accept_sampled": (_i, [_vp, _i, _i, _i, _vp, _vp, _vp, _vp, ctypes.c_float,
                                   ctypes.c_uint64, _vp, _vp, _vp, _vp, _i, _vp, _sz, _vp]),
    "ddtree_compact": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp]),
    "ddtree_verify_attn_spans": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i,
                                      ctypes.c_float, _i, _vp, _vp, _sz, _vp]),
    "ddtree_q4_store": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _i, _vp]),
    "ddtree_q4_append": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _i, _vp]),
    "ddtree_q4_load": (_i, [_vp, _vp, _vp, _vp, _i, _vp, _vp, _i, _i, _i, _i, _vp, _vp, _vp]),
    "ddtree_sample": (_i, [_vp, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "ddtree_accept_filtered": (_i, [_vp, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _vp, _sz,
                                    _vp]),
    "ddtree_verify_attn_q4_workspace_bytes": (_sz, [_i] * 6 + [ctypes.c_longlong]),
    "ddtree_verify_attn_q4": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i,
                                   ctypes.c_float, _i, _vp, _vp, _sz, _vp]),
    "ddtree_set_build_algorithm": (_i, [_i]),
    "ddtree_selftest_host": (_i, []),
    "ddtree_build_giveups": (_i, [ctypes.POINTER(ctypes.c_uint)]),
    "ddtree_build_handovers": (_i, [ctypes.POINTER(ctypes.c_uint)]),
    "ddtree_profile_enable": (_i, [ctypes.c_uint, _i]),
    "ddtree_profile_enable_every": (_i, [ctypes.c_uint, _i, _i]),
    "ddtree_profile_reset": (_i, []),
    "ddtree_profile_read": (_i, [_i, _vp, _i]),
}

KERNELS = {"topk_chunk": 0, "topk_merge": 1, "build": 2, "attn": 3, "attn_merge": 4,
           "accept_argmax": 5, "accept_walk": 6, "attn_generic": 7, "q4_write": 8, "q4_read": 9,
           "sample_scan": 10, "sample_pick": 11, "sample_steps": 12, "sample_gather": 13,
           "sample_again": 14}


class DDTreeError(RuntimeError):
    pass


def library_path() -> str:
    return _LIB_PATH


def load():
    """Load libddtree.so; raises if it has not been built (no CPU or eager fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise DDTreeError(f"{_LIB_PATH} is missing: build it with "
                              "`python -m paper_2604_12989_amd.build` first")
        lib = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def version() -> int:
    return int(load().ddtree_version())


def error_string(code: int) -> str:
    return load().ddtree_error_string(int(code)).decode()


def _check(code: int, what: str):
    if code != 0:
        raise DDTreeError(f"{what} failed: {error_string(code)} ({code})")


def _call(name, args, result, defer):
    """Run the C entry point now, or (defer=True) return a zero-argument callable that runs it
    with the arguments marshalled once: tight loops then pay one ctypes call per stage."""
    fn = getattr(_lib or load(), name)
    if not defer:
        rc = fn(*args)
        if rc != 0:
            _check(rc, name)
        return result

    # the callable holds raw pointers: the caller keeps the tensors alive while it is in use
    keep = (args, result)

    def run():
        rc = fn(*keep[0])
        if rc != 0:
            _check(rc, name)
        return keep[1]

    return run


def _keepalive(fn, *objs):
    def run():
        return fn()
    run.keep = objs
    return run


# A call's host time is the marshalling here plus the launches (1.5-2 us each).  A decoding round that does
# not defer its calls makes one per stage and layer, and the GPU waits for the host where a call takes
# longer than its kernels.  Hence plain integers for pointers (the argtypes convert them), results made from
# an input or from one another (empty_like 1.1 us, new_empty 1.7), the raw stream handle (a torch.cuda.Stream
# object takes 3.3 us) of the device that the C level of torch names (current_device() checks more: 0.4), and the
# address of a host array through its buffer (0.3 us; its ctypes object 1.1).  Each
# result has memory of its own: views of one allocation would be 2.9 us a round cheaper, but keeping one
# would keep all.  Per call, before and now, on one
# box: top-K 13.0 -> 12.3 us, build 18.2 -> 16.2, attention 16.6 -> 15.4, walk 16.4 -> 15.4, append 7.5 -> 6.4.
def _ptr(t):
    return None if t is None else t.data_ptr()


if hasattr(torch._C, "_cuda_getCurrentRawStream") and hasattr(torch._C, "_cuda_getDevice"):
    _raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice

    def _stream():
        return _raw_stream(_device())
else:
    def _stream():
        return torch.cuda.current_stream().cuda_stream


def _dev(t, dtype, what):
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.is_contiguous()):
        raise DDTreeError(f"{what}: expected a contiguous CUDA tensor of dtype {dtype}")
    return t


def _host_i32(values, n, what):
    """Host int32 array of n entries (the array itself where it is one already: a caller that defers
    a call may change its entries in place) and its address."""
    if not (type(values) is np.ndarray and values.dtype == np.int32 and values.flags.c_contiguous):
        values = np.ascontiguousarray(np.asarray(values, dtype=np.int32))
    if values.shape != (n,):
        raise DDTreeError(what)
    return values, _address(values)


def _address(values):
    if values.size > 0 and values.flags.writeable:
        return ctypes.addressof(ctypes.c_char.from_buffer(values))
    return values.ctypes.data


def workspace_bytes(batch, B, V, N, Hq, Hkv, D, max_sum_L) -> int:
    return int(load().ddtree_workspace_bytes(batch, B, V, N, Hq, Hkv, D, max_sum_L))


def verify_attn_workspace_bytes(batch, T, Hq, Hkv, D, dtype, sum_L):
    """Scratch that one verify_attn call uses for this shape and total cache length."""
    return int(load().ddtree_verify_attn_workspace_bytes(batch, T, Hq, Hkv, D, dtype, int(sum_L)))


class Workspace:
    """Device scratch sized by ddtree_workspace_bytes (plain torch allocation)."""

    def __init__(self, batch, B, V, N, Hq, Hkv, D, max_sum_L, device="cuda"):
        n = workspace_bytes(batch, B, V, N, Hq, Hkv, D, max_sum_L)
        if n == 0:
            raise DDTreeError("unsupported shape for ddtree_workspace_bytes")
        self.nbytes = n
        self.buf = torch.empty(n + 256, dtype=torch.uint8, device=device)
        off = (-self.buf.data_ptr()) % 256
        self.ptr = self.buf.data_ptr() + off


def _ws(ws):
    if ws is None:
        return None, 0
    return ws.ptr, ws.nbytes


def topk(logits, K, ws, topk_tok=None, topk_lp=None, defer=False):
    """logits fp32 [batch,B,V] (or [B,V]) -> (topk_tok int32, topk_lp fp32) [batch,B,K]."""
    _dev(logits, torch.float32, "logits")
    x = logits if logits.dim() == 3 else logits.unsqueeze(0)
    batch, B, V = x.shape
    if topk_tok is None:
        topk_tok = x.new_empty((batch, B, K), dtype=torch.int32)
    if topk_lp is None:
        topk_lp = x.new_empty((batch, B, K))
    p, n = _ws(ws)
    args = (_ptr(x), batch, B, V, K, _ptr(topk_tok), _ptr(topk_lp), p, n, _stream())
    return _call("ddtree_topk", args, (topk_tok, topk_lp), defer)


def build(topk_tok, topk_lp, N, root_token, ws=None, out=None, defer=False):
    """Returns dict(tokens, parent, depth, rank, node_score, ancestor_mask, n_nodes)."""
    _dev(topk_tok, torch.int32, "topk_tok")
    _dev(topk_lp, torch.float32, "topk_lp")
    _dev(root_token, torch.int32, "root_token")
    batch, B, K = topk_tok.shape
    T, W = N + 1, (N + 1 + 63) // 64
    if out is None:
        like, tokens = torch.empty_like, topk_tok.new_empty((batch, T))
        out = dict(tokens=tokens, parent=like(tokens), depth=like(tokens), rank=like(tokens),
                   node_score=topk_lp.new_empty((batch, T)),
                   ancestor_mask=topk_tok.new_empty((batch, T, W), dtype=torch.int64), n_nodes=topk_tok.new_empty((batch,)))
    p, n = _ws(ws)
    args = (_ptr(topk_tok), _ptr(topk_lp), batch, B, K, N, _ptr(root_token), _ptr(out["tokens"]),
            _ptr(out["parent"]), _ptr(out["depth"]), _ptr(out.get("rank")),
            _ptr(out.get("node_score")), _ptr(out["ancestor_mask"]), _ptr(out["n_nodes"]), p, n,
            _stream())
    return _call("ddtree_build", args, out, defer)


def verify_attn(q, k_cache, v_cache, k_tree, v_tree, ancestor_mask, kv_offset, batch, T, Hq, Hkv,
                D, softmax_scale, dtype, ws, out=None, defer=False):
    """q [batch*T,Hq,D]; k/v_cache [sum_L,Hkv,D]; k/v_tree [batch*T,Hkv,D]; mask int64 [batch,T,W];
    kv_offset: host int32 sequence of batch+1 entries."""
    tdt = torch.bfloat16 if dtype == DTYPE_BF16 else torch.float32
    for name, t in (("q", q), ("k_tree", k_tree), ("v_tree", v_tree)):
        _dev(t, tdt, name)
    if k_cache is not None:
        _dev(k_cache, tdt, "k_cache")
        _dev(v_cache, tdt, "v_cache")
    _dev(ancestor_mask, torch.int64, "ancestor_mask")
    off, off_p = _host_i32(kv_offset, batch + 1, "kv_offset must have batch+1 entries")
    if out is None:
        out = torch.empty_like(q)
    p, n = _ws(ws)
    args = (_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(k_tree), _ptr(v_tree), _ptr(ancestor_mask),
            off_p, batch, T, Hq, Hkv, D, softmax_scale, dtype, _ptr(out), p, n, _stream())
    run = _call("ddtree_verify_attn", args, out, defer)
    return _keepalive(run, off) if defer else run


def verify_attn_spans(q, k_cache, v_cache, k_tree, v_tree, ancestor_mask, kv_start, kv_len, batch, T, Hq,
                      Hkv, D, softmax_scale, dtype, ws, out=None, defer=False):
    """verify_attn with sequence s owning cache rows kv_start[s] .. kv_start[s] + kv_len[s] - 1
    (host int32 sequences of batch entries each; the spans need not touch)."""
    tdt = torch.bfloat16 if dtype == DTYPE_BF16 else torch.float32
    for name, t in (("q", q), ("k_tree", k_tree), ("v_tree", v_tree)):
        _dev(t, tdt, name)
    if k_cache is not None:
        _dev(k_cache, tdt, "k_cache")
        _dev(v_cache, tdt, "v_cache")
    _dev(ancestor_mask, torch.int64, "ancestor_mask")
    start, start_p = _host_i32(kv_start, batch, "kv_start and kv_len must have batch entries each")
    length, length_p = _host_i32(kv_len, batch, "kv_start and kv_len must have batch entries each")
    if out is None:
        out = torch.empty_like(q)
    p, n = _ws(ws)
    args = (_ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(k_tree), _ptr(v_tree), _ptr(ancestor_mask),
            start_p, length_p, batch, T, Hq, Hkv, D, softmax_scale, dtype, _ptr(out), p, n, _stream())
    run = _call("ddtree_verify_attn_spans", args, out, defer)
    return _keepalive(run, start, length) if defer else run


def accept(target_logits, tokens, parent, depth, n_nodes, B, ws, out=None, want_posterior=True,
           defer=False, temperature=None, seed=0):
    """target_logits fp32 [batch,T,V] -> dict(path [batch,B+1], n_accepted, bonus_token, posterior).
    temperature=None: greedy rule (ddtree_accept); a positive temperature: sampled selection
    (ddtree_accept_sampled) with the given 64-bit seed."""
    _dev(target_logits, torch.float32, "target_logits")
    batch, T, V = target_logits.shape
    if out is None:
        i32 = torch.int32
        n_accepted = target_logits.new_empty((batch,), dtype=i32)
        out = dict(path=target_logits.new_empty((batch, B + 1), dtype=i32), n_accepted=n_accepted,
                   bonus_token=torch.empty_like(n_accepted),
                   posterior=target_logits.new_empty((batch, T), dtype=i32) if want_posterior else None)
    p, n = _ws(ws)
    if temperature is not None:
        args = (_ptr(target_logits), batch, T, V, _ptr(tokens), _ptr(parent), _ptr(depth),
                _ptr(n_nodes), float(temperature), int(seed) & 0xFFFFFFFFFFFFFFFF,
                _ptr(out["path"]), _ptr(out["n_accepted"]), _ptr(out["bonus_token"]),
                _ptr(out.get("posterior")), B, p, n, _stream())
        return _call("ddtree_accept_sampled", args, out, defer)
    args = (_ptr(target_logits), batch, T, V, _ptr(tokens), _ptr(parent), _ptr(depth),
            _ptr(n_nodes), _ptr(out["path"]), _ptr(out["n_accepted"]), _ptr(out["bonus_token"]),
            _ptr(out.get("posterior")), B, p, n, _stream())
    return _call("ddtree_accept", args, out, defer)


def accept_noalloc(target_logits, tokens, parent, depth, n_nodes, B, out, defer=False):
    """ddtree_accept_noalloc: the greedy walk with its scratch in the library's static device
    array.  `out` (dict of path, n_accepted, bonus_token, posterior-or-None) is supplied by the
    caller: this path allocates nothing, here or in the library."""
    _dev(target_logits, torch.float32, "target_logits")
    batch, T, V = target_logits.shape
    args = (_ptr(target_logits), batch, T, V, _ptr(tokens), _ptr(parent), _ptr(depth),
            _ptr(n_nodes), _ptr(out["path"]), _ptr(out["n_accepted"]), _ptr(out["bonus_token"]),
            _ptr(out.get("posterior")), B, _stream())
    return _call("ddtree_accept_noalloc", args, out, defer)


def compact(k_tree, v_tree, path, n_accepted, dst_row, batch, T, B, Hkv, D, k_cache, v_cache):
    """Append the accepted tree rows of K and V to the caches in place."""
    dst, dst_p = _host_i32(dst_row, batch, "dst_row must have batch entries")
    _check(load().ddtree_compact(_ptr(k_tree), _ptr(v_tree), _ptr(path), _ptr(n_accepted), dst_p, batch, T, B,
                                 Hkv, D, k_tree.element_size(), _ptr(k_cache), _ptr(v_cache), _stream()),
           "ddtree_compact")


def _options(batch, temperature, top_k, top_p, min_p):
    """Sampling options as host arrays of batch entries (a scalar stands for all sequences) and their addresses."""
    def one(v, dtype, what):
        if not (type(v) is np.ndarray and v.dtype == dtype and v.flags.c_contiguous):
            v = np.asarray(v, dtype=dtype)
            v = np.full(batch, v, dtype) if v.ndim == 0 else np.ascontiguousarray(v)
        if v.shape != (batch,):
            raise DDTreeError(f"{what}: expected a number, or one for each of the {batch} sequences")
        return v
    arrays = (one(temperature, np.float32, "temperature"), one(top_k, np.int32, "top_k"), one(top_p, np.float32, "top_p"),
              one(min_p, np.float32, "min_p"))
    return arrays, tuple(_address(a) for a in arrays)


def sample(logits, uniforms, ws, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out=None, defer=False):
    """One token per row: logits fp32 [batch, T, V] (or [batch, V]), uniforms fp32 of a number a row -> int32 tokens like uniforms.
    Options: a number, or one for each sequence; temperature 0 is greedy, top_k 0, top_p 1 and min_p 0 are off."""
    _dev(logits, torch.float32, "logits")
    _dev(uniforms, torch.float32, "uniforms")
    if logits.dim() not in (2, 3) or uniforms.numel() * logits.shape[-1] != logits.numel():
        raise DDTreeError("logits must be [batch, T, V] or [batch, V], with one uniform a row")
    batch, T, V = logits.shape if logits.dim() == 3 else (logits.shape[0], 1, logits.shape[1])
    if out is None:
        out = torch.empty_like(uniforms, dtype=torch.int32)
    _dev(out, torch.int32, "out")
    if out.numel() != batch * T or len({t.get_device() for t in (logits, uniforms, out)}) != 1:
        raise DDTreeError("out: expected an entry a row, all tensors on one device")
    _current(logits.get_device())
    arrays, ptrs = _options(batch, temperature, top_k, top_p, min_p)
    p, n = _ws(ws)
    args = (_ptr(logits), batch, T, V, *ptrs, _ptr(uniforms), _ptr(out), p, n, _stream())
    run = _call("ddtree_sample", args, out, defer)
    return _keepalive(run, arrays) if defer else run


def accept_filtered(target_logits, tokens, parent, depth, n_nodes, B, uniforms, ws, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0,
                    out=None, want_posterior=True, defer=False):
    """accept() with the target's tokens selected as sample() does, one uniform fp32 [batch, T] a node."""
    _dev(target_logits, torch.float32, "target_logits")
    _dev(uniforms, torch.float32, "uniforms")
    batch, T, V = target_logits.shape
    if uniforms.numel() != batch * T or uniforms.get_device() != target_logits.get_device():
        raise DDTreeError("uniforms must be [batch, T], on the device of target_logits")
    for name, t, count in (("tokens", tokens, batch * T), ("parent", parent, batch * T), ("depth", depth, batch * T), ("n_nodes", n_nodes, batch)):
        _dev(t, torch.int32, name)
        if t.numel() != count or t.get_device() != target_logits.get_device():
            raise DDTreeError(f"{name}: expected {count} entries on the device of target_logits")
    _current(target_logits.get_device())
    if out is None:
        n_accepted = torch.empty_like(n_nodes)
        out = dict(path=n_nodes.new_empty((batch, B + 1)), n_accepted=n_accepted, bonus_token=torch.empty_like(n_accepted),
                   posterior=torch.empty_like(tokens) if want_posterior else None)
    else:
        for name, count in (("path", batch * (B + 1)), ("n_accepted", batch), ("bonus_token", batch), ("posterior", batch * T)):
            t = out.get(name)
            if t is None and name == "posterior":
                continue
            if _dev(t, torch.int32, name).numel() != count or t.get_device() != target_logits.get_device():
                raise DDTreeError(f"{name}: expected {count} entries on the device of target_logits")
    arrays, ptrs = _options(batch, temperature, top_k, top_p, min_p)
    p, n = _ws(ws)
    args = (_ptr(target_logits), batch, T, V, _ptr(tokens), _ptr(parent), _ptr(depth), _ptr(n_nodes), *ptrs, _ptr(uniforms),
            _ptr(out["path"]), _ptr(out["n_accepted"]), _ptr(out["bonus_token"]), _ptr(out.get("posterior")), B, p, n, _stream())
    run = _call("ddtree_accept_filtered", args, out, defer)
    return _keepalive(run, arrays) if defer else run


def _current(device):
    """The calls launch on the current device's stream."""
    if device != _device():
        raise DDTreeError(f"the tensors are on device {device}, which is not the current one")


class CacheQ4:
    """A KV cache in 4 bits (format: ddtree.h): codes uint8 [Hkv, rows, D/2] and scales uint8 [Hkv, rows, D/32] of K and V.
    CacheQ4.empty allocates one; the constructor takes the four tensors."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        for name, t in (("k_codes", k_codes), ("k_scales", k_scales), ("v_codes", v_codes), ("v_scales", v_scales)):
            _dev(t, torch.uint8, name)
        if k_codes.dim() != 3:
            raise DDTreeError("k_codes: expected [Hkv, rows, D/2]")
        Hkv, rows, half = k_codes.shape
        if half % 16 != 0 or v_codes.shape != k_codes.shape or k_scales.shape != (Hkv, rows, half // 16) or \
                v_scales.shape != k_scales.shape:
            raise DDTreeError("codes are [Hkv, rows, D/2] and scales [Hkv, rows, D/32], D a multiple of 32")
        if len({t.device for t in (k_codes, k_scales, v_codes, v_scales)}) != 1:
            raise DDTreeError("the tensors of a cache are on one device")
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        self.Hkv, self.rows, self.D, self.device = Hkv, rows, 2 * half, k_codes.get_device()
        self.row = torch.Size((Hkv, 2 * half))  # of a tensor of keys or values
        self.ptrs = (_ptr(k_codes), _ptr(k_scales), _ptr(v_codes), _ptr(v_scales))

    @classmethod
    def empty(cls, rows, Hkv, D, device="cuda"):
        def bytes_(width):
            return torch.empty((Hkv, rows, width), dtype=torch.uint8, device=device)
        return cls(bytes_(D // 2), bytes_(D // 32), bytes_(D // 2), bytes_(D // 32))


_ROW_DTYPE = {torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_FP32}


def _rows(t, cache, what):
    """A tensor of K or V rows that goes with the cache; its DTYPE_*."""
    dtype = _ROW_DTYPE.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if dtype is None or not t.is_cuda or t.shape[1:] != cache.row or not t.is_contiguous() or t.get_device() != cache.device:
        raise DDTreeError(f"{what}: expected a contiguous bfloat16 or float32 tensor [rows, {cache.Hkv}, {cache.D}] on the cache's device")
    _current(cache.device)
    return dtype


def q4_store(k, v, src_offset, dst_row, cache, defer=False):
    """Prompts into the cache: rows src_offset[s] .. src_offset[s+1] - 1 of k / v [rows, Hkv, D] become the rows from
    dst_row[s] on (host int32 sequences of batch+1 and batch entries)."""
    dtype = _rows(k, cache, "k")
    if _rows(v, cache, "v") != dtype or v.shape[0] != k.shape[0]:
        raise DDTreeError("k and v differ in rows or dtype")
    batch = len(dst_row)
    off, off_p = _host_i32(src_offset, batch + 1, "src_offset must have one entry more than dst_row")
    dst, dst_p = _host_i32(dst_row, batch, "dst_row must be one-dimensional")
    if batch and int(off[-1]) > k.shape[0]:
        raise DDTreeError("src_offset names rows past the end of k and v")
    args = (_ptr(k), _ptr(v), off_p, dst_p, batch, cache.Hkv, cache.D, dtype, *cache.ptrs, cache.rows, _stream())
    run = _call("ddtree_q4_store", args, cache, defer)
    return _keepalive(run, off, dst, k, v) if defer else run


def q4_append(k_tree, v_tree, path, n_accepted, dst_row, batch, T, B, cache, defer=False):
    """compact() into a 4-bit cache: the accepted tree rows are quantised behind each sequence."""
    dtype = _rows(k_tree, cache, "k_tree")
    if _rows(v_tree, cache, "v_tree") != dtype or v_tree.shape[0] != batch * T or k_tree.shape[0] != batch * T:
        raise DDTreeError("k_tree and v_tree: expected batch*T rows of one dtype")
    _dev(path, torch.int32, "path")
    _dev(n_accepted, torch.int32, "n_accepted")
    if path.numel() != batch * (B + 1) or n_accepted.numel() != batch:
        raise DDTreeError("path must be [batch, B+1] and n_accepted [batch]")
    dst, dst_p = _host_i32(dst_row, batch, "dst_row must have batch entries")
    args = (_ptr(k_tree), _ptr(v_tree), _ptr(path), _ptr(n_accepted), dst_p, batch, T, B, cache.Hkv, cache.D, dtype,
            *cache.ptrs, cache.rows, _stream())
    run = _call("ddtree_q4_append", args, cache, defer)
    return _keepalive(run, dst) if defer else run


def q4_load(cache, src_row, dst_offset, dtype=torch.bfloat16, out=None, defer=False):
    """Rows of the cache as tensors (k, v) [dst_offset[batch], Hkv, D] of dtype bfloat16 or float32: sequence s gives its
    rows from src_row[s] on as rows dst_offset[s] .. dst_offset[s+1] - 1."""
    batch = len(src_row)
    src, src_p = _host_i32(src_row, batch, "src_row must be one-dimensional")
    off, off_p = _host_i32(dst_offset, batch + 1, "dst_offset must have one entry more than src_row")
    if out is None:
        if dtype not in _ROW_DTYPE:
            raise DDTreeError("dtype: expected torch.bfloat16 or torch.float32")
        k = cache.k_codes.new_empty((int(off[-1]), cache.Hkv, cache.D), dtype=dtype)
        out = k, torch.empty_like(k)
    k, v = out
    code = _rows(k, cache, "k")
    if _rows(v, cache, "v") != code or min(k.shape[0], v.shape[0]) < int(off[-1]):
        raise DDTreeError("k and v differ in dtype, or have fewer rows than dst_offset names")
    args = (*cache.ptrs, cache.rows, src_p, off_p, batch, cache.Hkv, cache.D, code, _ptr(k), _ptr(v), _stream())
    run = _call("ddtree_q4_load", args, out, defer)
    return _keepalive(run, src, off) if defer else run


def verify_attn_q4_workspace_bytes(batch, T, Hq, Hkv, D, dtype, sum_L):
    """Scratch that one verify_attn_q4 call uses for this shape and total cache length."""
    return int(load().ddtree_verify_attn_q4_workspace_bytes(batch, T, Hq, Hkv, D, dtype, int(sum_L)))


def verify_attn_q4(q, cache, k_tree, v_tree, ancestor_mask, kv_start, kv_len, batch, T, Hq, Hkv, D, softmax_scale, dtype, ws,
                   out=None, defer=False):
    """verify_attn_spans over a 4-bit cache (CacheQ4); T = 1 is a plain decoding step."""
    if (cache.Hkv, cache.D) != (Hkv, D):
        raise DDTreeError("the cache has other KV heads or another head size")
    for name, t, heads in (("q", q, Hq), ("k_tree", k_tree, Hkv), ("v_tree", v_tree, Hkv)):
        _dev(t, torch.bfloat16 if dtype == DTYPE_BF16 else torch.float32, name)
        if t.numel() != batch * T * heads * D or t.get_device() != cache.device:
            raise DDTreeError(f"{name}: expected [batch*T, {heads}, {D}] on the cache's device")
    _dev(ancestor_mask, torch.int64, "ancestor_mask")
    if ancestor_mask.numel() != batch * T * ((T + 63) // 64) or ancestor_mask.get_device() != cache.device:
        raise DDTreeError("ancestor_mask must be [batch, T, ceil(T/64)], on the cache's device")
    _current(cache.device)
    start, start_p = _host_i32(kv_start, batch, "kv_start and kv_len must have batch entries each")
    length, length_p = _host_i32(kv_len, batch, "kv_start and kv_len must have batch entries each")
    if out is None:
        out = torch.empty_like(q)
    elif out.dtype != q.dtype or out.shape != q.shape or not out.is_contiguous() or out.get_device() != cache.device:
        raise DDTreeError("out: expected a contiguous tensor like q")
    p, n = _ws(ws)
    args = (_ptr(q), *cache.ptrs, cache.rows, _ptr(k_tree), _ptr(v_tree), _ptr(ancestor_mask), start_p, length_p, batch, T,
            Hq, Hkv, D, softmax_scale, dtype, _ptr(out), p, n, _stream())
    run = _call("ddtree_verify_attn_q4", args, out, defer)
    return _keepalive(run, start, length, cache) if defer else run


BUILD_AUTO, BUILD_POPS, BUILD_LEVELS = 0, 1, 2


def set_build_algorithm(algo):
    """Force one construction in ddtree_build (BUILD_POPS / BUILD_LEVELS) or let it choose (BUILD_AUTO)."""
    _check(load().ddtree_set_build_algorithm(int(algo)), "ddtree_set_build_algorithm")


def selftest_host():
    """Host-side self-check of the attention kernel's launch arithmetic (no GPU): 0 if it holds."""
    return int(load().ddtree_selftest_host())


def build_giveups():
    """Sequences (since load) that the levels handed to the pops."""
    n = ctypes.c_uint(0)
    _check(load().ddtree_build_giveups(ctypes.byref(n)), "ddtree_build_giveups")
    return int(n.value)


def build_handovers():
    """Sequences (since load) that the construction by deviations handed to the levels (no room, or no bound)."""
    n = ctypes.c_uint(0)
    _check(load().ddtree_build_handovers(ctypes.byref(n)), "ddtree_build_handovers")
    return int(n.value)


def profile_enable(kernels, capacity, every=1):
    """Time one launch in `every` of the named kernels (see KERNELS) with HIP events; [] switches it off."""
    mask = 0
    for k in kernels:
        mask |= 1 << KERNELS[k]
    _check(load().ddtree_profile_enable_every(mask, int(capacity), int(every)), "ddtree_profile_enable_every")


def profile_reset():
    _check(load().ddtree_profile_reset(), "ddtree_profile_reset")


def profile_read(kernel, max_records=1 << 16):
    """Elapsed milliseconds of the recorded launches of one kernel (synchronise first)."""
    buf = np.empty(max_records, np.float32)
    n = load().ddtree_profile_read(KERNELS[kernel], buf.ctypes.data_as(ctypes.c_void_p), max_records)
    if n < 0:
        _check(n, "ddtree_profile_read")
    return buf[:n].copy()
