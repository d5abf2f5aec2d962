"""ctypes binding of include/hydra_ops.h (argument marshalling only).

Arguments are torch CUDA tensors (device memory is PyTorch's job here); every
function enqueues the named C entry point on torch's current stream.
"""
from __future__ import annotations

import ctypes as C
import struct
from array import array

from .hydra import HydraError, lib

F32, BF16 = 0, 1
CACHE_INT8, CACHE_E4M3 = 0, 1
ROT_NONE, ROT_HALVES, ROT_NEIGHBOURS = 0, 1, 2
EPI_NONE, EPI_RELU, EPI_GELU = 0, 1, 2


class hydra_gemm_desc(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("dtype", "M", "N", "K", "x_kmajor", "w_kmajor", "ldx", "ldw", "ldo", "ldg", "ldr",
                                       "act", "out_f32", "tile", "G")] + \
               [(n, C.c_void_p) for n in ("X", "W", "bias", "out", "pre", "gate", "resid", "rowsum", "ws")] + \
               [("ws_bytes", C.c_size_t)]


# A small product takes less time than ctypes needs for its arguments: tables are made as one array of addresses and the
# descriptor is packed (3 tables of forward, bias and pre-activation: 4.1 -> 2.0 us, of which reading the addresses is 1.1).
_desc = struct.Struct("15i9PN").pack           # the fields of hydra_gemm_desc


_ready = False


def _L():
    global _ready
    L = lib()
    if not _ready:
        vp = pp = C.c_void_p                       # tables go by address, descriptors as bytes or by reference
        L.hydra_op_gemm.argtypes = [vp, vp]
        L.hydra_op_gemm_update.argtypes = [vp, C.c_int, pp, pp, pp, pp, vp, vp]
        L.hydra_op_colsum.argtypes = [C.c_int] * 5 + [pp, pp, pp, vp]
        L.hydra_op_colsum_part_floats.argtypes = [C.c_int, C.c_int]
        L.hydra_op_colsum_part_floats.restype = C.c_size_t
        L.hydra_op_colsum_noalloc.argtypes = [C.c_int] * 5 + [pp, pp, vp]
        L.hydra_op_colsum_noalloc_max_floats.argtypes = []
        L.hydra_op_colsum_noalloc_max_floats.restype = C.c_size_t
        L.hydra_op_gemm_split_k.argtypes = [C.c_int] * 3
        L.hydra_op_gemm_split_ws_bytes.argtypes = [C.c_int] * 4
        L.hydra_op_gemm_split_ws_bytes.restype = C.c_size_t
        L.hydra_op_softmax_ce.argtypes = [C.c_int] * 5 + [C.c_float, C.c_int, pp, vp, pp, pp, pp, vp]
        L.hydra_op_optim.argtypes = [C.c_int, C.c_size_t, C.c_int, pp, pp, pp, pp, pp, vp, vp]
        L.hydra_op_init_uniform.argtypes = [vp, C.c_size_t, C.c_uint64, C.c_uint64, C.c_float, vp]
        L.hydra_op_cast_bf16.argtypes = [vp, vp, C.c_size_t, vp]
        L.hydra_op_layernorm_fwd.argtypes = [C.c_int] * 4 + [C.c_float, C.c_int] + [pp] * 6 + [vp]
        L.hydra_op_layernorm_bwd.argtypes = [C.c_int] * 5 + [pp] * 10 + [vp]
        L.hydra_op_layernorm_part_floats.argtypes = [C.c_int, C.c_int]
        L.hydra_op_layernorm_part_floats.restype = C.c_size_t
        L.hydra_op_attention_fwd.argtypes = [C.c_int] * 7 + [C.c_float, C.c_int, pp, pp, pp, vp]
        L.hydra_op_attention_bwd.argtypes = [C.c_int] * 7 + [C.c_float, C.c_int] + [pp] * 6 + [vp]
        L.hydra_op_embed_fwd.argtypes = [C.c_int] * 6 + [vp, pp, pp, pp, vp]
        L.hydra_op_embed_bwd.argtypes = [C.c_int] * 8 + [vp, vp, pp, pp, pp, vp]
        L.hydra_op_cache_append.argtypes = [vp, vp]
        L.hydra_op_cache_attention.argtypes = [vp, vp]
        L.hydra_op_cache_attention_ws_bytes.argtypes = [vp, C.c_int]
        L.hydra_op_cache_attention_ws_bytes.restype = C.c_size_t
        L.hydra_op_cache_attention_plan.argtypes = [vp, C.c_int, vp]
        L.hydra_op_sample.argtypes = [C.c_int] * 6 + [pp, pp, vp, vp, vp, vp, pp, pp, vp]
        L.hydra_op_empty_launches.argtypes = [C.c_int, vp]
        L.hydra_ops_last_error.restype = C.c_char_p
        _ready = True
    return L


def _stream():
    """torch's current stream on the current device (the raw handle: building a Stream object costs several us)."""
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _tabs(*tables):
    """[keep, a, b, ...]: the addresses of all tables' tensors in one array, which the caller keeps over the call, and the address of
    each table in it (None for none)."""
    keep = array("Q", [x.data_ptr() for t in tables if t is not None for x in t])
    at, out = keep.buffer_info()[0], [keep]
    for t in tables:
        if t is None:
            out.append(None)
        else:
            out.append(at)
            at += 8 * len(t)
    return out


def _hp(hp_rows, problems):
    """Hyper-parameters of all problems as doubles, six to a problem, and their address: zeros where fewer are given, more are refused."""
    try:
        flat = array("d", [x for row in hp_rows for x in row])
    except TypeError:  # what only float() makes a number of
        flat = array("d", [float(x) for row in hp_rows for x in row])
    missing = 6 * problems - len(flat)
    if missing:
        if missing < 0:
            raise IndexError(f"{len(flat)} hyper-parameters for {problems} problems")
        flat.extend([0.0] * missing)
    return flat, flat.buffer_info()[0]


def _nbytes(ws):
    return 0 if ws is None else min(t.numel() * t.element_size() for t in ws)


def _check(st: int):
    if st != 0:
        raise HydraError(st, _L().hydra_ops_last_error().decode())


def hydra_op_gemm(dtype, M, N, K, X, W, out, *, x_kmajor, w_kmajor, ldx, ldw, ldo, bias=None, pre=None, gate=None,
                  resid=None, ldg=0, ldr=0, act=EPI_NONE, out_f32=False, tile=0, rowsum=None, ws=None):
    """ws: optional per-problem scratch tensors (uint8, hydra_op_gemm_split_ws_bytes bytes) that allow a split sum over k."""
    keep, *at = _tabs(X, W, bias, out, pre, gate, resid, rowsum, ws)
    d = _desc(dtype, M, N, K, int(x_kmajor), int(w_kmajor), ldx, ldw, ldo, ldg, ldr, act, int(out_f32), tile, len(X),
              *[a or 0 for a in at], _nbytes(ws))
    _check(_L().hydra_op_gemm(d, _stream()))


def hydra_op_gemm_split_k(M, N, K) -> int:
    return int(_L().hydra_op_gemm_split_k(M, N, K))


def hydra_op_gemm_split_ws_bytes(M, N, K, ldo) -> int:
    return int(_L().hydra_op_gemm_split_ws_bytes(M, N, K, ldo))


def hydra_op_gemm_update(dtype, M, N, K, X, W, opt, p, m, v, w16, hp_rows, *, ldx, ldw, ldo, out=None, tile=0, rowsum=None,
                         ws=None):
    """Weight gradient dW[M,N] = sum_k X(k,m) W(k,n) with the optimizer step of hydra_op_optim in its epilogue."""
    keep, tx, tw, to, tr, ts, tp, tm, tv, t16 = _tabs(X, W, out, rowsum, ws, p, m, v, w16)
    d = _desc(dtype, M, N, K, 0, 0, ldx, ldw, ldo, 0, 0, EPI_NONE, 1, tile, len(X), tx or 0, tw or 0, 0, to or 0, 0, 0, 0, tr or 0, ts or 0,
              _nbytes(ws))
    flat, hp = _hp(hp_rows, len(p))
    _check(_L().hydra_op_gemm_update(d, opt, tp, tm, tv, t16, hp, _stream()))


def hydra_op_colsum_part_floats(M, N) -> int:
    return int(_L().hydra_op_colsum_part_floats(M, N))


def hydra_op_colsum(dtype, M, N, ld, src, out, part=None):
    keep, *at = _tabs(src, out, part)
    _check(_L().hydra_op_colsum(dtype, M, N, ld, len(src), *at, _stream()))


def hydra_op_empty_launches(n: int):
    _check(_L().hydra_op_empty_launches(n, _stream()))


def hydra_op_colsum_noalloc(dtype, M, N, ld, src, out):
    keep, *at = _tabs(src, out)
    _check(_L().hydra_op_colsum_noalloc(dtype, M, N, ld, len(src), *at, _stream()))


def hydra_op_colsum_noalloc_max_floats() -> int:
    return int(_L().hydra_op_colsum_noalloc_max_floats())


def hydra_op_softmax_ce(dtype, M, Cn, ldz, lddz, inv_n, logits, labels, dz, rowloss, loss):
    keep, tz, *at = _tabs(logits, dz, rowloss, loss)
    _check(_L().hydra_op_softmax_ce(dtype, M, Cn, ldz, lddz, inv_n, len(logits), tz, labels.data_ptr(), *at, _stream()))


def hydra_op_optim(opt, n, p, g, m, v, w16, hp_rows):
    """hp_rows: per problem (lr, b1, b2, eps, bc1, bc2)."""
    keep, *at = _tabs(p, g, m, v, w16)
    flat, hp = _hp(hp_rows, len(p))
    _check(_L().hydra_op_optim(opt, n, len(p), *at, hp, _stream()))


def hydra_op_init_uniform(dst, n, seed, stream_id, a):
    _check(_L().hydra_op_init_uniform(C.c_void_p(dst.data_ptr()), n, C.c_uint64(seed), C.c_uint64(stream_id), a, _stream()))


def hydra_op_cast_bf16(src, dst, n):
    _check(_L().hydra_op_cast_bf16(C.c_void_p(src.data_ptr()), C.c_void_p(dst.data_ptr()), n, _stream()))


def hydra_op_layernorm_fwd(dtype, rows, d, ld, eps, x, y, gamma, beta, mean, rstd):
    keep, *at = _tabs(x, y, gamma, beta, mean, rstd)
    _check(_L().hydra_op_layernorm_fwd(dtype, rows, d, ld, eps, len(x), *at, _stream()))


def hydra_op_layernorm_part_floats(rows, d) -> int:
    return int(_L().hydra_op_layernorm_part_floats(rows, d))


def hydra_op_layernorm_bwd(dtype, rows, d, ld, x, dy, add, dx, gamma, mean, rstd, part, dgamma, dbeta):
    keep, *at = _tabs(x, dy, add, dx, gamma, mean, rstd, part, dgamma, dbeta)
    _check(_L().hydra_op_layernorm_bwd(dtype, rows, d, ld, len(x), *at, _stream()))


def hydra_op_attention_fwd(B, S, H, DH, ld_qkv, ld_o, causal, scale, qkv, o, lse):
    keep, *at = _tabs(qkv, o, lse)
    _check(_L().hydra_op_attention_fwd(B, S, H, DH, ld_qkv, ld_o, int(causal), scale, len(qkv), *at, _stream()))


def hydra_op_attention_bwd(B, S, H, DH, ld_qkv, ld_o, causal, scale, qkv, o, dout, lse, delta, dqkv):
    keep, *at = _tabs(qkv, o, dout, lse, delta, dqkv)
    _check(_L().hydra_op_attention_bwd(B, S, H, DH, ld_qkv, ld_o, int(causal), scale, len(qkv), *at, _stream()))


def hydra_op_embed_fwd(dtype, tokens, S, d, ld, ids, tok, pos, x):
    keep, *at = _tabs(tok, pos, x)
    _check(_L().hydra_op_embed_fwd(dtype, tokens, S, d, ld, len(x), ids.data_ptr(), *at, _stream()))


def hydra_op_embed_bwd(dtype, V, S, S_table, B, d, ld, row_ptr, positions, dx, dtok, dpos):
    keep, *at = _tabs(dx, dtok, dpos)
    _check(_L().hydra_op_embed_bwd(dtype, V, S, S_table, B, d, ld, len(dx), row_ptr.data_ptr(), positions.data_ptr(), *at, _stream()))


# All tables of a call lie in one array: one that is too short would be read on into the next.
def _one_per_model(G, *tables):
    for t in tables:
        if t is not None and len(t) != G:
            raise ValueError(f"a table of {len(t)} tensors for {G} models")


def _entries(t, n, dtype, name):
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{name} is contiguous {dtype} of at least {n} entries")


class Cache:
    """One layer's paged cache of G models: pools of 8-bit codes k, v [n_pages, HKV, page, DH] (lists of G tensors), their scales k_scale, v_scale
    [n_pages, HKV] fp32 and the page table [B, max_pages] int32 that the group shares.  A record of tensors and their addresses: what the
    cache holds is in the tensors alone.  Pools may be slices along their first dimension's stride (several layers in one tensor)."""

    def __init__(self, kind, k, v, k_scale, v_scale, page_table):
        import torch
        self._int32 = torch.int32
        self.kind, self.k, self.v, self.k_scale, self.v_scale, self.page_table = kind, k, v, k_scale, v_scale, page_table
        n_pages, hkv, page, dh = k[0].shape
        stride = k[0].stride(0)
        for t in (*k, *v):
            if t.shape != k[0].shape or t.element_size() != 1 or t.stride() != (stride, page * dh, dh, 1):
                raise ValueError("pools have one shape [n_pages, HKV, page, DH], one page stride and 1-byte codes, contiguous inside a page")
        if n_pages > 1 and stride < hkv * page * dh:
            raise ValueError("pages of a pool lie one behind the other")
        for t in (*k_scale, *v_scale):
            if tuple(t.shape) != (n_pages, hkv) or t.dtype is not torch.float32 or not t.is_contiguous():
                raise ValueError("scales are contiguous fp32 [n_pages, HKV]")
        if not len(k) == len(v) == len(k_scale) == len(v_scale):
            raise ValueError("k, v, k_scale and v_scale have one tensor per model")
        if page_table.dim() != 2 or page_table.dtype is not torch.int32 or not page_table.is_contiguous():
            raise ValueError("page_table is contiguous int32 [B, max_pages]")
        self.B, self.max_pages = page_table.shape
        self.HKV, self.page, self.DH, self.G = hkv, page, dh, len(k)
        self._head = (kind, self.B, hkv, dh, page, n_pages, self.max_pages, self.G)
        self._stride = stride if n_pages > 1 else 0
        self._table = page_table.data_ptr()
        self._keep, *self._at = _tabs(k, v, k_scale, v_scale)

    def fields(self, lens=None, q_ptr=None, n_tok=None, max_q=1, max_len=None):
        """The fields of a call's hydra_cache_desc."""
        if lens is not None and (lens.dtype is not self._int32 or lens.numel() < self.B or not lens.is_contiguous()):
            raise ValueError(f"lens is contiguous int32 of at least {self.B} entries")
        if q_ptr is not None and (q_ptr.dtype is not self._int32 or q_ptr.numel() <= self.B or not q_ptr.is_contiguous()):
            raise ValueError(f"q_ptr is contiguous int32 of at least {self.B + 1} entries")
        return (*self._head, self.B if n_tok is None else n_tok, max_q, self.max_pages * self.page if max_len is None else max_len, self._stride,
                self._table, 0 if lens is None else lens.data_ptr(), 0 if q_ptr is None else q_ptr.data_ptr(), *self._at)


# hydra_cache_desc, and with what an operator adds to it
_cache_desc, _append_desc, _attention_desc = (struct.Struct("11iN7P" + more).pack for more in ("", "5i3P", "4if4PN"))


def hydra_op_cache_append(cache, lens, H, ld_qkv, ld_q, qkv, q=None, *, rot=ROT_NONE, rot_dim=0, cos_sin=None, q_ptr=None, n_tok=None, max_q=1,
                          max_len=None):
    """q=None leaves the queries alone; max_len=None: as many tokens as the page table has room for."""
    if len(qkv) != cache.G or q is not None and len(q) != cache.G:
        raise ValueError(f"qkv and q have one tensor for each of {cache.G} models")
    keep, tqkv, tq = _tabs(qkv, q)
    d = _append_desc(*cache.fields(lens, q_ptr, n_tok, max_q, max_len), H, ld_qkv, ld_q, rot, rot_dim, 0 if cos_sin is None else cos_sin.data_ptr(), tqkv,
                     tq or 0)
    _check(_L().hydra_op_cache_append(d, _stream()))


def hydra_op_cache_attention_ws_bytes(cache, H, *, n_tok=None, max_q=1, max_len=None) -> int:
    return int(_L().hydra_op_cache_attention_ws_bytes(_cache_desc(*cache.fields(n_tok=n_tok, max_q=max_q, max_len=max_len)), H))


def hydra_op_cache_attention_plan(cache, H, *, n_tok=None, max_q=1, max_len=None):
    """(rows of a workgroup, its waves, runs of a sequence's tokens) of a call with enough scratch; 16 rows: the kernel for few rows."""
    plan = (C.c_int32 * 3)()
    _check(_L().hydra_op_cache_attention_plan(_cache_desc(*cache.fields(n_tok=n_tok, max_q=max_q, max_len=max_len)), H, plan))
    return tuple(plan)


def hydra_op_cache_attention(cache, lens, H, ld_q, ld_o, causal, scale, q, o, lse=None, *, ws=None, q_ptr=None, n_tok=None, max_q=1, max_len=None):
    """ws: optional per-model scratch tensors (uint8, hydra_op_cache_attention_ws_bytes bytes) that allow splitting a sequence's tokens."""
    _one_per_model(cache.G, q, o, lse, ws)
    keep, tq, to, tl, tw = _tabs(q, o, lse, ws)
    d = _attention_desc(*cache.fields(lens, q_ptr, n_tok, max_q, max_len), H, ld_q, ld_o, causal, scale, tq, to, tl or 0, tw or 0, _nbytes(ws))
    _check(_L().hydra_op_cache_attention(d, _stream()))


def hydra_op_sample(dtype, rows, V, ldz, ldu, logits, u, temperature, top_k, top_p, min_p, token, logprob=None):
    """temperature, top_p, min_p: fp32, top_k and every model's token: int32, of `rows` entries."""
    import torch
    _one_per_model(len(logits), u, token, logprob)
    for name, t, kind in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                          ("min_p", min_p, torch.float32), *(("token", t, torch.int32) for t in token)):
        _entries(t, rows, kind, name)
    keep, tz, tu, tt, tl = _tabs(logits, u, token, logprob)
    _check(_L().hydra_op_sample(dtype, rows, V, ldz, ldu, len(logits), tz, tu, temperature.data_ptr(), top_k.data_ptr(), top_p.data_ptr(),
                                min_p.data_ptr(), tt, tl, _stream()))
