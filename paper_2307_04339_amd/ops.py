"""Python view of the elastic operators: builds miriam_op_desc from torch tensors
(device memory only) and forwards to the C ABI.  No arithmetic happens here."""
from __future__ import annotations

import ctypes
import math

import torch

from . import _lib as L

TORCH_DTYPE = {torch.float32: L.F32, torch.float16: L.F16, torch.bfloat16: L.BF16}


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("operator tensors must live in device memory")
    return t.data_ptr()


# The current stream's handle without building a torch Stream object, which costs 2.7 us of a 6.4 us
# launch (0.2 us this way); the object where this torch build has no raw accessor.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_handle(stream):
    if stream is None:
        if _raw_stream is not None and _device is not None:
            return _raw_stream(_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


class ElasticOp:
    """One elastic operator over caller-owned device tensors."""

    _desc, _create = L.OpDesc, "miriam_op_create"

    def __init__(self, kind: int, dtype: torch.dtype, *, keep=(), **fields):
        lib = L.load()
        d = self._desc()
        d.kind = kind
        d.dtype = TORCH_DTYPE[dtype]
        for k, v in fields.items():
            if isinstance(v, torch.Tensor):
                v = _ptr(v)
            setattr(d, k, v)
        self.desc = d
        self._keep = tuple(keep)  # tensors borrowed by the op
        h = ctypes.c_void_p()
        self.handle = None
        L.check(getattr(lib, self._create)(ctypes.byref(d), ctypes.byref(h)), self._create)
        self.handle = h
        info = L.OpInfo()
        L.check(lib.miriam_op_query(h, ctypes.byref(info)), "miriam_op_query")
        self.info = info
        self.T = int(info.num_tiles)

    # --------------------------------------------------------------- launches
    def launch(self, begin: int, length: int, grid: int, block: int = 256, stream=None) -> None:
        L.check(L.load().miriam_elastic_launch(self.handle, begin, length, grid, block,
                                               _stream_handle(stream)), "miriam_elastic_launch")

    def launch_traced(self, begin, length, grid, block, owner_wg, owner_iter, count, stream=None,
                      wave_phys=None, wave_slot=None):
        def ptr(t):
            return None if t is None else ctypes.c_void_p(t.data_ptr())
        L.check(L.load().miriam_elastic_launch_traced(
            self.handle, begin, length, grid, block, _stream_handle(stream),
            ptr(owner_wg), ptr(owner_iter), ptr(count), ptr(wave_phys), ptr(wave_slot)),
            "miriam_elastic_launch_traced")

    def reset_counters(self, stream=None) -> None:
        """Clear the split-K arrival counters (stream-ordered) after a pass that did not cover
        the whole tile space."""
        L.check(L.load().miriam_op_reset_counters(self.handle, _stream_handle(stream)),
                "miriam_op_reset_counters")

    def variant(self, **changes) -> "ElasticOp":
        """A second op over the same tensors, from this op's descriptor with `changes` applied
        (for example flags=op.desc.flags | INDEX_MEMORY)."""
        lib = L.load()
        new = type(self).__new__(type(self))
        d = self._desc.from_buffer_copy(self.desc)
        for k, v in changes.items():
            setattr(d, k, v)
        new.desc = d
        new._keep = self._keep
        h = ctypes.c_void_p()
        new.handle = None
        L.check(getattr(lib, self._create)(ctypes.byref(d), ctypes.byref(h)), self._create)
        new.handle = h
        info = L.OpInfo()
        L.check(lib.miriam_op_query(h, ctypes.byref(info)), "miriam_op_query")
        new.info = info
        new.T = int(info.num_tiles)
        return new

    def run(self, stream=None) -> None:
        """Unsharded launch: the whole tile space at the op's full grid (one workgroup per
        tile, or the resident capacity for kernels that keep operands across tiles), block 256."""
        rc = L.load().miriam_op_run(self.handle, _stream_handle(stream))
        if rc < 0:
            L.check(rc, "miriam_op_run")

    def run_plan(self, shards, grids, blocks, stream=None) -> None:
        for (b, l), g, bl in zip(shards, grids, blocks):
            self.launch(b, l, g, bl, stream)

    def destroy(self) -> None:
        if self.handle:
            L.check(L.load().miriam_op_destroy(self.handle), "miriam_op_destroy")
            self.handle = None

    def __del__(self):
        try:
            if self.handle:
                L.load().miriam_op_destroy(self.handle)
        except Exception:
            pass


# ------------------------------------------------------------ constructors
def _epi(bias, bn, residual):
    flags = 0
    if bias is not None:
        flags |= L.EPI_BIAS
    if bn is not None:
        flags |= L.EPI_BN
    if residual is not None:
        flags |= L.EPI_RESIDUAL
    return flags


def conv2d(x, w, y, stride=1, pad=0, bias=None, bn=None, residual=None, act="none", eps=1e-5, tile=0,
           ksplit=0, memory_index=False):
    """x [N,H,W,C], w [K,KH,KW,C], y [N,Ho,Wo,K]; bias [K] f32; bn [4,K] f32.
    memory_index: output-row indices from a host-computed table instead of in-kernel division."""
    N, H, W, C = x.shape
    K, KH, KW, C2 = w.shape
    assert C2 == C
    return ElasticOp(L.OP_CONV2D, x.dtype, keep=(x, w, y, bias, bn, residual),
                     n=N, h=H, w=W, c=C, k=K, kh=KH, kw=KW, stride=stride, pad=pad, groups=1,
                     x=x, wt=w, y=y, bias=bias, bn=bn, residual=residual,
                     flags=_epi(bias, bn, residual) | (L.INDEX_MEMORY if memory_index else 0),
                     act=L.ACT_CODE[act], eps=eps, tile=tile, ksplit=ksplit)


def gemm(x, w, y, bias=None, residual=None, act="none", tile=0, ldx=0, ldw=0, ldy=0, m=None, n=None, k=None,
         ksplit=0, memory_index=False):
    """y[m][n] = act(x[m][:] . w[n][:] + bias + residual)."""
    M = m if m is not None else x.shape[0]
    Kk = k if k is not None else x.shape[-1]
    Nn = n if n is not None else w.shape[0]
    return ElasticOp(L.OP_GEMM, x.dtype, keep=(x, w, y, bias, residual),
                     m=M, nn=Nn, kk=Kk, ldx=ldx, ldw=ldw, ldy=ldy, x=x, wt=w, y=y, bias=bias,
                     residual=residual, flags=_epi(bias, None, residual) | (L.INDEX_MEMORY if memory_index else 0),
                     act=L.ACT_CODE[act], tile=tile, ksplit=ksplit)


def bgemm(x, w, y, m, n, k, batch, batch_div, ldx, ldw, ldy, sx=(0, 0), sw=(0, 0), sy=(0, 0),
          b_nmajor=False, tile=0):
    return ElasticOp(L.OP_BGEMM, x.dtype, keep=(x, w, y),
                     m=m, nn=n, kk=k, batch=batch, batch_div=batch_div, ldx=ldx, ldw=ldw, ldy=ldy,
                     sx0=sx[0], sx1=sx[1], sw0=sw[0], sw1=sw[1], sy0=sy[0], sy1=sy[1],
                     b_nmajor=1 if b_nmajor else 0, x=x, wt=w, y=y, tile=tile)


def dwconv(x, w, y, stride=1, pad=1, bias=None, bn=None, residual=None, act="none", eps=1e-5):
    """x [N,H,W,C], w [KH,KW,C], y [N,Ho,Wo,C]."""
    N, H, W, C = x.shape
    KH, KW, C2 = w.shape
    assert C2 == C
    return ElasticOp(L.OP_DWCONV, x.dtype, keep=(x, w, y, bias, bn, residual),
                     n=N, h=H, w=W, c=C, k=C, kh=KH, kw=KW, stride=stride, pad=pad, groups=C,
                     x=x, wt=w, y=y, bias=bias, bn=bn, residual=residual,
                     flags=_epi(bias, bn, residual), act=L.ACT_CODE[act], eps=eps)


def pool(x, y, k, stride, pad, mode="max"):
    N, H, W, C = x.shape
    kind = L.OP_POOL_MAX if mode == "max" else L.OP_POOL_AVG
    return ElasticOp(kind, x.dtype, keep=(x, y), n=N, h=H, w=W, c=C, k=C, kh=k, kw=k,
                     stride=stride, pad=pad, x=x, y=y)


def softmax(x, y, rows, n, scale=1.0, ldx=0, ldy=0):
    return ElasticOp(L.OP_SOFTMAX, x.dtype, keep=(x, y), m=rows, nn=n, ldx=ldx, ldy=ldy,
                     scale=scale, x=x, y=y)


def layernorm(x, gamma, beta, y, rows, n, residual=None, eps=1e-5):
    return ElasticOp(L.OP_LAYERNORM, x.dtype, keep=(x, gamma, beta, y, residual), m=rows, nn=n,
                     x=x, wt=gamma, bias=beta, y=y, residual=residual,
                     flags=L.EPI_RESIDUAL if residual is not None else 0, eps=eps)


def bn_act(x, y, rows, channels, bias=None, bn=None, residual=None, act="none", eps=1e-5):
    return ElasticOp(L.OP_BN_ACT, x.dtype, keep=(x, y, bias, bn, residual), m=rows, nn=channels,
                     x=x, y=y, bias=bias, bn=bn, residual=residual,
                     flags=_epi(bias, bn, residual), act=L.ACT_CODE[act], eps=eps)


# ------------------------------------------- operators over packed token rows
class SeqOp(ElasticOp):
    """An operator over packed token rows: launched, sharded and grouped into tasks as any other."""

    _desc, _create = L.SeqDesc, "miriam_seq_op_create"


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _rows(name, t, width=None, rows=None, dtype=None):
    """A tensor of rows whose values lie one after another: its row stride."""
    _need(t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1), f"{name}: rows of adjacent values expected")
    _need(width is None or t.shape[1] == width, f"{name}: rows of {width} values expected, got {t.shape[1]}")
    _need(rows is None or t.shape[0] == rows, f"{name}: {rows} rows expected, got {t.shape[0]}")
    _need(dtype is None or t.dtype == dtype, f"{name}: {dtype} expected, got {t.dtype}")
    # (the stride of a single row says nothing)
    _need(t.shape[0] <= 1 or t.stride(0) >= t.shape[1], f"{name}: rows that share memory (a broadcast tensor?)")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _vector(name, t, n, dtype):
    _need(t.dim() == 1 and t.shape[0] == n and t.dtype == dtype and t.is_contiguous(), f"{name}: {n} adjacent {dtype} values expected")


def _one_device(**tensors):
    first = None
    for name, t in tensors.items():
        if t is None:
            continue
        _need(t.is_cuda, f"{name}: operator tensors must live in device memory")
        first = first if first is not None else t.device
        _need(t.device == first, f"{name}: on {t.device}, others on {first}")
    _need(first.index == torch.cuda.current_device(), f"tensors on {first}, but the current device is {torch.cuda.current_device()}")


def _sequences(q_start, kv_len, page_table, k_cache, v_cache, dtype):
    """Descriptor fields of a batch and its cache (k_cache, v_cache: [pages, kv_heads, page, head_dim], any
    strides but the last)."""
    seqs = kv_len.shape[0]
    _vector("kv_len", kv_len, seqs, torch.int32)
    _vector("q_start", q_start, seqs + 1, torch.int32)
    f = dict(seqs=seqs, q_start=q_start, kv_len=kv_len)
    if k_cache is None:
        return f
    _need(k_cache.dim() == 4 and k_cache.shape == v_cache.shape and k_cache.stride() == v_cache.stride(),
          "caches: [pages, kv_heads, page, head_dim], both of the same shape and strides")
    _need(k_cache.dtype == dtype and v_cache.dtype == dtype, f"caches: {dtype} expected")
    _need(k_cache.shape[3] == 1 or k_cache.stride(3) == 1, "caches: the values of a head must be adjacent")
    _need(page_table.dim() == 2 and page_table.shape[0] == seqs and page_table.dtype == torch.int32 and
          (page_table.shape[1] <= 1 or page_table.stride(1) == 1), f"page_table: {seqs} rows of adjacent int32 expected")
    _need(seqs <= 1 or page_table.stride(0) >= page_table.shape[1], "page_table: rows that share memory (a broadcast tensor?)")
    f.update(kv_heads=k_cache.shape[1], page=k_cache.shape[2], pages=k_cache.shape[0], max_pages=page_table.shape[1],
             ldt=page_table.stride(0) if seqs > 1 else page_table.shape[1], page_table=page_table, k_cache=k_cache,
             v_cache=v_cache, cache_page=k_cache.stride(0), cache_head=k_cache.stride(1), cache_token=k_cache.stride(2))
    return f


def block_norm(x, y=None, *, residual=None, post=None, post_bias=None, gate=None, gate_act="none", scale=1.0, z=None,
               pre=None, pre_bias=None, norm="rms", eps=1e-5):
    """y = residual + scale * gate(N_post(x)), z = N_pre(that sum before its rounding to y); rows of x, residual,
    y and z; post, pre and the biases [n] f32.  norm: "rms" or "layer".  gate: [n] f32 (gate_act "none") or rows
    like x, taken as they are ("none") or through "silu" or "sigmoid".  y or z may be left out."""
    m, n = x.shape
    _one_device(x=x, y=y, residual=residual, post=post, post_bias=post_bias, gate=gate, z=z, pre=pre, pre_bias=pre_bias)
    _need(norm in ("rms", "layer"), f"unknown norm {norm!r}")
    f = dict(ldx=_rows("x", x))
    for name, key, t in (("residual", "ldr", residual), ("y", "ldy", y), ("z", "ldz", z)):
        if t is not None:
            f[key] = _rows(name, t, n, m, x.dtype)
    for name, t in (("post", post), ("post_bias", post_bias), ("pre", pre), ("pre_bias", pre_bias)):
        if t is not None:
            _vector(name, t, n, torch.float32)
    kind = L.GATE_NONE
    _need(gate_act in ("none", "silu", "sigmoid"), f"unknown gate activation {gate_act!r}")
    _need(gate is not None or gate_act == "none", "a gate activation without a gate")
    if gate is not None and gate.dim() == 1:
        _vector("gate", gate, n, torch.float32)
        _need(gate_act == "none", "a gate per channel has no activation")
        kind = L.GATE_CHANNEL
    elif gate is not None:
        f["ldg"] = _rows("gate", gate, n, m, x.dtype)
        kind = {"none": L.GATE_ROWS, "silu": L.GATE_SILU, "sigmoid": L.GATE_SIGMOID}[gate_act]
    return SeqOp(L.OP_BLOCK_NORM, x.dtype, keep=(x, y, residual, post, post_bias, gate, z, pre, pre_bias), tokens=m, n=n, x=x,
                 y=y, z=z, residual=residual, gate=gate, post=post, post_bias=post_bias, pre=pre, pre_bias=pre_bias,
                 gate_kind=kind, scale=scale, eps=eps, flags=L.SEQ_LAYER_NORM if norm == "layer" else 0, **f)


def rotary(x, y, freq, q_start, kv_len, *, heads, head_dim, kv_heads=0, k_cache=None, v_cache=None, page_table=None,
           interleaved=False, scale=1.0):
    """x [tokens, (heads + 2 kv_heads) * head_dim]: queries, keys and values of every token.  Queries, turned by
    their positions, go to y [tokens, heads * head_dim], turned keys and the values to the caches.  freq: f64
    [rot / 2] angles per position (rotary_freqs).  q_start [seqs + 1], kv_len [seqs] int32: the batch, read by
    every run.  kv_heads = 0: no cache, heads heads are turned."""
    _need((kv_heads > 0) == (k_cache is not None) == (v_cache is not None) == (page_table is not None),
          "kv_heads, k_cache, v_cache and page_table go together")
    _one_device(x=x, y=y, freq=freq, q_start=q_start, kv_len=kv_len, k_cache=k_cache, v_cache=v_cache, page_table=page_table)
    f = _sequences(q_start, kv_len, page_table, k_cache, v_cache, x.dtype)
    _need(kv_heads == f.get("kv_heads", 0) and (k_cache is None or k_cache.shape[3] == head_dim), "caches: kv_heads and head_dim differ")
    _vector("freq", freq, freq.shape[0], torch.float64)
    ldx = _rows("x", x, (heads + 2 * kv_heads) * head_dim)
    ldy = _rows("y", y, heads * head_dim, x.shape[0], x.dtype)
    return SeqOp(L.OP_ROTARY, x.dtype, keep=(x, y, freq, q_start, kv_len, k_cache, v_cache, page_table), tokens=x.shape[0],
                 heads=heads, head_dim=head_dim, rot=2 * freq.shape[0], x=x, y=y, freq=freq, ldx=ldx, ldy=ldy, scale=scale,
                 flags=L.SEQ_INTERLEAVED if interleaved else 0, **f)


def attention(q, k_cache, v_cache, y, q_start, kv_len, page_table, *, heads, scale=None, causal=True, window=0, max_q=None):
    """y = attention of the new tokens' queries q [tokens, heads * head_dim] over their sequences' cached keys
    (those of the new tokens among them).  scale: 1 / sqrt(head_dim) if None.  window > 0: of the keys up to
    a token's own only the last `window` (without causal all later ones, too).  max_q: most new tokens of one sequence (all rows if None); knowing that it is
    small gives the kernel for single tokens.  The arrays of a batch must not change during a pass."""
    _one_device(q=q, k_cache=k_cache, v_cache=v_cache, y=y, q_start=q_start, kv_len=kv_len, page_table=page_table)
    f = _sequences(q_start, kv_len, page_table, k_cache, v_cache, q.dtype)
    d = k_cache.shape[3]
    ldx = _rows("q", q, heads * d)
    ldy = _rows("y", y, heads * d, q.shape[0], q.dtype)
    _need(max_q is None or max_q >= 1, "max_q must be >= 1")
    _need(window >= 0, "window must be >= 0")
    return SeqOp(L.OP_ATTENTION, q.dtype, keep=(q, k_cache, v_cache, y, q_start, kv_len, page_table), tokens=q.shape[0],
                 heads=heads, head_dim=d, x=q, y=y, ldx=ldx, ldy=ldy, scale=1.0 / math.sqrt(d) if scale is None else scale,
                 flags=L.SEQ_CAUSAL if causal else 0, window=window, max_q=max_q or 0, **f)


def rotary_freqs(rot, base=10000.0, factor=1.0, original=0, low=1.0, high=32.0):
    """f64 [rot / 2] angles per position (host memory): base^(-2 j / rot), for a context stretched by `factor`.
    original > 0: by parts, untouched where a pair makes `high` turns or more over the original context, divided
    by the factor at `low` or fewer; original = 0: all divided."""
    out = torch.empty(max(rot // 2, 1), dtype=torch.float64)
    L.check(L.load().miriam_plan_rotary_freqs(rot, base, factor, original, low, high,
                                              ctypes.cast(out.data_ptr(), ctypes.POINTER(ctypes.c_double))),
            "miriam_plan_rotary_freqs")
    return out


def device_info():
    dd = L.DeviceDesc()
    L.check(L.load().miriam_device_query(ctypes.byref(dd)), "miriam_device_query")
    return dd
