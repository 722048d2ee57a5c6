"""Torch-facing wrapper of the C ABI.

Torch provides device memory and streams; each function below only turns
tensors into pointers and calls the library.  Names follow the C ABI:
``build_csr`` = taurus_build_csr, ``Layer`` = taurus_layer_init / push_chunk /
finalize / sampled_edges / destroy.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Sequence

import numpy as np
import torch

from . import _native as N
from .blockops import check_act, check_norm_args, label_log_probs, linear, residual_norm
from .rowops import _overlap, group_norm, grouped_linear, lookup_rows

_TORCH_DTYPE = {N.F32: torch.float32, N.BF16: torch.bfloat16, N.F16: torch.float16}


def torch_dtype(code: int):
    return _TORCH_DTYPE[code]


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _dev_ptr(t: torch.Tensor, dtype: torch.dtype, what: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def _buf_ptr(t: torch.Tensor, dtype: torch.dtype, what: str):
    """(pointer, on_host) of a device tensor or of a pinned host tensor."""
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if t.is_cuda:
        return t.data_ptr(), 0
    if not t.is_pinned():
        raise ValueError(f"{what} on the host must be pinned memory")
    return t.data_ptr(), 1


def hash_u64(seed: int, tag: int, *args: int) -> int:
    a = (ctypes.c_uint64 * max(1, len(args)))(*args)
    return int(N.lib().taurus_hash(seed & (2**64 - 1), tag, len(args), ctypes.cast(a, ctypes.c_void_p)))


def build_csr(n: int, src: torch.Tensor, dst: torch.Tensor, stream=None):
    """taurus_build_csr: device edge list (int32) -> (row_off int64[n+1], col_dst int32[e])."""
    e = src.numel()
    row_off = torch.empty(n + 1, dtype=torch.int64, device=src.device)
    col_dst = torch.empty(max(e, 1), dtype=torch.int32, device=src.device)[:e]
    N.check(N.lib().taurus_build_csr(n, e, _dev_ptr(src, torch.int32, "src"), _dev_ptr(dst, torch.int32, "dst"),
                                     row_off.data_ptr(), col_dst.data_ptr() if e else None,
                                     _stream_ptr(stream)), "taurus_build_csr")
    return row_off, col_dst


NOALLOC_MAX_EDGES = N.NOALLOC_MAX_EDGES


def build_csr_noalloc(n: int, src: torch.Tensor, dst: torch.Tensor, row_off: torch.Tensor, col_dst: torch.Tensor,
                      stream=None) -> None:
    """taurus_build_csr_noalloc: the CSR build into caller-allocated row_off
    (int64[n+1]) and col_dst (int32[e]) with no device allocation by the
    library or by this wrapper; at most NOALLOC_MAX_EDGES edges."""
    e = src.numel()
    if row_off.numel() != n + 1 or col_dst.numel() != e:
        raise ValueError("row_off must hold n + 1 and col_dst e entries")
    N.check(N.lib().taurus_build_csr_noalloc(n, e, _dev_ptr(src, torch.int32, "src"),
                                             _dev_ptr(dst, torch.int32, "dst"),
                                             _dev_ptr(row_off, torch.int64, "row_off"),
                                             _dev_ptr(col_dst, torch.int32, "col_dst") if e else None,
                                             _stream_ptr(stream)), "taurus_build_csr_noalloc")


def _graph(n: int, row_off: torch.Tensor, col_dst: torch.Tensor) -> N.Graph:
    e = col_dst.numel()
    return N.Graph(n, e, _dev_ptr(row_off, torch.int64, "row_off"), _dev_ptr(col_dst, torch.int32, "col_dst") if e else None)


def reorder(n: int, row_off: torch.Tensor, col_dst: torch.Tensor, stream=None) -> torch.Tensor:
    """taurus_reorder: degree/BFS order, new_of_old int32[n] on the device."""
    g = _graph(n, row_off, col_dst)
    out = torch.empty(n, dtype=torch.int32, device=row_off.device)
    N.check(N.lib().taurus_reorder(ctypes.byref(g), out.data_ptr(), _stream_ptr(stream)), "taurus_reorder")
    return out


def reorder_rcm(n: int, row_off: torch.Tensor, col_dst: torch.Tensor, stream=None) -> torch.Tensor:
    """taurus_reorder_rcm: RCMK order of the symmetrised graph, new_of_old int32[n] on the device."""
    g = _graph(n, row_off, col_dst)
    out = torch.empty(n, dtype=torch.int32, device=row_off.device)
    N.check(N.lib().taurus_reorder_rcm(ctypes.byref(g), out.data_ptr(), _stream_ptr(stream)), "taurus_reorder_rcm")
    return out


class TaOrder(NamedTuple):
    """taurus_reorder_ta's outputs: the order and positions on the device, and
    per update (index 0 = the bootstrap) C(pi) and J(pi) on the host."""
    pi: torch.Tensor         # int32[n], new ID of each vertex
    positions: torch.Tensor  # float64[n], r after the last update made
    spans: np.ndarray        # int64[iterations + 1]
    disp: np.ndarray         # float64[iterations + 1]
    done: int                # updates made


def reorder_ta(n: int, row_off: torch.Tensor, col_dst: torch.Tensor, pi0: Optional[torch.Tensor] = None,
               iterations: int = 5, stream=None) -> TaOrder:
    """taurus_reorder_ta: topology-aware order (Alg. 1) from bootstrap pi0
    (identity if None)."""
    g = _graph(n, row_off, col_dst)
    out = torch.empty(n, dtype=torch.int32, device=row_off.device)
    pos = torch.empty(n, dtype=torch.float64, device=row_off.device)
    spans = np.zeros(iterations + 1, dtype=np.int64)
    disp = np.zeros(iterations + 1, dtype=np.float64)
    done = ctypes.c_int32(0)
    p0 = None if pi0 is None else _dev_ptr(pi0, torch.int32, "pi0")
    N.check(N.lib().taurus_reorder_ta(ctypes.byref(g), p0, iterations, out.data_ptr(), pos.data_ptr(),
                                      spans.ctypes.data, disp.ctypes.data, ctypes.byref(done),
                                      _stream_ptr(stream)), "taurus_reorder_ta")
    return TaOrder(out, pos, spans, disp, done.value)


def relabel_graph(n: int, row_off: torch.Tensor, col_dst: torch.Tensor, new_of_old: torch.Tensor, stream=None):
    """taurus_relabel_graph: CSR of the graph with vertex v renamed new_of_old[v]."""
    g = _graph(n, row_off, col_dst)
    e = col_dst.numel()
    r2 = torch.empty(n + 1, dtype=torch.int64, device=row_off.device)
    c2 = torch.empty(max(e, 1), dtype=torch.int32, device=row_off.device)[:e]
    N.check(N.lib().taurus_relabel_graph(ctypes.byref(g), _dev_ptr(new_of_old, torch.int32, "new_of_old"),
                                         r2.data_ptr(), c2.data_ptr() if e else None, _stream_ptr(stream)),
            "taurus_relabel_graph")
    return r2, c2


def permute_rows(x: torch.Tensor, new_of_old: torch.Tensor, inverse: bool = False, stream=None) -> torch.Tensor:
    """taurus_permute_rows: rows of x [n][...] into the new numbering
    (out[new_of_old[v]] = x[v]), or back (inverse: out[v] = x[new_of_old[v]])."""
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous device tensor")
    n = x.shape[0]
    out = torch.empty_like(x)
    row_bytes = x[0].numel() * x.element_size() if n else 0
    N.check(N.lib().taurus_permute_rows(x.data_ptr(), out.data_ptr(), n, row_bytes,
                                        _dev_ptr(new_of_old, torch.int32, "new_of_old"), int(inverse),
                                        _stream_ptr(stream)), "taurus_permute_rows")
    return out


def release_cached_memory(nbytes: int = 0) -> int:
    """taurus_release_cached_memory: hand the library's cached device blocks
    back to the runtime, smallest first, until at least nbytes are freed (0:
    all).  Returns the bytes freed."""
    r = N.lib().taurus_release_cached_memory(int(nbytes))
    if r < 0:
        raise N.TaurusError(int(r), "taurus_release_cached_memory", N.last_error())
    return int(r)


def alloc_device(shape, dtype, device) -> torch.Tensor:
    """torch.empty, handing back as much of the library's cached memory as
    the allocation lacks (and retrying) when the device is out of memory."""
    try:
        return torch.empty(shape, dtype=dtype, device=device)
    except torch.OutOfMemoryError:
        need = int(np.prod(shape)) * torch.tensor([], dtype=dtype).element_size()
        free, _ = torch.cuda.mem_get_info(device)
        release_cached_memory(max(need - free, 0) + (1 << 30))
        torch.cuda.empty_cache()
        return torch.empty(shape, dtype=dtype, device=device)


_hip = None


def alloc_pinned(shape, dtype) -> torch.Tensor:
    """Pinned host tensor of exactly this size (hipHostMalloc; torch's pinned
    allocator rounds large blocks up to a power of two, which matters where
    pinned memory is capped).  Freed when the last tensor viewing it goes."""
    import weakref
    global _hip
    if _hip is None:
        _hip = ctypes.CDLL("libamdhip64.so")
        _hip.hipHostMalloc.restype = ctypes.c_int
        _hip.hipHostMalloc.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_size_t, ctypes.c_uint]
        _hip.hipHostFree.restype = ctypes.c_int
        _hip.hipHostFree.argtypes = [ctypes.c_void_p]
    nbytes = max(1, int(np.prod(shape)) * torch.tensor([], dtype=dtype).element_size())
    p = ctypes.c_void_p()
    rc = _hip.hipHostMalloc(ctypes.byref(p), nbytes, 0)
    if rc != 0 or not p.value:
        raise MemoryError(f"hipHostMalloc({nbytes}) failed ({rc})")
    buf = (ctypes.c_uint8 * nbytes).from_address(p.value)
    weakref.finalize(buf, _hip.hipHostFree, p.value)
    t = torch.frombuffer(buf, dtype=torch.uint8)
    return t[:nbytes].view(dtype).view(shape) if shape else t.view(dtype)


# eviction policies of a budgeted layer (taurus_eviction)
EVICTION = {"pending": N.EVICT_PENDING, "random": N.EVICT_RANDOM, "fifo": N.EVICT_FIFO, "lru": N.EVICT_LRU}


class Plan:
    """taurus_plan_create / taurus_plan_destroy: the per-graph structures
    (exact chunk index, in-edge lists for sampling) for one chunk size,
    shared by the layers over it and built by the first layer that needs
    each."""

    def __init__(self, n: int, row_off: torch.Tensor, col_dst: torch.Tensor, chunk: int, stream=None):
        self._h = ctypes.c_void_p()
        e = col_dst.numel()
        self.graph = N.Graph(n, e, _dev_ptr(row_off, torch.int64, "row_off"), col_dst.data_ptr() if e else None)
        self.chunk = chunk
        self._keep = (row_off, col_dst)
        N.check(N.lib().taurus_plan_create(ctypes.byref(self.graph), chunk, _stream_ptr(stream),
                                           ctypes.byref(self._h)), "taurus_plan_create")

    @property
    def handle(self):
        return self._h.value

    def destroy(self) -> None:
        if self._h:
            N.lib().taurus_plan_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class Layer:
    """One layer handle (taurus_layer_init ... taurus_layer_destroy)."""

    def __init__(self, n: int, row_off: torch.Tensor, col_dst: torch.Tensor, *, agg: int, d_in: int,
                 d_out: int, weight_cat: np.ndarray, bias: Optional[np.ndarray], out: torch.Tensor,
                 in_dtype: int = N.F32, out_dtype: int = N.F32, relu: bool = False, fanout: int = 0,
                 layer: int = 1, seed: int = 0, chunk: int = 65536, hbm_budget: int = 0,
                 hub_fraction: float = 0.0, stream=None, profile: int = 0, plan: "Plan" = None,
                 eviction: str = "pending", attn: Optional[np.ndarray] = None, d_hidden: int = 0,
                 weight2: Optional[np.ndarray] = None, bias2: Optional[np.ndarray] = None,
                 setup_stream=None):
        """setup_stream: a torch stream for the work the init enqueues (it
        then overlaps what `stream` still has queued, such as an earlier
        layer's chunks); the graph and plan must be ready on it."""
        self._h = ctypes.c_void_p()
        e = col_dst.numel()
        self.graph = N.Graph(n, e, _dev_ptr(row_off, torch.int64, "row_off"),
                             col_dst.data_ptr() if e else None)
        self._w = np.ascontiguousarray(weight_cat, dtype=np.float32)
        self._b = None if bias is None else np.ascontiguousarray(bias, dtype=np.float32)
        self._a = None if attn is None else np.ascontiguousarray(attn, dtype=np.float32).reshape(2, d_out)
        self._w2 = None if weight2 is None else np.ascontiguousarray(weight2, dtype=np.float32)
        self._b2 = None if bias2 is None else np.ascontiguousarray(bias2, dtype=np.float32)
        # the library reads these host arrays at init with the sizes the
        # descriptor implies: a short array would be read past its end
        hidden = d_hidden if agg == N.GIN_MLP else d_out       # accumulator width
        width = 2 * d_out if agg == N.SAGE_MEAN else hidden     # transform columns
        sizes = [(self._w, d_in * width, "weight_cat"), (self._b, hidden, "bias"),
                 (self._a, 2 * d_out if agg == N.GAT_ATT else None, "attn"),
                 (self._w2, d_hidden * d_out if agg == N.GIN_MLP else None, "weight2"),
                 (self._b2, d_out if agg == N.GIN_MLP else None, "bias2")]
        for arr, want, name in sizes:
            if arr is not None and want is not None and arr.size != want:
                raise ValueError(f"{name} has {arr.size} values; this layer needs {want}")
        self.out = out
        out_ptr, out_on_host = _buf_ptr(out, _TORCH_DTYPE[out_dtype], "out")
        self.n, self.d_in, self.d_out, self.chunk, self.in_dtype = n, d_in, d_out, chunk, in_dtype
        self.desc = N.LayerDesc(
            agg=agg, d_in=d_in, d_out=d_out, in_dtype=in_dtype, out_dtype=out_dtype, relu=int(relu),
            weight=self._w.ctypes.data, bias=None if self._b is None else self._b.ctypes.data,
            fanout=fanout, layer=layer, seed=seed & (2**64 - 1), chunk=chunk, hbm_budget=hbm_budget,
            hub_fraction=hub_fraction, out=out_ptr, out_on_host=out_on_host,
            stream=_stream_ptr(stream), profile=int(profile), plan=plan.handle if plan is not None else None,
            eviction=EVICTION[eviction] if isinstance(eviction, str) else int(eviction),
            attn=None if self._a is None else self._a.ctypes.data, d_hidden=d_hidden,
            weight2=None if self._w2 is None else self._w2.ctypes.data,
            bias2=None if self._b2 is None else self._b2.ctypes.data,
            setup_stream=None if setup_stream is None else setup_stream.cuda_stream)
        self._keep = (row_off, col_dst, plan, setup_stream)
        N.check(N.lib().taurus_layer_init(ctypes.byref(self.graph), ctypes.byref(self.desc),
                                          ctypes.byref(self._h)), "taurus_layer_init")

    def push_chunk(self, begin: int, end: int, x: torch.Tensor) -> None:
        """taurus_push_chunk with x = rows [begin, end), on the device or in
        pinned host memory (then it must stay unchanged until the next call)."""
        ptr, on_host = _buf_ptr(x, _TORCH_DTYPE[self.in_dtype], "x")
        # the library reads that many values behind the pointer
        if x.numel() < (end - begin) * self.d_in or (x.dim() == 2 and x.shape[1] != self.d_in):
            raise ValueError(f"x must hold rows [{begin}, {end}) of {self.d_in} values, got shape {tuple(x.shape)}")
        N.check(N.lib().taurus_push_chunk(self._h, begin, end, ptr, on_host), "taurus_push_chunk")

    def push_all(self, x: torch.Tensor, order: Optional[Sequence[int]] = None) -> None:
        """Stream every chunk of the full input x [n][d_in] (vertex order by default)."""
        nchunks = (self.n + self.chunk - 1) // self.chunk
        for j in (range(nchunks) if order is None else order):
            b, e = j * self.chunk, min((j + 1) * self.chunk, self.n)
            self.push_chunk(b, e, x[b:e])

    def stream(self, fill, ctx=None, threads: int = 2, ring: int = 0) -> dict:
        """taurus_stream_layer: the library's loader fills every chunk through
        fill (a C function address, or an N.FILL_FN callback) on `threads`
        host threads into a ring of pinned buffers and pushes them in order.
        ctx: a ctypes object (passed by address), an int address or None.
        Returns the loader's times."""
        fn = fill if isinstance(fill, int) else ctypes.cast(fill, ctypes.c_void_p).value
        if ctx is None or isinstance(ctx, int):
            cp = ctx
        else:
            cp = ctypes.addressof(ctx)
        st = N.StreamStats()
        N.check(N.lib().taurus_stream_layer(self._h, fn, cp, threads, ring, ctypes.byref(st)), "taurus_stream_layer")
        return st.as_dict()

    def finalize(self) -> dict:
        st = N.Stats()
        rc = N.lib().taurus_finalize(self._h, ctypes.byref(st))
        d = st.as_dict()
        if rc != N.OK:
            raise N.TaurusError(rc, "taurus_finalize", N.last_error())
        return d

    def reload_histogram(self, bins: int = 64) -> np.ndarray:
        """taurus_layer_reload_histogram: vertices reloaded exactly i times
        (i < bins - 1), then those reloaded bins - 1 times or more."""
        counts = np.zeros(bins, dtype=np.int64)
        N.check(N.lib().taurus_layer_reload_histogram(self._h, counts.ctypes.data, bins),
                "taurus_layer_reload_histogram")
        return counts

    def sampled_edges(self):
        """(mask_words uint64[ceil(e/64)], n_kept)."""
        words = np.zeros((self.graph.e + 63) // 64, dtype=np.uint64)
        kept = ctypes.c_int64()
        N.check(N.lib().taurus_sampled_edges(self._h, words.ctypes.data if words.size else None,
                                             ctypes.byref(kept)), "taurus_sampled_edges")
        return words, kept.value

    def destroy(self) -> None:
        if self._h:
            N.lib().taurus_layer_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def _check_norm(norm: Optional[dict]) -> None:
    unknown = set(norm or ()) - {"groups", "weight", "bias", "off", "eps", "act"}
    if unknown:
        raise ValueError(f"norm does not know {', '.join(sorted(unknown))}")


def _encode(x: torch.Tensor, encoder: dict, n: int, d_in: Optional[int], stream):
    """The first layer's input, at least n rows of d_in values: vertex v's
    features (x[v], or scale * x[ids[v]]), times its type's weight plus bias,
    normalised."""
    enc = dict(encoder)
    ids, scale, norm = enc.pop("ids", None), enc.pop("scale", 1.0), enc.pop("norm", None)
    off, weight, bias = enc.pop("off", None), enc.pop("weight", None), enc.pop("bias", None)
    if enc:
        raise ValueError(f"encoder does not know {', '.join(sorted(enc))}")
    if (off is None) != (weight is None) or (bias is not None and weight is None):
        raise ValueError("the encoder's linear map needs off and weight together")
    _check_norm(norm)
    rows, width = (x.shape[0] if ids is None else ids.numel()), (x.shape[-1] if weight is None else weight.shape[-1])
    if rows < n or (d_in is not None and width != d_in):
        raise ValueError(f"the encoder gives {rows} rows of {width} values; {n} vertices enter the first layer"
                         + (f" with {d_in} values each" if d_in is not None else ""))
    h = x if ids is None else lookup_rows(x, ids, scale, stream=stream)
    if weight is not None:
        h = grouped_linear(h, off, weight, bias, stream=stream)
    return h if norm is None else group_norm(h, stream=stream, **norm)


def _fits(t, shape, dtype, device, what: str) -> None:
    """An operator's array, checked before the layers that it comes after run
    (device None: not known)."""
    if not torch.is_tensor(t) or t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, got {getattr(t, 'dtype', type(t).__name__)}")
    if tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous with shape {shape}, got shape {tuple(t.shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"{what} must be on {device}, got {t.device}")


def _check_row_norm(norm: Optional[dict], d: int, device, what: str) -> None:
    for name in ("weight", "bias"):
        if norm is not None and norm.get(name) is not None:
            _fits(norm[name], (d,), torch.float32, device, f"{what}'s {name}")
    eps = 1e-5 if norm is None else norm.get("eps", 1e-5)
    if not 0 <= eps < float("inf"):
        raise ValueError(f"{what}'s eps {eps} is not in [0, inf)")


def _check_blocks(layers: list, stream_dtype, device):
    """The layers' norms and residual blocks fit what enters them (stream_dtype:
    the first layer's input; device: the graph's, None if not known).  Returns
    the type of the rows that leave the last."""
    rows_dtype = stream_dtype
    for spec in layers:
        _check_norm(spec.get("norm"))
        block = spec.get("residual")
        out_dtype = _TORCH_DTYPE[spec.get("out_dtype", N.F32)]
        if block is None:
            stream_dtype = rows_dtype = out_dtype
            continue
        unknown = set(block) - {"scale", "gate", "off", "post", "pre"}
        if unknown:
            raise ValueError(f"residual does not know {', '.join(sorted(unknown))}")
        check_norm_args(block.get("post"), "post")
        check_norm_args(block.get("pre"), "pre")
        if spec.get("norm") is not None:
            raise ValueError("a layer has a norm or a residual, whose post is the norm of its output")
        d = spec["d_out"]
        if spec["d_in"] != d:
            raise ValueError(f"a layer of {spec['d_in']} to {d} values has no residual")
        if d > N.RESIDUAL_MOST:
            raise ValueError(f"a residual has at most {N.RESIDUAL_MOST} channels, not {d}")
        if stream_dtype not in (out_dtype, torch.float32):
            raise ValueError(f"the residual stream is {stream_dtype}, the layer's output {out_dtype}")
        gate, off = block.get("gate"), block.get("off")
        if off is not None:
            _fits(off, (max(off.numel(), 1),), torch.int64, device, "off")
        if gate is not None:
            _fits(gate, (d,) if off is None else (off.numel() - 1, d), torch.float32, device, "gate")
        _check_row_norm(block.get("post"), d, device, "post")
        _check_row_norm(block.get("pre"), d, device, "pre")
        rows_dtype = stream_dtype if block.get("pre") is None else out_dtype
    return rows_dtype


def _check_places(x, layers: list, outs, n: int, head: bool, device) -> None:
    """What a residual or the head reads and writes lies on the graph's device,
    and a given output is one that a residual can write.  x: the rows that enter
    the first layer."""
    if device is None:
        return

    def here(t, what):
        if t.device != device:
            raise ValueError(f"{what} must be on {device}, where the graph is, got {t.device}: residuals and heads take "
                             "no rows from the host")

    rows, what = x, "x"
    for i, spec in enumerate(layers):
        out = outs[i] if outs is not None and i < len(outs) else None
        if spec.get("residual") is not None:
            here(rows, what)
            if out is not None:
                here(out, f"outs[{i}]")
                if tuple(out.shape) != (n, spec["d_out"]) or out.dtype != rows.dtype:
                    raise ValueError(f"outs[{i}] must hold the residual stream, {rows.dtype} of shape {(n, spec['d_out'])}, "
                                     f"got {out.dtype} of {tuple(out.shape)}")
                if _overlap(out, rows):
                    raise ValueError(f"outs[{i}] overlaps the rows that enter its block")
            else:
                out = rows
        elif out is None:  # made where x is
            out = torch.empty(0, dtype=_TORCH_DTYPE[spec.get("out_dtype", N.F32)], device=x.device)
        rows, what = out, f"outs[{i}]"
    if head:
        here(rows, what)


def _answer(h: torch.Tensor, head: dict, stream):
    """Log probabilities of the classes of rows h."""
    head = dict(head)
    maps = list(head.pop("linear", ()))
    for i, m in enumerate(maps):  # logits in fp32: 16 bits would make equal ones of different
        h = linear(h, stream=stream, out_dtype=torch.float32 if i + 1 == len(maps) else None, **m)
    return label_log_probs(h, head.pop("labels", None), stream=stream, **head)


def _check_head(head: dict, n: int, width: Optional[int], dtype, device) -> None:
    """The head fits n rows of `width` values (None: not known) of this type;
    device: the graph's, None if not known."""
    unknown = set(head) - {"linear", "labels", "scale", "top", "entropy"}
    if unknown:
        raise ValueError(f"head does not know {', '.join(sorted(unknown))}")
    for m in head["linear"]:
        unknown = set(m) - {"weight", "bias", "act"}
        if unknown or "weight" not in m:
            raise ValueError("head's linear maps have weight, bias and act, got " + ", ".join(sorted(m)))
        if m["weight"].dim() != 2 or width not in (None, m["weight"].shape[0]):
            raise ValueError(f"head's linear map of shape {tuple(m['weight'].shape)} takes no rows of {width} values")
        _fits(m["weight"], tuple(m["weight"].shape), dtype, device, "the weight of a head's linear map")
        width = m["weight"].shape[1]
        if m.get("bias") is not None:
            _fits(m["bias"], (width,), torch.float32, device, "the bias of a head's linear map")
        check_act(m.get("act", "none"))
    labels, top, scale = head.get("labels"), head.get("top", 0), head.get("scale", 1.0)
    if labels is not None and labels.numel() != n:
        raise ValueError(f"head has {labels.numel()} labels for {n} vertices")
    if labels is not None:
        _fits(labels, (n,), torch.int32, device, "labels")
    if width is not None and not 1 <= width <= N.CLASSES_MOST:
        raise ValueError(f"head answers with 1 to {N.CLASSES_MOST} classes, not {width}")
    most = N.TOP_MOST if width is None else min(width, N.TOP_MOST)
    if not 0 <= top <= most:
        raise ValueError(f"head's top {top} is not in [0, {most}]")
    if not 0 < scale < float("inf"):
        raise ValueError(f"head's scale {scale} is not positive and finite")


def run_layers(n: int, row_off: torch.Tensor, col_dst: torch.Tensor, x: torch.Tensor, layers: list,
               *, chunk: int, stream=None, profile: bool = False, outs: Optional[list] = None,
               encoder: Optional[dict] = None, head: Optional[dict] = None):
    """Layer-wise inference: layer l's output is layer l+1's input.

    ``layers`` holds dicts with keys agg, d_in, d_out, weight_cat, bias,
    in_dtype, out_dtype, relu, fanout, layer, seed, and optionally norm, a
    dict of group_norm's arguments (groups, weight, bias, off, eps, act) that
    is applied to the layer's output rows before the next layer takes them
    (the layer itself then usually has relu off).  encoder makes the first
    layer's input from x: a dict with off, weight and bias (vertices grouped
    by type, one linear map each: grouped_linear's), ids and scale (x is a
    table, vertex v's row scale * x[ids[v]]: lookup_rows') and norm, each
    optional; offsets must hold every vertex.

    A layer's residual makes a block of it: a dict of residual_norm's scale,
    gate, off, post and pre.  The rows that entered the block before (the first
    layer's input, or what the layer before put out) are the stream x, the
    layer's output is f; y = x + scale * gate * post(f) is the layer's output
    and the stream of the next block, and the next layer takes pre(y) (y
    without pre).  Offsets must hold every vertex.  The stream has the layers'
    out_dtype or fp32.  The rows that enter a block, its output and the rows that
    enter the head lie on the graph's device: x and outputs in host memory, as
    plain layers take them, go with neither.

    head answers with classes: a dict of linear (a list of dicts of linear's
    weight, bias and act, applied one after another to the last layer's rows,
    after its block's pre; none: the rows are the logits) and
    label_log_probs' labels, scale, top and entropy, each optional.  Its
    LabelLogProbs follows the layers' outputs.

    Returns (outputs, stats); the outputs are complete."""
    layers = list(layers)
    device = None if row_off is None else row_off.device
    rows_dtype = _check_blocks(layers, x.dtype, device)
    rows = x[:n] if encoder is None else torch.empty(0, dtype=x.dtype, device=x.device)  # an encoder's are new
    _check_places(rows, layers, outs, n, head is not None, device)
    if head is not None:
        head = dict(head, linear=list(head.get("linear", ())))
        _check_head(head, n, layers[-1]["d_out"] if layers else None, rows_dtype, device)
    h = x if encoder is None else _encode(x, encoder, n, layers[0]["d_in"] if layers else None, stream)
    results, stats = [], []
    block, norm, rows = None, None, h[:n]  # rows: the residual stream
    plan = Plan(n, row_off, col_dst, chunk, stream=stream)
    for i, spec in enumerate(layers):
        spec = dict(spec)
        norm, block = spec.pop("norm", None), spec.pop("residual", None)
        shape, dtype = (n, spec["d_out"]), _TORCH_DTYPE[spec.get("out_dtype", N.F32)]
        result = outs[i] if outs is not None and outs[i] is not None else torch.empty(
            shape, dtype=dtype if block is None else rows.dtype, device=x.device if block is None else rows.device)
        out = result if norm is None and block is None else torch.empty(shape, dtype=dtype, device=result.device)
        L = Layer(n, row_off, col_dst, out=out, chunk=chunk, stream=stream, profile=profile, plan=plan, **spec)
        L.push_all(h)
        stats.append(L.finalize())
        L.destroy()
        if norm is not None:
            out = group_norm(out, out=result, stream=stream, **norm)
        h = None
        if block is not None:
            out, h = residual_norm(rows, out, out=result, stream=stream, **block)
        results.append(out)
        rows = out
        h = out if h is None else h
    if plan is not None:
        plan.destroy()
    if head is not None:
        answer = _answer(h[:n], head, stream)
        if stream is not None:  # made on that stream, handed to the current one
            for t in answer:
                if t is not None:
                    t.record_stream(torch.cuda.current_stream(t.device))
        results.append(answer)
    if norm is not None or block is not None or head is not None:
        # these are only enqueued; finalize leaves a layer's rows complete
        (torch.cuda.current_stream(h.device) if stream is None else stream).synchronize()
    return results, stats
