"""Convenience wrappers used by the tests, the smoke check and the benchmark.

They only allocate device buffers with PyTorch, copy inputs in / results out and
call the C ABI through `binding`; no layer arithmetic happens here.
"""
import ctypes as C

import numpy as np
import torch

from . import binding as B


def _dev(a, dtype=torch.float32):
    if a is None:
        return None
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype=dtype)


def _tdtype(name):
    """Storage type of the tensor arguments: "f32", or "bf16" (values must already be
    bf16-representable, e.g. from synth.round_to_bf16, so the conversion is exact)."""
    return (B.RGNN_BF16, torch.bfloat16) if name == "bf16" else (B.RGNN_F32, torch.float32)


def _buf(nbytes):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device="cuda")


def _raw_stream(native):
    """device -> hipStream_t of its current stream: torch's own call where this torch has it (0.3 us, 2.7 with a Stream object), which is not in
    its documented interface."""
    return getattr(native, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


_raw = _raw_stream(torch._C)


def _stream():
    """hipStream_t of the current stream."""
    return _raw(torch.cuda.current_device())


class Graph:
    def __init__(self, N, R, src, dst, rel, ntype=None, T=1, rel_src_ntype=None, rel_dst_ntype=None):
        i32 = lambda a: None if a is None else np.ascontiguousarray(a, dtype=np.int32)
        torch.cuda.init()
        self.workspaces = {}
        self.handle = None
        self.N, self.R, self.T, self.E = int(N), int(R), int(T), len(src)
        self.handle = B.rgnn_graph_create(N, T, R, self.E, B.RGNN_COO, i32(src), i32(dst), i32(rel), i32(ntype),
                                          i32(rel_src_ntype), i32(rel_dst_ntype), B.RGNN_MEM_HOST)
        self.info = B.rgnn_graph_info(self.handle)
        self.P, self.Q = int(self.info.num_pairs), int(self.info.num_runs)
        self.workspaces = {}       # scratch buffers the autograd front end keeps per layer configuration

    def export(self, name):
        which = B.INDEX_NAMES.index(name)
        N, E, P, Q, R, T = self.N, self.E, self.P, self.Q, self.R, self.T
        length = {"in_ptr": N + 1, "pair_ptr": R + 1, "pair_src": P, "pair_rel": P, "run_ptr": Q + 1, "run_dst": Q,
                  "run_rel": Q, "dst_run_ptr": N + 1, "relrun_ptr": R + 1, "relrun_idx": Q, "out_ptr": P + 1,
                  "srcpair_ptr": N + 1, "srcpair_idx": P, "ntype_ptr": T + 1, "ntype_perm": N, "relrun_dst": Q,
                  "pair_sel_dst": P, "rel_src_type": R}.get(name, E)
        return B.rgnn_graph_export(self.handle, which, length)

    def close(self):
        self.workspaces.clear()
        if self.handle is not None:
            B.rgnn_graph_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class RgatLayer:
    """Device buffers for one RGAT layer call pair on a graph."""

    def __init__(self, graph, d, slope=0.2, dtype="f32", heads=1, flags=0, d_in=None):
        """d: output width; d_in: input width when it differs."""
        self.g, self.d, self.H = graph, d, heads
        k = d_in or d
        code, self.tdt = _tdtype(dtype)
        self.desc = B.make_desc(code, k, d, heads, slope, flags=flags)
        f, b, s = B.rgnn_workspace_bytes(graph.handle, B.RGNN_LAYER_RGAT, self.desc)
        self.ws = _buf(max(f, b))
        self.saved = _buf(s)
        N, R = graph.N, graph.R
        self.out = torch.empty(N, d, device="cuda")
        self.dX = torch.empty(N, k, device="cuda")
        self.dW = torch.empty(R, k, d, device="cuda")
        self.dw_s = torch.empty(R, d, device="cuda")
        self.dw_t = torch.empty(R, d, device="cuda")

    def load(self, X, W, w_s, w_t, dOut=None):
        t = self.tdt
        self.X, self.W, self.w_s, self.w_t, self.dOut = _dev(X, t), _dev(W, t), _dev(w_s, t), _dev(w_t, t), _dev(dOut, t)

    def fwd(self):
        B.rgnn_rgat_fwd(self.g.handle, self.desc, self.X, self.W, self.w_s, self.w_t, self.out, self.saved, self.ws,
                        _stream())

    def bwd(self):
        B.rgnn_rgat_bwd(self.g.handle, self.desc, self.X, self.W, self.w_s, self.w_t, self.out, self.saved, self.dOut,
                        self.dX, self.dW, self.dw_s, self.dw_t, self.ws, _stream())

    def saved_views(self):
        """The parts of `saved` where rows are kept per pair: Hs [P, d], s_dst [Q, heads], ms [N, heads, 2]."""
        P, Q, N, d, H = self.g.P, self.g.Q, self.g.N, self.d, self.H
        al = lambda n: (max(n, 1) * 4 + 255) // 256 * 256 // 4
        f32 = self.saved.view(torch.float32)
        hs = f32[: P * d].view(P, d)
        off = al(P * d)
        s_dst = f32[off: off + Q * H].view(Q, H)
        off += al(Q * H)
        return hs, s_dst, f32[off: off + 2 * N * H].view(N, H, 2)

    def grads(self):
        return dict(dX=self.dX, dW=self.dW, dw_s=self.dw_s, dw_t=self.dw_t)


class RgcnLayer:
    def __init__(self, graph, d, norm="in_degree_per_rel", act="none", self_loop=False, dtype="f32", flags=0, d_in=None):
        """d: output width; d_in: input width when it differs."""
        self.g, self.d, self.self_loop = graph, d, self_loop
        k = d_in or d
        code, self.tdt = _tdtype(dtype)
        self.desc = B.make_desc(code, k, d, 1, 0.0,
                                B.RGNN_NORM_IN_DEGREE_PER_REL if norm == "in_degree_per_rel" else B.RGNN_NORM_NONE,
                                B.RGNN_ACT_RELU if act == "relu" else B.RGNN_ACT_NONE, flags)
        f, b, s = B.rgnn_workspace_bytes(graph.handle, B.RGNN_LAYER_RGCN, self.desc)
        self.ws = _buf(max(f, b))
        self.saved = _buf(s)
        N, R = graph.N, graph.R
        self.out = torch.empty(N, d, device="cuda")
        self.dX = torch.empty(N, k, device="cuda")
        self.dW = torch.empty(R, k, d, device="cuda")
        self.dW0 = torch.empty(k, d, device="cuda") if self_loop else None

    def load(self, X, W, W0=None, dOut=None):
        t = self.tdt
        self.X, self.W, self.W0, self.dOut = _dev(X, t), _dev(W, t), _dev(W0, t), _dev(dOut, t)

    def fwd(self):
        B.rgnn_rgcn_fwd(self.g.handle, self.desc, self.X, self.W, self.W0, self.out, self.saved, self.ws, _stream())

    def bwd(self):
        B.rgnn_rgcn_bwd(self.g.handle, self.desc, self.X, self.W, self.W0, self.out, self.saved, self.dOut, self.dX,
                        self.dW, self.dW0, self.ws, _stream())

    def grads(self):
        g = dict(dX=self.dX, dW=self.dW)
        if self.self_loop:
            g["dW0"] = self.dW0
        return g


class HgtLayer:
    def __init__(self, graph, d, heads, with_mu=True, dtype="f32", flags=0):
        self.g, self.d, self.H = graph, d, heads
        code, self.tdt = _tdtype(dtype)
        self.desc = B.make_desc(code, d, d, heads, flags=flags)
        f, b, s = B.rgnn_workspace_bytes(graph.handle, B.RGNN_LAYER_HGT, self.desc)
        self.ws = _buf(max(f, b))
        self.saved = _buf(s)
        N, R, T, dh = graph.N, graph.R, graph.T, d // heads
        e = lambda *shape: torch.empty(*shape, device="cuda")
        self.out, self.dX = e(N, d), e(N, d)
        self.dWk, self.dWq, self.dWv, self.dWo = e(T, d, d), e(T, d, d), e(T, d, d), e(T, d, d)
        self.dWatt, self.dWmsg = e(R, heads, dh, dh), e(R, heads, dh, dh)
        self.dmu = e(R, heads) if with_mu else None

    def load(self, X, Wk, Wq, Wv, Wo, Watt, Wmsg, mu=None, dOut=None):
        (self.X, self.Wk, self.Wq, self.Wv, self.Wo, self.Watt, self.Wmsg, self.mu, self.dOut) = (
            _dev(a, self.tdt) for a in (X, Wk, Wq, Wv, Wo, Watt, Wmsg, mu, dOut))

    def fwd(self):
        B.rgnn_hgt_fwd(self.g.handle, self.desc, self.X, self.Wk, self.Wq, self.Wv, self.Wo, self.Watt, self.Wmsg,
                       self.mu, self.out, self.saved, self.ws, _stream())

    def bwd(self):
        B.rgnn_hgt_bwd(self.g.handle, self.desc, self.X, self.Wk, self.Wq, self.Wv, self.Wo, self.Watt, self.Wmsg,
                       self.mu, self.out, self.saved, self.dOut, self.dX, self.dWk, self.dWq, self.dWv, self.dWo,
                       self.dWatt, self.dWmsg, self.dmu, self.ws, _stream())

    def grads(self):
        g = dict(dX=self.dX, dWk=self.dWk, dWq=self.dWq, dWv=self.dWv, dWo=self.dWo, dWatt=self.dWatt,
                 dWmsg=self.dWmsg)
        if self.dmu is not None:
            g["dmu"] = self.dmu
        return g


class NormLayer:
    """Device buffers for one residual norm call pair on `rows` rows.  `x`, `residual`, `weight` (and `dOut`, `dSum`) are set by the
    caller; types "f32" or "bf16".  Without a residual, `total` is `x`'s type and the backward's `sum` is x."""

    def __init__(self, rows, width, x="f32", total="f32", out="f32", eps=1e-6, residual=True, flags=0):
        (cx, tx), (cs, ts), (co, to) = _tdtype(x), _tdtype(total), _tdtype(out)
        self.desc = B.make_norm_desc(rows, width, cx, cs, co, eps, flags)
        self.ws = _buf(B.rgnn_norm_workspace_bytes(self.desc))
        e = lambda t: torch.empty(rows, width, device="cuda", dtype=t)
        self.residual = self.dSum = None
        self.out, self.sum = e(to), e(ts) if residual else None
        # one buffer where the gradients of x and of the residual are of one type
        self.dResidual = e(ts) if residual else None
        self.dX = e(tx) if not residual or tx != ts else None
        self.dWeight = torch.empty(width, device="cuda")

    def fwd(self):
        B.rgnn_norm_fwd(self.desc, self.x, self.residual, self.weight, self.sum, self.out, _stream())

    def bwd(self):
        B.rgnn_norm_bwd(self.desc, self.sum, self.weight, self.dOut, self.dSum, self.dX, self.dResidual, self.dWeight, self.ws, _stream())


_ROW_TYPES = {torch.float32: B.RGNN_F32, torch.bfloat16: B.RGNN_BF16}
_STORED = {code: t for t, code in _ROW_TYPES.items()}


class _Checked:
    """A buffer that callers may put their own in the place of: its type, size, order and place are looked at when it is set.  want(owner): its type and number of
    elements.  (Reads find the tensor itself in the owner.)"""

    def __init__(self, want, optional=True):
        self.want, self.optional = want, optional

    def __set_name__(self, owner, name):
        self.name = name

    def __set__(self, owner, t):
        if t is owner.__dict__.get(self.name, self):
            return
        if t is not None or not self.optional:
            dtype, n = self.want(owner)
            if t is None or t.dtype != dtype or t.numel() != n or not t.is_cuda or not t.is_contiguous():
                raise TypeError(f"{type(owner).__name__}.{self.name}: {n} contiguous elements in {dtype} on the GPU are wanted"
                                + ("" if t is None else f", not {tuple(t.shape)} in {t.dtype}"))
        owner.__dict__[self.name] = t


class Rows8:
    """Buffers for `rows` rows held in 8 bits: `codes` int8 [rows, width], `scales` uint8 [rows, blocks of 32 columns].  Both may be replaced by the
    caller's own."""

    codes = _Checked(lambda r: (torch.int8, r.rows * r.width), optional=False)
    scales = _Checked(lambda r: (torch.uint8, r.rows * -(-r.width // 32)), optional=False)

    def __init__(self, rows, width):
        self.rows, self.width = rows, width
        self.codes = torch.empty(rows, width, device="cuda", dtype=torch.int8)
        self.scales = torch.empty(rows, -(-width // 32), device="cuda", dtype=torch.uint8)
        self._descs = {t: B.make_rows8_desc(rows, width, code) for t, code in _ROW_TYPES.items()}
        self._table = B.rows8(None, None)         # (filled in at each call)

    def _desc(self, x):
        if x.dtype not in self._descs or not x.is_cuda or not x.is_contiguous() or x.numel() != self.rows * self.width:
            raise TypeError(f"Rows8: {self.rows} contiguous rows of {self.width} in fp32 or bf16 on the GPU are wanted, not {tuple(x.shape)} in {x.dtype}")
        return self._descs[x.dtype]

    def tensors(self):
        self._table.codes, self._table.scales = self.codes.data_ptr(), self.scales.data_ptr()
        return self._table

    def pack(self, x):
        B.rgnn_rows8_pack(self._desc(x), x, self.tensors(), _stream())

    def unpack(self, x):
        B.rgnn_rows8_unpack(self._desc(x), self.tensors(), x, _stream())


class BlockNormLayer:
    """Device buffers for one junction call pair on `rows` rows: norm after a block, gate and residual scale by node type, norm before the next.  `a`, `s`
    (and `dOut`, `dSum`), the parameters and `types` (int32, with more than one) are set by the caller; types "f32" or "bf16".  held: the forward leaves
    a and s in 8 bits (`held_a`, `held_s`), and the backward reads them there."""

    _rows = lambda code: _Checked(lambda L: (_STORED[getattr(L.desc, code)], L.desc.rows * L.desc.width))
    a, s, dOut, dSum = _rows("a_dtype"), _rows("sum_dtype"), _rows("out_dtype"), _rows("sum_dtype")
    types = _Checked(lambda L: (torch.int32, L.desc.rows))
    w_after, w_before = (_Checked(lambda L: (torch.float32, L.desc.width)) for _ in range(2))
    gate = _Checked(lambda L: (torch.float32, L.desc.types * L.desc.width))
    scale = _Checked(lambda L: (torch.float32, L.desc.types))
    del _rows

    def __init__(self, rows, width, a="f32", total="f32", out="f32", types=1, eps=1e-6, held=False, flags=0):
        (ca, ta), (cs, ts), (co, to) = _tdtype(a), _tdtype(total), _tdtype(out)
        self.desc = B.make_block_norm_desc(rows, width, ca, cs, co, types, eps, flags)
        self.ws = _buf(B.rgnn_block_norm_workspace_bytes(self.desc))
        e = lambda *shape, t=torch.float32: torch.empty(*shape, device="cuda", dtype=t)
        self._table = B.block_norm_params()       # (filled in at each call)
        self.types = self.w_after = self.w_before = self.gate = self.scale = None
        self.a = self.s = self.dOut = self.dSum = None
        self.sum, self.out, self.dA, self.dS = e(rows, width, t=ts), e(rows, width, t=to), e(rows, width, t=ta), e(rows, width, t=ts)
        self.dWAfter, self.dWBefore, self.dGate, self.dScale = e(width), e(width), e(types, width), e(types)
        self.held_a, self.held_s = (Rows8(rows, width), Rows8(rows, width)) if held else (None, None)

    def _params(self):
        p, at = self._table, B._addr
        p.row_types, p.w_after, p.gate, p.scale, p.w_before = at(self.types), at(self.w_after), at(self.gate), at(self.scale), at(self.w_before)
        return p

    def _held(self):
        return (None, None) if self.held_a is None else (self.held_a.tensors(), self.held_s.tensors())

    def fwd(self):
        a8, s8 = self._held()
        B.rgnn_block_norm_fwd(self.desc, self._params(), self.a, self.s, self.sum, None if self.w_before is None else self.out, a8, s8, _stream())

    def bwd(self):
        a8, s8 = self._held()
        grads = B.block_norm_grads(*(g if p is not None else None for g, p in (
            (self.dWAfter, self.w_after), (self.dGate, self.gate), (self.dScale, self.scale), (self.dWBefore, self.w_before))))
        a, s = (self.a, self.s) if a8 is None else (None, None)
        B.rgnn_block_norm_bwd(self.desc, self._params(), a, s, a8, s8, self.dOut, self.dSum, self.dA, self.dS, grads, self.ws, _stream())


class FfnLayer:
    """Device buffers for one feed-forward block call pair on `rows` rows.  `X`, `Wg`, `Wu`, `Wd` (and `dOut`) are set by the caller; for `bwd_held`, the
    backward from rows in 8 bits, `held` (Rows8) instead of `X`."""

    def __init__(self, rows, width, hidden, dtype="f32", act="silu", flags=0):
        code, t = _tdtype(dtype)
        self.desc = B.make_ffn_desc(rows, width, hidden, code, B.RGNN_ACT_RELU if act == "relu" else B.RGNN_ACT_SILU, flags)
        self.ws = _buf(max(B.rgnn_ffn_workspace_bytes(self.desc)))
        e = lambda *shape: torch.empty(*shape, device="cuda", dtype=t)
        self.out, self.dX = e(rows, width), e(rows, width)
        self.dWg, self.dWu, self.dWd = e(width, hidden), e(width, hidden), e(hidden, width)

    def fwd(self):
        B.rgnn_ffn_fwd(self.desc, self.X, self.Wg, self.Wu, self.Wd, self.out, self.ws, _stream())

    def bwd(self):
        B.rgnn_ffn_bwd(self.desc, self.X, self.Wg, self.Wu, self.Wd, self.dOut, self.dX, self.dWg, self.dWu, self.dWd, self.ws, _stream())

    def bwd_held(self):
        if (self.held.rows, self.held.width) != (self.desc.rows, self.desc.width):
            raise ValueError(f"FfnLayer: held rows are [{self.held.rows}, {self.held.width}], not [{self.desc.rows}, {self.desc.width}]")
        B.rgnn_ffn_bwd_rows8(self.desc, self.held.tensors(), self.Wg, self.Wu, self.Wd, self.dOut, self.dX, self.dWg, self.dWu, self.dWd, self.ws, _stream())

    def grads(self):
        return dict(dX=self.dX, dWg=self.dWg, dWu=self.dWu, dWd=self.dWd)


def _dense(t):
    """Whether the tensor's elements fill one stretch of memory, in whatever order."""
    if t.is_contiguous():
        return True
    step = 1
    for stride, size in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n != 1):
        if stride != step:
            return False
        step *= size
    return True


_CLIP_TYPES = {torch.float32: B.RGNN_F32, torch.bfloat16: B.RGNN_BF16}


class GradClip:
    """The workspace, tables and result buffers for clipping tensors of the sizes and types of `like`, in place or into `clipped`."""

    def __init__(self, like, in_place=True):
        for t in like:
            if t.dtype not in _CLIP_TYPES or not t.is_cuda or not _dense(t):
                raise TypeError(f"GradClip takes dense fp32 or bf16 tensors on the GPU, not {t.dtype} of strides {t.stride()} on {t.device}")
        self._numel, self._types, self._devices = [t.numel() for t in like], [t.dtype for t in like], [t.get_device() for t in like]
        # (tensors that are not contiguous are taken by their exact layout)
        self._layouts = None if all(t.is_contiguous() for t in like) else [(t.shape, t.stride()) for t in like]
        self.ws = _buf(B.rgnn_clip_workspace_bytes(self._numel))
        self.sizes, self.dtypes = B.clip_tables(self._numel, [_CLIP_TYPES[t] for t in self._types])
        self.norm = torch.empty((), device="cuda")
        self.clipped = None if in_place else [torch.empty_like(t) for t in like]
        self._to = None if in_place else B.addresses(self.clipped)

    def _check(self, grads):
        if len(grads) != len(self._numel):
            raise ValueError(f"GradClip.clip: {len(grads)} tensors, made for {len(self._numel)}")
        if (list(map(torch.Tensor.numel, grads)) != self._numel or [t.dtype for t in grads] != self._types
                or list(map(torch.Tensor.get_device, grads)) != self._devices):
            raise ValueError("GradClip.clip: tensors of other sizes, types or devices than it is made for")
        if (not all(map(torch.Tensor.is_contiguous, grads)) if self._layouts is None
                else [(t.shape, t.stride()) for t in grads] != self._layouts):
            raise ValueError("GradClip.clip: tensors of another layout than it is made for")

    def clip(self, grads, max_norm):
        """`grads`: tensors of the sizes, types and layouts of `like`, in its order."""
        self._check(grads)
        given = (C.c_void_p * len(grads))(*map(torch.Tensor.data_ptr, grads))
        B.rgnn_clip_grad_norm(given, given if self._to is None else self._to, self.sizes, self.dtypes, max_norm, self.norm, self.ws, _stream())
