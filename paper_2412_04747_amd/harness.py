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


class FfnLayer:
    """Device buffers for one feed-forward block call pair on `rows` rows.  `X`, `Wg`, `Wu`, `Wd` (and `dOut`) are set by the caller."""

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
