"""PyTorch autograd front end of the layer library.

`rgat`, `rgcn` and `hgt` are differentiable functions of torch tensors that live on the GPU;
`RgatConv`, `RgcnConv` and `HgtConv` are `torch.nn.Module`s holding the parameters.  Forward and
backward are the C-ABI calls of `binding`; PyTorch only owns the memory, the stream and the
tape.  The layers are fp32 (the training protocol of the thesis' evaluation section: full-graph
training of a two-layer model with a negative-log-likelihood loss).

`residual_norm` and `gated_ffn` (`ResidualNorm`, `GatedFfn`) are what stands between the layers of a residual
model; they take fp32 or bf16 rows and need no graph (the layers here are fp32 only; the C calls also take bf16 rows).
`block_norm` (`BlockNorm`) joins a block's output to the residual stream: norm after the block, gate and residual scale by node type, norm
before the next block.  With held=True, `block_norm` and `gated_ffn` keep their rows for the backward in 8 bits (`pack_rows` has the
format) instead of the tensors themselves: results are the same, gradients are those of the held values.
`clip_grad_norm_` bounds the global norm of a model's gradients before the optimiser's step.

The workspace of a (layer kind, width, options) combination is allocated once per graph, kept on the
`Graph` object and dropped by `Graph.close()`; every call of that combination on the graph reuses it,
so such calls must not overlap on different streams.
"""
import math

import torch
from torch.autograd.function import once_differentiable

from . import binding as B
from .harness import Graph, _buf, _dense, _stream


def _bufs(graph, layer, desc, key):
    """(workspace, (forward size, saved size)) for a layer configuration on a graph.  The workspace lives in
    `graph.workspaces` (sized by rgnn_workspace_bytes for this very graph), so it can neither outlive
    the graph nor be handed to another one."""
    if graph.handle is None:
        raise RuntimeError("the graph has been closed")
    k = (layer,) + key
    if k not in graph.workspaces:
        f, b, s = B.rgnn_workspace_bytes(graph.handle, layer, desc)
        graph.workspaces[k] = (_buf(max(f, b)), (f, s))
    return graph.workspaces[k]


def _room(graph, layer, desc, key, keep):
    """(workspace, saved) of a forward call; keep: a backward may follow.  A call that keeps nothing takes the graph's workspace where
    it holds what `saved` would as well (RGCN's forward size covers that), otherwise one for its duration."""
    ws, (f, s) = _bufs(graph, layer, desc, key)
    if keep:
        return ws, _buf(s) if s else None
    need = f if layer == B.RGNN_LAYER_RGCN else (f + 255) // 256 * 256 + s
    return (ws if ws.numel() >= need else _buf(need)), None


def release(graph):
    """Drop the cached workspaces of a graph (Graph.close() does the same)."""
    graph.workspaces.clear()


def _f32(t):
    if t is None:
        return None
    if t.dtype != torch.float32 or not t.is_cuda:
        raise TypeError("rgnn autograd functions take fp32 CUDA tensors")
    return t.contiguous()


class _Rgat(torch.autograd.Function):
    @staticmethod
    def forward(ctx, graph, keep, slope, heads, X, W, w_s, w_t):
        X, W, w_s, w_t = _f32(X), _f32(W), _f32(w_s), _f32(w_t)
        d_in, d = W.shape[-2], W.shape[-1]
        desc = B.make_desc(B.RGNN_F32, d_in, d, heads, slope)
        ws, saved = _room(graph, B.RGNN_LAYER_RGAT, desc, (d_in, d, heads), keep)
        out = torch.empty(graph.N, d, device=X.device)
        B.rgnn_rgat_fwd(graph.handle, desc, X, W, w_s, w_t, out, saved, ws, _stream())
        ctx.graph, ctx.desc, ctx.ws, ctx.saved_buf = graph, desc, ws, saved
        ctx.save_for_backward(X, W, w_s, w_t, out)
        return out

    @staticmethod
    def backward(ctx, dOut):
        X, W, w_s, w_t, out = ctx.saved_tensors
        dOut = _f32(dOut)
        dX, dW, dws, dwt = (torch.empty_like(t) for t in (X, W, w_s, w_t))
        B.rgnn_rgat_bwd(ctx.graph.handle, ctx.desc, X, W, w_s, w_t, out, ctx.saved_buf, dOut, dX, dW, dws, dwt, ctx.ws,
                        _stream())
        return None, None, None, None, dX, dW, dws, dwt


class _Rgcn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, graph, keep, norm, act, X, W, W0):
        X, W, W0 = _f32(X), _f32(W), _f32(W0)
        d_in, d = W.shape[-2], W.shape[-1]
        desc = B.make_desc(B.RGNN_F32, d_in, d, 1, 0.0,
                           B.RGNN_NORM_IN_DEGREE_PER_REL if norm == "in_degree_per_rel" else B.RGNN_NORM_NONE,
                           B.RGNN_ACT_RELU if act == "relu" else B.RGNN_ACT_NONE)
        ws, saved = _room(graph, B.RGNN_LAYER_RGCN, desc, (d_in, d, norm, act), keep)
        out = torch.empty(graph.N, d, device=X.device)
        B.rgnn_rgcn_fwd(graph.handle, desc, X, W, W0, out, saved, ws, _stream())
        ctx.graph, ctx.desc, ctx.ws, ctx.saved_buf, ctx.has_w0 = graph, desc, ws, saved, W0 is not None
        ctx.save_for_backward(X, W, out, *([W0] if W0 is not None else []))
        return out

    @staticmethod
    def backward(ctx, dOut):
        X, W, out, *rest = ctx.saved_tensors
        W0 = rest[0] if ctx.has_w0 else None
        dOut = _f32(dOut)
        dX, dW = torch.empty_like(X), torch.empty_like(W)
        dW0 = torch.empty_like(W0) if W0 is not None else None
        B.rgnn_rgcn_bwd(ctx.graph.handle, ctx.desc, X, W, W0, out, ctx.saved_buf, dOut, dX, dW, dW0, ctx.ws, _stream())
        return None, None, None, None, dX, dW, dW0


class _Hgt(torch.autograd.Function):
    @staticmethod
    def forward(ctx, graph, X, Wk, Wq, Wv, Wo, Watt, Wmsg, mu):
        X, Wk, Wq, Wv, Wo, Watt, Wmsg, mu = (_f32(t) for t in (X, Wk, Wq, Wv, Wo, Watt, Wmsg, mu))
        d, H = Wk.shape[-1], Watt.shape[1]
        desc = B.make_desc(B.RGNN_F32, d, d, H)
        ws, (_, s) = _bufs(graph, B.RGNN_LAYER_HGT, desc, (d, H))
        out = torch.empty(graph.N, d, device=X.device)
        saved = _buf(s)
        B.rgnn_hgt_fwd(graph.handle, desc, X, Wk, Wq, Wv, Wo, Watt, Wmsg, mu, out, saved, ws, _stream())
        ctx.graph, ctx.desc, ctx.ws, ctx.saved_buf, ctx.has_mu = graph, desc, ws, saved, mu is not None
        ctx.save_for_backward(X, Wk, Wq, Wv, Wo, Watt, Wmsg, out, *([mu] if mu is not None else []))
        return out

    @staticmethod
    def backward(ctx, dOut):
        X, Wk, Wq, Wv, Wo, Watt, Wmsg, out, *rest = ctx.saved_tensors
        mu = rest[0] if ctx.has_mu else None
        dOut = _f32(dOut)
        g = [torch.empty_like(t) for t in (X, Wk, Wq, Wv, Wo, Watt, Wmsg)]
        dmu = torch.empty_like(mu) if mu is not None else None
        B.rgnn_hgt_bwd(ctx.graph.handle, ctx.desc, X, Wk, Wq, Wv, Wo, Watt, Wmsg, mu, out, ctx.saved_buf, dOut, *g, dmu,
                       ctx.ws, _stream())
        return (None, *g, dmu)


def _rows(*tensors):
    """The tensors (None stays) as the row operators take them: contiguous fp32 or bf16, on one GPU."""
    device = next(t.device for t in tensors if t is not None)
    for t in tensors:
        if t is not None and (t.dtype not in (torch.float32, torch.bfloat16) or not t.is_cuda or t.device != device):
            raise TypeError("rgnn row operators take fp32 or bf16 CUDA tensors on one device")
    return [t if t is None else _aligned(t) for t in tensors]


def _aligned(t):
    """The tensor, contiguous and from a 16-byte boundary on (a contiguous slice may start between two)."""
    return t.contiguous() if t.data_ptr() % 16 == 0 or not t.is_contiguous() else t.clone()


_CODES = {torch.float32: B.RGNN_F32, torch.bfloat16: B.RGNN_BF16}


def _code(dtype):
    if dtype not in _CODES:
        raise TypeError(f"rgnn row operators take and give fp32 or bf16, not {dtype}")
    return _CODES[dtype]


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, eps, out_dtype, x, residual, weight):
        ctx.set_materialize_grads(False)
        x, residual, weight = _rows(x, residual, weight)
        width = weight.numel()
        if weight.dim() != 1 or width == 0 or weight.dtype != torch.float32:
            raise TypeError("residual_norm: weight is a vector in fp32")
        if x.dim() < 1 or x.shape[-1] != width or (residual is not None and residual.shape != x.shape):
            raise ValueError(f"residual_norm: rows of {width} are wanted, got {tuple(x.shape)}"
                             + (f" and {tuple(residual.shape)}" if residual is not None else ""))
        with torch.cuda.device(x.device):
            total = torch.empty_like(residual) if residual is not None else None
            out = torch.empty(x.shape, dtype=out_dtype, device=x.device)
            kept = x if total is None else total
            ctx.desc = B.make_norm_desc(x.numel() // width, width, _code(x.dtype), _code(kept.dtype), _code(out_dtype), eps)
            B.rgnn_norm_fwd(ctx.desc, x, residual, weight, total, out, _stream())
        ctx.x_dtype, ctx.residual = x.dtype, residual is not None
        ctx.save_for_backward(kept, weight)
        return (out, total) if ctx.residual else out

    @staticmethod
    @once_differentiable
    def backward(ctx, dOut, dSum=None):
        kept, weight = ctx.saved_tensors
        if dOut is None:                   # only the sum was used
            if dSum is None:
                return None, None, None, None, None
            return None, None, dSum.to(ctx.x_dtype), dSum, None
        dOut, dSum = _rows(dOut, dSum)
        with torch.cuda.device(kept.device):
            need_x, need_r, need_w = ctx.needs_input_grad[2:]
            same = ctx.x_dtype == kept.dtype
            dX = torch.empty(kept.shape, dtype=ctx.x_dtype, device=kept.device) if need_x or (need_r and same) else None
            dR = torch.empty_like(kept) if need_r and not same else None
            dW = torch.empty_like(weight) if need_w else None
            ws = _buf(B.rgnn_norm_workspace_bytes(ctx.desc)) if need_w else None
            B.rgnn_norm_bwd(ctx.desc, kept, weight, dOut, dSum, dX, dR, dW, ws, _stream())
        return None, None, dX if need_x else None, (dX if same else dR) if need_r else None, dW


def _held(wanted):
    """Whether rows are to be held in 8 bits: only where a graph may be recorded.  (Within a Function's forward grad mode is off, and parameters ask for
    gradients whether or not there is one.)"""
    return bool(wanted) and torch.is_grad_enabled()


def _pack(x):
    """(codes, scales) of contiguous rows in 8 bits."""
    width = x.shape[-1]
    rows = x.numel() // width if width else 0
    codes = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    scales = torch.empty(*x.shape[:-1], -(-width // 32), dtype=torch.uint8, device=x.device)
    B.rgnn_rows8_pack(B.make_rows8_desc(rows, width, _code(x.dtype)), x, B.rows8(codes, scales), _stream())
    return codes, scales


@torch.no_grad()
def pack_rows(x):
    """Rows (the last dimension, up to 8192) in 8 bits: (codes, scales), int8 of x's shape and a uint8 for every 32 columns of a row.  A value stands
    for codes * 2^(scales - 133), off by at most half a step, 2^(scales - 134); the step is the least power of two with which the largest of the 32
    rounds to at most 127.  An infinity or NaN makes its 32 columns NaN."""
    x, = _rows(x)
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError(f"pack_rows: rows of one column at least are wanted, got {tuple(x.shape)}")
    with torch.cuda.device(x.device):
        return _pack(x)


@torch.no_grad()
def unpack_rows(codes, scales, dtype=torch.float32):
    """The rows that `pack_rows` gave, exact in fp32 and in bf16."""
    if codes.dtype != torch.int8 or scales.dtype != torch.uint8 or not codes.is_cuda or scales.device != codes.device:
        raise TypeError("unpack_rows: codes are int8 and scales uint8, on one GPU")
    if codes.dim() < 1 or codes.shape[-1] < 1 or scales.shape != (*codes.shape[:-1], -(-codes.shape[-1] // 32)):
        raise ValueError(f"unpack_rows: scales {tuple(scales.shape)} do not fit codes {tuple(codes.shape)}")
    code, width = _code(dtype), codes.shape[-1]
    with torch.cuda.device(codes.device):
        codes, scales = _aligned(codes), scales.contiguous()
        x = torch.empty(codes.shape, dtype=dtype, device=codes.device)
        B.rgnn_rows8_unpack(B.make_rows8_desc(codes.numel() // width, width, code), B.rows8(codes, scales), x, _stream())
    return x


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, eps, out_dtype, held, num_types, types, a, s, w_after, w_before, gate, scale):
        ctx.set_materialize_grads(False)
        a, s, types, w_after, w_before, gate, scale = (None if t is None else _aligned(t) for t in (a, s, types, w_after, w_before, gate, scale))
        width = a.shape[-1]
        with torch.cuda.device(a.device):
            ctx.desc = B.make_block_norm_desc(a.numel() // width, width, _code(a.dtype), _code(s.dtype), _code(out_dtype), num_types, eps)
            total = torch.empty_like(s)
            out = torch.empty(a.shape, dtype=out_dtype, device=a.device) if w_before is not None else None
            a8 = s8 = None
            ctx.held = held and any(ctx.needs_input_grad)
            if ctx.held:
                kept = [torch.empty(*a.shape[:-1], n, dtype=t, device=a.device) for _ in "as" for n, t in ((width, torch.int8), (-(-width // 32), torch.uint8))]
                a8, s8 = B.rows8(*kept[:2]), B.rows8(*kept[2:])
            B.rgnn_block_norm_fwd(ctx.desc, B.block_norm_params(types, w_after, gate, scale, w_before), a, s, total, out, a8, s8, _stream())
        ctx.types_of = a.dtype, s.dtype
        ctx.save_for_backward(types, w_after, w_before, gate, scale, *(kept if ctx.held else (a, s)))
        return (out, total) if out is not None else total

    @staticmethod
    @once_differentiable
    def backward(ctx, *grads):
        types, w_after, w_before, gate, scale, *kept = ctx.saved_tensors
        dOut, dSum = grads if w_before is not None else (None, *grads)
        if dOut is None and dSum is None:
            return (None,) * 11
        dOut, dSum = _rows(dOut, dSum)
        device = kept[0].device
        with torch.cuda.device(device):
            need = ctx.needs_input_grad[5:]
            shape = kept[0].shape
            dA, dS = (torch.empty(shape, dtype=t, device=device) if n else None for n, t in zip(need, ctx.types_of))
            dw = [torch.empty_like(t) if n else None for n, t in zip(need[2:], (w_after, w_before, gate, scale))]
            g = B.block_norm_grads(dw[0], dw[2], dw[3], dw[1])
            a8, s8 = (B.rows8(*kept[:2]), B.rows8(*kept[2:])) if ctx.held else (None, None)
            a, s = (None, None) if ctx.held else kept
            ws = _buf(B.rgnn_block_norm_workspace_bytes(ctx.desc)) if any(need[2:]) else None
            B.rgnn_block_norm_bwd(ctx.desc, B.block_norm_params(types, w_after, gate, scale, w_before), a, s, a8, s8, dOut, dSum, dA, dS, g, ws, _stream())
        return (None, None, None, None, None, dA, dS, *dw)


def block_norm(a, s, w_after=None, w_before=None, gate=None, scale=None, types=None, eps=1e-6, out_dtype=None, held=False):
    """Joins a block's output `a` to the residual stream `s`, over the last dimension:
        n = a / sqrt(mean(a^2) + eps) * w_after;   sum = scale[t] * s + gate[t] * n;   out = sum / sqrt(mean(sum^2) + eps) * w_before
    and returns (out, sum), or sum alone without w_before.  t = types (int32, a's shape without the last dimension); gate [width] or [types,
    width], scale [] or [types]; w_after, w_before [width]; all fp32.  What is not given is left out: the norm after the block, the gate (1), the scale (1),
    the norm before the next.  sum has s's type, out has out_dtype (fp32 or bf16; default: a's).  A row whose type is not one of the parameters' stands for
    nothing (a batch's padding): it is not read, and its results and gradients are zeros.
    HGT's skip connection: gate = sigmoid(p)[:, None].expand(-1, width), scale = 1 - sigmoid(p).
    held: a and s are kept for the backward in 8 bits (without a backward, nothing is packed)."""
    if out_dtype is not None and out_dtype not in _CODES:
        raise TypeError(f"block_norm: out_dtype is fp32 or bf16, not {out_dtype}")
    for t in (a, s):
        _code(t.dtype)
    if a.dim() < 1 or a.shape[-1] < 1 or s.shape != a.shape:
        raise ValueError(f"block_norm: rows of one shape are wanted, got {tuple(a.shape)} and {tuple(s.shape)}")
    width, counts = a.shape[-1], set()
    for name, t, dims in (("w_after", w_after, (1,)), ("w_before", w_before, (1,)), ("gate", gate, (1, 2)), ("scale", scale, (0, 1))):
        if t is None:
            continue
        if t.dtype != torch.float32:
            raise TypeError(f"block_norm: {name} is fp32, not {t.dtype}")
        if t.dim() not in dims or (name != "scale" and t.shape[-1] != width) or t.numel() == 0:
            raise ValueError(f"block_norm: {name} of shape {tuple(t.shape)} does not fit rows of {width}")
        if name in ("gate", "scale"):
            counts.add(t.numel() if name == "scale" else t.numel() // width)
    if len(counts) > 1:
        raise ValueError(f"block_norm: gate and scale are of {sorted(counts)} types")
    num_types = counts.pop() if counts else 1
    if types is None and num_types > 1:
        raise ValueError(f"block_norm: parameters of {num_types} types, but no types of the rows")
    if types is not None:
        if types.dtype != torch.int32:
            raise TypeError(f"block_norm: types are int32, not {types.dtype}")
        if types.shape != a.shape[:-1]:
            raise ValueError(f"block_norm: types of shape {tuple(types.shape)} for rows {tuple(a.shape)}")
    for t in (a, s, w_after, w_before, gate, scale, types):
        if t is not None and (not t.is_cuda or t.device != a.device):
            raise TypeError("block_norm takes tensors on one GPU")
    return _BlockNorm.apply(float(eps), out_dtype or a.dtype, _held(held), num_types, types, a, s, w_after, w_before, gate, scale)


class _GatedFfn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, act, held, X, Wg, Wu, Wd):
        X, Wg, Wu, Wd = _rows(X, Wg, Wu, Wd)
        if Wg.dim() != 2 or X.dim() < 1 or X.shape[-1] != Wg.shape[0] or Wu.shape != Wg.shape or Wd.shape != Wg.shape[::-1]:
            raise ValueError(f"gated_ffn: shapes {tuple(X.shape)}, {tuple(Wg.shape)}, {tuple(Wu.shape)}, {tuple(Wd.shape)} do not fit")
        if not X.dtype == Wg.dtype == Wu.dtype == Wd.dtype:
            raise TypeError("gated_ffn: rows and weights are of one type")
        width, hidden = Wg.shape
        with torch.cuda.device(X.device):
            ctx.desc = B.make_ffn_desc(X.numel() // width, width, hidden, _code(X.dtype),
                                       {"silu": B.RGNN_ACT_SILU, "relu": B.RGNN_ACT_RELU}[act])
            out = torch.empty_like(X)
            B.rgnn_ffn_fwd(ctx.desc, X, Wg, Wu, Wd, out, _buf(B.rgnn_ffn_workspace_bytes(ctx.desc)[0]), _stream())
            ctx.held = held and any(ctx.needs_input_grad)
            ctx.save_for_backward(Wg, Wu, Wd, *(_pack(X) if ctx.held else (X,)))
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dOut):
        Wg, Wu, Wd, *kept = ctx.saved_tensors
        dOut, = _rows(dOut)
        need_x, *need_w = ctx.needs_input_grad[2:]
        with torch.cuda.device(dOut.device):
            dX = torch.empty_like(dOut) if need_x else None
            g = [torch.empty_like(W) if any(need_w) else None for W in (Wg, Wu, Wd)]
            ws = _buf(B.rgnn_ffn_workspace_bytes(ctx.desc)[1])
            if ctx.held:
                B.rgnn_ffn_bwd_rows8(ctx.desc, B.rows8(*kept), Wg, Wu, Wd, dOut, dX, *g, ws, _stream())
            else:
                B.rgnn_ffn_bwd(ctx.desc, kept[0], Wg, Wu, Wd, dOut, dX, *g, ws, _stream())
        return (None, None, dX, *(t if n else None for t, n in zip(g, need_w)))


def residual_norm(x, weight, residual=None, eps=1e-6, out_dtype=None):
    """Residual addition and root-mean-square norm over the last dimension, s = x + residual, out = s / sqrt(mean(s^2) + eps) * weight:
    (out, s), or out alone without a residual.  s has the residual's type; out has out_dtype (fp32 or bf16; default: x's); weight is fp32."""
    if out_dtype is not None and out_dtype not in _CODES:
        raise TypeError(f"residual_norm: out_dtype is fp32 or bf16, not {out_dtype}")
    return _ResidualNorm.apply(float(eps), out_dtype or x.dtype, x, residual, weight)


def gated_ffn(X, Wg, Wu, Wd, act="silu", held=False):
    """Gated feed-forward block (act(X Wg) * (X Wu)) Wd over the last dimension; Wg, Wu [d, hidden], Wd [hidden, d], all of X's type.
    held: X is kept for the backward in 8 bits (without a backward, nothing is packed)."""
    if act not in ("silu", "relu"):
        raise ValueError(f"gated_ffn: unknown activation {act!r}")
    return _GatedFfn.apply(act, _held(held), X, Wg, Wu, Wd)


def _apart(t):
    """Whether no two of the tensor's elements share memory: each stride steps over all that the smaller ones reach."""
    reach = 0
    for stride, size in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n != 1):
        if stride <= reach:
            return t.numel() == 0
        reach += stride * (size - 1)
    return True


@torch.no_grad()
def clip_grad_norm_(parameters, max_norm, error_if_nonfinite=False):
    """Scales the gradients of `parameters` in place by min(1, max_norm / (norm + 1e-6)), norm the 2-norm of all of them together, and
    returns that norm (0-dim fp32 tensor on the GPU; nothing waits for it unless error_if_nonfinite).  Gradients are fp32 or bf16, on one
    GPU; contiguous ones that share memory are refused, and strided ones that begin at the same place.  Without any, a zero on the CPU."""
    if isinstance(parameters, torch.Tensor):
        parameters = [parameters]
    given = [p.grad for p in parameters if p.grad is not None]
    if not given:
        return torch.zeros(())
    for g in given:
        if g.layout != torch.strided or g.dtype not in _CODES or not g.is_cuda or g.device != given[0].device:
            raise TypeError("clip_grad_norm_ takes dense fp32 or bf16 gradients on one GPU")
    # (strided ones reach the library as copies, whose own memory it compares)
    strided = [g for g in given if not _dense(g)]
    for g in strided:
        if not _apart(g):
            raise RuntimeError(f"clip_grad_norm_: elements of a gradient share memory (shape {tuple(g.shape)}, strides {g.stride()})")
    if len({g.data_ptr() for g in strided if g.numel()}) < sum(g.numel() > 0 for g in strided):
        raise RuntimeError("clip_grad_norm_: two gradients share memory")
    with torch.cuda.device(given[0].device):
        grads = [g if _dense(g) else g.contiguous() for g in given] if strided else given
        sizes = [g.numel() for g in grads]
        norm = torch.empty((), device=given[0].device)
        dtypes, ws = [_code(g.dtype) for g in grads], _buf(B.rgnn_clip_workspace_bytes(sizes))
        if error_if_nonfinite:
            B.rgnn_clip_grad_norm(grads, None, sizes, dtypes, float(max_norm), norm, ws, _stream())
            if not torch.isfinite(norm):
                raise RuntimeError(f"the norm of the gradients is {norm.item()}, so that they cannot be clipped")
        B.rgnn_clip_grad_norm(grads, grads, sizes, dtypes, float(max_norm), norm, ws, _stream())
        torch.autograd.graph.increment_version([g for g, c in zip(given, grads) if c is g])
        if strided:
            for g, c in zip(given, grads):
                if c is not g:
                    g.copy_(c)
    return norm


def rgat(graph, X, W, w_s, w_t, slope=0.2, heads=1):
    """RGAT layer (listing of the single-headed RGAT layer in the thesis; with heads > 1 each head
    works on its slice of the d columns): out [N, d].  On a large graph a call outside grad mode may take another plan
    than one inside: the two agree up to rounding."""
    return _Rgat.apply(graph, torch.is_grad_enabled(), float(slope), int(heads), X, W, w_s, w_t)


def rgcn(graph, X, W, W0=None, norm="in_degree_per_rel", act="none"):
    """RGCN layer, Eq. (rgcn): out [N, d].  Inside and outside grad mode as with `rgat`."""
    return _Rgcn.apply(graph, torch.is_grad_enabled(), norm, act, X, W, W0)


def hgt(graph, X, Wk, Wq, Wv, Wo, Watt, Wmsg, mu=None):
    """HGT layer (figure "HGT and RGAT layer"): out [N, d]; heads = Watt.shape[1]."""
    return _Hgt.apply(graph, X, Wk, Wq, Wv, Wo, Watt, Wmsg, mu)


def _param(*shape, fan_in):
    return torch.nn.Parameter(torch.randn(*shape, device="cuda") / math.sqrt(fan_in))


class RgatConv(torch.nn.Module):
    def __init__(self, num_rels, d, slope=0.2, heads=1, d_in=None):
        """d: output width; d_in: input width when it differs (32 and 64 may be mixed)."""
        super().__init__()
        self.slope, self.heads = slope, heads
        k = d_in or d
        self.W, self.w_s, self.w_t = _param(num_rels, k, d, fan_in=k), _param(num_rels, d, fan_in=d), _param(num_rels, d, fan_in=d)

    def forward(self, graph, X):
        return rgat(graph, X, self.W, self.w_s, self.w_t, self.slope, self.heads)


class RgcnConv(torch.nn.Module):
    def __init__(self, num_rels, d, self_loop=True, norm="in_degree_per_rel", act="none", d_in=None):
        """d: output width; d_in: input width when it differs (32 and 64 may be mixed)."""
        super().__init__()
        self.norm, self.act = norm, act
        k = d_in or d
        self.W = _param(num_rels, k, d, fan_in=k)
        self.W0 = _param(k, d, fan_in=k) if self_loop else None

    def forward(self, graph, X):
        return rgcn(graph, X, self.W, self.W0, self.norm, self.act)


class HgtConv(torch.nn.Module):
    def __init__(self, num_ntypes, num_rels, d, heads, with_mu=True):
        super().__init__()
        dh = d // heads
        self.Wk, self.Wq, self.Wv, self.Wo = (_param(num_ntypes, d, d, fan_in=d) for _ in range(4))
        self.Watt, self.Wmsg = _param(num_rels, heads, dh, dh, fan_in=dh), _param(num_rels, heads, dh, dh, fan_in=dh)
        self.mu = torch.nn.Parameter(torch.ones(num_rels, heads, device="cuda")) if with_mu else None

    def forward(self, graph, X):
        return hgt(graph, X, self.Wk, self.Wq, self.Wv, self.Wo, self.Watt, self.Wmsg, self.mu)


class ResidualNorm(torch.nn.Module):
    def __init__(self, width, eps=1e-6, out_dtype=None):
        super().__init__()
        self.eps, self.out_dtype = eps, out_dtype
        self.weight = torch.nn.Parameter(torch.ones(width, device="cuda"))

    def forward(self, x, residual=None):
        return residual_norm(x, self.weight, residual, self.eps, self.out_dtype)


class BlockNorm(torch.nn.Module):
    """`block_norm` with its parameters: out, s = norm(a, s, types).  gate, scale: their first values, the same for all types and columns; after, before: whether
    there is a norm after the block and one before the next."""

    def __init__(self, width, num_types=1, gate=1.0, scale=1.0, after=True, before=True, eps=1e-6, out_dtype=None, held=False):
        super().__init__()
        self.eps, self.out_dtype, self.held = eps, out_dtype, held
        p = lambda value, *shape: torch.nn.Parameter(torch.full(shape, float(value), device="cuda"))
        self.weight_after = p(1, width) if after else None
        self.weight_before = p(1, width) if before else None
        self.gate, self.scale = p(gate, num_types, width), p(scale, num_types)

    def forward(self, a, s, types=None):
        return block_norm(a, s, self.weight_after, self.weight_before, self.gate, self.scale, types, self.eps, self.out_dtype, self.held)


class GatedFfn(torch.nn.Module):
    def __init__(self, width, hidden, act="silu", dtype=torch.float32, held=False):
        super().__init__()
        self.act, self.held = act, held
        p = lambda *shape, fan_in: torch.nn.Parameter(_param(*shape, fan_in=fan_in).detach().to(dtype))
        self.Wg, self.Wu = p(width, hidden, fan_in=width), p(width, hidden, fan_in=width)
        self.Wd = p(hidden, width, fan_in=hidden)

    def forward(self, X):
        return gated_ffn(X, self.Wg, self.Wu, self.Wd, self.act, self.held)


__all__ = ["Graph", "rgat", "rgcn", "hgt", "RgatConv", "RgcnConv", "HgtConv", "release", "residual_norm", "gated_ffn",
           "clip_grad_norm_", "ResidualNorm", "GatedFfn", "block_norm", "BlockNorm", "pack_rows", "unpack_rows"]
