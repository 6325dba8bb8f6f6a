"""Workloads of the operators that stand between the relational layers of a model and in its training step.

Three operators on the rows of all nodes: the residual addition with its root-mean-square norm (forward and backward), the gated
feed-forward block (forward and backward), and the global gradient norm with clipping over a model's tensors.  Node counts, widths
and storage types are those of the library's own workloads (`synth.config`, `bench.py`, `perf/cases.py`): from one node that is
scored online to full-graph training on two million nodes, widths 32, 64 and 128, fp32 or bf16 rows.

`run` computes an operator with elementary torch operations in fp32, or, with `own`, through the library.
"""
import math

import torch

own = False

EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _norm(name, mode, rows, width, x="f32", total="f32", out="f32", residual=True):
    c = dict(op="norm", mode=mode, rows=rows, width=width, x=x, total=total, out=out, residual=residual)
    return dict(c, name=name) if name else c


def _ffn(name, mode, rows, width, hidden, dtype="f32", act="silu"):
    c = dict(op="ffn", mode=mode, rows=rows, width=width, hidden=hidden, dtype=dtype, act=act)
    return dict(c, name=name) if name else c


def _clip(name, kind, layers, rels, width, hidden, embedding, share, dtype="f32", spread=3.0):
    c = dict(op="clip", kind=kind, layers=layers, rels=rels, width=width, hidden=hidden, embedding=embedding, share=share, dtype=dtype,
             spread=spread)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest call: the rows of one sampled neighbourhood, scored online
        _norm("norm_infer_tiny", "fwd", 17, 64),
        # a residual layer of the flagship graph, a million nodes of width 64, whose next layer takes bf16 rows
        _norm("norm_train_fwd_large", "fwd", 1000000, 64, out="bf16"),
        # its backward at the size of the HGT workload: rows, stream and gradients in bf16
        _norm("norm_train_bwd_large_bf16", "bwd", 2000000, 128, x="bf16", total="bf16", out="bf16"),
        # raw input features of an odd width are normed, nothing added: backward on a mid-size graph
        _norm("norm_features_bwd", "bwd", 30011, 349, residual=False),
        # one node scored online, the widest block
        _ffn("ffn_infer_one", "fwd", 1, 128, 512),
        # a mini-batch's seed nodes through a narrow block whose hidden width is 8/3 of the row
        _ffn("ffn_infer_small", "fwd", 1000, 32, 86),
        # full-graph inference of an HGT model with bf16 rows
        _ffn("ffn_infer_large_bf16", "fwd", 2000000, 128, 512, "bf16"),
        # full-graph training of the flagship's width in fp32
        _ffn("ffn_train_large", "bwd", 1000000, 64, 256),
        # training on a mid-size graph in bf16, an odd hidden width
        _ffn("ffn_train_mid_bf16", "bwd", 200017, 128, 341, "bf16"),
        # training step of a small two-layer RGAT model: six tensors of a few hundred KB
        _clip("clip_rgat_small", "rgat", 2, 50, 64, 0, 0, 0.5),
        # five HGT layers with their feed-forward blocks: fifty-five tensors, gradients in bf16
        _clip("clip_hgt_deep_bf16", "hgt", 5, 30, 128, 512, 0, 0.1, "bf16"),
        # a trained embedding of every node beside the layers' weights: the bytes of the embedding
        _clip("clip_embedding_large", "rgat", 2, 200, 64, 256, 1000000, 0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "ffn", "ffn", "clip"])
    types = rng.choice(["f32", "bf16"])
    if op == "norm":
        width = rng.choice([32, 64, 128, _log(rng, 1, 1024)])
        rows = _log(rng, 1, min(2e6, 256e6 / width))
        x, total, out = rng.choice([("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "f32", "bf16"), ("bf16", "f32", "bf16")])
        return _norm(None, rng.choice(["fwd", "bwd"]), rows, width, x, total, out, rng.random() < 0.75)
    if op == "ffn":
        width = rng.choice([32, 64, 128])
        mode = rng.choice(["fwd", "bwd"])
        hidden = _log(rng, 16, 512)
        rows = _log(rng, 1, min(1e6, 1.6e10 / (width * hidden) if mode == "bwd" else 1e6))
        return _ffn(None, mode, rows, width, hidden, types, rng.choice(["silu", "silu", "relu"]))
    return _clip(None, rng.choice(["rgat", "hgt"]), rng.randint(1, 5), _log(rng, 4, 200), rng.choice([32, 64, 128]),
                 rng.choice([0, _log(rng, 16, 512)]), rng.choice([0, _log(rng, 1000, 500000)]), rng.choice([0.1, 0.5, 2.0]), types,
                 rng.choice([0.0, 3.0]))


def _shapes(case):
    """The parameters of a model: per layer the relational weights, with a hidden width a norm and a feed-forward block too."""
    R, d, f = case["rels"], case["width"], case["hidden"]
    layer = [(R, d, d), (R, d), (R, d)] if case["kind"] == "rgat" else [(8, d, d)] * 4 + [(R, 4, d // 4, d // 4)] * 2 + [(R, 4)]
    block = [(d,), (d, f), (d, f), (f, d)] if f else []
    return [(case["embedding"], d)] * (case["embedding"] > 0) + (layer + block) * case["layers"]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype="f32"):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(TYPES[dtype])

    if case["op"] == "norm":
        n, d = case["rows"], case["width"]
        # the layers give nodes without incoming edges rows of zeros
        x = normal(n, d) * (torch.rand(n, 1, generator=g, device="cuda") > 0.05)
        s = {"case": case, "w": 1.0 + normal(d, scale=0.2)}
        if case["mode"] == "fwd":
            s["x"] = x.to(TYPES[case["x"]])
            s["r"] = normal(n, d, scale=2.0, dtype=case["total"]) if case["residual"] else None
        else:
            s["s"] = (x + normal(n, d, scale=2.0)).to(TYPES[case["total"]]) if case["residual"] else x.to(TYPES[case["x"]])
            s["dy"] = normal(n, d, scale=0.1, dtype=case["out"])
            s["ds"] = normal(n, d, scale=0.1, dtype=case["total"]) if case["residual"] else None
        return s
    if case["op"] == "ffn":
        n, d, f, t = case["rows"], case["width"], case["hidden"], case["dtype"]
        s = {"case": case, "x": normal(n, d, dtype=t), "wg": normal(d, f, scale=d ** -0.5, dtype=t),
             "wu": normal(d, f, scale=d ** -0.5, dtype=t), "wd": normal(f, d, scale=f ** -0.5, dtype=t)}
        if case["mode"] == "bwd":
            s["dy"] = normal(n, d, scale=0.1, dtype=t)
        return s
    # gradients of different tensors differ by orders of magnitude
    grads, square = [], 0.0
    for i, shape in enumerate(_shapes(case)):
        scale = 10.0 ** (-case["spread"] * (i % 5) / 4)
        grads.append(normal(*shape, scale=scale, dtype=case["dtype"]))
        square += scale * scale * grads[-1].numel()
    return {"case": case, "grads": grads, "max_norm": case["share"] * math.sqrt(square)}


# ---- the plain forms

def _plain_norm(s):
    w = s["w"]
    if s["case"]["mode"] == "fwd":
        x = s["x"].float()
        total = x if s["r"] is None else x + s["r"].float()
        out = total * torch.rsqrt((total * total).mean(1, keepdim=True) + EPS) * w
        out = out.to(TYPES[s["case"]["out"]])
        return {"out": out} if s["r"] is None else {"sum": total.to(s["r"].dtype), "out": out}
    t, dy = s["s"].float(), s["dy"].float()
    q = torch.rsqrt((t * t).mean(1, keepdim=True) + EPS)
    g = dy * w
    d = q * (g - t * (q * q * (g * t).mean(1, keepdim=True)))
    if s["ds"] is not None:
        d = d + s["ds"].float()
    return {"dx": d.to(s["s"].dtype), "dw": (dy * t * q).sum(0)}


def _plain_ffn(s):
    x, wg, wu, wd = s["x"].float(), s["wg"].float(), s["wu"].float(), s["wd"].float()
    t, silu = s["x"].dtype, s["case"]["act"] == "silu"
    a, u = x @ wg, x @ wu
    if silu:
        sig = 1.0 / (1.0 + torch.exp(-a))
        act = a * sig
    else:
        act = torch.where(a > 0, a, torch.zeros_like(a))
    if s["case"]["mode"] == "fwd":
        return {"out": ((act * u) @ wd).to(t)}
    dy = s["dy"].float()
    dh = dy @ wd.t()
    da = dh * u * (sig * (1.0 + a * (1.0 - sig)) if silu else (a > 0).float())
    du = dh * act
    return {"dx": (da @ wg.t() + du @ wu.t()).to(t), "dwg": (x.t() @ da).to(t), "dwu": (x.t() @ du).to(t),
            "dwd": ((act * u).t() @ dy).to(t)}


def _plain_clip(s):
    square = torch.stack([(g.float() * g.float()).sum(dtype=torch.float64) for g in s["grads"]]).sum()
    norm = torch.sqrt(square)
    c = torch.clamp(s["max_norm"] / (norm + EPS), max=1.0).float()
    return {"norm": norm.float(), "clipped": [(g.float() * c).to(g.dtype) for g in s["grads"]]}


# ---- the library's

def _own(s):
    from paper_2412_04747_amd import harness as H
    case = s["case"]
    if case["op"] == "norm":
        L = s.get("layer")
        if L is None:
            total = case["total"] if case["residual"] else case["x"]
            L = s["layer"] = H.NormLayer(case["rows"], case["width"], case["x"], total, case["out"], EPS, residual=case["residual"])
        L.weight = s["w"]
        if case["mode"] == "fwd":
            L.x, L.residual = s["x"], s["r"]
            L.fwd()
            return {"sum": L.sum, "out": L.out} if case["residual"] else {"out": L.out}
        L.sum, L.dOut, L.dSum = s["s"], s["dy"], s["ds"]
        L.bwd()
        return {"dx": L.dX if L.dResidual is None else L.dResidual, "dw": L.dWeight}
    if case["op"] == "ffn":
        L = s.get("layer")
        if L is None:
            L = s["layer"] = H.FfnLayer(case["rows"], case["width"], case["hidden"], case["dtype"], case["act"])
        L.X, L.Wg, L.Wu, L.Wd = s["x"], s["wg"], s["wu"], s["wd"]
        if case["mode"] == "fwd":
            L.fwd()
            return {"out": L.out}
        L.dOut = s["dy"]
        L.bwd()
        return {"dx": L.dX, "dwg": L.dWg, "dwu": L.dWu, "dwd": L.dWd}
    L = s.get("layer")
    if L is None:
        L = s["layer"] = H.GradClip(s["grads"], in_place=False)
    L.clip(s["grads"], s["max_norm"])
    return {"norm": L.norm, "clipped": L.clipped}


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "ffn": _plain_ffn, "clip": _plain_clip}[state["case"]["op"]](state)


def work(case):
    size = lambda t: 4 if t == "f32" else 2
    if case["op"] == "norm":
        n = case["rows"] * case["width"]
        total = size(case["total"]) if case["residual"] else 0
        if case["mode"] == "fwd":
            return {"bytes": n * (size(case["x"]) + 2 * total + size(case["out"])) + 4 * case["width"], "flops": 6 * n}
        read = total if case["residual"] else size(case["x"])
        return {"bytes": n * (2 * read + total + size(case["out"])) + 8 * case["width"], "flops": 14 * n}
    if case["op"] == "ffn":
        n, d, f, b = case["rows"], case["width"], case["hidden"], size(case["dtype"])
        if case["mode"] == "fwd":
            return {"bytes": b * (2 * n * d + 3 * d * f), "flops": 6 * n * d * f}
        return {"bytes": b * (3 * n * d + 6 * d * f), "flops": 16 * n * d * f}
    n = sum(math.prod(s) for s in _shapes(case))
    return {"bytes": 2 * n * size(case["dtype"]) + 4, "flops": 3 * n}


# ---- from the definitions, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        w = s["w"].double()
        if case["mode"] == "fwd":
            total = s["x"].double() if s["r"] is None else s["x"].double() + s["r"].double()
            out = total / (total.pow(2).mean(1) + EPS).sqrt()[:, None] * w
            return {"out": out} if s["r"] is None else {"sum": total, "out": out}
        # y_j = t_j w_j / m, m = sqrt(mean t^2 + eps): dy_j/dt_i = w_j (delta_ij / m - t_i t_j / (d m^3))
        t, dy = s["s"].double(), s["dy"].double()
        m = (t.pow(2).mean(1) + EPS).sqrt()[:, None]
        along = ((dy * w * t).sum(1) / t.shape[1])[:, None]
        d = dy * w / m - t * along / m.pow(3)
        return {"dx": d if s["ds"] is None else d + s["ds"].double(), "dw": torch.einsum("ij,ij->j", dy, t / m)}
    if case["op"] == "ffn":
        wg, wu, wd = s["wg"].double(), s["wu"].double(), s["wd"].double()
        rows, sums = [], [torch.zeros_like(v) for v in (wg, wu, wd)]
        for at in range(0, case["rows"], 1 << 17):
            x = s["x"][at:at + (1 << 17)].double()
            a, u = torch.mm(x, wg), torch.mm(x, wu)
            p = torch.sigmoid(a) if case["act"] == "silu" else (a > 0).double()
            if case["mode"] == "fwd":
                rows.append(torch.mm(a * p * u, wd))
                continue
            dy = s["dy"][at:at + (1 << 17)].double()
            dh = torch.mm(dy, wd.t().contiguous())
            slope = p + a * p * (1 - p) if case["act"] == "silu" else p
            da, du = dh * u * slope, dh * a * p
            rows.append(torch.mm(da, wg.t().contiguous()) + torch.mm(du, wu.t().contiguous()))
            for total, left, right in ((sums[0], x, da), (sums[1], x, du), (sums[2], a * p * u, dy)):
                total += torch.mm(left.t().contiguous(), right)
        out = torch.cat(rows)
        return {"out": out} if case["mode"] == "fwd" else {"dx": out, "dwg": sums[0], "dwu": sums[1], "dwd": sums[2]}
    norm = math.sqrt(sum(float(g.double().pow(2).sum()) for g in s["grads"]))
    c = min(1.0, s["max_norm"] / (norm + EPS))
    return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"), "clipped": [g.double() * c for g in s["grads"]]}
