"""Playback of recorded layers at a lower precision: 8-bit integers, or 4-bit floating point.

Alg. 1 of the paper replays a recorded layer's three products (Fwd, InGrad,
WgGrad) on a changed kernel and scores each output against the recorded one
(Err).  Here the changed kernel is the 8-bit layer, ``Linear8``, or the 4-bit
one, ``Linear4``: ``replay_layer`` scores the three products of one record;
``replay_norm`` a root-mean-square norm's output, rounded as the layer behind it
takes it, its residual stream and its gradients.  ``playback8`` scores those
of a list of records, and then ends the step as training does: the norm over all
weight gradients, by which they are clipped, for the recorded list and for the
replayed one, so that the scores also tell what the low-precision gradients change
in the step that the optimizer takes.

    python -m paper_2609_13544_gb300.playback8 --tokens 2048 --blocks 4
    python -m paper_2609_13544_gb300.playback8 --precision nvfp4 --norms

runs it on synthetic records (two linear layers a block, 1024 wide and 4096,
unless told otherwise; with --norms a norm in front of them) and prints the
scores as one line of JSON.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Any, List, Optional, Sequence

SCORES = ("n", "max_abs", "mean_abs", "var_abs", "mismatch")
PRECISIONS = ("i8", "mxfp4", "nvfp4")


@dataclass
class LayerRecord:
    """What a playback recorded of y = x weight^T + bias: the inputs of its three products and their outputs.
    Tensors have any leading dimensions; grad_weight may be of another type than the rest."""
    name: str
    x: Any             # [..., in]
    weight: Any        # [out, in]
    grad: Any          # dL/dy [..., out]
    y: Any             # [..., out]
    grad_x: Any        # [..., in]
    grad_weight: Any   # [out, in]
    bias: Optional[Any] = None  # float32 [out]


@dataclass
class NormRecord:
    """What a playback recorded of sum = x + residual, y = sum / sqrt(mean of squares + eps) weight: inputs, outputs, the
    gradients that came back to both and the ones that left.  Tensors have any leading dimensions."""
    name: str
    x: Any             # [..., cols]
    weight: Any        # [cols], of x's type or float32
    grad: Any          # dL/dy [..., cols]
    y: Any             # [..., cols]
    grad_x: Any        # of x and residual [..., cols]
    grad_weight: Any   # [cols]
    residual: Optional[Any] = None  # [..., cols]
    sum: Optional[Any] = None       # [..., cols]; None: not scored
    grad_sum: Optional[Any] = None  # dL/dsum beside the norm [..., cols]
    eps: float = 1e-6


def _score(h, golden, candidate, rtol: float, atol: float, stream) -> dict:
    from . import peat_compare, peat_topk_mean
    golden, candidate = golden.contiguous(), candidate.contiguous()
    stats, _ = peat_compare(h, golden, candidate, rtol, atol, stream)
    return {**{k: stats[k] for k in SCORES}, "top10_mean": peat_topk_mean(h, golden, candidate, stream=stream)["mean"]}


def _known(precision: str) -> None:
    if precision not in PRECISIONS:
        raise ValueError(f"unknown precision {precision!r}: one of {', '.join(PRECISIONS)}")


def replay_layer(h, rec: LayerRecord, rtol: float, atol: float = 0.0, stream=None, precision: str = "i8") -> tuple:
    """(scores of "fwd", "in_grad" and "wg_grad", the replayed weight gradient) of one record."""
    from . import Linear4, Linear8
    from .ops import _on
    _known(precision)
    layer = Linear8(h, rec.weight, stream) if precision == "i8" else Linear4(h, rec.weight, precision, stream)
    y = layer.forward(rec.x, rec.bias, stream)
    grad_x, grad_weight = layer.backward(rec.grad, rec.x, stream)
    with _on(stream):
        grad_weight = grad_weight.to(rec.grad_weight.dtype)
        scores = {key: _score(h, golden, got, rtol, atol, stream)
                  for key, golden, got in (("fwd", rec.y, y), ("in_grad", rec.grad_x, grad_x),
                                           ("wg_grad", rec.grad_weight, grad_weight))}
    return scores, grad_weight


def replay_norm(h, rec: NormRecord, rtol: float, atol: float = 0.0, stream=None, precision: str = "i8") -> tuple:
    """(scores of "fwd", "sum", "in_grad" and "wg_grad", the replayed weight gradient) of one record.  The output is
    rounded as the layer that takes it would round it: to 8 bits by row, or to 4 bits by blocks."""
    import torch
    from . import peat_quantize_f4_raw, peat_rmsnorm_backward, peat_rmsnorm_raw
    from .ops import _as_rows, _on
    _known(precision)
    cols = rec.weight.shape[0]
    with _on(stream):
        rows = lambda t: None if t is None else _as_rows(t, cols)
        x, residual = rows(rec.x), rows(rec.residual)
        new = lambda: torch.empty(x.shape, dtype=x.dtype, device=x.device)
        y, total = new(), new()
        rstd = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
        if precision == "i8":
            peat_rmsnorm_raw(h, x, rec.weight, rec.eps, residual, sum=total, values=y, rstd=rstd)
        else:
            peat_rmsnorm_raw(h, x, rec.weight, rec.eps, residual, sum=total, y=y, rstd=rstd)
            rounded = new()
            peat_quantize_f4_raw(h, y, precision, 0, values=rounded)
            y = rounded
        grad_x, grad_weight = peat_rmsnorm_backward(h, rows(rec.grad), total, rec.weight, rstd, rows(rec.grad_sum))
        grad_weight = grad_weight.to(rec.grad_weight.dtype)
        pairs = [("fwd", rec.y, y), ("sum", rec.sum, total), ("in_grad", rec.grad_x, grad_x),
                 ("wg_grad", rec.grad_weight, grad_weight)]
        scores = {key: _score(h, golden.reshape(got.shape), got, rtol, atol, stream) for key, golden, got in pairs
                  if golden is not None}
    return scores, grad_weight


def playback8(h, records: Sequence, rtol: float, atol: float = 0.0, max_norm: float = 1.0, unscale: float = 1.0,
              stream=None, precision: str = "i8") -> dict:
    """Every record (LayerRecord or NormRecord) replayed at a precision and scored, and the step's end.

    Returns {"layers": a dict of scores a record, "golden" and "replayed": the norm, clipping factor and bad
    elements of either list of weight gradients, "clipped": the scores of the clipped gradients}.  The records
    stay as they are."""
    import torch
    from . import GradList, peat_grad_clip
    from .ops import _on
    layers: List[dict] = []
    replayed = []
    for rec in records:
        replay = replay_norm if isinstance(rec, NormRecord) else replay_layer
        scores, grad = replay(h, rec, rtol, atol, stream, precision)
        layers.append({"name": rec.name, **scores})
        replayed.append(grad)
    with _on(stream):
        golden = [rec.grad_weight.contiguous() for rec in records]
        clipped = [torch.empty_like(g) for g in golden]
        ends = {"golden": peat_grad_clip(h, GradList(golden, clipped), max_norm, unscale=unscale, stream=stream),
                "replayed": peat_grad_clip(h, GradList(replayed), max_norm, unscale=unscale, stream=stream)}
        scores = [{"name": rec.name, **_score(h, g, r, rtol, atol, stream)}
                  for rec, g, r in zip(records, clipped, replayed)]
    return {"layers": layers, **{k: {f: v[f] for f in ("norm", "coef", "n_bad")} for k, v in ends.items()},
            "clipped": scores}


def _norm_record(name: str, normal, tokens: int, width: int) -> NormRecord:
    """A norm's record, computed in binary64."""
    x, residual = (3.0 * normal(tokens, width)).bfloat16(), normal(tokens, width).bfloat16()
    weight = 1.0 + 0.2 * normal(width)
    grad, grad_sum = ((normal(tokens, width) / tokens).bfloat16() for _ in range(2))
    total = (x.float() + residual.float()).bfloat16()
    s, d, w = total.double(), grad.double(), weight.double()
    rstd = 1.0 / (s.square().mean(1, keepdim=True) + 1e-6).sqrt()
    n, g = s * rstd, d * w
    grad_x = rstd * (g - n * (g * n).mean(1, keepdim=True)) + grad_sum.double()
    return NormRecord(name, x, weight, grad, (n * w).bfloat16(), grad_x.bfloat16(), (d * n).sum(0).float(), residual, total,
                      grad_sum)


def synthetic_records(tokens: int, width: int, hidden: int, blocks: int, seed: int, device="cuda",
                      norms: bool = False) -> List:
    """Records of two linear layers a block (width to hidden and back) in bfloat16, weight gradients in float32:
    normal activations, weights of variance 1 / in, output gradients of a size as training leaves them; with norms, a
    root-mean-square norm in front of each block."""
    import torch
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device=device)
    out = []
    for b in range(blocks):
        if norms:
            out.append(_norm_record(f"block{b}.norm", normal, tokens, width))
        for part, n_in, n_out in (("up", width, hidden), ("down", hidden, width)):
            x = normal(tokens, n_in).bfloat16()
            w = (normal(n_out, n_in) / n_in ** 0.5).bfloat16()
            grad = (normal(tokens, n_out) / tokens).bfloat16()
            bias = normal(n_out) * 0.02
            out.append(LayerRecord(f"block{b}.{part}", x, w, grad, (x.float() @ w.float().t() + bias).bfloat16(),
                                   grad @ w, grad.float().t() @ x.float(), bias))
    return out


def main(argv=None) -> dict:
    import argparse
    import json
    p = argparse.ArgumentParser(prog="python -m paper_2609_13544_gb300.playback8",
                                description="Layers replayed at a lower precision and scored; gradients clipped.")
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--width", type=int, default=1024)
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--blocks", type=int, default=4)
    p.add_argument("--rtol", type=float, default=2.0 ** -7)
    p.add_argument("--atol", type=float, default=0.0)
    p.add_argument("--max-norm", type=float, default=1.0)
    p.add_argument("--seed", type=int, default=0)
    p.add_argument("--precision", choices=PRECISIONS, default="i8")
    p.add_argument("--norms", action="store_true", help="a root-mean-square norm in front of each block")
    a = p.parse_args(argv)
    from . import Handle
    records = synthetic_records(a.tokens, a.width, a.hidden, a.blocks, a.seed, norms=a.norms)
    with Handle(0) as h:
        result = playback8(h, records, a.rtol, a.atol, a.max_norm, precision=a.precision)
    print(json.dumps(result))
    return result


if __name__ == "__main__":
    main()
