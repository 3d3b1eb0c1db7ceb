"""Playback of recorded linear layers in 8-bit integers.

Alg. 1 of the paper replays a recorded layer's three products (Fwd, InGrad,
WgGrad) on a changed kernel and scores each output against the recorded one
(Err).  Here the changed kernel is the 8-bit layer, ``Linear8``:
``replay_layer`` scores the three products of one record, ``playback8`` those
of a list of them, and then ends the step as training does: the norm over all
weight gradients, by which they are clipped, for the recorded list and for the
replayed one, so that the scores also tell what the 8-bit gradients change in
the step that the optimizer takes.

    python -m paper_2609_13544_gb300.playback8 --tokens 2048 --blocks 4

runs it on synthetic records (two linear layers a block, 1024 wide and 4096,
unless told otherwise) and prints the scores as one line of JSON.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Any, List, Optional, Sequence

SCORES = ("n", "max_abs", "mean_abs", "var_abs", "mismatch")


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


def _score(h, golden, candidate, rtol: float, atol: float, stream) -> dict:
    from . import peat_compare, peat_topk_mean
    golden, candidate = golden.contiguous(), candidate.contiguous()
    stats, _ = peat_compare(h, golden, candidate, rtol, atol, stream)
    return {**{k: stats[k] for k in SCORES}, "top10_mean": peat_topk_mean(h, golden, candidate, stream=stream)["mean"]}


def replay_layer(h, rec: LayerRecord, rtol: float, atol: float = 0.0, stream=None) -> tuple:
    """(scores of "fwd", "in_grad" and "wg_grad", the replayed weight gradient) of one record."""
    from . import Linear8
    from .ops import _on
    layer = Linear8(h, rec.weight, stream)
    y = layer.forward(rec.x, rec.bias, stream)
    grad_x, grad_weight = layer.backward(rec.grad, rec.x, stream)
    with _on(stream):
        grad_weight = grad_weight.to(rec.grad_weight.dtype)
        scores = {key: _score(h, golden, got, rtol, atol, stream)
                  for key, golden, got in (("fwd", rec.y, y), ("in_grad", rec.grad_x, grad_x),
                                           ("wg_grad", rec.grad_weight, grad_weight))}
    return scores, grad_weight


def playback8(h, records: Sequence[LayerRecord], rtol: float, atol: float = 0.0, max_norm: float = 1.0,
              unscale: float = 1.0, stream=None) -> dict:
    """Every record replayed and scored, and the step's end.

    Returns {"layers": a dict of scores a record, "golden" and "replayed": the norm, clipping factor and bad
    elements of either list of weight gradients, "clipped": the scores of the clipped gradients}.  The records
    stay as they are."""
    import torch
    from . import GradList, peat_grad_clip
    from .ops import _on
    layers: List[dict] = []
    replayed = []
    for rec in records:
        scores, grad = replay_layer(h, rec, rtol, atol, stream)
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


def synthetic_records(tokens: int, width: int, hidden: int, blocks: int, seed: int, device="cuda") -> List[LayerRecord]:
    """Records of two linear layers a block (width to hidden and back) in bfloat16, weight gradients in float32:
    normal activations, weights of variance 1 / in, output gradients of a size as training leaves them."""
    import torch
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device=device)
    out = []
    for b in range(blocks):
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
                                description="Linear layers replayed in 8-bit integers and scored; gradients clipped.")
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--width", type=int, default=1024)
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--blocks", type=int, default=4)
    p.add_argument("--rtol", type=float, default=2.0 ** -7)
    p.add_argument("--atol", type=float, default=0.0)
    p.add_argument("--max-norm", type=float, default=1.0)
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args(argv)
    from . import Handle
    records = synthetic_records(a.tokens, a.width, a.hidden, a.blocks, a.seed)
    with Handle(0) as h:
        result = playback8(h, records, a.rtol, a.atol, a.max_norm)
    print(json.dumps(result))
    return result


if __name__ == "__main__":
    main()
