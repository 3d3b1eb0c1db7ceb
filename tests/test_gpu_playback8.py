"""Playback of linear layers in 8 bits: the operators together, as a user runs them.

Tolerances.  An operand's rounding moves an element by at most half a step,
amax / 254 of its row or column, so a product of K terms moves by at most
  sum_k (|a| eb + |b| ea + ea eb),  ea = amax_a / 254, eb = amax_b / 254,
which is computed here in binary64; the output's own rounding adds 2^-8 of the
result for bfloat16, and the recorded output another (1.01 covers float32).
"""
import json

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h(peat_gpu):
    handle = peat_gpu.Handle(0)
    yield handle
    handle.close()


def bound(a, b):
    """Largest error of a [M, K] times b [N, K] rounded by row."""
    a, b = a.double().abs(), b.double().abs()
    ea, eb = a.amax(1) / 254, b.amax(1) / 254
    return a.sum(1)[:, None] * eb[None, :] + ea[:, None] * (b.sum(1) + a.shape[1] * eb)[None, :]


@pytest.mark.parametrize("tokens,width,hidden", [(1, 64, 40), (37, 96, 130), (520, 256, 1024)])
def test_playback8(peat_gpu, h, tokens, width, hidden):
    from paper_2609_13544_gb300 import playback8 as P
    import torch
    records = P.synthetic_records(tokens, width, hidden, 2, 5)
    kept = [{k: v.clone() for k, v in vars(r).items() if k != "name"} for r in records]
    got = P.playback8(h, records, 2.0 ** -7, 0.0, 0.25)
    assert [r["name"] for r in got["layers"]] == ["block0.up", "block0.down", "block1.up", "block1.down"]
    grads = []
    for rec, before, scores in zip(records, kept, got["layers"]):
        for k, v in before.items():
            assert torch.equal(getattr(rec, k), v)
        for key, golden, a, b in (("fwd", rec.y, rec.x, rec.weight), ("in_grad", rec.grad_x, rec.grad, rec.weight.t()),
                                  ("wg_grad", rec.grad_weight, rec.grad.t(), rec.x.t())):
            s = scores[key]
            slack = 2.0 ** -7 if golden.dtype == torch.bfloat16 else 1e-6
            size = a.double().abs() @ b.double().abs().t() + (0.1 if key == "fwd" else 0.0)
            assert s["n"] == golden.numel()
            assert 0.0 < s["mean_abs"] <= s["top10_mean"] <= s["max_abs"]
            assert s["max_abs"] <= 1.01 * float((bound(a, b) + slack * size).max())
        layer = peat_gpu.Linear8(h, rec.weight)
        grads.append(layer.weight_grad(rec.grad, rec.x))
    # the step's end, from its definition in 64 bits
    for key, ts in (("golden", [r.grad_weight for r in records]), ("replayed", grads)):
        norm = float(np.sqrt(sum(float((t.double() ** 2).sum()) for t in ts)))
        assert abs(got[key]["norm"] - norm) <= 40 * 2.0 ** -24 * norm and got[key]["n_bad"] == 0
        assert got[key]["coef"] == min(1.0, float(np.float32(0.25) / (np.float32(got[key]["norm"]) + np.float32(1e-6))))
    for rec, r, s in zip(records, grads, got["clipped"]):
        a = rec.grad_weight * got["golden"]["coef"]
        b = r * got["replayed"]["coef"]
        assert s["max_abs"] == float((a.double() - b.double()).abs().max())


def test_command(peat_gpu, capsys):
    from paper_2609_13544_gb300 import playback8 as P
    result = P.main(["--tokens", "40", "--width", "64", "--hidden", "128", "--blocks", "1"])
    assert json.loads(capsys.readouterr().out) == result
    assert len(result["layers"]) == 2 and result["golden"]["norm"] > 0


def test_other_stream(peat_gpu, h):
    """Everything on a given stream gives what the current one gives."""
    import torch
    from paper_2609_13544_gb300 import playback8 as P
    want = P.playback8(h, P.synthetic_records(65, 96, 64, 1, 9), 1e-2)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        records = P.synthetic_records(65, 96, 64, 1, 9)
    assert P.playback8(h, records, 1e-2, stream=s) == want
