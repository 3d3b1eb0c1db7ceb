"""Playback of layers in 4 bits, and of norms: the operators together, as a user runs them.

Tolerances.  The 4-bit values 1, 1.5, 2, 3, 4, 6 are at most half a step of a third (from 1 to 1.5, from 2 to 3) or a
quarter off a number between them: less than a third of it; and mxfp4's numbers above 6, below 8, come down to 6.  Below 1
the step is 0.5, off by 0.25 at most, with the block's largest number at 4 or more (mxfp4) or, its 8-bit scale off by a
sixteenth, at 5.6: less than an eighth of the row's largest.  So ea = max(|a| / 3, amax / 8) bounds an element's move, and a
product of K terms moves by at most sum_k (|a| eb + |b| ea + ea eb); the output's own rounding adds 2^-8 of the sum of
magnitudes for bfloat16, and the recorded output another (1.01 covers float32).
"""
import json

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h(peat_gpu):
    handle = peat_gpu.Handle(0)
    yield handle
    handle.close()


def moves(a):
    """Largest moves of a's elements, rounded by row (amax over the row bounds a block's)."""
    import torch
    a = a.double().abs()
    return torch.maximum(a / 3, (a.amax(1, keepdim=True) / 8).expand_as(a))


def bound(a, b):
    a, b = a.double().abs(), b.double().abs()
    ea, eb = moves(a), moves(b)
    return a @ eb.t() + ea @ b.t() + ea @ eb.t()


@pytest.mark.parametrize("precision", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("tokens,width,hidden", [(1, 64, 40), (37, 96, 130), (520, 256, 1024)])
def test_playback4(peat_gpu, h, precision, tokens, width, hidden):
    from paper_2609_13544_gb300 import playback8 as P
    import torch
    records = P.synthetic_records(tokens, width, hidden, 2, 5, norms=True)
    kept = [{k: v.clone() for k, v in vars(r).items() if isinstance(v, torch.Tensor)} for r in records]
    got = P.playback8(h, records, 2.0 ** -7, 0.0, 0.25, precision=precision)
    assert [r["name"] for r in got["layers"]] == [f"block{b}.{p}" for b in (0, 1) for p in ("norm", "up", "down")]
    for rec, before, scores in zip(records, kept, got["layers"]):
        for k, v in before.items():
            assert torch.equal(getattr(rec, k), v)
        if isinstance(rec, P.NormRecord):
            assert scores["sum"]["max_abs"] == 0.0 and set(scores) == {"name", "fwd", "sum", "in_grad", "wg_grad"}
            assert scores["fwd"]["n"] == rec.y.numel()
            assert scores["fwd"]["max_abs"] <= 1.01 * float((moves(rec.y) + 2.0 ** -7 * rec.y.double().abs()).max())
            size = rec.grad_x.double().abs().max() + rec.grad.double().abs().max() * 4
            assert scores["in_grad"]["max_abs"] <= 2.0 ** -7 * float(size)
            assert scores["wg_grad"]["max_abs"] <= (tokens + 8) * 2.0 ** -22 * float(rec.grad.double().abs().sum(0).max() * 6)
            continue
        for key, golden, a, b in (("fwd", rec.y, rec.x, rec.weight), ("in_grad", rec.grad_x, rec.grad, rec.weight.t()),
                                  ("wg_grad", rec.grad_weight, rec.grad.t(), rec.x.t())):
            s = scores[key]
            slack = 2.0 ** -7 if golden.dtype == torch.bfloat16 else 1e-6
            size = a.double().abs() @ b.double().abs().t() + (0.1 if key == "fwd" else 0.0)
            assert s["n"] == golden.numel()
            assert 0.0 < s["mean_abs"] <= s["top10_mean"] <= s["max_abs"]
            assert s["max_abs"] <= 1.01 * float((bound(a, b) + slack * size).max())


def test_norms_in_8_bits(peat_gpu, h):
    """A norm's replayed output is off by half a step of its row, 1 / 254 of the largest element, and the roundings to
    bfloat16 on both sides."""
    from paper_2609_13544_gb300 import playback8 as P
    rec = P.synthetic_records(130, 200, 64, 1, 3, norms=True)[0]
    scores, grad = P.replay_norm(h, rec, 2.0 ** -7)
    y = rec.y.double().abs()
    assert scores["fwd"]["max_abs"] <= 1.01 * float((y.amax(1, keepdim=True) / 254 + 2.0 ** -7 * y).max())
    assert scores["sum"]["max_abs"] == 0.0 and grad.shape == (200,)
    # any leading dimensions
    lead = lambda t: t if t is None or t.dim() == 1 else t.view(5, 26, -1)
    again = P.NormRecord(**{k: lead(v) if hasattr(v, "dim") else v for k, v in vars(rec).items()})
    assert P.replay_norm(h, again, 2.0 ** -7)[0] == scores


def test_command(peat_gpu, capsys):
    from paper_2609_13544_gb300 import playback8 as P
    for precision in ("mxfp4", "nvfp4", "i8"):
        result = P.main(["--tokens", "40", "--width", "64", "--hidden", "128", "--blocks", "1", "--precision", precision, "--norms"])
        assert json.loads(capsys.readouterr().out) == result
        assert len(result["layers"]) == 3 and result["golden"]["norm"] > 0


def test_unknown_precision(peat_gpu, h):
    from paper_2609_13544_gb300 import playback8 as P
    for rec in P.synthetic_records(3, 64, 40, 1, 1, norms=True)[:2]:
        replay = P.replay_norm if isinstance(rec, P.NormRecord) else P.replay_layer
        with pytest.raises(ValueError):
            replay(h, rec, 0.01, precision="fp4")


def test_other_stream(peat_gpu, h):
    """Everything on a given stream gives what the current one gives."""
    import torch
    from paper_2609_13544_gb300 import playback8 as P
    want = P.playback8(h, P.synthetic_records(65, 96, 64, 1, 9, norms=True), 1e-2, precision="nvfp4")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        records = P.synthetic_records(65, 96, 64, 1, 9, norms=True)
    assert P.playback8(h, records, 1e-2, stream=s, precision="nvfp4") == want
