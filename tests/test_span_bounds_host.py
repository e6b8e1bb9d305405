"""The element-wise bound for span attention: the emulated number formats keep it, and every second half term, the scale of the
probabilities and the reference of block-scaled rows is needed for that.  No GPU."""
import pytest
import torch

from tests import ref_span_bounds as E


def _quantised(x):
    scale = (x.abs().amax(-1, keepdim=True) / 32767).float()
    return torch.where(scale > 0, (x / scale.double()).round().clamp(-32767, 32767), 0.0), scale[:, 0]


def _data(kind, seed, scaled):
    g = torch.Generator().manual_seed(seed)
    hd = 128
    n, R = dict(plain=(200, 8), sink=(8200, 4), late=(220, 4))[kind]
    q = (torch.randn((R, hd), generator=g, dtype=torch.float64) * 1.5).float().double()
    k, v = (torch.randn((n, hd), generator=g, dtype=torch.float64) for _ in range(2))
    if kind == "sink":      # the first row takes most of the weight and is zero but for one element, the others have little weight and a mean of one
        q[1:] = q[0] * torch.tensor([[0.9], [1.1], [1.2]], dtype=torch.float64)
        q = q.float().double()
        k *= 0.02
        k[0] = q[0] / (q[0] ** 2).sum() * hd ** 0.5 * 12.0
        v = 1 + 0.1 * v
        v[0], v[0, 0] = 0, 1
    if kind == "late":      # a row in the middle of a wavefront's share takes all the weight; its values are far below the others'
        q[1:] = q[0]
        k[40] = q[0] / (q[0] ** 2).sum() * hd ** 0.5 * 60.0
        v *= 1e6
        v[40] = 10.0 ** -(seed % 3 - 1) * torch.randn(hd, generator=g, dtype=torch.float64)
    if not scaled:
        return q, k.half().double(), v.clamp(-60000, 60000).half().double(), None
    rows = [_quantised(k), _quantised(v)]
    return q, *(i * s.double()[:, None] for i, s in rows), rows


def _worst(kind, seed, scaled, mistake=None):
    """Largest error over its tolerance (both half terms, without their own rounding)."""
    q, k, v, rows = _data(kind, seed, scaled)
    got = E.emulate(q, k, v, len(k), rows, mistake).double()
    worst = 0.0
    for r in range(len(q)):
        out, _, _, tol = E.bound(q[r], k, v, v.abs().amax(-1) if scaled else None)
        worst = max(worst, float(((got[r] - out).abs() / tol).max()))
    return worst


@pytest.mark.parametrize("kind, scaled", [("plain", False), ("plain", True), ("sink", False), ("sink", True), ("late", True)])
def test_the_formats_keep_the_bound(kind, scaled):
    for seed in range(3):
        assert _worst(kind, seed, scaled) <= 1


@pytest.mark.parametrize("kind, scaled, mistake", [
    ("plain", False, "q"), ("plain", True, "q"), ("plain", False, "p"), ("plain", True, "p"), ("plain", True, "rows"),
    ("sink", False, "tail"), ("sink", True, "tail"), ("sink", False, "p"), ("late", True, "reference"), ("late", True, "rows")])
def test_the_bound_sees_what_is_missing(kind, scaled, mistake):
    for seed in range(3):
        assert _worst(kind, seed, scaled, mistake) > 1
