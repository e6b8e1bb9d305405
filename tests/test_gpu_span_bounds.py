"""Span attention against its definition in 64 bits, element by element: each output and each weight within what the formats and sums of
its own row allow (tests/ref_span_bounds.py; tests/test_span_bounds_host.py shows on the CPU that a second half term left out, probabilities split
at their own size or a stale reference of block-scaled rows are several times beyond that)."""
import math

import pytest
import torch

from tests.gpu_util import DEV
from tests import ref_span as R
from tests import ref_span_bounds as E
from tests.test_gpu_span_ops import _i32, _ops, _rnd, _run_span

pytestmark = pytest.mark.gpu


def _check(cache, q, lens, T, nsplit=0, span=None, weights=True):
    q = q.float().double()
    k, v = cache.values(0), cache.values(1)
    want, hi, both, add, add_tol = E.attend(q, k, v, lens, T, cache.block_scaled, span)
    w0 = torch.rand((cache.B, cache.Hkv, cache.S), generator=torch.Generator().manual_seed(6)) * 0.1
    weight = w0.to(DEV) if weights else None
    out, lo = _run_span(cache, q, lens, T, nsplit, span, weight)
    there = ~want.isnan()
    assert ((out - want).abs() <= hi)[there].all(), float(((out - want).abs() / hi)[there].max())
    assert ((out + lo - want).abs() <= both)[there].all(), float(((out + lo - want).abs() / both)[there].max())
    assert (out[~there] == 7.0).all() and (lo[~there] == 7.0).all()
    if weights:      # the query rows of a kv head are added up in fp32, at most T * Hq / Hkv of them, and to what was there
        ref = w0.double() + add
        tol = add_tol + (math.sqrt(T * q.shape[2] / cache.Hkv) * 4 * add + 2 * ref) * R.F32_STEP
        assert ((weight.cpu().double() - ref).abs() <= tol).all()
        assert torch.equal(weight.cpu()[add == 0], w0[add == 0])


SHAPES = [(1, 4, 1), (3, 4, 1), (6, 4, 1), (6, 8, 1), (2, 8, 2)]       # T, Hq, Hkv: 4, 12, 24, 48 query rows of a kv head (two workgroups), 8


@pytest.mark.parametrize("nsplit", [1, 3])
@pytest.mark.parametrize("block_scaled", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv", SHAPES)
def test_rows_with_little_weight_each(T, Hq, Hkv, block_scaled, nsplit):
    """The first row takes most of the weight and is zero but for one element, thousands of others share the rest: a bounded cache's usual shape."""
    hd, n = 128, 8200
    S = n + 8
    g = torch.Generator().manual_seed(T + Hq)
    q0 = (_rnd(g, 1, 1, 1, hd) * 1.5).expand(1, T, Hq, hd) * (0.9 + 0.05 * torch.arange(T * Hq, dtype=torch.float64).view(1, T, Hq, 1) % 0.4)
    k, v = _rnd(g, 1, Hkv, S, hd) * 0.02, 1 + 0.1 * _rnd(g, 1, Hkv, S, hd)
    k[:, :, 0] = q0[0, 0, 0] / (q0[0, 0, 0] ** 2).sum() * hd ** 0.5 * 12.0
    v[:, :, 0], v[:, :, 0, 0] = 0, 1
    _check(R.Cache(k, v, block_scaled), q0, [n - T], T, nsplit)


@pytest.mark.parametrize("at", [40, 300])
@pytest.mark.parametrize("block_scaled", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv", SHAPES)
def test_a_late_row_of_small_values_takes_all_the_weight(T, Hq, Hkv, block_scaled, at):
    """A row behind the first tile of a wavefront's share dominates and holds values far below those of the rows before it."""
    hd, n = 128, 520
    g = torch.Generator().manual_seed(T * Hq + at)
    q = (_rnd(g, 1, 1, 1, hd) * 1.5).expand(1, T, Hq, hd)
    for small in (10.0, 0.1, 0.01):
        k, v = _rnd(g, 1, Hkv, n + T, hd), _rnd(g, 1, Hkv, n + T, hd) * (1e6 if block_scaled else 1e4)
        k[:, :, at] = q[0, 0, 0] / (q[0, 0, 0] ** 2).sum() * hd ** 0.5 * 60.0
        v[:, :, at] = small * _rnd(g, 1, Hkv, hd)
        _check(R.Cache(k, v, block_scaled), q, [n], T, 1)


@pytest.mark.parametrize("T,Hq,Hkv", SHAPES)
def test_values_below_the_normal_numbers(T, Hq, Hkv):
    """Block-scaled rows whose scale is a subnormal number, alone and beside rows of ordinary size."""
    hd, n = 64, 150
    g = torch.Generator().manual_seed(T * Hq)
    k, v, q = _rnd(g, 2, Hkv, n + T, hd), _rnd(g, 2, Hkv, n + T, hd) * 1e-36, _rnd(g, 2, T, Hq, hd)
    v[1, :, ::5] *= 1e36
    _check(R.Cache(k, v, True), q, [n, n - 70], T)


@pytest.mark.parametrize("block_scaled", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,nsplit", [(1, 4, 1, 1), (3, 4, 1, 1), (6, 4, 1, 1), (12, 4, 1, 1), (2, 4, 1, 2), (6, 4, 1, 2)])
def test_not_a_number_comes_out_as_one(T, Hq, Hkv, nsplit, block_scaled):
    """A NaN in a query, a K or a V row makes the queries that hold or see it NaN, and no others differ in a bit."""
    hd, n = 128, 270
    g = torch.Generator().manual_seed(T)
    k, v, q = _rnd(g, 2, Hkv, n + T, hd), _rnd(g, 2, Hkv, n + T, hd), _rnd(g, 2, T, Hq, hd)
    clean, clean_lo = _run_span(R.Cache(k, v, block_scaled), q, [n, n - 9], T, nsplit)
    bad = q.clone()
    bad[0, T - 1, 2, 5] = float("nan")
    hit = torch.zeros((2, T, Hq), dtype=torch.bool)
    hit[0, T - 1, 2] = True
    for name, at in (("q", 0), ("inf", 0), ("k", 40), ("v", 40), ("k", n + T - 1), ("v", n + T - 1)):
        cache = R.Cache(k, v, block_scaled)
        if name == "inf":
            bad[0, T - 1, 2, 5] = -float("inf")
        if name in "kv":
            i = "kv".index(name)
            if block_scaled:
                cache.scales[i][0, 0, at] = float("nan")
            else:
                cache.rows[i][0, 0, at] = float("nan")
            hit = torch.zeros((2, T, Hq), dtype=torch.bool)
            hit[0, max(0, at - n):] = True
        out, lo = _run_span(cache, q if name in "kv" else bad, [n, n - 9], T, nsplit)
        assert out[hit].isnan().all() and lo[hit].isnan().all(), (name, at)
        assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lo[~hit], clean_lo[~hit]), (name, at)


@pytest.mark.parametrize("block_scaled", [False, True])
def test_an_infinite_value_is_no_finite_result(block_scaled):
    T, Hq, hd, n = 3, 4, 64, 100
    g = torch.Generator().manual_seed(2)
    k, v, q = _rnd(g, 1, 1, n + T, hd), _rnd(g, 1, 1, n + T, hd), _rnd(g, 1, T, Hq, hd)
    for sign in (1, -1):
        for at in (5, n, n + 2):
            cache = R.Cache(k, v, block_scaled)
            if block_scaled:
                cache.scales[1][0, 0, at] = sign * float("inf")
            else:
                cache.rows[1][0, 0, at] = sign * float("inf")
            out, _ = _run_span(cache, q, [n], T)
            sees = out[0, max(0, at - n):]
            # NaN, or saturated with the sign of the value; a row whose scale is infinite has values of both signs
            assert (sees.isnan() | (sees == sign * 65504)).all() and (not block_scaled or sees.isnan().all())
            if block_scaled:
                cache = R.Cache(k, v, True)
                cache.scales[0][0, 0, at] = sign * float("inf")
                assert _run_span(cache, q, [n], T)[0][0, max(0, at - n):].isnan().all()


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("nsplit", [2, 5, 64])
@pytest.mark.parametrize("block_scaled,page", [(False, 0), (True, 16)])
@pytest.mark.parametrize("T,Hq,Hkv,hd", [(1, 4, 2, 128), (2, 8, 2, 64), (3, 8, 2, 128), (6, 8, 2, 64), (8, 4, 1, 128), (11, 8, 1, 64)])
def test_splits_of_every_number_of_query_rows(T, Hq, Hkv, hd, block_scaled, page, nsplit, weights):
    """2, 8, 12, 24, 32 and 88 query rows of a kv head (three workgroups), the rows of a sequence on several workgroups."""
    B, S = 3, 432
    g = torch.Generator().manual_seed(T + nsplit)
    cache = R.Cache(_rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd), block_scaled, page)
    _check(cache, _rnd(g, B, T, Hq, hd, std=1.5), [S - T, 0, 130], T, nsplit, [T, T, max(1, T - 1)], weights)


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("block_scaled", [False, True])
@pytest.mark.parametrize("T,Hq", [(2, 4), (3, 4), (6, 4)])
def test_page_lists_longer_than_a_wavefront(T, Hq, block_scaled, weights):
    """A wavefront's share of 16-row pages passes 64, 128 and 192 entries of its list; lengths that end just behind a refill."""
    B, hd, S, page = 4, 64, 13120, 16
    g = torch.Generator().manual_seed(T)
    cache = R.Cache(_rnd(g, B, 1, S, hd), _rnd(g, B, 1, S, hd), block_scaled, page)
    _check(cache, _rnd(g, B, T, Hq, hd), [S - T, 4 * 1024 + 1, 4097 + 128, 8 * 1024 + 17], T, 1, None, weights)


@pytest.mark.parametrize("nsplit", [0, 1, 4])
@pytest.mark.parametrize("block_scaled,page", [(False, 64), (True, 0)])
def test_a_chunk_of_a_prompt_over_a_cached_prefix(block_scaled, page, nsplit):
    B, T, Hq, Hkv, hd, S = 2, 70, 8, 2, 128, 640
    g = torch.Generator().manual_seed(nsplit)
    cache = R.Cache(_rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd), block_scaled, page)
    _check(cache, _rnd(g, B, T, Hq, hd), [S - T, 37], T, nsplit, [T, 51])


@pytest.mark.parametrize("block_scaled", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,hd", [(1, 4, 4, 64), (2, 16, 2, 128), (5, 8, 2, 128), (9, 16, 4, 64)])
def test_each_result_within_its_own_bound(T, Hq, Hkv, hd, block_scaled):
    """Ordinary rows: the second half terms of queries, probabilities and integer rows decide whether this holds."""
    for n in (3, 40, 300):
        g = torch.Generator().manual_seed(n + T)
        k, v = _rnd(g, 1, Hkv, n + T, hd), _rnd(g, 1, Hkv, n + T, hd)
        _check(R.Cache(k, v, block_scaled), _rnd(g, 1, T, Hq, hd, std=1.5), [n], T)
