"""Steps of several tokens over a bounded cache -- rl_op_rope_append_at, rl_op_span_attention, rl_op_evict_rows,
rl_op_verify_drafts -- against their definitions in 64 bits (tests/ref_span.py), alone and as the loop they make together.

Tolerances, from the formats: an output rounded to half is off by 2^-11 of its value; a score by ref_span.score_error, so a
probability by twice that relatively (numerator and sum) plus the exponential's own 2^-20, and an output by as much of the largest
|v|; fp32 sums by 2^-24 of the terms per addition.  Eviction moves values and verification returns whole numbers: equal."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_util import DEV
from tests import ref_span as R

pytestmark = pytest.mark.gpu


def _ops():
    from paper_2406_14088_amd import ops
    return ops


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _rnd(g, *shape, std=1.0):
    return torch.randn(shape, generator=g, dtype=torch.float64) * std


# ------------------------------------------------------------------------------------------------------------ span attention
def _run_span(cache, q, lens, T, nsplit=0, span=None, weight=None, want_lo=True):
    B, _, Hq, hd = q.shape
    ops = _ops()
    d_q = q.reshape(B * T, Hq * hd).to(torch.float32).to(DEV)
    out = torch.full((B * T, Hq * hd), 7.0, dtype=torch.float16, device=DEV)
    lo = torch.full_like(out, 7.0) if want_lo else None
    n = ops.span_attention_ws_floats(B, T, Hq, cache.Hkv, hd, cache.S, nsplit, weight is not None)
    ws = torch.full((max(n, 1),), float("nan"), device=DEV)
    ops.span_attention(d_q, cache.rows[0], cache.rows[1], _i32(lens), out, ws, T, Hq, cache.Hkv, hd, cache.S, nsplit=nsplit,
                       d_span=None if span is None else _i32(span), out_lo=lo, weight=weight, **cache.args())
    torch.cuda.synchronize()
    shape = (B, T, Hq, hd)
    return out.cpu().double().view(shape), None if lo is None else lo.cpu().double().view(shape)


def _check_span(cache, q, lens, T, nsplit=0, span=None, weights=True):
    q = q.float().double()
    k, v = cache.values(0), cache.values(1)
    want, add, valid = R.attend(q, k, v, lens, T, span)
    g = torch.Generator().manual_seed(5)
    w0 = torch.rand((cache.B, cache.Hkv, cache.S), generator=g)
    weight = w0.to(DEV) if weights else None
    out, lo = _run_span(cache, q, lens, T, nsplit, span, weight)
    seen = torch.zeros((cache.B, cache.S), dtype=torch.bool)
    for b in range(cache.B):
        seen[b, : max(0, min(int(lens[b]), cache.S)) + T] = True
    ks, vs = (torch.where(seen[:, None, :, None], x, 0.0) for x in (k, v))
    ds = 2 * R.score_error(q, ks, cache.hd) + 2.0 ** -20
    vmax = float(vs.nan_to_num(0, 0, 0).abs().max())
    sel = valid[..., None, None].expand_as(want)
    assert torch.equal(torch.isfinite(out)[sel], torch.isfinite(want)[sel])
    fine = sel & torch.isfinite(want)
    err = (out - want).abs()[fine]
    assert (err <= R.HALF_STEP * want.abs()[fine] + ds * vmax + 2.0 ** -25).all(), float(err.max())
    err2 = (out + lo - want).abs()[fine]
    assert (err2 <= ds * vmax + 2.0 ** -22 * want.abs()[fine] + 2.0 ** -25).all(), float(err2.max())
    assert (out[~sel] == 7.0).all() and (lo[~sel] == 7.0).all()           # rows without a token stay as they were
    if weights:
        got = weight.cpu().double()
        ref = w0.double() + add
        ok = torch.isfinite(add)
        g_heads = q.shape[2] // cache.Hkv
        assert ((got - ref).abs()[ok] <= (ds + 4 * math.sqrt(T * g_heads) * R.F32_STEP) * add[ok] + 2 * R.F32_STEP * ref.abs()[ok]).all()
        untouched = add == 0
        assert torch.equal(got[untouched], w0.double()[untouched])         # rows that nobody sees keep their weight
    return out


SPAN_CASES = [
    # B, T, Hq, Hkv, hd, S, lens
    (1, 1, 4, 4, 128, 16, [0]),                      # a single row: its own
    (2, 1, 4, 4, 64, 48, [0, 46]),
    (3, 4, 8, 2, 128, 80, [0, 1, 75]),
    (2, 5, 4, 4, 128, 272, [255, 267]),              # more rows than a tile, an end inside one
    (2, 5, 16, 2, 64, 160, [31, 155]),
    (1, 8, 16, 1, 128, 336, [320]),                  # 128 query rows of one kv head
    (2, 3, 6, 2, 128, 64, [17, 33]),                 # three heads per kv head
    (1, 2, 64, 1, 64, 96, [90]),                     # 64 heads per kv head
    (5, 1, 64, 8, 128, 208, [200, 0, 15, 16, 100]),  # single tokens, grouped heads
    (2, 33, 4, 2, 128, 96, [0, 60]),                 # a span longer than what was there
    (2, 16, 8, 8, 64, 1040, [1000, 3]),
]


@pytest.mark.parametrize("page", [0, 16, 32])
@pytest.mark.parametrize("block_scaled", [False, True])
@pytest.mark.parametrize("case", SPAN_CASES)
def test_span_attention(case, block_scaled, page):
    B, T, Hq, Hkv, hd, S, lens = case
    S = -(-S // max(page, 1)) * max(page, 1)
    g = torch.Generator().manual_seed(B * 100 + T)
    k, v = _rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd)
    for b in range(B):                               # what lies behind the last sequence's rows must not matter
        k[b, :, lens[b] + T:] = float("nan")
        v[b, :, lens[b] + T:] = float("inf")
    if block_scaled:                                 # rows of very different magnitude, and a row of zeros
        mag = torch.rand((B, 1, S, 1), generator=g, dtype=torch.float64) * 6 - 3
        v = v * 10.0 ** mag
        v[:, :, 3] = 0
        k[:, :, 5] = 0
        k, v = k.nan_to_num(0, 0, 0), v.nan_to_num(0, 0, 0)
    cache = R.Cache(k, v, block_scaled, page, seed=B + S)
    _check_span(cache, _rnd(g, B, T, Hq, hd, std=1.5), lens, T)


@pytest.mark.parametrize("nsplit", [1, 2, 3, 7, 64])
@pytest.mark.parametrize("block_scaled", [False, True])
def test_span_attention_splits_join(nsplit, block_scaled):
    B, T, Hq, Hkv, hd, S = 3, 3, 8, 2, 128, 256
    g = torch.Generator().manual_seed(nsplit)
    cache = R.Cache(_rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd), block_scaled)
    _check_span(cache, _rnd(g, B, T, Hq, hd, std=2.0), [250, 0, 100], T, nsplit)


@pytest.mark.parametrize("T,Hq,hd", [(1, 16, 128), (2, 10, 64), (2, 16, 128), (4, 8, 64)])
@pytest.mark.parametrize("block_scaled", [False, True])
def test_span_attention_weights_of_long_unsplit_sequences(T, Hq, hd, block_scaled):
    # scores of 8 (up to 8 query rows: 16) tiles of 32 rows stay in a wavefront's registers, four wavefronts share a sequence: either side of 2048 and 1024 rows
    lens = [2600, 2048 - T, 2048, 1024 - T, 1025, 1]
    B, Hkv, S = len(lens), 2, 2608
    g = torch.Generator().manual_seed(T * hd + Hq)
    cache = R.Cache(_rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd), block_scaled)
    _check_span(cache, _rnd(g, B, T, Hq, hd, std=1.5), lens, T, 1)


@pytest.mark.parametrize("T,Hq", [(3, 4), (4, 8), (8, 8)])
@pytest.mark.parametrize("page", [0, 16])
def test_span_attention_weights_of_ragged_spans(T, Hq, page):
    B, Hkv, hd, S = 6, 2, 128, 160                     # query rows behind a sequence's last token add nothing to its weights
    g = torch.Generator().manual_seed(T)
    cache = R.Cache(_rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd), False, page)
    _check_span(cache, _rnd(g, B, T, Hq, hd), [0, 150, 31, 32, 100, 7], T, span=[1, T, 0, T - 1, 2, T + 3])


@pytest.mark.parametrize("T,Hq", [(1, 64), (2, 64), (4, 64), (5, 64)])
def test_span_attention_weights_of_many_sequences(T, Hq):
    B, Hkv, hd, S = 65, 8, 64, 96                      # more kv heads than workgroups of four wavefronts run at once
    g = torch.Generator().manual_seed(T)
    cache = R.Cache(_rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd), False)
    _check_span(cache, _rnd(g, B, T, Hq, hd), torch.randint(0, S - T + 1, (B,), generator=g).tolist(), T)


@pytest.mark.parametrize("page", [0, 64])
def test_span_attention_of_ragged_spans(page):
    B, T, Hq, Hkv, hd, S = 5, 6, 8, 2, 128, 128
    g = torch.Generator().manual_seed(3)
    cache = R.Cache(_rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd), page=page)
    _check_span(cache, _rnd(g, B, T, Hq, hd), [10, 64, 0, 122, 31], T, span=[0, 6, 1, 3, -4])
    _check_span(cache, _rnd(g, B, T, Hq, hd), [-3, 126, 128, 500, 31], T, span=[2, 6, 2, 1, 99])    # clamped to the capacity


def test_span_attention_peaks_and_large_scores():
    """One key takes all the weight, late and early; scores of several hundred."""
    B, T, Hq, Hkv, hd, S = 2, 2, 4, 2, 128, 200
    g = torch.Generator().manual_seed(8)
    for at in (0, 63, 150, 197):
        k, v = _rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd)
        q = _rnd(g, B, T, Hq, hd)
        k[:, :, at] = q[:, 0].view(B, Hkv, -1, hd)[:, :, 0] * 30
        _check_span(R.Cache(k, v), q, [198, 196], T)
        v[:, :, at] *= 1e-6                                                # the row that matters has the smallest scale
        _check_span(R.Cache(k, v, block_scaled=True), q, [198, 196], T)


@pytest.mark.parametrize("block_scaled", [False, True])
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_span_attention_not_finite_rows_reach_only_who_sees_them(block_scaled, what, bad):
    B, T, Hq, Hkv, hd, S = 2, 5, 4, 2, 128, 96
    g = torch.Generator().manual_seed(4)
    k, v = _rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd)
    cache = R.Cache(k, v, block_scaled)
    i = 0 if what == "k" else 1
    (cache.scales[i] if block_scaled else cache.rows[i])[0, 1, 70 + 3] = bad       # the row of token 3 of sequence 0, kv head 1
    q = _rnd(g, B, T, Hq, hd)
    out, _ = _run_span(cache, q, [70, 40], T)
    clean = R.Cache(k, v, block_scaled)
    want, _ = _run_span(clean, q, [70, 40], T)
    assert torch.equal(out[1], want[1]) and torch.equal(out[0, :, :2], want[0, :, :2]) and torch.equal(out[0, :3], want[0, :3])
    if what == "v" or bad != float("-inf"):
        sees = out[0, 3:, 2:]
        # a saturated half stands for a value beyond the type; -inf scores only where q . k says so
        assert what == "k" and not block_scaled or not torch.isfinite(sees).any() or (sees.abs() >= 65504).any()


def test_span_attention_lowest_values_and_ties():
    """Keys of the lowest half and equal scores everywhere: weights are 1 / n."""
    B, T, Hq, Hkv, hd, S = 1, 3, 4, 4, 64, 64
    g = torch.Generator().manual_seed(9)
    k = torch.zeros((B, Hkv, S, hd), dtype=torch.float64)
    v = _rnd(g, B, Hkv, S, hd)
    _check_span(R.Cache(k, v), _rnd(g, B, T, Hq, hd), [50], T)
    k[..., 0] = -65504.0
    q = torch.zeros((B, T, Hq, hd), dtype=torch.float64)
    q[..., 0] = 1.0
    _check_span(R.Cache(k, v), q, [50], T)


def test_span_attention_of_one_token_agrees_with_decode_attention():
    ops = _ops()
    B, Hq, Hkv, hd, S = 4, 32, 8, 128, 320
    g = torch.Generator().manual_seed(10)
    k, v, q = _rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd), _rnd(g, B, 1, Hq, hd)
    cache = R.Cache(k, v)
    got, got_lo = _run_span(cache, q, [300, 0, 17, 255], 1)
    out = torch.zeros((B, Hq * hd), dtype=torch.float16, device=DEV)
    lo = torch.zeros_like(out)
    ops.decode_attention(q.float().view(B, -1).to(DEV), cache.rows[0], cache.rows[1], _i32([300, 0, 17, 255]), out, None, B, Hq, Hkv, hd, S, 1,
                         len_stride=1, out_lo=lo)
    both = 2 * (2 * R.score_error(q, k, hd) + 2.0 ** -20) * float(v.abs().max())
    assert ((got + got_lo).view(B, -1) - (out.cpu().double() + lo.cpu().double())).abs().max() <= both


def test_span_attention_long_cache_offsets():
    """A pool whose element offsets pass 2^31, with the rows in use at its end, and a contiguous cache of more than 4 GB."""
    ops = _ops()
    Hkv, hd, page, T, Hq = 8, 128, 64, 2, 8
    n_pages = (1 << 31) // (Hkv * page * hd) + 40
    pool = [torch.zeros((n_pages, Hkv, page, hd), dtype=torch.float16, device=DEV) for _ in range(2)]
    g = torch.Generator().manual_seed(11)
    n = 200
    k, v, q = (_rnd(g, 1, h, r, hd) for h, r in ((Hkv, 256), (Hkv, 256), (T, Hq)))
    table = torch.arange(n_pages - 4, n_pages, dtype=torch.int32)[None]
    for x, p in ((k, pool[0]), (v, pool[1])):
        p[-4:] = x.to(torch.float16).view(Hkv, 4, page, hd).transpose(0, 1).to(DEV)
    out = torch.zeros((T, Hq * hd), dtype=torch.float16, device=DEV)
    ws = torch.empty(max(1, ops.span_attention_ws_floats(1, T, Hq, Hkv, hd, 256, 0, False)), device=DEV)
    ops.span_attention(q.float().view(T, -1).to(DEV), pool[0], pool[1], _i32([n]), out, ws, T, Hq, Hkv, hd, 256, table=table.to(DEV), page_size=page)
    kk, vv = k.to(torch.float16).double(), v.to(torch.float16).double()
    want, _, _ = R.attend(q.float().double(), kk, vv, [n], T)
    tol = (2 * R.score_error(q, kk, hd) + 2.0 ** -20) * float(vv.abs().max())
    err = (out.cpu().double().view(want.shape) - want).abs()
    assert (err <= tol + R.HALF_STEP * want.abs()).all()
    # the same memory as one slab per (sequence, kv head): the last sequence of 33
    S = n_pages * page // 33
    slab = [p.view(-1)[: 33 * Hkv * S * hd].view(33, Hkv, S, hd) for p in pool]
    for x, p in ((k, slab[0]), (v, slab[1])):
        p[32, :, :256] = x[0].to(torch.float16).to(DEV)
    qs = q.float().view(1, T, -1).expand(33, T, Hq * hd).reshape(33 * T, -1).contiguous().to(DEV)
    outs = torch.zeros((33 * T, Hq * hd), dtype=torch.float16, device=DEV)
    ws = torch.empty(max(1, ops.span_attention_ws_floats(33, T, Hq, Hkv, hd, S, 1, False)), device=DEV)
    ops.span_attention(qs, slab[0], slab[1], _i32([n] * 33), outs, ws, T, Hq, Hkv, hd, S, nsplit=1)
    err = (outs[-T:].cpu().double().view(want.shape) - want).abs()
    assert (err <= tol + R.HALF_STEP * want.abs()).all()


# -------------------------------------------------------------------------------------------------------------- append
APPEND_CASES = [
    # B, T, Hq, Hkv, hd, rot, style, nsplit, S, slots, positions
    (1, 1, 4, 4, 64, 64, 1, 1, 16, [0], [0]),
    (3, 4, 8, 2, 128, 128, 1, 3, 64, [0, 17, 60], [0, 400, 90]),
    (2, 5, 4, 4, 128, 64, 0, 2, 48, [3, 31], [2000, 31]),
    (2, 7, 6, 2, 64, 16, 0, 1, 48, [40, 0], [40, 1234]),
    (2, 3, 16, 1, 128, 8, 1, 1, 32, [0, 29], [5, 29]),
    (1, 130, 4, 2, 64, 32, 1, 4, 160, [11], [1800]),
]


def _table(rot, n, base=10000.0, **kw):
    tab = torch.zeros((n, rot // 2, 2), device=DEV)
    _ops().build_rope_table_scaled(tab, n, rot, base, **kw)
    return tab


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("block_scaled", [False, True])
@pytest.mark.parametrize("case", APPEND_CASES)
def test_rope_append_at(case, block_scaled, page):
    B, T, Hq, Hkv, hd, rot, style, nsplit, S, slots, poss = case
    g = torch.Generator().manual_seed(T)
    k0, v0 = _rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd)
    cache = R.Cache(k0, v0, block_scaled, page)
    before = [r.clone() for r in cache.rows]
    heads = Hq + 2 * Hkv
    qkv = _rnd(g, nsplit, B * T, heads * hd).float()
    tab = _table(rot, 2200)
    weight, row_pos = torch.rand((B, Hkv, S), device=DEV) + 1, torch.full((B, Hkv, S), -9, dtype=torch.int32, device=DEV)
    w0, r0 = weight.cpu(), row_pos.cpu()
    qf, qh, ql = torch.zeros((B * T, Hq * hd), device=DEV), *(torch.zeros((B * T, Hq * hd), dtype=torch.float16, device=DEV) for _ in range(2))
    _ops().rope_append_at(qkv.to(DEV), nsplit, B * T * heads * hd, T, _i32(poss), _i32(slots), tab, style, rot, Hq, Hkv, hd, S, cache.rows[0],
                          cache.rows[1], q_f32=qf, q_f16=qh, q_f16_lo=ql, weight=weight, row_pos=row_pos, **cache.args())
    torch.cuda.synchronize()
    x = qkv.double().sum(0).view(B, T, heads, hd)
    mag = qkv.double().abs().sum(0).view(B, T, heads, hd).amax(-1, keepdim=True)
    pos = torch.tensor(poss)[:, None] + torch.arange(T)
    y = x.clone()
    y[:, :, : Hq + Hkv] = R.rotate(x[:, :, : Hq + Hkv], pos[:, :, None].expand(B, T, Hq + Hkv), R.frequencies(rot, 10000.0), rot, style)
    # a pair: nsplit - 1 additions, two products with a rounded cosine and sine, one sum, on values up to mag each
    tol = (nsplit + 6) * R.F32_STEP * 2 * mag
    assert ((qf.cpu().double().view(B, T, Hq, hd) - y[:, :, :Hq]).abs() <= tol[:, :, :Hq]).all()
    assert torch.equal(qh, qf.clamp(-65504, 65504).to(torch.float16))
    assert torch.equal(ql, (qf - qh.float()).to(torch.float16))
    k, v = cache.values(0), cache.values(1)
    touched = torch.zeros((B, S), dtype=torch.bool)
    for b in range(B):
        at = slots[b] + torch.arange(T)
        touched[b, at] = True
        for got, h0 in ((k, Hq), (v, Hq + Hkv)):
            ref, t = y[b, :, h0:h0 + Hkv].transpose(0, 1), tol[b, :, h0:h0 + Hkv].transpose(0, 1)
            err = (got[b][:, at] - ref).abs()
            if block_scaled:      # half a unit of the row's scale, which is its largest magnitude / 32767
                assert (err <= 0.501 * ref.abs().amax(-1, keepdim=True) / 32767 + 2 * t).all()
            else:
                assert (err <= R.HALF_STEP * ref.abs() + t + 2.0 ** -25).all()
        assert (weight[b].cpu()[:, at] == 0).all()
        assert (row_pos[b].cpu()[:, at] == (poss[b] + torch.arange(T)).to(torch.int32)).all()
    # everything else is as it was, bit for bit (rows behind the last slot and spare pages among it)
    idx = cache.index()[touched[:, None].expand(B, Hkv, S)]
    for now, old in zip(cache.rows, before):
        a, b_ = (r.view(torch.int16).cpu().view(-1, hd).clone() for r in (now, old))
        a[idx], b_[idx] = 0, 0
        assert torch.equal(a, b_)
    keep = ~touched[:, None].expand(B, Hkv, S)
    assert torch.equal(weight.cpu()[keep], w0[keep]) and torch.equal(row_pos.cpu()[keep], r0[keep])


def test_rope_append_at_skips_what_has_no_place():
    """Slots outside the cache, positions outside the table and tokens behind a sequence's span leave everything as it was."""
    B, T, Hq, Hkv, hd, S = 6, 3, 4, 2, 64, 32
    g = torch.Generator().manual_seed(2)
    cache = R.Cache(_rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd))
    before = [cache.raw(0).clone(), cache.raw(1).clone()]
    qkv = _rnd(g, B * T, (Hq + 2 * Hkv) * hd).float().to(DEV)
    q = torch.full((B * T, Hq * hd), 9.0, device=DEV)
    slots, poss, span = [31, -1, 5, 5, 5, 5], [0, 0, 98, -2, 0, 0], [3, 3, 3, 3, 0, 2]
    rows = {(0, 0): 31, (1, 1): 0, (1, 2): 1, (2, 0): 5, (2, 1): 6, (3, 2): 7, (5, 0): 5, (5, 1): 6}    # (sequence, token): slot
    _ops().rope_append_at(qkv, 1, 0, T, _i32(poss), _i32(slots), _table(64, 100), 1, 64, Hq, Hkv, hd, S, cache.rows[0], cache.rows[1], q_f32=q,
                          d_span=_i32(span))
    q = q.cpu().view(B, T, -1)
    for b in range(B):
        hit = {s for (bb, _), s in rows.items() if bb == b}
        for t in range(T):
            assert (q[b, t] != 9.0).any() if (b, t) in rows else (q[b, t] == 9.0).all()
        for j in range(S):
            same = all(torch.equal(cache.raw(i)[b, :, j], before[i][b, :, j]) for i in range(2))
            assert same == (j not in hit), (b, j)


def test_rope_append_at_agrees_with_rope_append():
    """Slot = position, whole heads, contiguous: the same bits as the append that has one number for both."""
    ops = _ops()
    B, T, Hq, Hkv, hd, S = 2, 4, 8, 2, 128, 64
    g = torch.Generator().manual_seed(6)
    for style in (0, 1):
        for bs in (False, True):
            a, b = (R.Cache(torch.zeros(B, Hkv, S, hd), torch.zeros(B, Hkv, S, hd), bs) for _ in range(2))
            qkv = _rnd(g, 2, B * T, (Hq + 2 * Hkv) * hd).float().to(DEV)
            tab = torch.zeros((S, hd // 2, 2), device=DEV)
            ops.build_rope_table(tab, S, hd, 10000.0)
            assert torch.equal(tab, _table(hd, S))
            qa, qb = torch.zeros((B * T, Hq * hd), device=DEV), torch.zeros((B * T, Hq * hd), device=DEV)
            start = _i32([7, 33])
            ops.rope_append(qkv, 2, qkv[0].numel(), B * T, T, 0, start, tab, style, Hq, Hkv, hd, S, qa, None, a.rows[0], a.rows[1], pos_stride=1,
                            kscale=a.scales[0], vscale=a.scales[1])
            ops.rope_append_at(qkv, 2, qkv[0].numel(), T, start, start, tab, style, hd, Hq, Hkv, hd, S, b.rows[0], b.rows[1], q_f32=qb, **b.args())
            assert torch.equal(qa, qb) and all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(a.rows, b.rows))
            if bs:
                assert all(torch.equal(x, y) for x, y in zip(a.scales, b.scales))


def test_block_scaled_append_of_zeros_and_of_large_rows():
    B, T, Hq, Hkv, hd, S = 1, 2, 2, 2, 64, 16
    cache = R.Cache(torch.ones(B, Hkv, S, hd), torch.ones(B, Hkv, S, hd), True)
    qkv = torch.zeros((T, (Hq + 2 * Hkv) * hd), device=DEV)
    qkv[1] = 3e30
    _ops().rope_append_at(qkv, 1, 0, T, _i32([0]), _i32([4]), _table(64, 8), 1, 64, Hq, Hkv, hd, S, cache.rows[0], cache.rows[1], **cache.args())
    assert (cache.values(1)[:, :, 4] == 0).all()
    assert ((cache.values(1)[:, :, 5] / 3e30 - 1).abs() < 2e-5).all()


@pytest.mark.parametrize("kw", [dict(kind=0), dict(kind=1, factor=8.0), dict(kind=2, factor=4.0), dict(kind=3, factor=8.0, orig_len=512, low=1.0, high=4.0)])
def test_scaled_rope_table(kw):
    rot, n, base = 64, 20000, 500000.0
    tab = _table(rot, n, base, **kw).cpu().double()
    f = R.frequencies(rot, base, kw["kind"], kw.get("factor", 1.0), kw.get("orig_len", 0), kw.get("low", 1.0), kw.get("high", 32.0))
    ang = torch.arange(n, dtype=torch.float64)[:, None] * torch.tensor(f, dtype=torch.float64)
    # one rounding to fp32 of a value up to 1; the angle in fp64 is exact to 2^-52 of itself
    assert ((tab[..., 0] - ang.cos()).abs() <= R.F32_STEP + n * 2.0 ** -50).all() and ((tab[..., 1] - ang.sin()).abs() <= R.F32_STEP + n * 2.0 ** -50).all()


# ------------------------------------------------------------------------------------------------------------- eviction
def _evict(cache, weight, lens, keep, recent, pos=None, inplace=False):
    ops = _ops()
    B, Hkv, S, hd = cache.B, cache.Hkv, cache.S, cache.hd
    w = weight.to(DEV)
    wo = w if inplace else torch.full_like(w, -5.0)
    p = None if pos is None else pos.to(DEV)
    po = p if inplace or p is None else torch.full_like(p, -5)
    d_len = _i32(lens)
    d_out = d_len if inplace else torch.full_like(d_len, -5)
    ws = torch.full((max(1, ops.evict_rows_ws_bytes(B, Hkv, S, keep)),), 255, dtype=torch.uint8, device=DEV)
    ops.evict_rows(cache.rows[0], cache.rows[1], w, wo, d_len, d_out, ws, Hkv, hd, S, keep, recent, pos=p, pos_out=po, **cache.args())
    torch.cuda.synchronize()
    return wo.cpu(), None if po is None else po.cpu(), d_out.cpu().tolist()


def _check_evict(B, Hkv, hd, S, lens, keep, recent, weight, pos, block_scaled=False, page=0, inplace=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    if block_scaled:
        cache = R.Cache(_rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd), True, page)
    else:   # every bit pattern of a half: values are moved, not computed
        cache = R.Cache(_rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd), False, page)
        for i in range(2):
            cache.rows[i].view(torch.int16).copy_(torch.randint(-32768, 32768, cache.rows[i].shape, generator=g, dtype=torch.int32).to(torch.int16))
    before = [r.view(torch.int16).cpu().clone() for r in cache.rows]
    scales = [None if s is None else s.cpu().clone() for s in cache.scales]
    wo, po, out_len = _evict(cache, weight, lens, keep, recent, pos, inplace)
    idx = cache.index()
    want = [r.view(-1, hd).clone() for r in before]
    want_s = [None if s is None else s.view(-1).clone() for s in scales]
    for b in range(B):
        n = min(max(lens[b], 0), S)
        assert out_len[b] == min(n, keep)
        for h in range(Hkv):
            src = R.evict(weight[b, h].tolist(), None if pos is None else pos[b, h].tolist(), lens[b], S, keep, recent)
            at, of = idx[b, h, : len(src)], idx[b, h, torch.tensor(src, dtype=torch.long)]
            for i in range(2):
                want[i][at] = before[i].view(-1, hd)[of]
                if scales[i] is not None:
                    want_s[i][at] = scales[i].view(-1)[of]
            s = torch.tensor(src, dtype=torch.long)
            assert torch.equal(wo[b, h, : len(src)].view(torch.int32), weight[b, h][s].view(torch.int32))
            rest = weight[b, h, len(src):] if inplace else torch.full((S - len(src),), -5.0)
            assert torch.equal(wo[b, h, len(src):].view(torch.int32), rest.view(torch.int32))
            if pos is not None:
                assert torch.equal(po[b, h, : len(src)], pos[b, h][s])
                assert torch.equal(po[b, h, len(src):], pos[b, h, len(src):] if inplace else torch.full((S - len(src),), -5, dtype=torch.int32))
    for i in range(2):
        assert torch.equal(cache.rows[i].view(torch.int16).cpu().view(-1, hd), want[i])
        if scales[i] is not None:
            assert torch.equal(cache.scales[i].cpu().view(-1).view(torch.int32), want_s[i].view(torch.int32))


EVICT_CASES = [
    # B, Hkv, hd, S, lens, keep, recent
    (1, 1, 64, 16, [16], 1, 0),
    (1, 1, 64, 16, [16], 1, 1),
    (4, 2, 128, 80, [0, 1, 40, 80], 40, 10),         # nothing to do, nothing there, exactly full
    (3, 3, 64, 208, [200, 67, 208], 64, 64),         # recent rows only
    (2, 4, 128, 1104, [1100, 1025], 1000, 0),
    (2, 2, 128, 1040, [1040, 700], 16, 7),
    (1, 2, 64, 5008, [5001], 2500, 300),
]


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("form", [(False, 0), (False, 16), (True, 0), (True, 16)])
@pytest.mark.parametrize("case", EVICT_CASES)
def test_evict_rows(case, form, inplace):
    B, Hkv, hd, S, lens, keep, recent = case
    g = torch.Generator().manual_seed(S)
    weight = torch.randn((B, Hkv, S), generator=g).exp()
    pos = torch.argsort(torch.rand((B, Hkv, S), generator=g), -1).to(torch.int32) + 1000
    _check_evict(B, Hkv, hd, S, lens, keep, recent, weight, pos if inplace or form[1] else None, form[0], form[1], inplace)


@pytest.mark.parametrize("kind", ["equal", "few", "special", "negative", "nan"])
def test_evict_rows_ties_and_special_weights(kind):
    B, Hkv, hd, S, keep = 2, 2, 64, 400, 150
    g = torch.Generator().manual_seed(1)
    w = torch.randn((B, Hkv, S), generator=g)
    if kind == "equal":
        w = torch.zeros_like(w)
    if kind == "few":                                # ties everywhere, zeros of both signs among them
        w = torch.randint(-1, 3, w.shape, generator=g).float() * 0.5
        w[:, :, ::7] = -0.0
    if kind == "special":
        w[:, :, ::3], w[:, :, 1::9], w[:, :, 2::11], w[:, :, 5::13] = float("nan"), float("inf"), float("-inf"), 1e-45
    if kind == "negative":
        w = -w.abs() * 1e30
    if kind == "nan":
        w[:] = float("nan")
    for recent in (0, 30):
        _check_evict(B, Hkv, hd, S, [400, 333], keep, recent, w, None)
        pos = torch.argsort(torch.rand((B, Hkv, S), generator=g), -1).to(torch.int32)
        _check_evict(B, Hkv, hd, S, [400, 333], keep, recent, w, pos, inplace=True)


def test_evict_rows_positions_at_the_ends_of_their_type():
    B, Hkv, hd, S = 1, 1, 64, 48
    w = torch.rand((B, Hkv, S), generator=torch.Generator().manual_seed(2))
    pos = torch.arange(S, dtype=torch.int32).view(B, Hkv, S) - 2 ** 31          # the lowest positions of the type
    _check_evict(B, Hkv, hd, S, [48], 20, 20, w, pos)
    pos = (torch.arange(S, dtype=torch.int64) + 2 ** 31 - S).to(torch.int32).view(B, Hkv, S)
    _check_evict(B, Hkv, hd, S, [48], 20, 5, w, pos)
    _check_evict(B, Hkv, hd, S, [48], 20, 20, w, torch.zeros_like(pos))         # the same position everywhere: all count as recent


def test_evict_rows_of_long_slabs():
    g = torch.Generator().manual_seed(3)
    S = 70000
    w = torch.rand((1, 1, S), generator=g) ** 4
    pos = torch.randperm(S, generator=g).to(torch.int32).view(1, 1, S)
    _check_evict(1, 1, 64, S, [69999], 30000, 1000, w, pos)
    _check_evict(1, 1, 64, S, [69999], 40000, 0, w, None)


# --------------------------------------------------------------------------------------------------------- verification
def _verify(target, draft, drafts, u, temperature, span=None, logp=True, pad=0):
    ops = _ops()
    B, T = drafts.shape
    V = target.shape[-1]

    def put(x):
        if x is None:
            return None
        wide = torch.full((x.shape[0] * x.shape[1], V + pad), float("nan"), device=DEV)
        wide[:, :V] = x.reshape(-1, V).to(DEV)
        return wide[:, :V]

    acc, tok = torch.full((B,), -7, dtype=torch.int32, device=DEV), torch.full((B, T + 1), -7, dtype=torch.int32, device=DEV)
    lp = torch.full((B, T + 1), -7.0, device=DEV) if logp else None
    ws = torch.full((max(1, ops.verify_drafts_ws_bytes(B, T, V)),), 255, dtype=torch.uint8, device=DEV)
    ops.verify_drafts(put(target), drafts.to(torch.int32).to(DEV), None if u is None else u.to(DEV), acc, tok, ws, temperature, draft=put(draft),
                      d_span=None if span is None else _i32(span), logp=lp)
    torch.cuda.synchronize()
    return acc.cpu().tolist(), tok.cpu().tolist(), None if lp is None else lp.cpu().double()


def _check_verify(target, draft, drafts, u, temperature, span=None, pad=0):
    B, T = drafts.shape
    acc, tok, lp = _verify(target, draft, drafts, u, temperature, span, pad=pad)
    for b in range(B):
        n = T if span is None else min(max(span[b], 0), T)
        a, t, l = R.verify(target[b].double(), None if draft is None else draft[b].double(), drafts[b], None if u is None else u[b].double(), n, temperature)
        assert acc[b] == a and tok[b] == t, (b, acc[b], a, tok[b], t)
        want = torch.tensor(l, dtype=torch.float64)
        assert torch.equal(lp[b].isnan(), want.isnan())                  # greedy choice from a row whose largest value is not finite
        fine = ~want.isnan()
        assert ((lp[b] - want).abs() <= R.F32_STEP * want.abs() + 1e-9)[fine].all()
    return acc


def _drafting(B, T, V, seed, spread=2.5, apart=0.6, heat=1.0):
    g = torch.Generator().manual_seed(seed)
    d = torch.randn((B, T, V), generator=g) * spread
    t = torch.cat([d, torch.randn((B, 1, V), generator=g) * spread], 1) + torch.randn((B, T + 1, V), generator=g) * apart
    noise = -torch.log(-torch.log(torch.rand((B, T, V), generator=g).clamp(1e-9, 1 - 1e-7)))
    drafts = (d / heat + noise).argmax(-1)
    return t, d, drafts, torch.rand((B, T + 1), generator=g)


@pytest.mark.parametrize("V", [1, 2, 63, 1024, 1025, 4099, 32000])
@pytest.mark.parametrize("T", [1, 4])
@pytest.mark.parametrize("temperature", [0.0, 0.7, 1.0])
def test_verify_drafts(V, T, temperature):
    B = 6
    t, d, drafts, u = _drafting(B, T, V, V + T, heat=temperature or 0.05)
    _check_verify(t, d, drafts, u, temperature)
    _check_verify(t, None, drafts, u, temperature, span=[0, 1, T, T + 5, -2, T])
    _check_verify(t, d, drafts, u, temperature, span=[T, 0, 1, T, T, T], pad=3)


def test_verify_drafts_borders():
    """Draws at 0 and next to 1, certain tokens, tokens without probability, ids outside the vocabulary, the same distribution."""
    B, T, V = 8, 3, 300
    t, d, drafts, u = _drafting(B, T, V, 5)
    last = float(np.nextafter(np.float32(1), np.float32(0)))
    for value in (0.0, last):
        acc = _check_verify(t, d, drafts, torch.full_like(u, value), 1.0)
        _check_verify(t, None, drafts, torch.full_like(u, value), 1.0)
    same = torch.cat([d, d[:, :1]], 1)
    assert _check_verify(same, d, drafts, torch.full_like(u, last), 1.0) == [T] * B      # equal distributions accept everything
    out = drafts.clone()
    out[0, 0], out[1, 1], out[2, 2], out[3, 0] = -1, V, 2 ** 31 - 1, -2 ** 31
    _check_verify(t, d, out, u, 1.0)
    _check_verify(t, None, out, u, 1.0)
    _check_verify(t, None, out, None, 0.0)
    cut = torch.full_like(t, float("-inf"))                                              # one possible token a row
    cut[:, :, 17] = 1.0
    _check_verify(cut, d, drafts, u, 1.0)
    _check_verify(cut, None, torch.full_like(drafts, 17), u, 1.0)
    top = t.clone()
    top[:, :, V // 2:] = float("-inf")                                                   # half of the vocabulary is masked
    _check_verify(top, d, drafts, u, 0.9)
    big = t * 1e4                                                                        # peaks: everything else underflows
    _check_verify(big, d, drafts, u, 1.0)
    _check_verify(big, d * 1e4, drafts, u, 2.5)


@pytest.mark.parametrize("greedy", [False, True])
def test_verify_drafts_rows_that_cannot_be_used(greedy):
    B, T, V = 6, 3, 500
    t, d, drafts, u = _drafting(B, T, V, 6, apart=0.0)
    if greedy:
        drafts = t[:, :T].argmax(-1)
    u[:, :T] = 0.0
    t[0, 0, 3] = float("nan")
    t[1, 2, 499] = float("nan")
    t[2, 3, 0] = float("nan")
    t[3, 1] = float("-inf")
    t[4, 1, 8] = float("inf")
    d[5, 1, 77] = float("nan")
    _check_verify(t, d, drafts, u, 0.0 if greedy else 1.0)
    _check_verify(t, None, drafts, u, 0.0 if greedy else 1.0)


def test_verify_drafts_greedy_ties_go_to_the_lowest_index():
    B, T, V = 3, 2, 1000
    t = torch.zeros((B, T + 1, V))
    t[0, :, [5, 600]] = 2.0
    t[1, :, [0, 999]] = 2.0
    drafts = torch.tensor([[5, 5], [0, 999], [0, 1]])
    _check_verify(t, None, drafts, None, 0.0)


def test_verify_drafts_many_draws_follow_the_target():
    """The tokens that come out are distributed as the target's own: 20000 sequences, five tokens; chi-squared below the
    0.9999 quantile of 4 degrees of freedom (23.5)."""
    B, V = 20000, 5
    g = torch.Generator().manual_seed(12)
    t, d = torch.tensor([0.3, -1.0, 0.9, 0.0, -0.4]), torch.tensor([1.0, 0.2, -0.5, 0.0, 0.7])
    drafts = torch.multinomial(torch.softmax(d, 0), B, replacement=True, generator=g)[:, None]
    _, tok, _ = _verify(t.expand(B, 2, V).contiguous(), d.expand(B, 1, V).contiguous(), drafts, torch.rand((B, 2), generator=g), 1.0)
    count = torch.bincount(torch.tensor(tok)[:, 0], minlength=V).double()
    want = torch.softmax(t.double(), 0) * B
    assert float(((count - want) ** 2 / want).sum()) < 23.5


# ------------------------------------------------------------------------------------------------------------- together
class _Loop:
    """One layer of a program that decodes with drafted tokens over a bounded cache."""

    def __init__(self, block_scaled, page, B=3, T=4, Hq=8, Hkv=2, hd=64, S=96, V=50):
        g = torch.Generator().manual_seed(77)
        self.dims = B, T, Hq, Hkv, hd, S, V
        self.cache = R.Cache(_rnd(g, B, Hkv, S, hd), _rnd(g, B, Hkv, S, hd), block_scaled, page)
        ops = self.ops = _ops()
        z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device=DEV)                 # noqa: E731
        self.weight, self.row_pos = z(B, Hkv, S), z(B, Hkv, S, dt=torch.int32)
        self.len, self.pos = _i32([20, 25, 40]), _i32([20, 25, 40])
        self.row_pos[:] = torch.arange(S, device=DEV, dtype=torch.int32)
        self.qkv, self.q = z(B * T, (Hq + 2 * Hkv) * hd), z(B * T, Hq * hd)
        self.out = z(B * T, Hq * hd, dt=torch.float16)
        self.tab = _table(32, 4096, kind=1, factor=4.0)
        self.head = (_rnd(g, V, Hq * hd) * 0.5).float().to(DEV)
        self.drafts, self.u = z(B, T - 1, dt=torch.int32), z(B, T)
        self.accepted, self.tokens, self.logp = z(B, dt=torch.int32), z(B, T, dt=torch.int32), z(B, T)
        self.ws = z(max(1, ops.span_attention_ws_floats(B, T, Hq, Hkv, hd, S, 0, True)))
        self.ews = z(max(1, ops.evict_rows_ws_bytes(B, Hkv, S, 48)), dt=torch.uint8)
        self.vws = z(max(1, ops.verify_drafts_ws_bytes(B, T - 1, V)), dt=torch.uint8)

    def step(self):
        B, T, Hq, Hkv, hd, S, V = self.dims
        ops, c = self.ops, self.cache
        ops.rope_append_at(self.qkv, 1, 0, T, self.pos, self.len, self.tab, 0, 32, Hq, Hkv, hd, S, c.rows[0], c.rows[1], q_f32=self.q,
                           weight=self.weight, row_pos=self.row_pos, **c.args())
        ops.span_attention(self.q, c.rows[0], c.rows[1], self.len, self.out, self.ws, T, Hq, Hkv, hd, S, weight=self.weight, **c.args())
        self.logits = self.out.float() @ self.head.t()
        ops.verify_drafts(self.logits, self.drafts, self.u, self.accepted, self.tokens, self.vws, 0.9, logp=self.logp)
        self.len += self.accepted + 1
        self.pos += self.accepted + 1
        ops.evict_rows(c.rows[0], c.rows[1], self.weight, self.weight, self.len, self.len, self.ews, Hkv, hd, S, 48, 12, pos=self.row_pos,
                       pos_out=self.row_pos, **c.args())

    def feed(self, seed):
        g = torch.Generator().manual_seed(seed)
        B, T, Hq, Hkv, hd, S, V = self.dims
        self.qkv.copy_(_rnd(g, *self.qkv.shape).float())
        self.drafts.copy_(torch.randint(0, V, self.drafts.shape, generator=g, dtype=torch.int32))
        self.u.copy_(torch.rand(self.u.shape, generator=g) * 0.3)

    def state(self):
        return [x.clone() for x in (self.out, self.tokens, self.accepted, self.logp, self.weight, self.row_pos, self.len, self.pos, *self.cache.rows)]


@pytest.mark.parametrize("form", [(False, 0), (True, 16)])
def test_the_loop_they_make_together(form):
    """40 steps: the cache reaches its bound and is evicted from again and again.  Each step's results against the definitions on the
    state that the step found (so that a rounding decides no later choice)."""
    L = _Loop(*form)
    B, T, Hq, Hkv, hd, S, V = L.dims
    evicted = 0
    for step in range(40):
        L.feed(step)
        len0, pos0, w0, r0 = L.len.cpu(), L.pos.cpu(), L.weight.cpu().double(), L.row_pos.cpu()
        k0 = [L.cache.values(i) for i in range(2)]
        L.step()
        torch.cuda.synchronize()
        x = L.qkv.cpu().double().view(B, T, Hq + 2 * Hkv, hd)
        p = pos0[:, None] + torch.arange(T)
        y = R.rotate(x[:, :, : Hq + Hkv], p[:, :, None].expand(B, T, Hq + Hkv), R.frequencies(32, 10000.0, 1, 4.0), 32, 0)
        k, v = k0
        for b in range(B):
            at = int(len0[b]) + torch.arange(T)
            k[b][:, at], v[b][:, at] = y[b, :, Hq:].transpose(0, 1), x[b, :, Hq + Hkv:].transpose(0, 1)
            w0[b][:, at] = 0
            r0[b][:, at] = p[b].to(torch.int32)
        want, add, _ = R.attend(y[:, :, :Hq], k, v, len0.tolist(), T)
        out = L.out.cpu().double().view(want.shape)
        # cache rows carry a rounding of their own here: 2^-11 of k moves a score by |q||k| 2^-11 / sqrt(hd) at most
        ds = 2 * float(y[:, :, :Hq].norm(dim=-1).max() * k.norm(dim=-1).max()) / math.sqrt(hd) * R.HALF_STEP
        assert ((out - want).abs() <= (ds + 2 * R.HALF_STEP) * float(v.abs().max())).all()
        logits = L.logits.cpu().double().view(B, T, V)
        lens = []
        for b in range(B):
            a, t, l = R.verify(logits[b], None, L.drafts[b].tolist(), L.u[b].cpu().double(), T - 1, 0.9)
            assert L.accepted[b] == a and L.tokens[b].tolist() == t
            lens.append(int(len0[b]) + a + 1)
        assert L.pos.tolist() == [int(pos0[b]) + lens[b] - int(len0[b]) for b in range(B)]
        assert L.len.tolist() == [min(n, 48) for n in lens]
        w1, r1 = L.weight.cpu().double(), L.row_pos.cpu()
        for b in range(B):
            evicted += lens[b] > 48
            for h in range(Hkv):
                kept = set(r1[b, h, : int(L.len[b])].tolist())
                had = r0[b, h, : lens[b]].tolist()
                assert kept <= set(had) and len(kept) == int(L.len[b])
                assert set(sorted(had)[-12:]) <= kept                       # the recent rows stay
                by_pos = {q: j for j, q in enumerate(had)}
                full = w0[b, h] + add[b, h]
                for j, q in enumerate(r1[b, h, : int(L.len[b])].tolist()):   # weights follow their rows
                    assert abs(float(w1[b, h, j]) - float(full[by_pos[q]])) <= (ds + 1e-5) * float(full[by_pos[q]]) + 1e-6
                out_w = [float(full[by_pos[q]]) for q in had if q not in kept]
                in_w = [float(full[by_pos[q]]) for q in kept if q not in set(sorted(had)[-12:])]
                if out_w and in_w:
                    assert max(out_w) <= min(in_w) * (1 + 2 * ds + 1e-4) + 1e-5
    assert evicted > 20


def test_the_loop_captured_and_replayed():
    """The whole step as a graph: every replay equals the eager step bit for bit, with eager work and waits in between."""
    a, b = _Loop(False, 16), _Loop(False, 16)
    for L in (a, b):
        L.feed(0)
        L.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    keep = [x.clone() for x in (b.weight, b.row_pos, b.len, b.pos, *b.cache.rows)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.step()
    for x, y in zip((b.weight, b.row_pos, b.len, b.pos, *b.cache.rows), keep):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))             # capturing runs nothing
    for step in range(1, 9):
        for L in (a, b):
            L.feed(step)
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))
        torch.zeros(1 << 20, device=DEV).sum().item()


def test_two_streams_at_once():
    """Two loops on two streams with buffers of their own give what each gives alone."""
    alone, one, two = _Loop(True, 0), _Loop(True, 0), _Loop(True, 0)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for step in range(6):
        for L in (alone, one, two):
            L.feed(step)
        alone.step()
        torch.cuda.synchronize()
        for L, s in zip((one, two), streams):
            with torch.cuda.stream(s):
                L.step()
        torch.cuda.synchronize()
        for x, y, z in zip(alone.state(), one.state(), two.state()):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16)) and torch.equal(x.view(torch.int16), z.view(torch.int16))


# ------------------------------------------------------------------------------------------------------------- refusals
def test_operands_that_do_not_fit_are_refused():
    from paper_2406_14088_amd import RlGenError
    L = _Loop(False, 0)
    B, T, Hq, Hkv, hd, S, V = L.dims
    ops, c = L.ops, L.cache
    span = dict(q=L.q, kc=c.rows[0], vc=c.rows[1], d_len=L.len, out=L.out, ws=L.ws, T=T, Hq=Hq, Hkv=Hkv, hd=hd, S=S)
    ev = dict(kc=c.rows[0], vc=c.rows[1], weight=L.weight, weight_out=L.weight, d_len=L.len, d_len_out=None, ws=L.ews, Hkv=Hkv, hd=hd, S=S, keep=48, recent=4)
    ap = dict(qkv=L.qkv, nsplit=1, split_stride=0, T=T, d_pos=L.pos, d_slot=L.len, rope_tab=L.tab, rope_style=0, rot_dim=32, Hq=Hq, Hkv=Hkv, hd=hd, S=S,
              kc=c.rows[0], vc=c.rows[1])
    L.logits = torch.zeros((B * T, V), device=DEV)
    ve = dict(target=L.logits, drafts=L.drafts, u=L.u, accepted=L.accepted, tokens=L.tokens, ws=L.vws, temperature=1.0)
    bad = [
        (ops.span_attention, span, dict(q=L.q[:-1])), (ops.span_attention, span, dict(q=L.q.half())), (ops.span_attention, span, dict(S=S + 1)),
        (ops.span_attention, span, dict(d_len=L.len.long())), (ops.span_attention, span, dict(out=L.out.cpu())), (ops.span_attention, span, dict(T=0)),
        (ops.span_attention, span, dict(T=S + 1, q=torch.zeros(B * (S + 1) * Hq * hd, device=DEV), out=torch.zeros(B * (S + 1) * Hq * hd, device=DEV).half())),
        (ops.span_attention, span, dict(Hq=7)), (ops.span_attention, span, dict(hd=96)), (ops.span_attention, span, dict(nsplit=65)),
        (ops.span_attention, span, dict(kc=c.rows[0].transpose(1, 2))), (ops.span_attention, span, dict(kscale=torch.ones(B * Hkv * S, device=DEV))),
        (ops.span_attention, span, dict(weight=L.weight[:, :1])), (ops.span_attention, span, dict(table=L.len.view(B, 1), page_size=24)),
        (ops.span_attention, span, dict(table=L.len.view(B, 1), page_size=16)), (ops.span_attention, span, dict(weight=L.weight, ws=L.ws[:8])),
        (ops.evict_rows, ev, dict(keep=0)), (ops.evict_rows, ev, dict(keep=S + 1)), (ops.evict_rows, ev, dict(recent=49)), (ops.evict_rows, ev, dict(recent=-1)),
        (ops.evict_rows, ev, dict(pos=L.row_pos)), (ops.evict_rows, ev, dict(ws=L.ews[:1])), (ops.evict_rows, ev, dict(weight_out=L.weight.double())),
        (ops.rope_append_at, ap, dict(rot_dim=0)), (ops.rope_append_at, ap, dict(rot_dim=12)), (ops.rope_append_at, ap, dict(rot_dim=72)),
        (ops.rope_append_at, ap, dict(rope_style=2)), (ops.rope_append_at, ap, dict(nsplit=2, split_stride=L.qkv.numel())), (ops.rope_append_at, ap, dict(nsplit=0)),
        (ops.rope_append_at, ap, dict(q_f16_lo=L.out)), (ops.rope_append_at, ap, dict(d_slot=L.len[:1])), (ops.rope_append_at, ap, dict(split_stride=2)),
        (ops.verify_drafts, ve, dict(target=L.logits[:-1])), (ops.verify_drafts, ve, dict(target=L.logits.t().contiguous().t())), (ops.verify_drafts, ve, dict(u=None)),
        (ops.verify_drafts, ve, dict(temperature=float("nan"))), (ops.verify_drafts, ve, dict(draft=L.logits[:, :-1])), (ops.verify_drafts, ve, dict(tokens=L.tokens[:, :-1])),
        (ops.verify_drafts, ve, dict(temperature=float("inf"))), (ops.verify_drafts, ve, dict(ws=L.vws[:1])),
    ]
    for i, (fn, good, change) in enumerate(bad):
        with pytest.raises((RlGenError, AttributeError)):
            fn(**{**good, **change})
            print("not refused:", i, change.keys())
    torch.cuda.synchronize()


def test_empty_batches_enqueue_nothing():
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device=DEV)                     # noqa: E731
    none, half, f, raw = z(0, dt=torch.int32), z(0, dt=torch.float16), z(0), z(4096, dt=torch.uint8)
    ops = _ops()
    ops.rope_append_at(f, 1, 0, 3, none, none, z(4, 32, 2), 1, 64, 4, 2, 64, 32, half, half)
    ops.span_attention(f, half, half, none, half, None, 3, 4, 2, 64, 32)
    ops.evict_rows(half, half, f, f, none, none, raw, 2, 64, 32, 16, 4)
    ops.verify_drafts(z(0, 10), z(0, 3, dt=torch.int32), f, none, none, raw, 1.0)
    torch.cuda.synchronize()
