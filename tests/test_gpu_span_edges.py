"""Edges of the operators for steps of several tokens that their own tests leave out: numbers that are none, the long paths of draft
verification, workspaces of larger batches, operands that do not fit."""
import pytest
import torch

from tests.gpu_util import DEV
from tests import ref_span as R
from tests.test_gpu_span_ops import _check_verify, _drafting, _i32, _ops, _rnd, _table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd,rot,style", [(64, 64, 1), (128, 64, 0), (128, 128, 1)])
@pytest.mark.parametrize("block_scaled", [False, True])
def test_append_keeps_not_a_number(block_scaled, hd, rot, style):
    """A NaN in a query, key or value reaches the elements it turns with (block-scaled: its row) and nothing else differs in a bit."""
    B, T, Hq, Hkv, S = 2, 3, 4, 2, 32
    g = torch.Generator().manual_seed(hd + rot)
    heads = Hq + 2 * Hkv
    clean = _rnd(g, B * T, heads, hd).float()
    bad = clean.clone()
    hit = torch.zeros((B * T, heads, hd), dtype=torch.bool)
    for m, head, e in ((1, 2, 5), (2, Hq + 1, 7), (4, Hq + Hkv, hd - 1), (5, Hq, hd - 2)):
        bad[m, head, e] = float("nan")
        hit[m, head, e] = True
        if head < Hq + Hkv and e < rot:                                  # the other element of the pair
            hit[m, head, e ^ 1 if style == 0 else (e + rot // 2) % rot] = True
    got = []
    for x in (clean, bad):
        cache = R.Cache(torch.zeros(B, Hkv, S, hd), torch.zeros(B, Hkv, S, hd), block_scaled)
        qf, qh, ql = torch.zeros((B * T, Hq * hd), device=DEV), *(torch.zeros((B * T, Hq * hd), dtype=torch.float16, device=DEV) for _ in range(2))
        _ops().rope_append_at(x.view(B * T, -1).to(DEV), 1, 0, T, _i32([3, 40]), _i32([2, 20]), _table(rot, 64), style, rot, Hq, Hkv, hd, S, cache.rows[0],
                              cache.rows[1], q_f32=qf, q_f16=qh, q_f16_lo=ql, **cache.args())
        got.append(([t.cpu().view(B * T, Hq, hd) for t in (qf, qh, ql)], cache))
    for a, b in zip(got[0][0], got[1][0]):
        assert b[hit[:, :Hq]].isnan().all() and torch.equal(a[~hit[:, :Hq]], b[~hit[:, :Hq]])
    for i, h0 in ((0, Hq), (1, Hq + Hkv)):
        a, b = (c.values(i) for _, c in got)
        where = torch.zeros(a.shape, dtype=torch.bool)
        for m in range(B * T):
            where[m // T, :, [2, 20][m // T] + m % T] = hit[m, h0:h0 + Hkv]
        if block_scaled:
            where = where.any(-1, keepdim=True).expand_as(where)
        assert b[where].isnan().all() and torch.equal(a[~where], b[~where])


def test_workspaces_of_a_large_batch_serve_every_smaller_one():
    ops = _ops()
    V, B, T = 32000, 40, 6
    g = torch.Generator().manual_seed(1)
    logits = torch.randn((B * (T + 1), V), generator=g).to(DEV)
    drafts, u = torch.randint(0, V, (B, T), generator=g, dtype=torch.int32).to(DEV), torch.rand((B, T + 1), generator=g).to(DEV)
    ws = torch.empty(ops.verify_drafts_ws_bytes(B, T, V), dtype=torch.uint8, device=DEV)
    for b in (40, 33, 17, 11, 10, 9, 5, 1):
        for t in (6, 5, 2, 1):
            outs = []
            for w in (ws, torch.empty(ops.verify_drafts_ws_bytes(b, t, V), dtype=torch.uint8, device=DEV)):
                acc, tok = torch.zeros(b, dtype=torch.int32, device=DEV), torch.zeros((b, t + 1), dtype=torch.int32, device=DEV)
                ops.verify_drafts(logits[: b * (t + 1)], drafts[:b, :t].contiguous(), u[:b, : t + 1].contiguous(), acc, tok, w, 1.0, draft=logits[:b * t] * 0.9)
                outs.append((acc, tok))
            assert all(torch.equal(x, y) for x, y in zip(*outs))
    B, T, Hq, Hkv, hd, S = 48, 12, 16, 4, 64, 2048
    k, v = torch.randn((2, B, Hkv, S, hd), generator=g).to(torch.float16).to(DEV)
    q = torch.randn((B * T, Hq * hd), generator=g).to(DEV)
    for weights in (False, True):
        ws = torch.empty(ops.span_attention_ws_floats(B, T, Hq, Hkv, hd, S, 0, weights), device=DEV)
        for b in (48, 33, 32, 16, 7, 2, 1):
            for t in (12, 8, 5, 4, 2, 1):
                lens = torch.randint(0, S - t, (b,), generator=g, dtype=torch.int32).to(DEV)
                outs = []
                for w in (ws, torch.empty(ops.span_attention_ws_floats(b, t, Hq, Hkv, hd, S, 0, weights), device=DEV)):
                    out, weight = torch.zeros((b * t, Hq * hd), dtype=torch.float16, device=DEV), torch.zeros((b, Hkv, S), device=DEV)
                    ops.span_attention(q[: b * t], k, v, lens, out, w, t, Hq, Hkv, hd, S, weight=weight if weights else None)
                    outs.append((out, weight))
                assert all(torch.equal(x, y) for x, y in zip(*outs))


def test_operands_that_are_missing_or_do_not_belong_together():
    """All refused on the host, with the library's error."""
    from paper_2406_14088_amd import RlGenError
    ops = _ops()
    B, T, Hq, Hkv, hd, S, V = 2, 3, 4, 2, 64, 32, 50
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device=DEV)                     # noqa: E731
    c = R.Cache(torch.zeros(B, Hkv, S, hd), torch.zeros(B, Hkv, S, hd), True, 16)
    pool = dict(kc=c.rows[0], vc=c.rows[1], **c.args())
    flat = dict(kc=z(B, Hkv, S, hd, dt=torch.float16), vc=z(B, Hkv, S, hd, dt=torch.float16))
    i = z(B, dt=torch.int32)
    ap = dict(qkv=z(2, B * T, (Hq + 2 * Hkv) * hd), nsplit=2, split_stride=B * T * (Hq + 2 * Hkv) * hd, T=T, d_pos=i, d_slot=i, rope_tab=z(8, 32, 2), rope_style=0, rot_dim=64,
              Hq=Hq, Hkv=Hkv, hd=hd, S=S)
    sp = dict(q=z(B * T, Hq * hd), d_len=i, out=z(B * T, Hq * hd, dt=torch.float16), ws=z(1), T=T, Hq=Hq, Hkv=Hkv, hd=hd, S=S)
    ev = dict(weight=z(B, Hkv, S), weight_out=z(B, Hkv, S), d_len=i, d_len_out=None, ws=z(1 << 16, dt=torch.uint8), Hkv=Hkv, hd=hd, S=S, keep=16, recent=4)
    ve = dict(target=z(B * (T + 1), V), drafts=z(B, T, dt=torch.int32), u=z(B, T + 1), accepted=i, tokens=z(B, T + 1, dt=torch.int32), ws=z(1 << 16, dt=torch.uint8), temperature=1.0)
    wrap = 1 << 32
    bad = [(ops.rope_append_at, {**ap, **flat}, [dict(qkv=None), dict(d_pos=None), dict(d_slot=None), dict(rope_tab=None), dict(kc=None), dict(vc=None), dict(split_stride=-4),
                                                 dict(split_stride=4 - (1 << 64)), dict(T=T - wrap), dict(T=T + wrap), dict(S=S - wrap), dict(Hq=Hq - wrap)]),
           (ops.span_attention, {**sp, **flat}, [dict(q=None), dict(d_len=None), dict(out=None), dict(kc=None), dict(vc=None), dict(T=T - wrap), dict(S=S - wrap), dict(weight=z(B, Hkv, S)),
                                                 dict(ws=None, weight=z(B, Hkv, S)), dict(hd=hd - wrap)]),
           (ops.evict_rows, {**ev, **flat}, [dict(weight=None), dict(weight_out=None), dict(d_len=None), dict(ws=None), dict(kc=None), dict(keep=wrap + 16), dict(recent=wrap),
                                             dict(recent=4 - wrap)]),
           (ops.verify_drafts, ve, [dict(target=None), dict(drafts=None), dict(u=None), dict(accepted=None), dict(tokens=None), dict(ws=None), dict(drafts=i), dict(target=z(V))])]
    short = [dict(vc=c.rows[1][:-1]), dict(kscale=c.scales[0][:-1]), dict(vscale=c.scales[1][:-1]), dict(kc=None), dict(S=S - wrap), dict(S=S + wrap), dict(table=c.d_table[:1]),
             dict(table=c.d_table[:, :1].contiguous())]
    bad += [(fn, {**a, **pool}, short) for fn, a in ((ops.rope_append_at, ap), (ops.span_attention, sp), (ops.evict_rows, ev))]
    for fn, good, changes in bad:
        for change in changes:
            with pytest.raises(RlGenError):
                fn(**{**good, **change})
                print("not refused:", fn.__name__, change)
    torch.cuda.synchronize()


# ---------------------------------------------------------------------------------------------- draft verification, long paths
def _drawn(u, where):
    """u whose last entry puts the draw near the start, the middle or the end of what is left to draw from."""
    u = u.clone()
    u[:, -1] = {"first": 1e-4, "middle": 0.5, "last": 1 - 2.0 ** -24}[where]
    return u


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("form", ["sampled", "onehot", "greedy"])
@pytest.mark.parametrize("B,T,V", [(14, 4, 32000), (1, 1, 128256), (2, 3, 131073), (1, 5, 300001), (33, 1, 32003), (3, 200, 67), (2, 256, 300), (520, 1, 4000)])
def test_verify_drafts_long_paths(B, T, V, form, where):
    """Chunks of 2048 logits (14 x 5 rows of 32000, 131073, 300001 and 520 x 2 of 4000), more than 64 chunks to join (128256: 251 of 512; 131073
    and 300001: 65 and 147 of 2048), more drafted tokens than the wavefronts that put them out (200, 256)."""
    t, d, drafts, u = _drafting(B, T, V, V + T, spread=1.0 if V < 1000 else 2.5, apart=0.1 if T > 100 else 0.6, heat=0.02 if form == "greedy" else 0.8)
    u = _drawn(u, where)
    if T > 100:          # most drafts are accepted, a sequence ends late or at its end
        u[:, :-1] *= 0.5
        if form != "sampled":
            drafts = t[:, :T].argmax(-1)
            drafts[0, T - 7] = (drafts[0, T - 7] + 1) % V
            u[:, :-1] *= 1e-3
    elif B > 1:          # rejected at once, later, not at all
        u[0, 0], u[-1, :T] = 1 - 2.0 ** -24, 0.0
    acc = _check_verify(t, None if form == "onehot" else d, drafts, u, 0.0 if form == "greedy" else 0.8, span=None if where == "middle" else [T - i % 2 * (T > 1) for i in range(B)])
    if T > 100:
        assert max(acc) > 192


def test_append_of_rows_below_the_normal_numbers():
    """A block-scaled row whose largest magnitude has no reciprocal within fp32: zeros stay zeros, the rest is off by at most that magnitude."""
    B, T, Hq, Hkv, hd, S = 1, 4, 2, 2, 64, 16
    cache = R.Cache(torch.ones(B, Hkv, S, hd), torch.ones(B, Hkv, S, hd), True)
    g = torch.Generator().manual_seed(3)
    x = _rnd(g, T, Hq + 2 * Hkv, hd).float()
    x[:, :, ::3] = 0
    x *= torch.tensor([1e-42, 1e-36, 3e-31, 1e-28])[:, None, None]
    _ops().rope_append_at(x.view(T, -1).to(DEV), 1, 0, T, _i32([0]), _i32([4]), _table(64, 8), 1, 64, Hq, Hkv, hd, S, cache.rows[0], cache.rows[1], **cache.args())
    v, want = cache.values(1)[0, :, 4:4 + T].transpose(0, 1), x[:, Hq + Hkv:].double()
    top = want.abs().amax(-1, keepdim=True)
    assert (v[want == 0] == 0).all()
    assert ((v - want).abs() <= torch.where(top > 2.0 ** -100, 0.51 * top / 32767, top)).all()
