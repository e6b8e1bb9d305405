"""Host side of the span operators: arguments that are refused before anything is launched, and workspace sizes.  No GPU."""
import ctypes as C

import pytest

E_NULL, E_SHAPE, E_CAPACITY = -1, -2, -3
P = 4096            # an aligned address that is never read


@pytest.fixture(scope="module")
def L():
    from paper_2406_14088_amd import binding
    return binding.lib()


def _append(L, **kw):
    a = dict(qkv=P, nsplit=1, stride=0, B=2, T=3, pos=P, slot=P, span=None, tab=P, tab_rows=10, style=1, rot=64, Hq=4, Hkv=2, hd=64, S=32, qf=None, qh=None,
             ql=None, kc=P, vc=P, ks=None, vs=None, table=None, ts=0, page=0, w=None, rp=None, st=None)
    assert set(kw) <= set(a)
    return L.rl_op_rope_append_at(*{**a, **kw}.values())


def _span(L, **kw):
    a = dict(q=P, kc=P, vc=P, ks=None, vs=None, table=None, ts=0, page=0, len=P, span=None, out=P, lo=None, w=None, ws=None, wsn=0, B=2, T=3, Hq=4, Hkv=2, hd=64,
             S=32, nsplit=1, st=None)
    assert set(kw) <= set(a)
    return L.rl_op_span_attention(*{**a, **kw}.values())


def _evict(L, **kw):
    a = dict(kc=P, vc=P, ks=None, vs=None, table=None, ts=0, page=0, w=P, wo=P, pos=None, po=None, len=P, lo=None, ws=P, wsn=1 << 20, B=2, Hkv=2, hd=64, S=32, keep=16,
             recent=4, st=None)
    assert set(kw) <= set(a)
    return L.rl_op_evict_rows(*{**a, **kw}.values())


def _verify(L, **kw):
    a = dict(t=P, ldt=100, d=None, ldd=0, drafts=P, u=P, span=None, B=2, T=3, V=100, temp=1.0, acc=P, tok=P, lp=None, ws=P, wsn=1 << 20, st=None)
    assert set(kw) <= set(a)
    return L.rl_op_verify_drafts(*{**a, **kw}.values())


@pytest.mark.parametrize("call, names", [(_append, ("qkv", "pos", "slot", "tab", "kc", "vc")), (_span, ("q", "kc", "vc", "len", "out")),
                                         (_evict, ("kc", "vc", "w", "wo", "len", "ws")), (_verify, ("t", "drafts", "u", "acc", "tok", "ws"))])
def test_missing_operands(L, call, names):
    for n in names:
        assert call(L, **{n: None}) == E_NULL, n


def test_operands_that_go_together(L):
    for call in (_append, _span, _evict):
        assert call(L, ks=P) == E_NULL and call(L, vs=P) == E_NULL
        assert call(L, table=P, ts=1, page=16) == E_SHAPE          # 16 of 32 rows
        for page in (0, 8, 24, 8192, -16):
            assert call(L, table=P, ts=100, page=page) == E_SHAPE
        assert call(L, hd=96) == E_SHAPE and call(L, Hkv=0) == E_SHAPE and call(L, S=0) == E_SHAPE and call(L, B=-1) == E_SHAPE
        assert call(L, kc=P + 2) == E_SHAPE and call(L, vc=P + 8) == E_SHAPE
    assert _append(L, ql=P) == E_NULL and _evict(L, pos=P) == E_NULL
    assert _span(L, w=P) == E_NULL                                 # weights need a workspace
    assert _span(L, w=P, ws=P, wsn=L.rl_op_span_attention_ws_floats(2, 3, 4, 2, 64, 32, 1, 1) - 1) == E_CAPACITY
    assert _span(L, ws=P, nsplit=2, wsn=L.rl_op_span_attention_ws_floats(2, 3, 4, 2, 64, 32, 2, 0) - 1) == E_CAPACITY
    assert _evict(L, wsn=L.rl_op_evict_rows_ws_bytes(2, 2, 32, 16) - 1) == E_CAPACITY
    assert _verify(L, wsn=L.rl_op_verify_drafts_ws_bytes(2, 3, 100) - 1) == E_CAPACITY


def test_sizes_and_options(L):
    for kw in (dict(rot=0), dict(rot=4), dict(rot=12), dict(rot=72), dict(style=2), dict(style=-1), dict(nsplit=0), dict(stride=2), dict(T=0), dict(Hq=0),
               dict(tab_rows=0), dict(B=1 << 20, T=1 << 12), dict(qkv=P + 4), dict(qf=P + 4), dict(qh=P + 2)):
        assert _append(L, **kw) == E_SHAPE, kw
    for kw in (dict(T=0), dict(T=33), dict(Hq=3), dict(Hq=130), dict(nsplit=-1), dict(nsplit=65), dict(q=P + 4), dict(out=P + 2), dict(ws=P + 4),
               dict(B=1 << 24, T=32)):
        assert _span(L, **kw) == E_SHAPE, kw
    for kw in (dict(keep=0), dict(keep=33), dict(recent=-1), dict(recent=17), dict(ws=P + 4)):
        assert _evict(L, **kw) == E_SHAPE, kw
    for kw in (dict(T=0), dict(T=257), dict(V=0), dict(ldt=99), dict(d=P, ldd=99), dict(temp=float("nan")), dict(temp=float("inf")), dict(temp=1e-40),
               dict(B=-1), dict(B=1 << 30), dict(ws=P + 4)):
        assert _verify(L, **kw) == E_SHAPE, kw
    assert _verify(L, B=1, T=1, V=(1 << 30) + 1, ldt=1 << 31, wsn=1 << 40) == E_SHAPE  # behind it a chunk's first index would pass 31 bits
    assert L.rl_op_verify_drafts_ws_bytes(1, 1, (1 << 30) + 1) == 0 < L.rl_op_verify_drafts_ws_bytes(1, 1, 1 << 30)
    assert _verify(L, temp=0.0, u=None, ws=None) == E_NULL


def test_rope_table_refusals(L):
    f = L.rl_op_build_rope_table_scaled
    assert f(None, 1, 64, 1e4, 0, 1.0, 0, 1.0, 32.0) == E_NULL
    for a in ((0, 64, 1e4, 0, 1.0, 0, 1.0, 32.0), (4, 63, 1e4, 0, 1.0, 0, 1.0, 32.0), (4, 64, 0.0, 0, 1.0, 0, 1.0, 32.0), (4, 64, 1e4, 4, 1.0, 0, 1.0, 32.0),
              (4, 64, 1e4, 1, 0.5, 0, 1.0, 32.0), (4, 2, 1e4, 2, 2.0, 0, 1.0, 32.0), (4, 64, 1e4, 3, 2.0, 0, 1.0, 32.0), (4, 64, 1e4, 3, 2.0, 512, 4.0, 4.0),
              (4, 64, float("nan"), 0, 1.0, 0, 1.0, 32.0), (4, 64, 1e4, 1, float("inf"), 0, 1.0, 32.0)):
        assert f(P, *a) == E_SHAPE, a


def test_workspace_sizes_of_what_is_refused_are_zero(L):
    assert L.rl_op_span_attention_ws_floats(2, 3, 3, 2, 64, 32, 1, 1) == 0
    assert L.rl_op_span_attention_ws_floats(2, 3, 4, 2, 64, 32, 1, 1) > 0
    assert L.rl_op_evict_rows_ws_bytes(2, 2, 32, 33) == 0 and L.rl_op_evict_rows_ws_bytes(2, 2, 32, 16) > 0
    assert L.rl_op_verify_drafts_ws_bytes(2, 0, 10) == 0 and L.rl_op_verify_drafts_ws_bytes(2, 3, 10) > 0
    assert L.rl_op_evict_rows_ws_bytes(1 << 10, 64, 1 << 20, 1 << 19) > 1 << 32      # sizes beyond 32 bits


def test_launches_of_2_to_the_32_threads_are_refused(L):
    """Where the first kernel of a call cannot be launched the next ones would read what it did not write."""
    assert _append(L, B=1 << 20, T=16) == E_SHAPE
    assert _evict(L, B=1 << 22, Hkv=2) == E_SHAPE and _evict(L, B=1 << 21, Hkv=2, S=8192, wsn=1 << 40) == E_SHAPE
    assert L.rl_op_evict_rows_ws_bytes(1 << 22, 2, 32, 16) == 0 < L.rl_op_evict_rows_ws_bytes((1 << 22) - 1, 2, 32, 16)
    assert _verify(L, B=9 << 20, T=1, V=10, wsn=1 << 50) == E_SHAPE and _verify(L, B=6 << 20, T=1, V=10, d=P, ldd=10, wsn=1 << 50) == E_SHAPE
    assert L.rl_op_verify_drafts_ws_bytes(9 << 20, 1, 10) == 0 < L.rl_op_verify_drafts_ws_bytes((8 << 20) - 1, 1, 10)
    assert _span(L, B=1 << 17, T=1, Hq=16, Hkv=16, S=64, nsplit=16, ws=P, wsn=1 << 50) == E_SHAPE
    assert _span(L, B=1 << 16, T=32, Hq=8, Hkv=8, S=1 << 16, w=P, ws=P, wsn=1 << 60) == E_SHAPE      # the second kernel's
    assert L.rl_op_span_attention_ws_floats(1 << 17, 1, 16, 16, 64, 64, 16, 1) == 0 < L.rl_op_span_attention_ws_floats(1 << 17, 1, 16, 16, 64, 64, 15, 1)


def test_a_workspace_for_the_largest_step_serves_smaller_ones(L):
    """A generation loop sizes its workspaces once, and its batch shrinks as sequences end."""
    for V in (10, 1024, 32000, 128256, 600000):
        for T in (1, 3, 5, 16, 40):
            sizes = [L.rl_op_verify_drafts_ws_bytes(B, T, V) for B in range(0, 70)]
            assert sizes == sorted(sizes), (V, T)
        sizes = [L.rl_op_verify_drafts_ws_bytes(12, T, V) for T in range(1, 257)]
        assert sizes == sorted(sizes), V
    for weights in (0, 1):
        for nsplit in (0, 1, 3):
            for Hq, Hkv, hd in ((32, 8, 128), (32, 32, 128), (64, 8, 64), (7, 1, 64), (600, 300, 64)):
                for S in (100, 600, 4096, 100000):
                    for T in (1, 2, 4, 8, 9, 33):
                        sizes = [L.rl_op_span_attention_ws_floats(B, T, Hq, Hkv, hd, S, nsplit, weights) for B in range(0, 70)]
                        assert sizes == sorted(sizes), (weights, nsplit, Hq, Hkv, hd, S, T)
                    sizes = [L.rl_op_span_attention_ws_floats(5, T, Hq, Hkv, hd, S, nsplit, weights) for T in range(1, 100)]
                    assert sizes == sorted(sizes), (weights, nsplit, Hq, Hkv, hd, S)
    sizes = [L.rl_op_evict_rows_ws_bytes(B, 8, 2112, 2048) for B in range(70)]
    assert sizes == sorted(sizes)


def test_partials_that_lie_nowhere_are_refused(L):
    """A negative distance of partials, as a size, would be read in front of the operand."""
    for stride in (2 ** 64 - 4, 2 ** 64 - 4096, 2 ** 63, 2 ** 61):
        assert _append(L, nsplit=2, stride=stride) == E_SHAPE
