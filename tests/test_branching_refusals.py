"""What the calls of branching sequences refuse, on the host: no kernel is launched, and the made-up device addresses are never followed."""
import ctypes

import pytest
import torch

from paper_2511_18871_amd import binding as B
from tests.test_rollout_refusals import BAD_CACHES, INVALID, P, UNSUPPORTED, WORKSPACE, cache, ints

FAR = [0x100000 * (i + 1) for i in range(8)]


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def tree(lib, c=None, q=P, o=P, lse=P, hq=4, ng=2, n=3, Gs=ints(1, 2), new=ints(3, 0, 40), anc=P, ms=2, pt=P, pw=2, pl=P, rt=P, rw=2, rl=P, scale=0.1, ws=P, bytes=1 << 28):
    return lib.sp_attn_tree_decode(cache() if c is None else c, q, o, lse, hq, ng, n, Gs, new, anc, ms, pt, pw, pl, rt, rw, rl, scale, ws, bytes, None)


def test_tree_refuses(lib):
    for kw, status in BAD_CACHES[1:]:
        assert tree(lib, c=cache(**kw)) == status, kw
    for kw in (dict(q=None), dict(o=None), dict(lse=None), dict(q=0x1004), dict(o=0x1008), dict(lse=0x1002), dict(hq=3), dict(hq=0), dict(ng=0), dict(n=0), dict(n=4),
               dict(Gs=ints(4, -1)), dict(Gs=None), dict(new=None), dict(new=ints(1, -1, 1)), dict(new=ints(1, 1025, 1)), dict(ms=1), dict(ms=-1), dict(anc=None), dict(anc=0x1002), dict(pt=None),
               dict(pl=None), dict(pw=0), dict(pw=-1), dict(rt=None), dict(rw=0), dict(rl=None), dict(rl=0x1001), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
               dict(scale=float("nan")), dict(scale=3e38), dict(rw=2 ** 31 - 1)):
        assert tree(lib, **kw) == INVALID, kw
    need = lib.sp_attn_tree_decode_workspace_bytes(2, 3, 43, 4, 2, 128, B.SP_BF16)
    assert 256 < need < 1 << 28
    for kw in (dict(ws=None), dict(ws=0x1008), dict(bytes=0), dict(bytes=need - 1)):
        assert tree(lib, **kw) == WORKSPACE, kw
    assert tree(lib, new=ints(0, 0, 0), anc=None, ms=0) == B.SP_OK       # no row, no launch
    for bad in ((0, 1, 1, 4, 2, 128, 0), (1, 0, 1, 4, 2, 128, 0), (1, 1, -1, 4, 2, 128, 0), (1, 1, 1 << 31, 4, 2, 128, 0), (1, 1, 1, 3, 2, 128, 0), (1, 1, 1, 4, 2, 96, 0), (1, 1, 1, 4, 2, 128, 9)):
        assert lib.sp_attn_tree_decode_workspace_bytes(*bad) == 0


def keep(lib, c=None, layers=1, stride=0, n=2, t=FAR[0], w=3, lens=FAR[1], kept=FAR[2], kw=5, nk=FAR[3], out=FAR[4]):
    return lib.sp_attn_cache_keep(cache() if c is None else c, layers, stride, n, t, w, lens, kept, kw, nk, out, None)


def test_keep_refuses(lib):
    for kw, status in BAD_CACHES[1:]:
        assert keep(lib, c=cache(**kw)) == status, kw
    for kw in (dict(layers=0), dict(layers=-1), dict(layers=2), dict(layers=2, stride=4 * 16 * 2 * 128 - 8), dict(layers=2, stride=4 * 16 * 2 * 128 + 4), dict(layers=2, stride=-(1 << 40)),
               dict(layers=50001, stride=1 << 20), dict(layers=3, stride=(1 << 62)), dict(n=0), dict(w=0), dict(kw=-1), dict(t=None), dict(lens=None), dict(kept=None), dict(nk=None), dict(out=None),
               dict(t=FAR[0] + 2), dict(out=FAR[4] + 1), dict(out=FAR[1]), dict(out=FAR[1] + 4), dict(out=FAR[3] - 4), dict(out=FAR[0] + 20), dict(out=FAR[2] + 36)):
        assert keep(lib, **kw) == INVALID, kw


def fit(lib, refs=FAR[0], pages=10, page=16, n=2, t=FAR[1], w=3, lens=FAR[2], miss=FAR[3], ws=FAR[4], bytes=1 << 20):
    return lib.sp_attn_pages_fit(refs, pages, page, n, t, w, lens, miss, ws, bytes, None)


def test_fit_refuses(lib):
    for kw in (dict(refs=None), dict(refs=FAR[0] + 1), dict(pages=0), dict(pages=1 << 31), dict(n=0), dict(w=0), dict(t=None), dict(lens=None), dict(lens=FAR[2] + 2), dict(miss=FAR[3] + 3),
               dict(t=FAR[0] + 36), dict(lens=FAR[0]), dict(lens=FAR[1] + 20), dict(miss=FAR[0] + 8), dict(miss=FAR[1] + 20), dict(miss=FAR[2] + 4)):
        assert fit(lib, **kw) == INVALID, kw
    for page in (8, 48, 512, 0, -16):
        assert fit(lib, page=page) == UNSUPPORTED
    need = lib.sp_attn_pages_workspace_bytes(10, 2)
    for kw in (dict(ws=None), dict(ws=FAR[4] + 8), dict(bytes=need - 1)):
        assert fit(lib, **kw) == WORKSPACE, kw
    assert [lib.sp_attn_pages_workspace_bytes(*x) for x in ((0, 1), (1, 0), (1 << 31, 1), (-1, 1))] == [0] * 4


def fork(lib, c=None, layers=1, stride=0, refs=FAR[0], n=2, parents=FAR[1], ns=3, st=FAR[2], sw=4, sl=FAR[3], t=FAR[4], w=5, out=FAR[5], flags=0, ws=FAR[6], bytes=1 << 20):
    return lib.sp_attn_cache_fork(cache() if c is None else c, layers, stride, refs, n, parents, ns, st, sw, sl, t, w, out, flags, ws, bytes, None)


def test_fork_refuses(lib):
    for kw, status in BAD_CACHES[1:]:
        assert fork(lib, c=cache(**kw)) == status, kw
    for kw in (dict(layers=0), dict(layers=2), dict(layers=40000, stride=1 << 20), dict(refs=None), dict(parents=None), dict(st=None), dict(sl=None), dict(t=None), dict(out=None), dict(n=0), dict(ns=0),
               dict(sw=0), dict(w=0), dict(refs=FAR[0] + 1), dict(out=FAR[5] + 2), dict(t=FAR[2] + 44), dict(out=FAR[3] + 8), dict(out=FAR[1]), dict(t=FAR[0] - 36), dict(out=FAR[4] + 36),
               dict(t=FAR[1]), dict(sl=FAR[0] + 12), dict(flags=8), dict(flags=32)):
        assert fork(lib, **kw) == INVALID, kw
    need = lib.sp_attn_pages_workspace_bytes(4, 2)
    for kw in (dict(ws=None), dict(ws=FAR[6] + 8), dict(bytes=need - 1)):
        assert fork(lib, **kw) == WORKSPACE, kw


def test_the_binding_refuses():
    k = torch.zeros(2, 4, 2, 16, 64)
    layers, one = B.KvLayers(k, k.clone()), B.KvCache(k[0], k[1])
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    calls = [
        lambda: B.KvLayers(k[0], k[0]), lambda: B.KvLayers(k, k[:1]), lambda: B.KvLayers(k.transpose(0, 1), k.transpose(0, 1)), lambda: B.KvLayers(k[:0], k[:0]),
        lambda: B.KvLayers(k.expand(2, 4, 2, 16, 64)[:1].expand(3, -1, -1, -1, -1), k[:1].expand(3, -1, -1, -1, -1)), lambda: B.KvLayers(k, k.bfloat16()),
        lambda: B.sp_attn_tree_decode(one, torch.zeros(3, 4, 32), None, [3], None, None, None, i32(1, 2), i32(1), 0.1),
        lambda: B.sp_attn_tree_decode(one, torch.zeros(3, 4, 64), None, [2], None, None, None, i32(1, 2), i32(1), 0.1),
        lambda: B.sp_attn_tree_decode(one, torch.zeros(3, 4, 64), None, [3], i32(2, 1), None, None, i32(1, 2), i32(1), 0.1),
        lambda: B.sp_attn_tree_decode(one, torch.zeros(3, 4, 64), None, [3], torch.zeros(3, 1), None, None, i32(1, 2), i32(1), 0.1),
        lambda: B.sp_attn_tree_decode(one, torch.zeros(3, 4, 64), None, [3], None, i32(1, 1), None, i32(1, 2), i32(1), 0.1),
        lambda: B.sp_attn_tree_decode(one, torch.zeros(3, 4, 64), None, [3], None, None, None, i32(1, 2), i32(2), 0.1),
        lambda: B.sp_attn_tree_decode(one, torch.zeros(3, 4, 64), None, [3], None, None, None, i32(1, 2), i32(1), 0.1),          # not on a GPU
        lambda: B.sp_attn_cache_keep(layers, i32(2, 3), i32(3), i32(3, 1), i32(3)), lambda: B.sp_attn_cache_keep(layers, i32(3, 3), i32(3), i32(3), i32(3)),
        lambda: B.sp_attn_cache_keep(layers, i32(3, 3), i32(3), i32(3, 1), i32(2)), lambda: B.sp_attn_cache_keep(layers, i32(3, 3), i32(3), i32(3, 1), i32(3).long()),
        lambda: B.sp_attn_pages_fit(i32(4, 2), 16, i32(3, 3), i32(3)), lambda: B.sp_attn_pages_fit(i32(4), 16, i32(2, 3), i32(3)),
        lambda: B.sp_attn_pages_fit(i32(4), 16, i32(3, 6)[:, ::2], i32(3)), lambda: B.sp_attn_pages_fit(i32(4), 16, i32(3, 3), i32(3), missing=i32(2)),
        lambda: B.sp_attn_cache_fork(layers, i32(5), i32(2), i32(3, 2), i32(3), i32(2, 2)), lambda: B.sp_attn_cache_fork(layers, i32(4), i32(2), i32(2, 2), i32(3), i32(2, 2)),
        lambda: B.sp_attn_cache_fork(layers, i32(4), i32(2), i32(3, 2), i32(3), i32(3, 2)),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(B.SpAttnError) as e:
            call()
        assert e.value.status == INVALID, i
    for call in (lambda: B.sp_attn_decode(layers, torch.zeros(1, 2, 64), None, None, None, i32(1, 1), i32(1), 0.1),
                 lambda: B.sp_attn_cache_append(layers, torch.zeros(1, 2, 64), torch.zeros(1, 2, 64), i32(1, 1), i32(1), 1e4)):
        with pytest.raises(AttributeError):                              # a call for one layer
            call()
    layers.k = torch.zeros(2, 5, 2, 16, 64)
    with pytest.raises(B.SpAttnError):
        layers._ref
