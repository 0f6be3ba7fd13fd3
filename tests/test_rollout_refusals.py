"""What the rollout calls refuse, on the host: no kernel is launched, and the made-up device addresses are never followed."""
import ctypes

import pytest
import torch

from paper_2511_18871_amd import binding as B

P = 0x1000
INVALID, UNSUPPORTED, WORKSPACE = B.SP_ERR_INVALID_ARG, B.SP_ERR_UNSUPPORTED, B.SP_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def ints(*xs):
    return (ctypes.c_int32 * max(1, len(xs)))(*xs)


def cache(k=P, v=P, n_pages=4, page=16, hkv=2, d=128, dtype=B.SP_BF16):
    return ctypes.byref(B._KvCacheStruct(k, v, n_pages, page, hkv, d, dtype))


BAD_CACHES = [(None, INVALID), (dict(k=None), INVALID), (dict(v=0x1008), INVALID), (dict(n_pages=0), INVALID), (dict(n_pages=1 << 31), INVALID),
              (dict(hkv=0), INVALID), (dict(page=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED), (dict(page=512), UNSUPPORTED), (dict(page=-16), UNSUPPORTED),
              (dict(d=96), UNSUPPORTED), (dict(dtype=5), UNSUPPORTED)]


def append(lib, q=P, qs=512, q_out=P, hq=4, k=P, ks=256, k_out=None, v=P, vs=256, n=2, new=None, tables=P, width=3, lens=P, base=None, lens_out=0x2000,
           rope=1e4):
    return lib.sp_attn_cache_append(cache(), q, qs, q_out, hq, k, ks, k_out, v, vs, n, new, tables, width, lens, base, lens_out, rope, None)


def test_append_refuses(lib):
    for kw, status in BAD_CACHES:
        c = None if kw is None else cache(**kw)
        assert lib.sp_attn_cache_append(c, None, 0, None, 0, P, 256, None, P, 256, 1, None, P, 1, P, None, None, 1e4, None) == status, kw
    for kw in (dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(q=0x1008), dict(k_out=0x1002), dict(hq=0), dict(ks=255), dict(ks=128), dict(vs=250), dict(qs=511),
               dict(qs=516), dict(n=0), dict(n=-1), dict(width=0), dict(tables=None), dict(lens=None), dict(lens=0x1001), dict(base=0x1002), dict(lens_out=P), dict(rope=1.0),
               dict(rope=float("nan")), dict(rope=float("inf")), dict(new=ints(1, -1)), dict(new=ints(2 ** 31 - 1, 2 ** 31 - 1)), dict(k_out=P, ks=512), dict(q=0x4000, q_out=0x4000, qs=1024)):
        assert append(lib, **kw) == INVALID, kw
    assert lib.sp_attn_cache_append(cache(), None, 0, None, 4, P, 256, None, P, 256, 1, None, P, 1, P, None, None, 1e4, None) == INVALID      # heads without q
    assert b"n_q_heads" in lib.sp_attn_last_error()


def decode(lib, c=None, q=P, o=P, lse=P, hq=4, ng=2, n=3, Gs=ints(1, 2), pt=P, pw=2, pl=P, rt=P, rw=2, rl=P, scale=0.1, ws=P, bytes=1 << 24):
    return lib.sp_attn_decode(cache() if c is None else c, q, o, lse, hq, ng, n, Gs, pt, pw, pl, rt, rw, rl, scale, ws, bytes, None)


def test_decode_refuses(lib):
    for kw, status in BAD_CACHES[1:]:
        assert decode(lib, c=cache(**kw)) == status, kw
    for kw in (dict(q=None), dict(o=None), dict(lse=None), dict(q=0x1004), dict(o=0x1008), dict(lse=0x1002), dict(hq=3), dict(hq=0), dict(ng=0), dict(n=0), dict(n=4), dict(Gs=ints(4, -1)),
               dict(Gs=None), dict(pt=None), dict(pl=None), dict(pw=0), dict(pw=-1), dict(rt=None), dict(rw=0), dict(rl=None), dict(rl=0x1001), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("inf")), dict(scale=float("nan")), dict(rw=2 ** 31 - 1), dict(ng=2 ** 30, n=2 ** 30, Gs=None)):
        assert decode(lib, **kw) == INVALID, kw
    for kw in (dict(ws=None), dict(ws=0x1008), dict(bytes=0), dict(bytes=B.decode_workspace_bytes(2, 3, 4, 2, 128, B.SP_BF16) - 1)):
        assert decode(lib, **kw) == WORKSPACE, kw
    for bad in ((0, 1, 4, 2, 128, 0), (1, 0, 4, 2, 128, 0), (1, 1, 3, 2, 128, 0), (1, 1, 4, 2, 96, 0), (1, 1, 4, 2, 128, 9)):
        assert B.decode_workspace_bytes(*bad) == 0
    small, large = (B.decode_workspace_bytes(g, n, 40, 8, 128, B.SP_BF16) for g, n in ((1, 1), (64, 1024)))
    assert 256 < small <= large < 1 << 31


def rules(rep=1.0, pres=0.0, freq=0.0, temp=1.0, bias=None):
    return ctypes.byref(B._LogitRulesStruct(rep, pres, freq, temp, bias))


BAD_RULES = [dict(rep=0.0), dict(rep=-1.0), dict(rep=float("inf")), dict(rep=1e-45), dict(temp=0.0), dict(temp=float("nan")), dict(temp=1e-45), dict(pres=float("nan")), dict(freq=float("inf")), dict(bias=0x1002)]


def adjust(lib, z=P, zs=100, out=P, os=100, V=100, r=None, mask=None, ms=4, ng=2, n=3, Gs=ints(1, 2), pt=P, ps=5, pl=P, rt=P, rs=5, rl=P, dtype=B.SP_BF16):
    return lib.sp_attn_adjust_logits(z, zs, out, os, V, rules() if r is None else r, mask, ms, ng, n, Gs, pt, ps, pl, rt, rs, rl, dtype, None)


def test_adjust_refuses(lib):
    for kw in BAD_RULES:
        assert adjust(lib, r=rules(**kw)) == INVALID, kw
    for kw in (dict(z=None), dict(out=None), dict(z=0x1004), dict(out=0x1008), dict(V=0), dict(V=-1), dict(V=(1 << 30) + 1), dict(zs=99), dict(os=99, out=0x2000), dict(os=104), dict(mask=0x1001), dict(mask=P, ms=3),
               dict(ng=0), dict(n=0), dict(n=5), dict(Gs=None), dict(Gs=ints(-1, 4)), dict(pt=None), dict(pl=None), dict(rt=None), dict(rl=None), dict(ps=-1), dict(rs=-1), dict(pl=0x1002)):
        assert adjust(lib, **kw) == INVALID, kw
    assert adjust(lib, dtype=4) == UNSUPPORTED
    assert lib.sp_attn_adjust_logits(P, 100, P, 100, 100, None, None, 0, 1, 1, None, None, 0, None, None, 0, None, 0, None) == INVALID


def test_adjusted_logprob_refuses(lib):
    one, g, r = ints(4), ints(1), ints(3)
    assert lib.sp_attn_adjusted_logprob_workspace_bytes(7, 1, 1, 151936) > lib.sp_attn_loss_workspace_bytes(7, 1, 1)
    for bad in ((0, 1, 1, 9), (7, 0, 1, 9), (7, 1, 1, 0), (7, 1, 1, (1 << 30) + 1)):
        assert lib.sp_attn_adjusted_logprob_workspace_bytes(*bad) == 0
    def fwd(z=P, y=P, t=P, logp=P, lse=P, V=100, ru=None, mask=None, ms=4, ng=1, resp=r, dtype=B.SP_F32, flags=0, ws=P, bytes=1 << 20):
        return lib.sp_attn_adjusted_logprob_fwd(z, y, t, logp, lse, V, rules() if ru is None else ru, mask, ms, ng, one, g, resp, dtype, flags, ws, bytes, None)
    def bwd(z=P, y=P, t=P, lse=P, up=P, dz=P, V=100, ru=None, mask=None, ms=4, dtype=B.SP_F32, flags=0, ws=P, bytes=1 << 20):
        return lib.sp_attn_adjusted_logprob_bwd(z, y, t, lse, up, dz, V, rules() if ru is None else ru, mask, ms, 1, one, g, r, dtype, flags, ws, bytes, None)
    for kw in BAD_RULES:
        assert fwd(ru=rules(**kw)) == INVALID and bwd(ru=rules(**kw)) == INVALID
    for kw in (dict(z=None), dict(z=0x1004), dict(y=None), dict(y=0x1002), dict(t=None), dict(lse=None), dict(lse=0x1002), dict(V=0), dict(mask=P, ms=3), dict(flags=1), dict(flags=16)):
        assert fwd(**kw) == INVALID and bwd(**kw) == INVALID, kw
    for kw in (dict(logp=None), dict(ng=0), dict(resp=None), dict(resp=ints(-1))):
        assert fwd(**kw) == INVALID, kw
    for kw in (dict(up=None), dict(dz=None), dict(dz=0x1008)):
        assert bwd(**kw) == INVALID, kw
    assert fwd(dtype=3) == UNSUPPORTED and bwd(dtype=3) == UNSUPPORTED
    for kw in (dict(ws=None), dict(bytes=64), dict(ws=0x1008)):
        assert fwd(**kw) == WORKSPACE and bwd(**kw) == WORKSPACE


def refused(f, *args, **kw):
    with pytest.raises(B.SpAttnError) as e:
        f(*args, **kw)
    return e.value.status == INVALID


def test_binding_refuses_what_a_pointer_does_not_show():
    k = torch.zeros(4, 2, 16, 64)
    assert refused(B.KvCache, k, k.double()) and refused(B.KvCache, k, k[:3]) and refused(B.KvCache, k.transpose(1, 2), k.transpose(1, 2)) and refused(B.KvCache, k[0], k[0])
    with pytest.raises(TypeError):
        B.KvCache(k.half(), k.half())
    c = B.KvCache(k, k.clone())
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    x, q = torch.zeros(3, 2, 64), torch.zeros(3, 4, 64)
    good = dict(q=q, pos_base=i32(3))
    for a, kw in (((x[:2], x, i32(3, 2), i32(3)), {}), ((x, x[:2], i32(3, 2), i32(3)), {}), ((x.bfloat16(), x, i32(3, 2), i32(3)), {}), ((x, x, i32(3, 2).long(), i32(3)), {}),
                  ((x, x, i32(2, 2), i32(3)), {}), ((x, x, i32(3, 4)[:, ::2], i32(3)), {}), ((x, x, i32(3, 2), i32(3).float()), {}), ((x.transpose(0, 1).contiguous().transpose(0, 1), x, i32(3, 2), i32(3)), {}),
                  ((x, x, i32(3, 2), i32(3)), dict(new_lens=[1, 1])), ((x, x, i32(3, 2), i32(3)), dict(new_lens=[1, 1, 2])), ((x, x, i32(3, 2), i32(3)), dict(q=q[:2])),
                  ((x, x, i32(3, 2), i32(3)), dict(q=q, q_out=q.bfloat16())), ((x, x, i32(3, 2), i32(3)), dict(q_out=q)), ((x, x, i32(3, 2), i32(3)), dict(k_out=q)),
                  ((x, x, i32(3, 2), i32(3)), dict(lens_out=i32(2))), ((x, x, i32(3, 2), i32(3)), dict(pos_base=i32(2))), ((x, x, i32(3, 2), i32(3)), good)):      # the last: not on a GPU
        assert refused(B.sp_attn_cache_append, c, *a, 1e4, **kw), (a, kw)
    d = lambda **kw: refused(B.sp_attn_decode, c, kw.get("q", q), kw.get("Gs", [1, 2]), kw.get("pt", i32(2, 3)), kw.get("pl", i32(2)), kw.get("rt", i32(3, 3)), kw.get("rl", i32(3)), 0.1, **kw.get("more", {}))
    for kw in (dict(q=q.bfloat16()), dict(q=q[:, :, :32]), dict(q=q[:, ::2]), dict(Gs=[1, 2, 0]), dict(pt=i32(3, 3)), dict(pl=i32(3)), dict(rt=i32(2, 3)), dict(rl=i32(2)), dict(rl=i32(3).long()),
               dict(more=dict(o=q.bfloat16())), dict(more=dict(lse=torch.zeros(3, 4))), {}):
        assert d(**kw), kw
    z, rules_ = torch.zeros(3, 40), B.LogitRules(bias=torch.zeros(40))
    assert refused(B.LogitRules, bias=torch.zeros(40).double()) and refused(B.LogitRules, bias=torch.zeros(80)[::2])
    a = lambda **kw: refused(B.sp_attn_adjust_logits, kw.get("z", z), kw.get("r", rules_), kw.get("Gs", [1, 2]), kw.get("pt", i32(2, 5)), kw.get("pl", i32(2)), kw.get("rt", i32(3, 5)), kw.get("rl", i32(3)), mask=kw.get("mask"))
    for kw in (dict(z=z.t().contiguous().t()), dict(r=B.LogitRules(bias=torch.zeros(41))), dict(pt=i32(3, 5)), dict(pl=None), dict(rt=None), dict(rl=i32(2)), dict(mask=i32(2, 2)), dict(mask=i32(3, 2).float()), {}):
        assert a(**kw), kw
    t = i32(7)
    zz = torch.zeros(7, 40)
    f = lambda z_=zz, y=t, tok=t, pl=[4], rl=[3], **kw: refused(B.sp_attn_adjusted_logprob_fwd, z_, y, tok, rules_, pl, [1], rl, **kw)
    assert f(z_=zz[:6]) and f(rl=[4]) and f(y=t.long()) and f(tok=t[:6]) and f(mask=i32(6, 2)) and f(logp=torch.zeros(6)) and f()
    b = lambda lse=torch.zeros(7), g=torch.zeros(7), **kw: refused(B.sp_attn_adjusted_logprob_bwd, zz, t, t, lse, g, rules_, [4], [1], [3], **kw)
    assert b(lse=torch.zeros(6)) and b(g=torch.zeros(7).double()) and b(dlogits=zz.bfloat16()) and b(dlogits=zz[:6]) and b()
