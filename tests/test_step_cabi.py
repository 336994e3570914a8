"""Refusals of the decode step's entry points, and the checks of their binding, without a GPU."""
import ctypes
import math

import pytest
import torch


@pytest.fixture(scope="module")
def vt():
    from paper_2603_05210_b200.build import build
    build()
    import paper_2603_05210_b200 as vt
    vt.lib()
    return vt


FAKE = 0x10000        # a non-NULL, 256-byte aligned address that is never dereferenced on the host
BIG = 1 << 40


def heads(vt, ptr=FAKE, token=4096, head=128):
    from paper_2603_05210_b200.binding import _VtHeads
    return _VtHeads(ptr, token, head)


def cache(vt, **kw):
    from paper_2603_05210_b200.binding import _VtCacheStruct
    a = dict(k=FAKE, v=FAKE, page_table=FAKE, lens=FAKE, k_page_stride=16384, k_token_stride=1024, k_head_stride=128, v_page_stride=16384,
             v_token_stride=1024, v_head_stride=128, table_stride=64, n_pages=100, page_size=16, heads=8, head_dim=128, B=4, max_pages=64)
    a.update(kw)
    return _VtCacheStruct(**a)


def ref(x):
    return None if x is None else ctypes.byref(x)


def test_table_refuses(vt):
    def call(**kw):
        a = dict(t=FAKE, rot=128, base=1e4, scaling=4, factor=8.0, low=1.0, high=32.0, orig=8192.0)
        a.update(kw)
        return vt.lib().vt_rope_table(a["t"], a["rot"], a["base"], a["scaling"], a["factor"], a["low"], a["high"], a["orig"], None)
    assert call(t=None) == vt.VT_ERR_NULL
    for bad in (dict(rot=0), dict(rot=24), dict(rot=1040), dict(rot=-16), dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(scaling=5),
                dict(scaling=-1), dict(factor=0.0), dict(factor=math.inf), dict(scaling=1, factor=-2.0), dict(low=0.0), dict(low=40.0), dict(high=math.nan),
                dict(orig=0.0), dict(scaling=3, low=4.0, high=4.0), dict(scaling=3, orig=math.inf)):
        assert call(**bad) == vt.VT_ERR_SHAPE, bad
    assert call(t=FAKE + 4) == vt.VT_ERR_ALIGN


def rope(vt, **kw):
    a = dict(q=heads(vt), k=heads(vt), pos=FAKE, table=FAKE, N=5, Hq=32, Hkv=8, D=128, rot=128, amp=1.0, options=0, qo=heads(vt), ko=heads(vt))
    a.update(kw)
    return vt.lib().vt_rope(ref(a["q"]), ref(a["k"]), a["pos"], a["table"], a["N"], a["Hq"], a["Hkv"], a["D"], a["rot"], a["amp"], a["options"],
                            ref(a["qo"]), ref(a["ko"]), None)


def test_rope_refuses(vt):
    for bad in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(pos=None), dict(table=None), dict(q=heads(vt, None)), dict(ko=heads(vt, None))):
        assert rope(vt, **bad) == vt.VT_ERR_NULL, bad
    for bad in (dict(N=-1), dict(Hq=0), dict(Hkv=-1), dict(D=120), dict(D=0), dict(D=2048), dict(rot=144), dict(rot=8), dict(rot=0), dict(amp=math.nan),
                dict(amp=math.inf), dict(options=4), dict(q=heads(vt, token=4100)), dict(qo=heads(vt, head=4)), dict(k=heads(vt, token=0)),
                dict(ko=heads(vt, head=-128)), dict(Hq=1 << 20)):
        assert rope(vt, **bad) == vt.VT_ERR_SHAPE, bad
    for bad in (dict(q=heads(vt, FAKE + 8)), dict(k=heads(vt, FAKE + 2)), dict(qo=heads(vt, FAKE + 8)), dict(ko=heads(vt, FAKE + 8)), dict(pos=FAKE + 1),
                dict(table=FAKE + 4)):
        assert rope(vt, **bad) == vt.VT_ERR_ALIGN, bad
    assert rope(vt, N=0) == vt.VT_OK and rope(vt, N=0, Hkv=0, k=None, ko=None, pos=None, q=heads(vt, None)) == vt.VT_OK


BAD_CACHES = (dict(n_pages=0), dict(page_size=0), dict(page_size=4), dict(page_size=24), dict(page_size=96), dict(page_size=192), dict(page_size=-128), dict(heads=0),
              dict(B=0), dict(max_pages=0), dict(table_stride=-1), dict(k_page_stride=0), dict(k_token_stride=1028), dict(k_head_stride=-128),
              dict(v_page_stride=7), dict(v_token_stride=4), dict(v_head_stride=0))


def append(vt, **kw):
    a = dict(q=heads(vt), k=heads(vt), v=heads(vt), pos=FAKE, cu=FAKE, table=FAKE, N=5, Hq=32, rot=128, amp=1.0, options=0, qo=heads(vt), cache=cache(vt))
    a.update(kw)
    return vt.lib().vt_rope_append(ref(a["q"]), ref(a["k"]), ref(a["v"]), a["pos"], a["cu"], a["table"], a["N"], a["Hq"], a["rot"], a["amp"],
                                   a["options"], ref(a["qo"]), ref(a["cache"]), None)


def test_append_refuses(vt):
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(qo=None), dict(cu=None), dict(pos=None), dict(table=None), dict(cache=None),
                dict(v=heads(vt, None)), *(dict(cache=cache(vt, **{n: None})) for n in ("k", "v", "page_table", "lens"))):
        assert append(vt, **bad) == vt.VT_ERR_NULL, bad
    for bad in (dict(N=-1), dict(Hq=0), dict(rot=144), dict(amp=math.nan), dict(options=2), dict(v=heads(vt, token=12)),
                *(dict(cache=cache(vt, **c)) for c in BAD_CACHES), dict(cache=cache(vt, head_dim=120)), dict(cache=cache(vt, head_dim=64))):
        assert append(vt, **bad) == vt.VT_ERR_SHAPE, bad
    for bad in (dict(v=heads(vt, FAKE + 8)), dict(cu=FAKE + 2), dict(cache=cache(vt, k=FAKE + 8)), dict(cache=cache(vt, v=FAKE + 2)),
                dict(cache=cache(vt, lens=FAKE + 1)), dict(cache=cache(vt, page_table=FAKE + 2))):
        assert append(vt, **bad) == vt.VT_ERR_ALIGN, bad
    assert append(vt, N=0) == vt.VT_OK


def attend(vt, **kw):
    a = dict(q=heads(vt), cu=FAKE, cache=cache(vt), mask=FAKE, words=2, N=5, Hq=32, most=60, scale=0.1, out=heads(vt), lse=FAKE, ws=FAKE, n=BIG)
    a.update(kw)
    return vt.lib().vt_tree_attention(ref(a["q"]), a["cu"], ref(a["cache"]), a["mask"], a["words"], a["N"], a["Hq"], a["most"], a["scale"],
                                      ref(a["out"]), a["lse"], a["ws"], a["n"], None)


def test_attention_refuses(vt):
    for bad in (dict(q=None), dict(cu=None), dict(out=None), dict(cache=None), dict(q=heads(vt, None)), dict(out=heads(vt, None)),
                dict(cache=cache(vt, lens=None))):
        assert attend(vt, **bad) == vt.VT_ERR_NULL, bad
    for bad in (dict(words=0), dict(words=-1), dict(N=-1), dict(Hq=0), dict(Hq=33), dict(Hq=8 * 136), dict(most=0), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=math.nan), dict(scale=math.inf), dict(q=heads(vt, token=4)), dict(out=heads(vt, head=0)),
                *(dict(cache=cache(vt, **c)) for c in BAD_CACHES), dict(cache=cache(vt, head_dim=96)), dict(cache=cache(vt, head_dim=256))):
        assert attend(vt, **bad) == vt.VT_ERR_SHAPE, bad
    for bad in (dict(q=heads(vt, FAKE + 8)), dict(out=heads(vt, FAKE + 8)), dict(cu=FAKE + 1), dict(mask=FAKE + 2), dict(lse=FAKE + 2),
                dict(cache=cache(vt, k=FAKE + 8))):
        assert attend(vt, **bad) == vt.VT_ERR_ALIGN, bad
    need = vt.vt_tree_attention_workspace_bytes(32, 8, 128, 60)
    for bad in (dict(ws=None), dict(ws=FAKE + 16), dict(n=need - 1)):
        assert attend(vt, **bad) == vt.VT_ERR_WORKSPACE, bad
    assert attend(vt, N=0) == vt.VT_OK


def test_workspace_sizes(vt):
    size = vt.vt_tree_attention_workspace_bytes
    for bad in ((0, 1, 64, 1), (3, 2, 64, 1), (1, 0, 64, 1), (1, 1, 96, 1), (129, 1, 64, 1), (1, 1, 64, 0)):
        assert size(*bad) == 0, bad
    assert size(32, 8, 128, 1) < size(32, 8, 128, 60) < size(32, 8, 128, 64) == size(32, 8, 128, 10 ** 6)
    assert size(32, 8, 128, 1) % 256 == 0 and size(32, 8, 128, 1) < 2 << 20


def test_mask_refuses(vt):
    def call(parents=FAKE, cu=FAKE, lens=FAKE, N=5, B=2, mask=FAKE, words=1, positions=FAKE):
        return vt.lib().vt_tree_mask(parents, cu, lens, N, B, mask, words, positions, None)
    for bad in (dict(parents=None), dict(cu=None), dict(mask=None, positions=None)):
        assert call(**bad) == vt.VT_ERR_NULL, bad
    for bad in (dict(N=-1), dict(B=0), dict(words=0)):
        assert call(**bad) == vt.VT_ERR_SHAPE, bad
    for bad in (dict(parents=FAKE + 1), dict(mask=FAKE + 2), dict(lens=FAKE + 2)):
        assert call(**bad) == vt.VT_ERR_ALIGN, bad
    assert call(N=0) == vt.VT_OK


def verify(vt, **kw):
    a = dict(P=FAKE, ld=32000, tokens=FAKE, parents=FAKE, cu=FAKE, ua=FAKE, us=FAKE, Q=FAKE, ldq=4000, ids=FAKE, d2t=FAKE, N=9, B=2, V=32000, Vd=4000,
             most=8, n=FAKE, path=FAKE, out=FAKE)
    a.update(kw)
    return vt.lib().vt_verify_tokens(a["P"], a["ld"], a["tokens"], a["parents"], a["cu"], a["ua"], a["us"], a["Q"], a["ldq"], a["ids"], a["d2t"], a["N"],
                                     a["B"], a["V"], a["Vd"], a["most"], a["n"], a["path"], a["out"], None)


def test_verify_refuses(vt):
    for name in ("P", "tokens", "parents", "cu", "ua", "us", "ids", "n", "path", "out"):
        assert verify(vt, **{name: None}) == vt.VT_ERR_NULL, name
    for bad in (dict(N=-1), dict(B=0), dict(V=0), dict(most=0), dict(most=1025), dict(ld=31999), dict(Vd=0), dict(ldq=3999), dict(V=393217, ld=1 << 20),
                dict(V=4194305, ld=1 << 23, Q=None)):
        assert verify(vt, **bad) == vt.VT_ERR_SHAPE, bad
    for name in ("P", "tokens", "parents", "cu", "ua", "us", "Q", "ids", "d2t", "n", "path", "out"):
        assert verify(vt, **{name: FAKE + 2}) == vt.VT_ERR_ALIGN, name


def test_binding_refuses_host_tensors_and_wrong_types(vt, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    rope = vt.VtRope(torch.zeros(32, dtype=torch.int64), 64, False, 1.0)
    with pytest.raises(ValueError):
        vt.vt_rope(x, None, i, rope)
    with pytest.raises(TypeError):
        vt.vt_rope(x.float(), None, i, rope)
    with pytest.raises(ValueError):
        vt.vt_rope_table(64, scaling="longer")
    with pytest.raises(ValueError):
        vt.VtCache(torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16), i[None], i[:1])
    with pytest.raises(TypeError):
        vt.VtCache(torch.zeros(3, 16, 2, 64), torch.zeros(3, 16, 2, 64), i[None], i[:1])
    with pytest.raises(ValueError):
        vt.vt_tree_mask(i, i, 4)
    with pytest.raises(ValueError):
        vt.vt_verify_tokens(torch.zeros(4, 9), i, i, i, torch.zeros(4), torch.zeros(1), max_tokens=3)


def test_docstrings_say_where_time_outs_and_bad_pages_are_seen(vt):
    assert "vt_last_status" in vt.vt_tree_attention.__doc__
