"""Refusals of the paged cache and draw calls, before any launch (no GPU)."""
import ctypes as C

import numpy as np
import pytest

from paper_2602_20217_amd import _lib as K

P = 4096  # a pointer that no refused call follows


def cache(**kw):
    d = dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=8, page=64, block=16, hkv=2, hd=128,
             kind=K.KS_E4M3)
    d.update(kw)
    return K.PagedCache(*[d[f] for f, _ in K.PagedCache._fields_])


def rows(**kw):
    d = dict(B=2, rows=6, row_start=P, pos0=P, table=P, table_ld=4, max_rows=3, max_len=100,
             err=None)
    d.update(kw)
    return K.PagedRows(*[d[f] for f, _ in K.PagedRows._fields_])


def append(c, r, q=P, ldq=8 * 128, k=P, ldk=256, v=P, ldv=256, qo=P, ldqo=8 * 128, hq=8,
           dtype=K.KS_BF16, rope=P, rope_rows=512):
    K.ks_paged_append(C.byref(c) if c else None, C.byref(r) if r else None, q, ldq, k, ldk, v, ldv,
                      qo, ldqo, hq, dtype, rope, rope_rows, None)


def attend(c, r, q=P, ldq=8 * 128, out=P, ldo=8 * 128, hq=8, dtype=K.KS_BF16, scale=0.1, lse=None,
           ws=P, ws_bytes=1 << 40):
    K.ks_paged_attention(C.byref(c) if c else None, C.byref(r) if r else None, q, ldq, out, ldo,
                         hq, dtype, scale, lse, ws, ws_bytes, None)


BAD_CACHE = [dict(kind=K.KS_F32), dict(kind=7), dict(hd=96), dict(hd=256), dict(hkv=0),
             dict(n_pages=0), dict(page=8), dict(page=48), dict(page=2048), dict(block=8),
             dict(block=48), dict(block=128), dict(k=None), dict(v=None), dict(k_scale=None),
             dict(v_scale=None), dict(k=P + 8), dict(v=P + 4)]
BAD_ROWS = [dict(B=-1), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(B=(1 << 20) + 1),
            dict(row_start=None), dict(pos0=None), dict(table=None), dict(table_ld=0),
            dict(max_rows=0), dict(max_len=0)]


@pytest.mark.parametrize("bad", BAD_CACHE + BAD_ROWS, ids=str)
def test_bad_caches_and_rows(bad):
    c, r = (cache(**bad), rows()) if bad in BAD_CACHE else (cache(), rows(**bad))
    for call in (append, attend):
        with pytest.raises(K.KsError) as e:
            call(c, r)
        assert e.value.status == K.KS_EINVAL and K.last_error()


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(k=None), dict(v=None), dict(qo=None),
                                dict(hq=0), dict(ldk=255), dict(ldv=0), dict(ldq=1023),
                                dict(ldqo=1000), dict(ldq=2048), dict(rope=P + 4),
                                dict(rope_rows=0)], ids=str)
def test_bad_append(kw):
    with pytest.raises(K.KsError) as e:
        append(cache(), rows(), **kw)
    assert e.value.status == K.KS_EINVAL


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(q=None), dict(out=None), dict(hq=0),
                                dict(hq=7), dict(hq=2 * 129), dict(ldq=1023), dict(ldo=0),
                                dict(q=P + 2), dict(out=P + 8), dict(ldq=1025), dict(ldo=1028),
                                dict(scale=float("nan")), dict(scale=float("inf"))], ids=str)
def test_bad_attention(kw):
    with pytest.raises(K.KsError) as e:
        attend(cache(), rows(), **kw)
    assert e.value.status == K.KS_EINVAL


def test_attention_workspace():
    c, r = cache(), rows(max_len=100000, table_ld=2000)
    n = K.ks_paged_attention_workspace_bytes(C.byref(c), 2, 6, 8, 3, 100000)
    assert n > 256
    for kw in (dict(ws=None), dict(ws_bytes=n - 1)):
        with pytest.raises(K.KsError) as e:
            attend(c, r, **kw)
        assert e.value.status == K.KS_ENOMEM
    with pytest.raises(K.KsError) as e:
        attend(c, r, ws=P + 8)
    assert e.value.status == K.KS_EINVAL
    for bad in ((2, 6, 7, 3, 100), (2, 6, 8, 0, 100), (2, 6, 8, 3, 0), (-1, 6, 8, 3, 100)):
        assert K.ks_paged_attention_workspace_bytes(C.byref(c), *bad) == 0
    assert K.ks_paged_attention_workspace_bytes(None, 2, 6, 8, 3, 100) == 0


def test_nothing_to_do():
    for r in (rows(B=0), rows(rows=0)):
        append(cache(), r)
        attend(cache(), r)
    p = K.DrawParams(None, None, None, None, None)
    K.ks_sample_draw(None, K.KS_F32, 0, 10, 10, C.byref(p), None, None, None, None, 0, None)


def test_null_structures():
    for call in (append, attend):
        for c, r in ((None, rows()), (cache(), None)):
            with pytest.raises(K.KsError) as e:
                call(c, r)
            assert e.value.status == K.KS_EINVAL
    with pytest.raises(K.KsError):
        K.ks_use_paged(None, None, None, 0)


def test_bad_draw():
    p = K.DrawParams(None, None, None, None, P)
    n = K.ks_sample_draw_workspace_bytes(4, 1000)
    assert n > 0

    def call(logits=P, dtype=K.KS_F32, rows=4, vocab=1000, ld=1000, p=p, tok=P, ws=P, nb=n):
        K.ks_sample_draw(logits, dtype, rows, vocab, ld, C.byref(p) if p else None, tok, None, None,
                         ws, nb, None)

    for kw in (dict(logits=None), dict(dtype=2), dict(rows=-1), dict(rows=65536), dict(vocab=0),
               dict(vocab=524289, ld=600000), dict(ld=999), dict(p=None), dict(tok=None),
               dict(ws=None), dict(ws=P + 4), dict(logits=P + 2),
               dict(p=K.DrawParams(None, None, None, None, None))):
        with pytest.raises(K.KsError) as e:
            call(**kw)
        assert e.value.status == K.KS_EINVAL, kw
    with pytest.raises(K.KsError) as e:
        call(nb=n - 1)
    assert e.value.status == K.KS_ENOMEM
    for bad in ((-1, 1000), (65536, 1000), (4, 0), (4, 524289)):
        assert K.ks_sample_draw_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("hkv,G", [(1, 1), (2, 4), (8, 4), (8, 1), (1, 128), (4, 16)])
def test_workspace_of_bounds_is_enough_below_them(hkv, G):
    """Fewer sequences, rows or positions than a workspace was asked for never need more,
    though they may be split more finely."""
    rng = np.random.RandomState(hkv * G)
    c = cache(hkv=hkv)
    f = lambda *a: K.ks_paged_attention_workspace_bytes(C.byref(c), a[0], a[1], hkv * G, *a[2:])
    for _ in range(500):
        top = [int(2 ** rng.uniform(0, e)) for e in (8, 12, 11, 18)]
        for _ in range(10):
            low = [rng.randint(1, t + 1) for t in top]
            assert f(*low) <= f(*top), (top, low)


def test_cache_kinds():
    from paper_2602_20217_amd.engine import DeviceModel
    with pytest.raises(ValueError, match="cache must be"):
        DeviceModel(None, 128, cache="fp8")
