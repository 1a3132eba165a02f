"""The serving operators without a GPU: refusals of the C entry points and of the
binding before any device work, sizes, and the oracle's own pins."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import pipeline, serve
from paper_2608_18147_amd import ecasq

FAKE = 0x100000  # aligned, never read: every call below is refused on the host


def _cache(**kw):
    c = ecasq._kv_struct(1, 0, 2, 128, 16, 3, 4, 9, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [dict(dt=0), dict(dt=3), dict(coded=2), dict(heads=0), dict(heads=1025),
              dict(head_dim=96), dict(head_dim=512), dict(page_size=8), dict(page_size=24),
              dict(page_size=1 << 17), dict(batch=0), dict(batch=65536), dict(max_pages=0),
              dict(n_pages=0), dict(max_pages=1 << 30)]
BAD_POINTERS = [dict(k=None), dict(v=None), dict(table=None), dict(lens=None), dict(k=FAKE + 8),
                dict(coded=1), dict(coded=1, k_books=FAKE, v_books=FAKE + 2)]


@pytest.mark.parametrize("args", [(0, 5, 32), (5, 0, 32), (5, 5, 0), (5, 5, 31), (5, 5, 48),
                                  (5, 5, -32), ((1 << 24) + 1, 5, 32), (5, (1 << 24) + 1, 32),
                                  (1 << 24, 1 << 17, 32), (5, 5, 1 << 25)])
def test_weights_sizes_refused(args):
    assert ecasq.lib().ecasq_weights_size(*args) == 0


@pytest.mark.parametrize("n_out,n_in,group", [(1, 1, 32), (16, 128, 32), (17, 129, 64),
                                              (1000, 4100, 96), (5, 7, 1 << 24)])
def test_weights_size(n_out, n_in, group):
    tiles = -(-n_out // 16)
    want = 256 + tiles * -(-n_in // 128) * 1024 + tiles * -(-n_in // group) * 32
    assert ecasq.lib().ecasq_weights_size(n_out, n_in, group) == want


def test_products_refused():
    L = ecasq.lib()
    size = L.ecasq_weights_size(20, 200, 64)

    def pack(sym=FAKE, cb=FAKE, t=16, sc=FAKE, dt=1, n_out=20, n_in=200, group=64, to=FAKE,
             nb=size):
        return L.ecasq_weights_pack(sym, cb, t, sc, dt, n_out, n_in, group, None, to, nb)

    for kw in (dict(sym=None), dict(cb=None), dict(t=0), dict(t=17), dict(sc=None),
               dict(sc=FAKE + 1), dict(dt=0), dict(dt=3), dict(n_out=0), dict(group=33),
               dict(to=None), dict(to=FAKE + 8), dict(nb=size - 1)):
        assert pack(**kw) == ecasq.ECASQ_EINVAL, kw

    def vec(w=FAKE, dt=2, n_out=20, n_in=200, group=64, x=FAKE, m=1, step=200, y=FAKE):
        return L.ecasq_matvec(w, dt, n_out, n_in, group, x, m, step, None, y)

    for kw in (dict(w=None), dict(w=FAKE + 4), dict(dt=0), dict(x=None), dict(x=FAKE + 1),
               dict(y=None), dict(y=FAKE + 1), dict(m=0), dict(m=-1), dict(m=(1 << 20) + 1),
               dict(step=199), dict(n_in=0), dict(group=16)):
        assert vec(**kw) == ecasq.ECASQ_EINVAL, kw


@pytest.mark.parametrize("kw", BAD_CACHES + BAD_POINTERS)
def test_caches_refused(kw):
    L, c = ecasq.lib(), _cache(**kw)
    r = ctypes.byref(c)
    big = 1 << 40
    assert L.ecasq_kv_write(r, FAKE, 256, FAKE, 256, 1, FAKE, None, None, FAKE, FAKE, FAKE, FAKE,
                            16, 0, None, None) == ecasq.ECASQ_EINVAL
    assert L.ecasq_kv_attention(r, FAKE, 1024, 2, 1.0, None, None, FAKE, FAKE,
                                big) == ecasq.ECASQ_EINVAL
    assert L.ecasq_kv_evict(r, 4, 1, FAKE, FAKE, FAKE, None, FAKE, big) == ecasq.ECASQ_EINVAL
    if kw in BAD_CACHES:
        assert L.ecasq_kv_attention_workspace(r, 2, 0) == 0
        assert L.ecasq_kv_evict_workspace(r, 4) == 0


def test_cache_calls_refused():
    L, c = ecasq.lib(), _cache()
    r = ctypes.byref(c)

    def write(k=FAKE, ks=256, v=FAKE, vs=256, rows=1, starts=FAKE, c=r, books=(None,) * 4, s=0,
              hats=(None, None)):
        return L.ecasq_kv_write(c, k, ks, v, vs, rows, starts, None, None, *books, s, 0, *hats)

    for kw in (dict(k=None), dict(k=FAKE + 1), dict(v=None), dict(ks=255), dict(vs=255),
               dict(rows=0), dict(rows=(1 << 30) + 1), dict(starts=None), dict(c=None),
               dict(hats=(FAKE, FAKE)), dict(hats=(FAKE, None))):
        assert write(**kw) == ecasq.ECASQ_EINVAL, kw
    coded = _cache(coded=1, k_books=FAKE, v_books=FAKE)
    for kw in (dict(), dict(books=(FAKE, FAKE, FAKE, None), s=16), dict(books=(FAKE,) * 4, s=1),
               dict(books=(FAKE,) * 4, s=33), dict(books=(FAKE,) * 4, s=16, hats=(FAKE, None))):
        assert write(c=ctypes.byref(coded), **kw) == ecasq.ECASQ_EINVAL, kw

    size = L.ecasq_kv_attention_workspace(r, 4, 1)
    assert size >= L.ecasq_kv_attention_workspace(r, 4, 0) > 0
    for heads in (0, 1, 3, 130):
        assert L.ecasq_kv_attention_workspace(r, heads, 0) == 0

    def attend(q=FAKE, step=512, heads=4, scale=0.1, out=FAKE, ws=FAKE, nb=size, c=r):
        return L.ecasq_kv_attention(c, q, step, heads, scale, FAKE, None, out, ws, nb)

    for kw in (dict(q=None), dict(q=FAKE + 1), dict(step=511), dict(heads=3), dict(heads=130),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=1e300),
               dict(out=None), dict(out=FAKE + 8), dict(ws=None), dict(ws=FAKE + 16),
               dict(c=None)):
        assert attend(**kw) == ecasq.ECASQ_EINVAL, kw
    assert attend(nb=size - 1) == ecasq.ECASQ_EWORKSPACE

    size = L.ecasq_kv_evict_workspace(r, 8)

    def evict(keep=8, recent=2, m=FAKE, p=FAKE, n=FAKE, ws=FAKE, nb=size, c=r):
        return L.ecasq_kv_evict(c, keep, recent, m, p, n, None, ws, nb)

    for kw in (dict(keep=0), dict(recent=-1), dict(recent=9), dict(m=None), dict(p=None),
               dict(n=None), dict(ws=None), dict(ws=FAKE + 16), dict(c=None)):
        assert evict(**kw) == ecasq.ECASQ_EINVAL, kw
    for kw in (dict(mass=None), dict(pos=None)):
        assert evict(c=ctypes.byref(_cache(**kw))) == ecasq.ECASQ_EINVAL, kw
    assert evict(nb=size - 1) == ecasq.ECASQ_EWORKSPACE


def test_binding_refuses_host_tensors():
    h = torch.zeros(4, 2, 16, 128, dtype=torch.float16)
    table, lens = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        ecasq.ecasq_kv_cache(h, h, table, lens)
    with pytest.raises(TypeError):
        ecasq.ecasq_weights_pack(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(16),
                                 torch.zeros(4, 2, dtype=torch.float16), 32)


def test_rounding_of_rows_is_the_roundings_rule():
    """One row's symbols by the oracle of ecasq_quantize, its counter word aside."""
    g = np.random.default_rng(0)
    x = g.standard_normal((1, 128)).astype(np.float16).astype(np.float64)
    q = np.sort(x[0])[np.linspace(0, 127, 9).astype(int)]
    got = serve.round_rows(x, q[None, :], [9], 2 ** 33 + 5, 0)[0]
    want, _, _ = pipeline.quantize(x[0].astype(np.float32), q, 2 ** 33 + 5)
    np.testing.assert_array_equal(got, want)


def test_eviction_by_hand():
    c = dict(k=np.zeros((1, 1, 16, 64)), table=np.zeros((1, 1), dtype=np.int32),
             lens=np.array([6]), mass=np.zeros((1, 1, 16)), pos=np.zeros((1, 1, 16), np.int32))
    c["mass"][0, 0, :6] = [5, 1, np.nan, 4, 1, 0]
    c["pos"][0, 0, :6] = [0, 1, 2, 3, 4, 5]
    # kept of 6: slot 5 (newest), 0, 3, then the first of the two of weight 1
    mass, pos, lens, moves = serve.evict(c, 4, 1)
    assert moves == [(0, 0, 5, 2)] and lens[0] == 4
    np.testing.assert_array_equal(mass[0, 0, :4], [5, 1, 0, 4])
    np.testing.assert_array_equal(pos[0, 0, :4], [0, 1, 5, 3])


def test_attention_of_equal_keys_is_the_mean():
    c = dict(k=np.ones((2, 1, 16, 64)), v=np.arange(2 * 16 * 64.0).reshape(2, 1, 16, 64),
             table=np.array([[1, 0]]), lens=np.array([20]))
    out, mass, _, _ = serve.attention(c, np.ones((1, 2, 64)), 0.3)
    want = np.concatenate((c["v"][1, 0], c["v"][0, 0, :4])).mean(0)
    np.testing.assert_allclose(out[0], [want, want], rtol=1e-14)
    np.testing.assert_allclose(mass[0, 0], [0.1] * 20 + [0.0] * 12, rtol=1e-14)


def test_sizes_of_one_launch():
    """What one launch cannot cover is refused."""
    L = ecasq.lib()
    r = ctypes.byref(_cache(batch=65535, heads=17))
    assert L.ecasq_kv_attention_workspace(r, 17, 0) == 0 == L.ecasq_kv_evict_workspace(r, 5)
    c = _cache(batch=65535, heads=8, max_pages=16, page_size=128)  # 2^30 slots of heads, less 2^14
    assert L.ecasq_kv_attention_workspace(ctypes.byref(c), 8, 1) > 0
    assert L.ecasq_kv_attention_workspace(ctypes.byref(c), 8 * 16, 0) > 0
    assert L.ecasq_kv_attention_workspace(ctypes.byref(c), 8 * 17, 0) == 0
    c.max_pages = 17
    r = ctypes.byref(c)
    assert L.ecasq_kv_attention_workspace(r, 8, 0) > 0
    assert L.ecasq_kv_attention_workspace(r, 8, 1) == 0 == L.ecasq_kv_evict_workspace(r, 5)
    big = 1 << 62
    assert L.ecasq_kv_attention(r, FAKE, 1024, 8, 1.0, FAKE, None, FAKE, FAKE,
                                big) == ecasq.ECASQ_EINVAL
    assert L.ecasq_kv_evict(r, 4, 1, FAKE, FAKE, FAKE, None, FAKE, big) == ecasq.ECASQ_EINVAL
    c = _cache()
    assert L.ecasq_kv_write(ctypes.byref(c), FAKE, 256, FAKE, 256, (1 << 23) + 1, FAKE, None, None,
                            None, None, None, None, 0, 0, None, None) == ecasq.ECASQ_EINVAL
