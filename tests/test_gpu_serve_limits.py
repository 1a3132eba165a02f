"""The serving operators at the ends of what the header allows: the most sequences, heads, slots of a
page and of a table; numbers below the types' normal range; every call on a stream that is
given.  Tolerances as in test_gpu_serve.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import serve
from paper_2608_18147_amd import ecasq
from tests.test_gpu_serve import (TYPES, _check_product, _need_gpu, _np, _weights, check_attention,
                                  make_cache, on_gpu)

pytestmark = pytest.mark.gpu


def _part(c, batch):
    """The sequences `batch` of a cache's arrays."""
    return {k: v[batch] if k in ("table", "lens", "mass", "pos") else v for k, v in c.items()}


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("batch,heads,group,page", [(65535, 2, 2, 16), (4, 1024, 1, 16), (1024, 1, 64, 32)])
def test_many_sequences_and_heads(batch, heads, group, page, coded):
    """A write of a token each, attention with weights and an eviction; some sequences by 64 bits."""
    _need_gpu()
    print("[case] many", batch, heads, group, coded, flush=True)
    dim, dtype, keep = 64, torch.bfloat16, 9
    g = torch.Generator().manual_seed(batch + heads)
    lens = torch.randint(0, page, (batch,), generator=g, dtype=torch.int32)
    some = torch.unique(torch.cat((torch.tensor([0, 1, batch - 1]),
                                   torch.randint(0, batch, (9,), generator=g))))
    c = dict(table=torch.randperm(batch, generator=g).to(torch.int32)[:, None].contiguous(), lens=lens,
             mass=torch.rand((batch, heads, page), generator=g),
             pos=torch.arange(page, dtype=torch.int32).repeat(batch, heads, 1))
    shape = (batch, heads, page)
    for name in ("k", "v"):
        if coded:
            c[name] = torch.randint(0, 256, shape + (dim // 2,), generator=g, dtype=torch.uint8)
            c[name + "_books"] = torch.randn(shape + (16,), generator=g, dtype=torch.float32).to(dtype)
        else:
            c[name] = torch.randn(shape + (dim,), generator=g, dtype=torch.float32).to(dtype)
    kv = on_gpu(c)
    kv.lens += 1
    rows = torch.randn((batch, heads, dim), generator=g).to(dtype).cuda()
    starts = torch.arange(batch + 1, dtype=torch.int32, device="cuda")
    kw = {}
    if coded:
        books = torch.linspace(-5, 5, 16, dtype=torch.float64, device="cuda").repeat(batch * heads, 1)
        t = torch.full((batch * heads,), 16, dtype=torch.int32, device="cuda")
        kw = dict(k_codebooks=books, k_counts=t, v_codebooks=books, v_counts=t, seed=5,
                  k_hat=torch.zeros_like(rows), v_hat=torch.zeros_like(rows))
    ecasq.ecasq_kv_write(kv, rows, rows, starts, **kw)
    now = {n: getattr(kv, n).cpu() for n in c}
    assert torch.equal(now["lens"], lens + 1)
    at = c["table"][some, 0].long()
    for name in ("k", "v"):
        want = (kw[name + "_hat"] if coded else rows)[some.cuda()].cpu()
        got = now[name][at[:, None], torch.arange(heads)[None], lens[some].long()[:, None]]
        if coded:
            got = torch.stack((got & 15, got >> 4), -1).flatten(2).long()
            x = now[name + "_books"][at[:, None], torch.arange(heads)[None], lens[some].long()[:, None]]
            got = x.gather(2, got)
        assert torch.equal(got, want)
    q = torch.randn((batch, heads * group, dim), generator=g).to(dtype)
    mass = torch.full_like(kv.mass, -1.0)
    out = ecasq.ecasq_kv_attention(kv, q.cuda(), mass_out=mass)
    base = now["mass"]
    check_attention(out[some.cuda()], _part(now, some), q[some], dim ** -0.5, _np(mass[some.cuda()]),
                    _np(base[some]))
    kv.mass.copy_(torch.where(mass < 0, kv.mass, mass))
    before = {n: getattr(kv, n).cpu() for n in c}
    ecasq.ecasq_kv_evict(kv, keep, 3)
    part = {k: _np(v) if v.is_floating_point() else v.numpy() for k, v in _part(before, some).items()}
    mass, pos, left, moves = serve.evict(part, keep, 3)
    assert torch.equal(kv.lens.cpu(), (lens + 1).clamp(max=keep))
    for i, b in enumerate(some.tolist()):
        n = int(left[i])
        np.testing.assert_array_equal(kv.pos[b, :, :n].cpu().numpy(), pos[i, :, :n])
        np.testing.assert_array_equal(_np(kv.mass[b, :, :n]), mass[i, :, :n])
    for i, h, f, t in moves[::7]:
        p = int(c["table"][some[i], 0])
        assert torch.equal(kv.k[p, h, t].cpu(), before["k"][p, h, f])
        assert torch.equal(kv.v[p, h, t].cpu(), before["v"][p, h, f])


@pytest.mark.parametrize("coded", [False, True])
def test_the_largest_page(coded):
    _need_gpu()
    print("[case] page of 65536", coded, flush=True)
    c = make_cache([70000, 3], 1, 64, 65536, torch.float16, coded)
    c["mass"] = torch.randint(0, 50000, c["mass"].shape,
                              generator=torch.Generator().manual_seed(1)).float()
    kv = on_gpu(c)
    q = torch.randn(2, 2, 64, generator=torch.Generator().manual_seed(2)).half()
    out = ecasq.ecasq_kv_attention(kv, q.cuda())
    small = {k: v[1:] if k in ("table", "lens", "mass", "pos") else v for k, v in c.items()}
    check_attention(out[1:], small, q[1:], 0.125)
    # the same rows on pages of 64 slots, bit for bit
    d = dict(lens=c["lens"])
    first, second = c["table"][0].tolist()
    other = int(c["table"][1, 0])
    for name in c:
        if name in ("k", "v", "k_books", "v_books"):
            x = torch.cat((c[name][first, 0], c[name][second, 0], c[name][other, 0]))
            d[name] = x.reshape(-1, 1, 64, x.shape[-1])
    d["table"] = torch.full((2, 2048), -1, dtype=torch.int32)
    d["table"][0] = torch.arange(2048)
    d["table"][1, :1024] = 2048 + torch.arange(1024)
    assert torch.equal(ecasq.ecasq_kv_attention(on_gpu(d), q.cuda()), out)
    ecasq.ecasq_kv_evict(kv, 40000, 100)
    mass, pos, lens, moves = serve.evict({k: _np(v) if v.is_floating_point() else v.numpy()
                                          for k, v in c.items()}, 40000, 100)
    assert kv.lens.tolist() == [40000, 3] == lens.tolist()
    np.testing.assert_array_equal(kv.pos[0, 0, :40000].cpu().numpy(), pos[0, 0, :40000])
    np.testing.assert_array_equal(_np(kv.mass[0, 0, :40000]), mass[0, 0, :40000])
    k = kv.k.cpu()
    for _, _, f, t in moves[::501]:
        (a, b), (e, g) = (divmod(s, 65536) for s in (f, t))
        assert torch.equal(k[int(c["table"][0, e]), 0, g], c["k"][int(c["table"][0, a]), 0, b])


def test_the_widest_table():
    """2^30 slots in a table, of which two pages are there."""
    _need_gpu()
    print("[case] widest table", flush=True)
    c = make_cache([900, 0], 2, 64, 64, torch.bfloat16, False)
    q = torch.randn(2, 6, 64, generator=torch.Generator().manual_seed(2)).bfloat16()
    wide = torch.full((2, (1 << 30) // 64), -1, dtype=torch.int32)
    wide[:, : c["table"].shape[1]] = c["table"]
    kv = on_gpu({"table": wide, **{k: c[k] for k in ("k", "v", "lens")}})
    out = ecasq.ecasq_kv_attention(kv, q.cuda())
    check_attention(out, c, q, 0.125)
    kv.lens[1] = (1 << 30) - 5  # no page but those of the first slots: none of this sequence
    assert torch.all(ecasq.ecasq_kv_attention(kv, q.cuda())[1] == 0)


@pytest.mark.parametrize("dtype", TYPES)
def test_numbers_below_the_normal_range(dtype):
    _need_gpu()
    print("[case] subnormal", dtype, flush=True)
    tiny = torch.finfo(dtype).tiny
    # products: entries of x, and the codebook's values
    sym, cb, sc = _weights(40, 300, 64, dtype)
    x = (torch.randn(3, 300, generator=torch.Generator().manual_seed(1)) * tiny / 8).to(dtype)
    assert (x != 0).any() and (x.abs() < tiny).all()
    for c, y in ((cb, x), ((cb * tiny / 8).to(dtype).double(), torch.ones_like(x) * 4)):
        w = ecasq.ecasq_weights_pack(sym.cuda(), c.cuda(), sc.cuda(), 64)
        _check_product(ecasq.ecasq_matvec(w, y.cuda()), sym, c, sc, 64, y)
    for coded in (False, True):
        c = make_cache([50, 700], 2, 64, 16, dtype, coded)
        name = "v_books" if coded else "v"
        c[name] = (c[name].float() * tiny / 8).to(dtype)
        q = torch.randn(2, 4, 64, generator=torch.Generator().manual_seed(2)).to(dtype)
        out = ecasq.ecasq_kv_attention(on_gpu(c), q.cuda())
        assert (out != 0).any()
        check_attention(out, c, q, 0.125)


def test_every_call_on_a_given_stream():
    """The current stream is another one, which is kept busy: results are the given stream's."""
    _need_gpu()
    side = torch.cuda.Stream()
    dtype = torch.float16
    sym, cb, sc = [x.cuda() for x in _weights(64, 256, 32, dtype)]
    c = make_cache([100, 30], 2, 64, 16, dtype, True, max_pages=8)
    kvs = [on_gpu(c) for _ in range(2)]
    g = torch.Generator().manual_seed(1)
    x = torch.randn(3, 256, generator=g).to(dtype).cuda()
    q = torch.randn(2, 4, 128, generator=g).to(dtype).cuda()[:, :, :64]  # copied by the call
    rows = torch.randn(3, 2, 128, generator=g).to(dtype).cuda()[:, :, ::2]
    starts = torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda")
    books = torch.linspace(-4, 4, 16, dtype=torch.float64, device="cuda").repeat(6, 1)
    t = torch.full((6,), 16, dtype=torch.int32, device="cuda")
    busy = torch.randn(4096, 4096, device="cuda")
    got = []
    torch.cuda.synchronize()
    for kv, kw in zip(kvs, ({}, dict(stream=side))):
        for _ in range(8):
            busy = torch.tanh(busy)
        w = ecasq.ecasq_weights_pack(sym, cb, sc, 32, **kw)
        y = ecasq.ecasq_matvec(w, x, **kw)
        ecasq.ecasq_kv_write(kv, rows, rows, starts, None, books, t, books, t, seed=3, **kw)
        a = ecasq.ecasq_kv_attention(kv, q, mass_out=kv.mass, **kw)
        ecasq.ecasq_kv_evict(kv, 20, 4, **kw)
        side.synchronize() if kw else torch.cuda.synchronize()
        got.append((w.packed, y, a, kv.k, kv.v, kv.k_books, kv.v_books, kv.mass, kv.pos, kv.lens))
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(torch.nan_to_num(a.float(), 7.0), torch.nan_to_num(b.float(), 7.0))
    with pytest.raises(ValueError, match="stream"):
        ecasq.ecasq_matvec(w, x, stream=type("S", (), {"device": torch.device("cuda", 7)})())
