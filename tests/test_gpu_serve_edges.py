"""The serving operators where their kernels change course: matrices of more
columns than a workgroup holds, more tiles than a round, rows above 16; lengths at
the borders of the chunks that attention is split into, tables much longer than
the sequences, head groups of every size; heads at the sizes where eviction keeps
its keys elsewhere; rounding of infinities, NaN and codebooks at the edges of the
32-bit comparison; calls on two streams at once, and two graphs that are replayed
in turn.  Tolerances as in test_gpu_serve.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import serve
from paper_2608_18147_amd import ecasq
from tests.test_gpu_serve import (F, TYPES, _check_evict, _check_product, _e, _np, _weights,
                                  check_attention, make_cache, on_gpu, oracle_cache)

pytestmark = pytest.mark.gpu


def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n_out,n_in,group", [
    (16, 40, 9000, 64),     # more than 64 blocks: x read again, or from LDS for few rows
    (7, 300, 10017, 96),
    (3, 700, 8200, 128),
    (1, 33, 20000, 128),
    (20, 5000, 8321, 256),  # two tiles to a part of x, two groups of rows
    (4, 9000, 8193, 32),
    (2, 13000, 384, 32),    # several rounds of tiles
    (1, 70001, 40, 32),
    (9, 17000, 1100, 128),
    (100, 70, 5000, 64),
])
def test_products_large(m, n_out, n_in, group, dtype):
    _need_gpu()
    print("[case] product", m, n_out, n_in, group, dtype, flush=True)
    sym, cb, sc = _weights(n_out, n_in, group, dtype)
    x = torch.randn(m, n_in, generator=torch.Generator().manual_seed(n_in)).to(dtype)
    w = ecasq.ecasq_weights_pack(sym.cuda(), cb.cuda(), sc.cuda(), group)
    y = ecasq.ecasq_matvec(w, x.cuda())
    _check_product(y, sym, cb, sc, group, x)
    for r in {0, m // 2, m - 1}:  # the same bits for a row by itself, and for some of them
        assert torch.equal(ecasq.ecasq_matvec(w, x[r].cuda()), y[r])
    assert torch.equal(ecasq.ecasq_matvec(w, x[: (m + 1) // 2].cuda()), y[: (m + 1) // 2])


@pytest.mark.parametrize("n_in", [127, 8195])
def test_products_padding_is_harmless(n_in):
    """Every value but one infinite: what fills up tiles takes the finite one; and a
    whole codebook of NaN gives NaN."""
    _need_gpu()
    n_out, m = 19, 3
    cb = torch.full((16,), float("inf"), dtype=torch.float64)
    cb[11] = 0.5
    sym = torch.full((n_out, n_in), 11, dtype=torch.uint8)
    sym[18, 0] = 0
    sc = torch.ones(n_out, -(-n_in // 32)).half()
    x = torch.randn(m, n_in).half()
    w = ecasq.ecasq_weights_pack(sym.cuda(), cb.cuda(), sc.cuda(), 32)
    y = ecasq.ecasq_matvec(w, x.cuda()).cpu()
    assert torch.isinf(y[:, 18]).all()
    cb[:] = 0.5
    _check_product(y[:, :18], sym[:18], cb, sc[:18], 32, x)
    w = ecasq.ecasq_weights_pack(sym.cuda(), torch.full((3,), float("nan")), sc.cuda(), 32)
    assert torch.isnan(ecasq.ecasq_matvec(w, x.cuda())).all()


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("lens", [[256, 255, 257, 512, 1], [1023, 1024, 1025, 0, 640]])
def test_attention_at_chunk_borders(lens, coded):
    """A table of 4096 slots, most of them never used."""
    _need_gpu()
    print("[case] chunks", lens, coded, flush=True)
    c = make_cache(lens, 2, 64, 32, torch.bfloat16, coded, max_pages=128)
    q = torch.randn(len(lens), 6, 64).to(torch.bfloat16)
    kv = on_gpu(c)
    mass = torch.zeros_like(kv.mass)
    out = ecasq.ecasq_kv_attention(kv, q.cuda(), mass_out=mass)
    check_attention(out, c, q, 0.125, _np(mass), _np(c["mass"]))


@pytest.mark.parametrize("group", [1, 2, 3, 7, 15, 16, 17, 31, 33])
def test_attention_groups(group):
    _need_gpu()
    c = make_cache([37, 300], 2, 128, 16, torch.float16, group % 2 == 1)
    q = torch.randn(2, 2 * group, 128).half()
    print("[case] group", group, flush=True)
    kv = on_gpu(c)
    mass = torch.zeros_like(kv.mass)
    out = ecasq.ecasq_kv_attention(kv, q.cuda(), mass_out=mass)
    check_attention(out, c, q, 128 ** -0.5, _np(mass), _np(c["mass"]))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_many_small_weights(dtype):
    """One slot far above 6000 others whose weights together count: sums and products
    of weights around 2^-20 of the largest."""
    _need_gpu()
    n, dim, page = 6001, 64, 64
    c = make_cache([n], 1, dim, page, dtype, False)
    q = torch.ones(1, 1, dim).to(dtype)
    for s in range(n):
        at = int(c["table"][0, s // page]), 0, s % page
        c["k"][at] = 0.0
        c["v"][at] = 1.0 if s else -1.0
        if s == 1234:
            c["k"][at] = 0.75
            c["v"][at] = 0.0
    print("[case] small weights", dtype, flush=True)
    for scale in (0.15, 0.25, 0.29):  # the peak at 7, 12 and 14
        out = ecasq.ecasq_kv_attention(on_gpu(c), q.cuda(), scale=scale)
        check_attention(out, c, q, scale)


@pytest.mark.parametrize("slots,lens,keep,recent", [
    (4096, [4096, 4095], 2000, 10), (4112, [4112, 4000], 100, 7), (32768, [32768], 9, 3),
    (32784, [32784, 100], 30000, 29999), (4096, [4096], 4096, 1), (4096, [4096], 4095, 0),
])
def test_evict_sizes(slots, lens, keep, recent):
    _need_gpu()
    print("[case] evict", slots, lens, keep, recent, flush=True)
    c = make_cache(lens, 2, 64, 16, torch.bfloat16, False, max_pages=slots // 16)
    g = torch.Generator().manual_seed(slots)
    c["mass"] = torch.rand(c["mass"].shape, generator=g) ** 20
    c["mass"][0] = torch.randint(0, 5, c["mass"][0].shape, generator=g).float()  # ties all over
    _check_evict(c, keep, recent, in_place=False)
    _check_evict(c, keep, recent, in_place=True)


def test_evict_extreme_positions_and_weights():
    _need_gpu()
    c = make_cache([200, 200], 1, 64, 16, torch.float16, False)
    c["pos"][0, 0, ::2] = -2 ** 31
    c["pos"][0, 0, 1::2] = 2 ** 31 - 1
    c["pos"][1] = -2 ** 31
    c["mass"][0] = torch.tensor([1e-45, -1e-45, 3e38, -3e38, 0.0]).repeat(1, 42)[:, :208]
    print("[case] evict extremes", flush=True)
    for keep, recent in ((150, 150), (150, 0), (20, 1)):
        _check_evict(c, keep, recent, in_place=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_write_of_special_values_and_books(dim, dtype):
    """Entries outside the codebook's range, infinities and NaN; intervals of no width,
    of a denormal's and beyond the floats; values a hair from entries."""
    _need_gpu()
    print("[case] write specials", dim, dtype, flush=True)
    g = torch.Generator().manual_seed(dim)
    x = torch.randn(6, 1, dim, generator=g).to(dtype)
    x[0, 0, :8] = torch.tensor([float("inf"), float("-inf"), float("nan"), 1e4, -1e4, 0.0, -0.0, 1.0])
    x[1] = torch.where(x[1] > 0, torch.ones_like(x[1]), -torch.ones_like(x[1]))
    books = torch.zeros(6, 16, dtype=torch.float64)
    books[0, :4] = torch.tensor([-2.0, -0.5, 0.25, 2.0])
    books[1, :5] = torch.tensor([-1.0, -1.0, 1.0 - 1e-12, 1.0, 1.0], dtype=torch.float64)
    books[2, :3] = torch.tensor([-1e-320, 0.0, 1e-320], dtype=torch.float64)
    books[3, :4] = torch.tensor([-1e300, -1e39, 1e39, 1e300], dtype=torch.float64)
    books[4, :16] = torch.linspace(-3, 3, 16, dtype=torch.float64) * (1 + 1e-9)
    books[5, :2] = torch.tensor([0.0, 2.0 ** -110], dtype=torch.float64)
    t = torch.tensor([4, 5, 3, 4, 16, 2], dtype=torch.int32)
    c = make_cache([6], 1, dim, 16, dtype, True)
    kv = on_gpu(c)
    hat = torch.zeros_like(x).cuda()
    starts = torch.tensor([0, 6], dtype=torch.int32).cuda()
    xd, bd, td = x.cuda(), books.cuda(), t.cuda()
    ecasq.ecasq_kv_write(kv, xd, xd, starts, k_codebooks=bd, k_counts=td, v_codebooks=bd, v_counts=td,
                         seed=3, k_hat=hat, v_hat=torch.zeros_like(hat))
    page = int(c["table"][0, 0])
    for name, word in (("k", 2), ("v", 3)):
        sym = torch.from_numpy(serve.round_rows(_np(x.reshape(6, dim)), books.numpy(), t.numpy(), 3,
                                                word))
        two = (sym[:, 0::2] | (sym[:, 1::2] << 4)).to(torch.uint8)
        assert torch.equal(getattr(kv, name).cpu()[page, 0, :6], two), name
        want = torch.where(torch.arange(16)[None, :] < t[:, None], books, 0.0).to(dtype)
        assert torch.equal(getattr(kv, name + "_books").cpu()[page, 0, :6], want)
        if name == "k":
            assert torch.equal(hat.cpu().reshape(6, dim), books.gather(1, sym).to(dtype))


def test_codebooks_are_rounded_once():
    """Values that come out differently if a double goes through a float on its way to
    16 bits: half a step and a bit."""
    _need_gpu()
    for dtype, step in ((torch.float16, 2.0 ** -10), (torch.bfloat16, 2.0 ** -7)):
        tie = 1.0 + step / 2
        cb = torch.tensor([tie - 2.0 ** -40, tie, tie + 2.0 ** -40], dtype=torch.float64)
        want = torch.tensor([1.0, 1.0, 1.0 + step])
        sym = torch.arange(3, dtype=torch.uint8).repeat_interleave(1)[:, None]
        w = ecasq.ecasq_weights_pack(sym.cuda(), cb, torch.ones(3, 1, dtype=dtype).cuda(), 32)
        y = ecasq.ecasq_matvec(w, torch.ones(1, 1, dtype=dtype).cuda())
        assert torch.equal(y.float().cpu()[0], want), dtype


def test_two_streams_at_once():
    """The same calls on two streams, interleaved without a wait between them."""
    _need_gpu()
    c = make_cache([700, 2000, 30], 2, 128, 64, torch.float16, True)
    kvs = [on_gpu(c) for _ in range(2)]
    sym, cb, sc = _weights(512, 1024, 64, torch.float16)
    w = ecasq.ecasq_weights_pack(sym.cuda(), cb.cuda(), sc.cuda(), 64)
    q = [torch.randn(3, 8, 128).half().cuda() for _ in range(8)]
    x = [torch.randn(3, 1024).half().cuda() for _ in range(8)]

    def calls(kv, k):
        a = ecasq.ecasq_kv_attention(kv, q[k], mass_out=kv.mass)
        y = ecasq.ecasq_matvec(w, x[k])
        if k == 4:
            ecasq.ecasq_kv_evict(kv, 400, 40)
        return a, y

    want_kv = on_gpu(c)
    want = [calls(want_kv, k) for k in range(8)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    print("[case] two streams", flush=True)
    for k in range(8):
        for s in range(2):
            with torch.cuda.stream(streams[s]):
                got[s].append(calls(kvs[s], k))
    torch.cuda.synchronize()
    for s in range(2):
        for a, b in zip(want, got[s]):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        for name in ("k", "v", "mass", "pos", "lens"):
            assert torch.equal(getattr(kvs[s], name), getattr(want_kv, name)), name


def test_two_graphs_in_turn():
    """Two captured calls with workspaces, replayed in turn with eager calls between."""
    _need_gpu()
    caches = [make_cache([900, 5], 2, 64, 16, torch.bfloat16, True, seed=s) for s in range(2)]
    kvs = [on_gpu(c) for c in caches]
    qs = [torch.randn(2, 4, 64).bfloat16().cuda() for _ in range(2)]
    outs = [torch.zeros_like(kv.mass) for kv in kvs]
    for kv, q in zip(kvs, qs):
        ecasq.ecasq_kv_attention(kv, q, mass_out=torch.zeros_like(kv.mass))
    torch.cuda.synchronize()
    graphs, got = [], []
    for kv, q, m in zip(kvs, qs, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(ecasq.ecasq_kv_attention(kv, q, mass_out=m))
        graphs.append(g)
    print("[case] two graphs", flush=True)
    for turn in range(6):
        for q in qs:
            q.copy_(torch.randn(2, 4, 64).bfloat16())
        for g in graphs if turn % 2 else graphs[::-1]:
            g.replay()
        for k in range(2):
            m = torch.zeros_like(outs[k])
            eager = ecasq.ecasq_kv_attention(kvs[k], qs[k], mass_out=m)
            assert torch.equal(eager, got[k]) and torch.equal(m, outs[k]), (turn, k)
            check_attention(got[k], caches[k], qs[k].cpu(), 0.125)
