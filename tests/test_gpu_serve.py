"""The serving operators on the GPU against plain 64-bit forms (oracle/serve.py).

Tolerances, with e = finfo(type).eps / 2 the largest relative rounding of a
16-bit type and f = 2^-23 twice that of fp32 (a matrix instruction's additions
may round more than once):
  products   e |y| for the result, f (n_in + groups + 2) sum|terms| for the sums,
             half the type's smallest step below its normal range
  attention  a score is off by at most ds = f (dim + 4) sum|terms|, an unnormalised
             weight by ds + 2^-20 (exponential) and e (its rounding for the matrix
             instructions), the sums by f (slots + 8); numerator and denominator
             both, times the weighted absolute values, and e |out|
  writes and evictions are exact
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import serve
from paper_2608_18147_amd import ecasq

pytestmark = pytest.mark.gpu

TYPES = [torch.float16, torch.bfloat16]
F = 2.0 ** -23


def _np(x):
    return x.double().cpu().numpy()


def _e(dtype):
    return torch.finfo(dtype).eps / 2


def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# ---------------------------------------------------------------------------
# Products


def _weights(n_out, n_in, group, dtype, t=16, seed=0):
    g = torch.Generator().manual_seed(seed + 7 * n_out + n_in)
    sym = torch.randint(0, t, (n_out, n_in), generator=g).to(torch.uint8)
    cb = torch.randn(t, generator=g).sort()[0].to(dtype).double()
    sc = (torch.rand((n_out, -(-n_in // group)), generator=g) + 0.1).to(dtype)
    return sym, cb, sc


def _check_product(y, sym, cb, sc, group, x):
    want, terms = serve.matvec(sym.numpy(), cb.numpy(), _np(sc), group, _np(x))
    e, tiny = _e(y.dtype), torch.finfo(y.dtype).tiny
    tol = e * np.abs(want) + e * tiny + F * (x.shape[-1] + sc.shape[1] + 2) * terms * (1 + e)
    err = np.abs(_np(y).reshape(want.shape) - want)
    assert np.all(err <= tol), float((err / tol).max())


PRODUCTS = [(1, 1, 1, 32), (1, 16, 128, 128), (3, 17, 129, 32), (16, 33, 31, 64),
            (17, 40, 300, 96), (65, 20, 257, 256), (1, 5, 5000, 128), (2, 1000, 64, 4096),
            (5, 100, 4100, 64), (1, 4096, 640, 160), (33, 130, 1024, 32), (130, 24, 160, 128),
            (1, 7, 16384, 32), (1, 20000, 96, 32), (4, 257, 2049, 2048), (1, 48, 8193, 512)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n_out,n_in,group", PRODUCTS)
def test_products(m, n_out, n_in, group, dtype):
    _need_gpu()
    print("[case] product", m, n_out, n_in, group, dtype, flush=True)
    sym, cb, sc = _weights(n_out, n_in, group, dtype)
    x = torch.randn(m, n_in, generator=torch.Generator().manual_seed(m)).to(dtype)
    w = ecasq.ecasq_weights_pack(sym.cuda(), cb.cuda(), sc.cuda(), group)
    y = ecasq.ecasq_matvec(w, x.cuda())
    assert y.shape == (m, n_out) and y.dtype == dtype
    _check_product(y, sym, cb, sc, group, x)
    # the same bits on a second run, and for each row by itself
    assert torch.equal(ecasq.ecasq_matvec(w, x.cuda()), y)
    assert torch.equal(ecasq.ecasq_matvec(w, x[m // 2].cuda()), y[m // 2])


@pytest.mark.parametrize("dtype", TYPES)
def test_products_of_strided_and_unaligned_rows(dtype):
    _need_gpu()
    m, n_out, n_in, group = 5, 50, 333, 64
    sym, cb, sc = _weights(n_out, n_in, group, dtype, t=11)
    wide = torch.full((m, 700), float("nan")).to(dtype)
    for at in (0, 1, 8, 101):
        x = torch.randn(m, n_in).to(dtype)
        big = wide.clone()
        big[:, at:at + n_in] = x
        big = big.cuda()
        w = ecasq.ecasq_weights_pack(sym.cuda(), cb.cuda(), sc.cuda(), group)
        print("[case] strided", at, dtype, flush=True)
        _check_product(ecasq.ecasq_matvec(w, big[:, at:at + n_in]), sym, cb, sc, group, x)
        store = torch.full((m * n_out + 3,), 7.0, dtype=dtype, device="cuda")
        out = store[1:-2].view(m, n_out)  # not aligned to more than its type
        ecasq.ecasq_matvec(w, x.cuda(), out=out)
        _check_product(out, sym, cb, sc, group, x)
        assert store[0] == 7 and store[-1] == 7 and store[-2] == 7
    # transposed storage and a leading shape
    xt = torch.randn(n_in, 6).to(dtype)
    y = ecasq.ecasq_matvec(w, xt.cuda().t().reshape(2, 3, n_in))
    assert y.shape == (2, 3, n_out)
    _check_product(y, sym, cb, sc, group, xt.t())
    assert ecasq.ecasq_matvec(w, torch.empty(0, n_in, dtype=dtype, device="cuda")).shape == (0, n_out)


@pytest.mark.parametrize("dtype", TYPES)
def test_products_with_nan_inf_and_large_symbols(dtype):
    _need_gpu()
    m, n_out, n_in, group = 20, 37, 200, 32
    sym, cb, sc = _weights(n_out, n_in, group, dtype, t=6)
    sym[3, 5], sym[4, 6] = 6, 255  # count as the last value
    x = torch.randn(m, n_in).to(dtype)
    clean = x.clone()
    x[3, 7], x[17, 199] = float("nan"), float("inf")
    sc[9, 2] = float("inf")
    w = ecasq.ecasq_weights_pack(sym.cuda(), cb.cuda(), sc.cuda(), group)
    y = ecasq.ecasq_matvec(w, x.cuda()).cpu()
    assert torch.isnan(y[3]).all() and not torch.isfinite(y[17].float()).any()
    assert not torch.isfinite(y[:, 9].float()).any()
    rows = [r for r in range(m) if r not in (3, 17)]
    cols = [o for o in range(n_out) if o != 9]
    _check_product(y[rows][:, cols], sym[cols], cb, sc[cols], group, clean[rows])
    # a codebook with an infinite value that no symbol of the first rows uses
    cb2 = cb.clone()
    cb2[5] = float("inf")
    sym2 = sym.clamp(max=4)
    sym2[36, :] = 5
    sc2 = sc.clone()
    sc2[9, 2] = 1
    w = ecasq.ecasq_weights_pack(sym2.cuda(), cb2.cuda(), sc2.cuda(), group)
    y = ecasq.ecasq_matvec(w, clean.cuda()).cpu()
    assert not torch.isfinite(y[:, 36].float()).any()
    cb2[5] = 0
    _check_product(y[:, :36], sym2[:36], cb2, sc2[:36], group, clean)
    cb3 = cb.clone()
    cb3[0] = float("inf")  # the value that fills up tiles and blocks
    w = ecasq.ecasq_weights_pack(sym.clamp(min=1).cuda(), cb3.cuda(), sc2.cuda(), group)
    y = ecasq.ecasq_matvec(w, clean.cuda()).cpu()
    cb3[0] = 0
    _check_product(y, sym.clamp(min=1), cb3, sc2, group, clean)


# ---------------------------------------------------------------------------
# The cache


def make_cache(lens, heads, dim, page, dtype, coded, seed=0, max_pages=None, spare=2, first=0):
    """A cache (on the GPU, and its arrays for the oracle) with random rows in the
    slots in use, NaN everywhere else, and its pages in random order from `first`."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-max(0, n) // page) for n in lens]
    width = max_pages or max(1, max(need))
    need = [min(n, width) for n in need]
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=g)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = 0
    c = {}
    nan = float("nan")
    if coded:
        for name in ("k", "v"):
            c[name] = torch.randint(0, 256, (n_pages, heads, page, dim // 2), generator=g,
                                    dtype=torch.uint8)
            c[name + "_books"] = torch.full((n_pages, heads, page, 16), nan).to(dtype)
    else:
        for name in ("k", "v"):
            c[name] = torch.full((n_pages, heads, page, dim), nan).to(dtype)
    for b, n in enumerate(need):
        for i in range(n):
            p = int(order[at])
            at += 1
            table[b, i] = p
            used = min(page, lens[b] - i * page)
            for name in ("k", "v"):
                if coded:
                    c[name + "_books"][p, :, :used] = torch.randn(
                        (heads, used, 16), generator=g).sort(-1)[0].to(dtype)
                else:
                    c[name][p, :, :used] = torch.randn((heads, used, dim), generator=g).to(dtype)
    c["table"], c["lens"] = table, torch.tensor(lens, dtype=torch.int32)
    slots = width * page
    c["mass"] = torch.rand((len(lens), heads, slots), generator=g)
    c["pos"] = torch.arange(slots, dtype=torch.int32).expand(len(lens), heads, slots).contiguous()
    return c


def on_gpu(c):
    d = {k: v.cuda() for k, v in c.items()}
    return ecasq.ecasq_kv_cache(**d)


def oracle_cache(c):
    return {k: (v.numpy() if v.dtype in (torch.uint8, torch.int32, torch.float32) else _np(v))
            for k, v in c.items()}


def check_attention(out, c, q, scale, got_mass=None, base_mass=None):
    want, mass, absolute, terms = serve.attention(oracle_cache(c), _np(q), scale)
    e = _e(out.dtype)
    n = np.array([max(1, serve.length(oracle_cache(c), b)) for b in range(q.shape[0])])[:, None]
    dw = 2 * F * (q.shape[2] + 4) * terms + 2.0 ** -20 + F * (n + 8)  # a weight, relative
    tol = (2 * dw + e)[..., None] * absolute + e * np.abs(want) + e * torch.finfo(out.dtype).tiny
    got = _np(out)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bad = np.isnan(want)
    err = np.where(bad, 0, np.abs(got - want))
    assert np.all(err <= np.where(bad, np.inf, tol)), float(np.nanmax(err / tol))
    if got_mass is not None:
        group = q.shape[1] // mass.shape[1]
        off = 2 * dw.reshape(dw.shape[0], -1, group).max(-1)[..., None] * mass
        for b in range(q.shape[0]):
            k = serve.length(oracle_cache(c), b)
            total = base_mass[b, :, :k] + mass[b, :, :k]
            err = np.abs(got_mass[b, :, :k] - total)
            assert np.all(err <= off[b, :, :k] + F * total + 1e-38), b


CACHES = [
    # lens, heads, group, dim, page
    ([1], 1, 1, 64, 16),
    ([1, 0, 17, 16, 15], 2, 4, 128, 16),
    ([33, 31, 32], 3, 5, 128, 32),
    ([200, 3, 64], 2, 8, 64, 64),
    ([130, 129], 1, 16, 256, 48),
    ([70, 0], 2, 3, 256, 16),
    ([1000], 1, 20, 128, 128),
    ([500, 77], 1, 64, 64, 16),
    ([2600, 1, 2500], 2, 1, 128, 64),
    ([-5, 40], 2, 2, 128, 16),
    ([0, 0], 1, 2, 64, 16),
]


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,heads,group,dim,page", CACHES)
def test_attention(lens, heads, group, dim, page, dtype, coded):
    _need_gpu()
    print("[case] attention", lens, heads, group, dim, page, dtype, coded, flush=True)
    c = make_cache(lens, heads, dim, page, dtype, coded, seed=sum(lens))
    q = torch.randn(len(lens), heads * group, dim, generator=torch.Generator().manual_seed(3)).to(dtype)
    kv = on_gpu(c)
    out = ecasq.ecasq_kv_attention(kv, q.cuda())
    check_attention(out, c, q, dim ** -0.5)
    # with the weights: the same result, and slots past the length as they were
    mass_out = torch.full_like(kv.mass, -3.0)
    again = ecasq.ecasq_kv_attention(kv, q.cuda(), mass_out=mass_out)
    assert torch.equal(out, again)
    check_attention(again, c, q, dim ** -0.5, _np(mass_out), _np(c["mass"]))
    for b in range(len(lens)):
        assert torch.all(mass_out[b, :, max(0, lens[b]):] == -3.0)
    # in place, and a scale of its own
    ecasq.ecasq_kv_attention(kv, q.cuda(), mass_out=kv.mass)
    for b in range(len(lens)):
        n = max(0, lens[b])
        assert torch.equal(kv.mass[b, :, :n], mass_out[b, :, :n])
        assert torch.equal(kv.mass[b, :, n:].cpu(), c["mass"][b, :, n:])
    check_attention(ecasq.ecasq_kv_attention(kv, q.cuda(), scale=-0.7), c, q, -0.7)
    check_attention(ecasq.ecasq_kv_attention(kv, q.cuda(), scale=0.0), c, q, 0.0)


@pytest.mark.parametrize("coded", [False, True])
def test_attention_holes_and_lengths_past_the_table(coded):
    """Table entries that are no page, in the middle and everywhere; lens past the
    table; query rows apart and unaligned; no mass in the cache."""
    _need_gpu()
    dtype, dim, page = torch.float16, 128, 16
    c = make_cache([100, 90, 50, 20], 2, dim, page, dtype, coded)
    c["table"][0, 2] = -1
    c["table"][0, 4] = c["k"].shape[0]
    c["table"][1, :] = 2 ** 31 - 1
    c["table"][3, 0] = -2 ** 31
    c["lens"][2] = 10 ** 9  # the table's capacity: pages that are -1 past the 50th slot's
    page_id = int(c["table"][2, 3])
    for name in ("k", "v"):  # the rest of that page is in use now
        x = c[name + "_books"] if coded else c[name]
        x[page_id] = torch.where(torch.isnan(x[page_id]), torch.zeros_like(x[page_id]), x[page_id])
    q = torch.randn(4, 4, dim).to(dtype)
    wide = torch.zeros(4, 4 * dim + 77, dtype=dtype)
    wide[:, 5:5 + 4 * dim] = q.reshape(4, -1)
    qv = wide.cuda()[:, 5:5 + 4 * dim].view(4, 4, dim)
    kv = on_gpu({k: v for k, v in c.items() if k not in ("mass", "pos")})
    print("[case] holes", coded, flush=True)
    mass = torch.zeros(kv._slots_shape, device="cuda")
    out = ecasq.ecasq_kv_attention(kv, qv, mass_out=mass)
    check_attention(out, c, q, dim ** -0.5, _np(mass), np.zeros(mass.shape))
    assert torch.all(out[1] == 0) and torch.all(mass[1] == 0)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_infinite_and_large_scores(dtype):
    _need_gpu()
    print("[case] infinite", dtype, flush=True)
    dim, page = 64, 16
    c = make_cache([40, 40, 40, 40, 40], 1, dim, page, dtype, False)
    q = torch.ones(5, 2, dim).to(dtype)

    def row(b, s):
        return int(c["table"][b, s // page]), 0, s % page

    for s in range(40):
        c["k"][row(0, s)] = float("-inf")       # every score -inf: zeros
        if s != 21:
            c["k"][row(1, s)] = float("-inf")   # all but one: that row
        c["k"][row(3, s)] = 300.0 * (s - 20)    # scores a long way apart
    c["v"][row(2, 7)] = float("nan")            # a NaN that is read
    c["k"][row(4, 3)] = float("nan")
    out = ecasq.ecasq_kv_attention(on_gpu(c), q.cuda())
    assert torch.all(out[0] == 0)
    assert torch.equal(out[1, 0].cpu(), c["v"][row(1, 21)])
    assert torch.equal(out[3, 1].cpu(), c["v"][row(3, 39)])
    assert torch.isnan(out[2]).all() and torch.isnan(out[4]).all()


@pytest.mark.parametrize("coded,dtype,group", [(False, torch.bfloat16, 4), (True, torch.float16, 8)])
def test_attention_long(coded, dtype, group):
    """Lengths that are split, one much longer than the others, on pages past the
    first 2^32 bytes of the cache."""
    _need_gpu()
    lens, heads, dim, page = [40001, 700, 20011], 2, 128, 64
    c = make_cache(lens, heads, dim, page, dtype, coded, spare=0)
    n = c["k"].shape[0]
    far = (5 << 30) // (c["k"][0].numel() * c["k"].element_size())
    d = {}
    for k, v in c.items():
        if k in ("k", "v"):
            d[k] = torch.empty((far + n,) + v.shape[1:], dtype=v.dtype, device="cuda")
            d[k][far:] = v.cuda()
        elif k in ("k_books", "v_books"):
            d[k] = torch.empty((far + n,) + v.shape[1:], dtype=v.dtype, device="cuda")
            d[k][far:] = v.cuda()
        else:
            d[k] = v.cuda()
    d["table"] = torch.where(d["table"] >= 0, d["table"] + far, d["table"])
    print("[case] long", coded, dtype, far, flush=True)
    q = torch.randn(3, heads * group, dim, generator=torch.Generator().manual_seed(5)).to(dtype)
    kv = ecasq.ecasq_kv_cache(**d)
    mass = torch.zeros_like(kv.mass)
    out = ecasq.ecasq_kv_attention(kv, q.cuda(), mass_out=mass)
    # the oracle takes rows one by one: the plain form in torch's 64 bits instead
    tol_e = _e(dtype)
    for b, length in enumerate(lens):
        at = c["table"][b, :-(-length // page)].long()
        for h in range(heads):
            rows = []
            for name in ("k", "v"):
                x = c[name][at, h].reshape(-1, c[name].shape[-1])[:length]
                if coded:
                    book = c[name + "_books"][at, h].reshape(-1, 16)[:length].double()
                    x = book.gather(1, torch.stack((x & 15, x >> 4), -1).flatten(1).long())
                rows.append(x.double())
            z = q[b, h * group:(h + 1) * group].double() @ rows[0].T.contiguous() * dim ** -0.5
            p = torch.softmax(z, 1)
            ds = 2 * F * (dim + 4) * float((q[b].double().abs().max() * rows[0].abs().sum(1)).max()
                                           * dim ** -0.5) + 2.0 ** -20 + F * (length + 8)
            want = p @ rows[1]
            tol = (2 * ds + tol_e) * (p @ rows[1].abs()) + tol_e * want.abs()
            got = out[b, h * group:(h + 1) * group].double().cpu()
            assert torch.all((got - want).abs() <= tol)
            w = p.sum(0)
            total = c["mass"][b, h, :length].double() + w
            assert torch.all((mass[b, h, :length].double().cpu() - total).abs()
                             <= 2 * ds * w + F * total)
    for _ in range(2):
        assert torch.equal(ecasq.ecasq_kv_attention(kv, q.cuda()), out)


def test_attention_many_sequences():
    _need_gpu()
    lens = [(37 * i) % 90 for i in range(300)]
    c = make_cache(lens, 2, 64, 16, torch.bfloat16, True)
    q = torch.randn(300, 4, 64).to(torch.bfloat16)
    print("[case] many sequences", flush=True)
    check_attention(ecasq.ecasq_kv_attention(on_gpu(c), q.cuda()), c, q, 0.125)


def _codebooks(x, g, s=16):
    """Codebooks of values of the rows, 1 to 16 of them, a few rows without one."""
    n, d = x.shape
    t = torch.randint(1, 17, (n,), generator=g, dtype=torch.int32)
    t = torch.minimum(t, torch.tensor(s, dtype=torch.int32))
    books = torch.full((n, s), float("nan"), dtype=torch.float64)
    for r in range(n):
        at = torch.linspace(0, d - 1, int(t[r])).round().long()
        books[r, : int(t[r])] = x[r].double().sort()[0][at]
    t[n // 3], t[n // 2] = 0, 17
    return books, t


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,dim,page,counts,lens,s", [
    (2, 128, 16, [3, 0, 1, 20], [3, 5, 17, 30], 16),
    (1, 64, 32, [1, 1], [1, 64], 32),
    (3, 256, 16, [7, 2], [40, 2], 20),
    (5, 64, 16, [4, 9, 0], [2, 1000, -4], 16),  # slots below 0 and past the table: left out
])
def test_write(heads, dim, page, counts, lens, s, dtype, coded):
    _need_gpu()
    print("[case] write", heads, dim, page, counts, dtype, coded, flush=True)
    g = torch.Generator().manual_seed(dim + heads)
    c = make_cache([min(max(n, 1), 64) for n in lens], heads, dim, page, dtype, coded, max_pages=4,
                   seed=1)
    c["lens"] = torch.tensor(lens, dtype=torch.int32)
    c["table"][0, 2:] = -1
    kv = on_gpu(c)
    rows = sum(counts) + 2  # two rows that no sequence has
    starts = torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32)
    fused = torch.randn(rows, 3 * heads * dim + 5, generator=g).to(dtype)
    k = fused[:, 1:1 + heads * dim].view(rows, heads, dim)
    v = fused[:, 3 + heads * dim:3 + 2 * heads * dim].view(rows, heads, dim)
    fd = fused.cuda()
    kd = fd[:, 1:1 + heads * dim].view(rows, heads, dim)
    vd = fd[:, 3 + heads * dim:3 + 2 * heads * dim].view(rows, heads, dim)
    seed = 2 ** 63 + 12345
    where = serve.new_slots(oracle_cache(c), starts.numpy(), rows)
    want = {name: c[name].clone() for name in c}
    kw, hats = {}, {}
    if coded:
        for name, x, word in (("k", k, 2), ("v", v, 3)):
            books, t = _codebooks(x.reshape(rows * heads, dim), g, s)
            kw[name + "_codebooks"], kw[name + "_counts"] = books.cuda(), t.cuda()
            sym = serve.round_rows(_np(x.reshape(rows * heads, dim)), books.numpy(), t.numpy(), seed,
                                   word)
            good = (t >= 1) & (t <= min(s, 16))
            full = torch.zeros(rows * heads, 16, dtype=torch.float64)
            m = min(16, s)
            full[:, :m] = torch.where(torch.arange(m)[None, :] < t[:, None], books[:, :m], 0.0)
            full[~good] = float("nan")
            hat = full.gather(1, torch.from_numpy(sym)).to(dtype).reshape(rows, heads, dim)
            hats[name] = hat
            for i, at in enumerate(where):
                p = serve.place(oracle_cache(c), *at) if at else None
                if p is not None:
                    two = torch.from_numpy(sym).reshape(rows, heads, dim)[i]
                    want[name][p[0], :, p[1]] = (two[:, 0::2] | (two[:, 1::2] << 4)).to(torch.uint8)
                    want[name + "_books"][p[0], :, p[1]] = full.reshape(rows, heads, 16)[i].to(dtype)
            kw[name + "_hat"] = torch.full((rows, heads, dim), 5.0, dtype=dtype, device="cuda")
        kw["seed"] = seed
    else:
        for i, at in enumerate(where):
            p = serve.place(oracle_cache(c), *at) if at else None
            if p is not None:
                want["k"][p[0], :, p[1]], want["v"][p[0], :, p[1]] = k[i], v[i]
    for positions in (None, torch.arange(rows, dtype=torch.int32) + 1000):
        for i, at in enumerate(where):
            if at:
                want["mass"][at[0], :, at[1]] = 0
                want["pos"][at[0], :, at[1]] = at[1] if positions is None else int(positions[i])
        ecasq.ecasq_kv_write(kv, kd, vd, starts.cuda(), positions=None if positions is None else
                             positions.cuda(), **kw)
        for name in want:
            got = getattr(kv, name).cpu()
            assert got.dtype == want[name].dtype
            if got.is_floating_point():  # NaN included, bit for bit
                same = (got == want[name]) | (torch.isnan(got) & torch.isnan(want[name]))
                assert torch.all(same), name
            else:
                assert torch.equal(got, want[name]), name
    for name, hat in hats.items():
        got = kw[name + "_hat"].cpu()
        for i, at in enumerate(where):
            p = serve.place(oracle_cache(c), *at) if at else None
            if p is None:
                assert torch.all(got[i] == 5.0)
            else:
                assert torch.all((got[i] == hat[i]) | (torch.isnan(got[i]) & torch.isnan(hat[i])))


def test_write_many_sequences_and_no_rows():
    _need_gpu()
    n = 200
    c = make_cache([5] * n, 2, 64, 16, torch.float16, False)
    c["lens"] = torch.full((n,), 6, dtype=torch.int32)
    kv = on_gpu(c)
    k, v = torch.randn(n, 2, 64).half(), torch.randn(n, 2, 64).half()
    starts = torch.arange(n + 1, dtype=torch.int32).cuda()
    print("[case] write 200 sequences", flush=True)
    ecasq.ecasq_kv_write(kv, k.cuda(), v.cuda(), starts)
    at = c["table"][:, 0].long()
    assert torch.equal(kv.k.cpu()[at, :, 5], k) and torch.equal(kv.v.cpu()[at, :, 5], v)
    before = kv.k.clone()
    ecasq.ecasq_kv_write(kv, k[:0].cuda(), v[:0].cuda(), torch.zeros_like(starts))
    assert torch.equal(torch.nan_to_num(kv.k), torch.nan_to_num(before))


def _check_evict(c, keep, recent, in_place):
    kv = on_gpu(c)
    o = oracle_cache(c)
    mass, pos, lens, moves = serve.evict(o, keep, recent)
    want = {k: c[k].clone() for k in c if k.startswith(("k", "v"))}
    for b, h, f, t in moves:
        pf, pt = serve.place(o, b, f), serve.place(o, b, t)
        if pf is None or pt is None:
            continue
        for name in want:
            want[name][pt[0], h, pt[1]] = c[name][pf[0], h, pf[1]]
    if in_place:
        ecasq.ecasq_kv_evict(kv, keep, recent)
        got = kv.mass, kv.pos, kv.lens
    else:
        got = torch.full_like(kv.mass, -9.0), torch.full_like(kv.pos, -9), torch.zeros_like(kv.lens)
        ecasq.ecasq_kv_evict(kv, keep, recent, *got)
        for b in range(len(lens)):
            mass[b, :, lens[b]:], pos[b, :, lens[b]:] = -9.0, -9
        for name in ("mass", "pos", "lens"):
            assert torch.equal(torch.nan_to_num(getattr(kv, name).cpu().float()),
                               torch.nan_to_num(c[name].float()))
    np.testing.assert_array_equal(got[2].cpu().numpy(), lens)
    np.testing.assert_array_equal(got[1].cpu().numpy(), pos)
    np.testing.assert_array_equal(got[0].cpu().numpy(), mass)
    for name in want:
        g = getattr(kv, name).cpu()
        same = g == want[name]
        if g.is_floating_point():
            same |= torch.isnan(g) & torch.isnan(want[name])
        assert torch.all(same), name


@pytest.mark.parametrize("coded,dtype", [(False, torch.float16), (True, torch.bfloat16)])
@pytest.mark.parametrize("lens,heads,dim,page,keep,recent", [
    ([1, 2, 0], 1, 64, 16, 1, 0),
    ([20, 16, 17, 40], 2, 128, 16, 16, 4),
    ([100, 99, 3], 3, 64, 32, 50, 50),
    ([65, 65, 65], 2, 256, 16, 64, 1),
    ([1500, 1025, 1024], 2, 64, 64, 700, 100),
    ([3000], 1, 128, 16, 2999, 0),
    ([50], 1, 64, 16, 1, 1),
    ([30, 40], 1, 64, 16, 1000, 10),
    ([5000, 4097], 2, 64, 128, 4096, 512),
])
def test_evict(lens, heads, dim, page, keep, recent, dtype, coded):
    _need_gpu()
    print("[case] evict", lens, heads, dim, page, keep, recent, coded, flush=True)
    for case in range(4):
        c = make_cache(lens, heads, dim, page, dtype, coded, seed=case)
        g = torch.Generator().manual_seed(case)
        if case == 1:  # many ties, signs and specials
            c["mass"] = torch.randint(-2, 3, c["mass"].shape, generator=g).float() * 0.5
            c["mass"][..., ::7] = float("nan")
            c["mass"][..., 3::11] = float("inf")
            c["mass"][..., 5::13] = float("-inf")
            c["mass"][..., 6::17] = -0.0
        elif case == 2:  # every weight the same; positions in any order, some alike
            c["mass"][:] = 0.25
            c["pos"] = torch.randint(-50, 2 ** 31 - 1, c["pos"].shape, generator=g, dtype=torch.int32)
            c["pos"][..., ::3] = 2 ** 31 - 1
        elif case == 3:  # falling weights: the first slots stay; tiny and large
            c["mass"] = (2.0 ** -(torch.arange(c["mass"].shape[-1]) % 150)).float().expand(
                c["mass"].shape).contiguous()
            c["pos"] = torch.flip(c["pos"], (-1,)).contiguous()
        _check_evict(c, keep, recent, in_place=case % 2 == 0)


def test_evict_without_pages_and_twice():
    _need_gpu()
    c = make_cache([100, 100], 2, 64, 16, torch.float16, False)
    c["table"][0, 1], c["table"][0, 5] = -1, 10 ** 6
    print("[case] evict holes", flush=True)
    _check_evict(c, 40, 3, in_place=True)
    kv = on_gpu(c)
    ecasq.ecasq_kv_evict(kv, 40, 3)
    before = [x.clone() for x in (kv.k, kv.mass, kv.pos, kv.lens)]
    ecasq.ecasq_kv_evict(kv, 40, 3)  # nothing left to give up
    for x, y in zip(before, (kv.k, kv.mass, kv.pos, kv.lens)):
        assert torch.equal(torch.nan_to_num(x.float()), torch.nan_to_num(y.float()))


def test_evict_long():
    """A hundred thousand slots a head, many of equal weight."""
    _need_gpu()
    lens, heads, keep, recent = [100003, 70000], 2, 33333, 1000
    c = make_cache(lens, heads, 64, 128, torch.float16, False)
    g = torch.Generator().manual_seed(1)
    c["mass"] = torch.randint(0, 3000, c["mass"].shape, generator=g).float() ** 2
    print("[case] evict long", flush=True)
    _check_evict(c, keep, recent, in_place=False)
