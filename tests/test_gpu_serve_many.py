"""Calls large enough that a workgroup or a wavefront goes round again: coded writes of hundreds
of tokens (a wavefront rounds several units, keys and values, the next one read ahead), products
of more tiles than a round over columns that are read in turns, and of more rows than a launch.
Writes exactly as oracle/serve.py, products by the tolerances of test_gpu_serve.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import serve
from paper_2608_18147_amd import ecasq
from tests.test_gpu_serve import TYPES, _check_product, _need_gpu, _np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
# tokens and heads for which a workgroup has one, two and more units of 128 entries to a wavefront
@pytest.mark.parametrize("rows,heads,dim", [(600, 9, 64), (1100, 9, 64), (1100, 1, 64), (600, 5, 128),
                                            (1100, 5, 128), (1030, 16, 128), (600, 3, 256),
                                            (1100, 3, 256), (260, 8, 256)])
def test_coded_writes_of_many_tokens(rows, heads, dim, dtype):
    _need_gpu()
    print("[case] write", rows, heads, dim, dtype, flush=True)
    g = torch.Generator().manual_seed(rows + heads + dim)
    page, counts = 32, [rows // 2 + 5, 0, rows - rows // 2 - 5 - 2]  # two rows that nobody has
    before = [7, 3, 40]  # slots in use already
    lens = [a + b for a, b in zip(counts, before)]
    width = -(-max(lens) // page)
    n_pages = 3 * width + 1
    table = torch.randperm(n_pages, generator=g)[: 3 * width].to(torch.int32).reshape(3, width)
    table[0, 4] = -1  # a page that is missing
    starts = torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32)
    fused = torch.randn(rows, 2 * heads * dim + 3, generator=g).to(dtype)
    x = {"k": fused[:, 1:1 + heads * dim], "v": fused[:, 2 + heads * dim:2 + 2 * heads * dim]}
    fd = fused.cuda()
    xd = {"k": fd[:, 1:1 + heads * dim], "v": fd[:, 2 + heads * dim:2 + 2 * heads * dim]}
    seed = 2 ** 62 + 99
    kw, want = dict(seed=seed), {}
    c = dict(table=table, lens=torch.tensor(lens, dtype=torch.int32),
             mass=torch.rand(3, heads, width * page, generator=g),
             pos=torch.full((3, heads, width * page), -7, dtype=torch.int32))
    for name, word in (("k", 2), ("v", 3)):
        flat = x[name].reshape(rows * heads, dim)
        t = torch.randint(2, 17, (rows * heads,), generator=g, dtype=torch.int32)
        at = torch.arange(16)[None, :] * (dim - 1) // (t[:, None] - 1)
        books = flat.double().sort(-1)[0].gather(1, at.clamp_(max=dim - 1))
        books[torch.arange(16)[None, :] >= t[:, None]] = float("nan")
        # rows without a codebook, one value, too many, in between
        for first, count in ((3, 0), (4, 17), (10, 1), (11, -1)):
            t[first::29] = count
        books[10::29, 1:] = float("nan")
        sym = torch.from_numpy(serve.round_rows(_np(flat), books.numpy(), t.numpy(), seed, word))
        good = (t >= 1) & (t <= 16)
        full = torch.where(torch.arange(16)[None, :] < t[:, None], books, 0.0)
        full[~good] = float("nan")
        want[name + "_hat"] = full.gather(1, sym).to(dtype).reshape(rows, heads, dim)
        want[name] = (sym[:, 0::2] | (sym[:, 1::2] << 4)).to(torch.uint8).reshape(rows, heads, -1)
        want[name + "_books"] = full.to(dtype).reshape(rows, heads, 16)
        kw[name + "_codebooks"], kw[name + "_counts"] = books.cuda(), t.cuda()
        kw[name + "_hat"] = torch.full((rows, heads, dim), 5.0, dtype=dtype, device="cuda")
        c[name] = torch.full((n_pages, heads, page, dim // 2), 0xEE, dtype=torch.uint8)
        c[name + "_books"] = torch.full((n_pages, heads, page, 16), 3.0).to(dtype)
    kv = ecasq.ecasq_kv_cache(**{k: v.cuda() for k, v in c.items()})
    ecasq.ecasq_kv_write(kv, xd["k"].view(rows, heads, dim), xd["v"].view(rows, heads, dim),
                         starts.cuda(), **kw)
    o = {k: v.numpy() for k, v in c.items() if k in ("table", "lens", "k")}
    left_out = []
    for i, at in enumerate(serve.new_slots(o, starts.numpy(), rows)):
        if at is not None:
            c["mass"][at[0], :, at[1]], c["pos"][at[0], :, at[1]] = 0.0, at[1]
        place = serve.place(o, *at) if at is not None else None
        if place is None:
            left_out.append(i)
            continue
        for name in ("k", "v", "k_books", "v_books"):
            c[name][place[0], :, place[1]] = want[name][i]
    assert 2 < len(left_out) <= 2 + page
    for name in ("k", "v", "k_books", "v_books", "mass", "pos"):
        got = getattr(kv, name).cpu()
        same = got == c[name]
        if got.is_floating_point():
            same |= torch.isnan(got) & torch.isnan(c[name])
        assert same.all(), (name, int((~same).sum()))
    for name in ("k_hat", "v_hat"):
        want[name][left_out] = 5.0
        got = kw[name].cpu()
        assert ((got == want[name]) | (torch.isnan(got) & torch.isnan(want[name]))).all(), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n_out,n_in,group", [(5, 33000, 8300, 128), (16, 40009, 8200, 96),
                                                (7, 17000, 9999, 32)])
def test_products_of_many_tiles_in_turns(m, n_out, n_in, group, dtype):
    """More than 8192 columns, rows of x that do not fit in LDS, more tiles than a round."""
    _need_gpu()
    print("[case] turns", m, n_out, n_in, group, dtype, flush=True)
    g = torch.Generator(device="cuda").manual_seed(n_out)
    sym = torch.randint(0, 16, (n_out, n_in), dtype=torch.uint8, device="cuda", generator=g)
    cb = torch.randn(16, device="cuda", generator=g).sort()[0].to(dtype).double()
    sc = (torch.rand(n_out, -(-n_in // group), device="cuda", generator=g) + 0.1).to(dtype)
    x = torch.randn(m, n_in, device="cuda", generator=g).to(dtype)
    w = ecasq.ecasq_weights_pack(sym, cb, sc, group)
    y = ecasq.ecasq_matvec(w, x)
    # each row by itself, from LDS, has the same bits; some of the outputs by 64 bits
    for r in range(m):
        assert torch.equal(ecasq.ecasq_matvec(w, x[r]), y[r]), r
    for at in (slice(0, 33), slice(16 * 256 * 4 - 5, 16 * 256 * 4 + 40), slice(n_out // 2, n_out // 2 + 33),
               slice(n_out - 41, n_out)):
        at = slice(at.start, min(at.stop, n_out))
        _check_product(y[:, at], sym[at].cpu(), cb.cpu(), sc[at].cpu(), group, x.cpu())


@pytest.mark.parametrize("dtype", TYPES)
def test_products_of_more_rows_than_a_launch(dtype):
    _need_gpu()
    m, n_out, n_in, group = (1 << 19) + 21, 3, 8, 32
    print("[case] rows", m, dtype, flush=True)
    g = torch.Generator().manual_seed(1)
    sym = torch.randint(0, 16, (n_out, n_in), generator=g).to(torch.uint8)
    cb = torch.randn(16, generator=g).sort()[0].to(dtype).double()
    sc = (torch.rand(n_out, 1, generator=g) + 0.1).to(dtype)
    x = torch.randn(m, n_in + 1, generator=g).to(dtype)
    w = ecasq.ecasq_weights_pack(sym.cuda(), cb.cuda(), sc.cuda(), group)
    xd = x.cuda()
    for part in (xd[:, :n_in], xd[:, 1:]):  # rows an odd number of entries apart
        y = ecasq.ecasq_matvec(w, part)
        assert y.shape == (m, n_out)
        _check_product(y, sym, cb, sc, group, part.cpu())
