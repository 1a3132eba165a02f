"""The serving operators past 2^32 bytes: writes and evictions on far pages, where they
have to leave what they leave on near ones, bit for bit; a packed matrix and rows of x that
lie as far."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_18147_amd import ecasq
from tests.test_gpu_serve import TYPES, _check_product, _need_gpu, make_cache, on_gpu

pytestmark = pytest.mark.gpu


def _far(c):
    """The cache on pages behind 5 GiB, and how many come first."""
    n = c["k"].shape[0]
    far = (5 << 30) // (c["k"][0].numel() * c["k"].element_size())
    d = {}
    for k, v in c.items():
        if k in ("k", "v", "k_books", "v_books"):
            d[k] = torch.empty((far + n,) + v.shape[1:], dtype=v.dtype, device="cuda")
            d[k][far:] = v.cuda()
        else:
            d[k] = v.cuda()
    d["table"] = torch.where(d["table"] >= 0, d["table"] + far, d["table"])
    return ecasq.ecasq_kv_cache(**d), far


def _same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), 77.0), torch.nan_to_num(b.float(), 77.0))


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_writes_and_evictions_on_far_pages(dtype, coded):
    _need_gpu()
    heads, dim, page, lens = 3, 128, 32, [130, 64, 0, 200]
    c = make_cache(lens, heads, dim, page, dtype, coded, seed=3)
    near, (far, first) = on_gpu(c), _far(c)
    print("[case] far", dtype, coded, first, flush=True)
    counts = torch.tensor([3, 64, 0, 7])
    starts = torch.cat((torch.zeros(1), counts.cumsum(0))).int().cuda()
    rows = int(counts.sum())
    g = torch.Generator().manual_seed(1)
    k, v = [torch.randn(rows, heads, dim, generator=g).to(dtype).cuda() for _ in range(2)]
    kw = {}
    if coded:
        books = torch.linspace(-5, 5, 16, dtype=torch.float64).repeat(rows * heads, 1).cuda()
        t = torch.full((rows * heads,), 16, dtype=torch.int32, device="cuda")
        kw = dict(k_codebooks=books, k_counts=t, v_codebooks=books, v_counts=t, seed=4)
    before = near.k.clone()
    for kv in (near, far):
        ecasq.ecasq_kv_write(kv, k, v, starts, **kw)
    assert not _same(near.k, before)
    for step in range(2):
        for name in ("k", "v", "k_books", "v_books"):
            a, b = getattr(near, name), getattr(far, name)
            assert a is None or _same(a, b[first:]), (step, name)
        for name in ("mass", "pos", "lens"):
            assert torch.equal(getattr(near, name), getattr(far, name)), (step, name)
        before = near.k.clone()
        if step == 0:
            for kv in (near, far):
                ecasq.ecasq_kv_evict(kv, 70, 20)
            assert near.lens.tolist() == [70, 64, 0, 70] and not _same(near.k, before)


@pytest.mark.parametrize("dtype", TYPES)
def test_products_of_a_matrix_past_4_gib(dtype):
    _need_gpu()
    n_out, n_in, group, m, last = (1 << 20) + 9, 8200, 512, 3, 41
    print("[case] far matrix", dtype, flush=True)
    torch.manual_seed(2)
    sym = torch.randint(0, 16, (n_out, n_in), dtype=torch.uint8, device="cuda")
    cb = torch.randn(16, device="cuda").sort()[0].to(dtype).double()
    sc = (torch.rand(n_out, -(-n_in // group), device="cuda") + 0.1).to(dtype)
    w = ecasq.ecasq_weights_pack(sym, cb, sc, group)
    assert w.packed.numel() > 1 << 32
    # rows of x more than 2^31 bytes apart
    x = torch.empty(m, (1 << 30) + 24, dtype=dtype, device="cuda")[:, 5:5 + n_in]
    x.copy_(torch.randn(m, n_in))
    y = ecasq.ecasq_matvec(w, x)
    for at in (slice(0, last), slice(n_out // 2, n_out // 2 + last), slice(n_out - last, n_out)):
        _check_product(y[:, at], sym[at].cpu(), cb.cpu(), sc[at].cpu(), group, x.cpu())
