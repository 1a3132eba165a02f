"""Products of rows of x that begin between two dwords, by many rows and few, whole
blocks and ends, columns that one wavefront holds or that are read in turns."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_18147_amd import ecasq
from tests.test_gpu_serve import TYPES, _check_product, _need_gpu, _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 5, 6, 16, 23])
@pytest.mark.parametrize("n_out,n_in,group", [(20, 9, 32), (33, 130, 64), (40, 513, 32),
                                              (17, 4101, 96), (150, 8191, 128), (35, 9999, 128),
                                              (50, 17000, 32)])
def test_rows_between_dwords(n_out, n_in, group, m, dtype):
    _need_gpu()
    print("[case] odd", n_out, n_in, group, m, dtype, flush=True)
    sym, cb, sc = _weights(n_out, n_in, group, dtype)
    w = ecasq.ecasq_weights_pack(sym.cuda(), cb.cuda(), sc.cuda(), group)
    g = torch.Generator().manual_seed(m + n_in)
    x = torch.randn(m, n_in, generator=g).to(dtype)
    want = ecasq.ecasq_matvec(w, x.cuda())
    _check_product(want, sym, cb, sc, group, x)
    for step in (n_in, n_in + 1, n_in + 8):
        for first in (0, 1, 2, 7):
            # NaN around the rows
            buf = torch.full((first + m * step + 8,), float("nan")).to(dtype).cuda()
            rows = buf[first:first + m * step].view(m, step)[:, :n_in]
            rows.copy_(x)
            assert torch.equal(ecasq.ecasq_matvec(w, rows), want), (step, first)
