"""Attention over value rows that hold infinities and NaN.  Finite results by the tolerances
of test_gpu_serve.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import serve
from paper_2608_18147_amd import ecasq
from tests.test_gpu_serve import F, TYPES, _e, _need_gpu, _np, make_cache, on_gpu, oracle_cache

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def _check(out, c, q, scale):
    o = oracle_cache(c)
    with np.errstate(invalid="ignore"):
        want, _, absolute, terms = serve.attention(o, _np(q), scale)
    got, e = _np(out), _e(out.dtype)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_array_equal(np.where(np.isinf(got), got, 0.0), np.where(np.isinf(want), want, 0.0))
    n = np.array([max(1, serve.length(o, b)) for b in range(q.shape[0])])[:, None, None]
    with np.errstate(invalid="ignore"):
        dw = (2 * F * (q.shape[2] + 4) * terms)[..., None] + 2.0 ** -20 + F * (n + 8)
        tol = (2 * dw + e) * absolute + e * np.abs(want) + e * torch.finfo(out.dtype).tiny
        ok = ~np.isfinite(want) | (np.abs(got - want) <= tol)
    assert ok.all(), int((~ok).sum())
    return want


def _row(c, b, s):
    return int(c["table"][b, s // c["k"].shape[2]]), slice(None), s % c["k"].shape[2]


def _set_keys(c, b, s, value):
    c["k_books" if "k_books" in c else "k"][_row(c, b, s)] = value


def _set_value(c, b, s, entry, value):
    """The entry (all entries of symbol `entry` % 16 where rows are coded) of every head's row."""
    if "v_books" in c:
        c["v_books"][_row(c, b, s) + (entry % 16,)] = value
    else:
        c["v"][_row(c, b, s) + (entry,)] = value


def _query(batch, heads, dim, dtype, seed=3):
    """Positive entries: the sign of a key row that is all alike is its score's."""
    g = torch.Generator().manual_seed(seed)
    return (torch.rand((batch, heads, dim), generator=g) + 0.1).to(dtype)



@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_no_weight_at_all_is_zero(dtype, coded):
    """Scores that are all -inf give zeros, whatever the values hold; a part of the slots
    without weight hands on their NaN."""
    _need_gpu()
    print("[case] no weight", dtype, coded, flush=True)
    lens, dim = [40, 2600, 2600, 1], 64
    c = make_cache(lens, 1, dim, 16, dtype, coded)
    for b in (0, 1, 3):
        for s in range(lens[b]):
            _set_keys(c, b, s, -INF)
        for e, value in ((1, NAN), (2, INF), (3, -INF)):
            _set_value(c, b, lens[b] // 2, e, value)
            _set_value(c, b, 0, e, value)
    for s in range(600):  # (whole chunks of them)
        _set_keys(c, 2, s, -INF)
    _set_value(c, 2, 100, 4, NAN)
    q = _query(4, 3, dim, dtype)
    mass = torch.zeros(4, 1, 2608, device="cuda")
    out = ecasq.ecasq_kv_attention(on_gpu({**c, "mass": torch.zeros(mass.shape)}), q.cuda(), mass_out=mass)
    for b in (0, 1, 3):
        assert torch.all(out[b] == 0) and torch.all(mass[b] == 0), b
    want = _check(out[2:3], {**c, "table": c["table"][2:3], "lens": c["lens"][2:3]}, q[2:3], dim ** -0.5)
    assert np.isnan(want).any() and np.isfinite(want).any()
