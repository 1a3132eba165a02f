"""Attention over value rows that hold infinities, NaN and numbers near the type's
largest, where its products of unnormalised weights in two parts pass the floats or multiply
zeros and infinities: the result is the definition's, sum p_t V_t in 64 bits, an infinity
where that has one.  Finite results by the tolerances of test_gpu_serve.py."""
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


# lens, heads, group, dim, page: one chunk, and several that are joined
SHAPES = [([40, 1, 300, 33], 2, 3, 64, 16), ([40, 90], 1, 20, 128, 32), ([17, 250], 2, 4, 256, 16),
          ([3000, 5, 1111], 1, 5, 128, 64), ([2500], 2, 2, 64, 16), ([2600], 1, 17, 256, 128)]


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,heads,group,dim,page", SHAPES)
def test_infinite_and_nan_values(lens, heads, group, dim, page, dtype, coded):
    _need_gpu()
    print("[case] infinite values", lens, heads, group, dim, dtype, coded, flush=True)
    c = make_cache(lens, heads, dim, page, dtype, coded, seed=dim + len(lens))
    for b, n in enumerate(lens):
        last = n - 1
        _set_value(c, b, last // 3, 1, INF)
        _set_value(c, b, last, 2, -INF)
        _set_value(c, b, last // 2, 3, INF)  # both signs: NaN
        _set_value(c, b, 0, 3, -INF) if n > 1 else None
        _set_value(c, b, last // 4, 4, NAN)
        if n > 30:
            # slots of next to no weight: 2^-50 to 2^-400 of the others'
            for k, slot in enumerate((7, 12, 29, last - 3)):
                _set_keys(c, b, slot, (-1.0, -4.0, -8.0, -2.0)[k] * 2 ** (dim == 64))
                _set_value(c, b, slot, 5 + k, INF if k % 2 else -INF)
            # a score of -inf: no weight at all, and no number from an infinity
            _set_keys(c, b, 20, -INF)
            _set_value(c, b, 20, 9, INF)
    q = _query(len(lens), heads * group, dim, dtype)
    kv = on_gpu(c)
    for scale in (dim ** -0.5, 0.5):
        mass = torch.zeros_like(kv.mass)
        out = ecasq.ecasq_kv_attention(kv, q.cuda(), scale=scale, mass_out=mass)
        want = _check(out, c, q, scale)
        assert np.isposinf(want).any() and np.isneginf(want).any() and np.isfinite(want).any()
        again = ecasq.ecasq_kv_attention(kv, q.cuda(), scale=scale)
        assert torch.equal(torch.nan_to_num(again, 7.0), torch.nan_to_num(out, 7.0))
        # the weights do not know of the values
        _, weights, _, terms = serve.attention(oracle_cache({**c, "v" + "_books" * coded: torch.zeros_like(
            c["v" + "_books" * coded])}), _np(q), scale)
        got = _np(mass) - np.where(_np(mass) != 0, _np(c["mass"]), 0.0)
        off = 4 * F * (dim + 4) * terms.max() + 2.0 ** -19 + 2 * F * (max(lens) + 8)
        live = np.arange(kv.slots)[None, None, :] < np.array(lens)[:, None, None]
        assert np.all(np.abs(got - weights)[np.broadcast_to(live, got.shape)] <= off * group + F)


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,heads,group,dim,page", SHAPES)
def test_values_near_the_largest(lens, heads, group, dim, page, dtype, coded):
    """Sums of unnormalised weights times values pass the floats in bf16; the weighted means do
    not.  Equal scores, scores that rise and fall, values of one sign and of both."""
    _need_gpu()
    print("[case] large values", lens, heads, group, dim, dtype, coded, flush=True)
    most = torch.finfo(dtype).max
    c = make_cache(lens, heads, dim, page, dtype, coded, seed=dim)
    name = "v_books" if coded else "v"
    sign = torch.where(c[name].float() < 0, -1.0, 1.0)
    part = c[name][..., :8]  # (entries 0 to 7, or symbols)
    c[name] = torch.where(torch.isnan(c[name]), c[name], (sign * most).to(dtype))
    c[name][..., :8] = torch.where(torch.isnan(part), part, torch.full_like(part, most))
    q = _query(len(lens), heads * group, dim, dtype)
    for scale in (0.0, dim ** -0.5, 0.7):
        out = ecasq.ecasq_kv_attention(on_gpu(c), q.cuda(), scale=scale)
        assert torch.isfinite(out).all(), scale
        assert np.isfinite(_check(out, c, q, scale)).all()


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
