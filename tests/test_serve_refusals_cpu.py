"""Refusals of the serving operators that need no GPU: results over their operands,
and numbers that a 32-bit argument would cut."""
import ctypes
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2608_18147_amd import ecasq

FAKE = 0x10000000  # aligned, never read: every call below is refused on the host


@pytest.mark.parametrize("m,step", [(1, 200), (3, 200), (3, 320)])
def test_products_over_their_operands_refused(m, step):
    n_out, n_in = 20, 200
    ends = 2 * ((m - 1) * step + n_in)
    for y in (FAKE, FAKE + ends - 2, FAKE - 2 * m * n_out + 2):
        assert ecasq.lib().ecasq_matvec(FAKE, 1, n_out, n_in, 64, FAKE, m, step, None,
                                        y) == ecasq.ECASQ_EINVAL, hex(y)


def test_attention_over_its_query_refused():
    c = ecasq._kv_struct(1, 0, 2, 128, 16, 3, 4, 9, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, FAKE)
    L, r = ecasq.lib(), ctypes.byref(c)
    size, row = L.ecasq_kv_attention_workspace(r, 4, 0), 4 * 128
    for step in (row, 2 * row):
        ends = 2 * (2 * step + row)
        for out in (FAKE, FAKE + ends - 16, FAKE - 2 * 3 * row + 16):
            assert L.ecasq_kv_attention(r, FAKE, step, 4, 0.1, None, None, out, FAKE,
                                        size) == ecasq.ECASQ_EINVAL, hex(out)


def test_attention_scale_past_a_float_refused():
    """The scale times log2(e) is no float."""
    c = ecasq._kv_struct(1, 0, 2, 128, 16, 3, 4, 9, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, FAKE)
    L, r = ecasq.lib(), ctypes.byref(c)
    size = L.ecasq_kv_attention_workspace(r, 4, 0)
    for scale in (3e38, -3e38):
        assert L.ecasq_kv_attention(r, FAKE, 512, 4, scale, None, None, 2 * FAKE, FAKE,
                                    size) == ecasq.ECASQ_EINVAL


@pytest.mark.parametrize("keep,recent", [((1 << 32) + 1, 0), (-(1 << 32) + 1, 0), (1 << 31, 0),
                                         (4, 1 << 32), (4, -(1 << 33))])
def test_eviction_of_cut_numbers_refused(keep, recent):
    with pytest.raises(ValueError, match="32-bit"):
        ecasq.ecasq_kv_evict(types.SimpleNamespace(mass=1, pos=1), keep, recent)
