"""The uniforms of a coded write: the same for the same seed, whatever the cache, and others for
others; and rounded means that come near the rows over many seeds, as they do only if those
give independent uniforms."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_18147_amd import ecasq

pytestmark = pytest.mark.gpu


def test_seeds():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rows, heads, dim, dtype = 30, 2, 64, torch.float16
    g = torch.Generator().manual_seed(1)
    x = torch.randn(rows, heads, dim, generator=g).clamp(-2.9, 2.9).to(dtype).cuda()
    books = torch.linspace(-3, 3, 16, dtype=torch.float64).to(dtype).double().repeat(
        rows * heads, 1).cuda()
    t = torch.full((rows * heads,), 16, dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, rows], dtype=torch.int32, device="cuda")

    def rounded(seed):
        kv = ecasq.ecasq_kv_cache(
            *[torch.zeros(2, heads, 16, dim // 2, dtype=torch.uint8, device="cuda") for _ in "kv"],
            torch.arange(2, dtype=torch.int32, device="cuda").reshape(1, 2),
            torch.tensor([rows], dtype=torch.int32, device="cuda"),
            *[torch.zeros(2, heads, 16, 16, dtype=dtype, device="cuda") for _ in "kv"])
        hats = torch.zeros_like(x), torch.zeros_like(x)
        ecasq.ecasq_kv_write(kv, x, x, starts, k_codebooks=books, k_counts=t, v_codebooks=books,
                             v_counts=t, seed=seed, k_hat=hats[0], v_hat=hats[1])
        return hats

    k, v = rounded(7)
    again = rounded(7)
    assert torch.equal(k, again[0]) and torch.equal(v, again[1])
    assert not torch.equal(k, v)
    n, layers = 200, 4
    mean = torch.zeros(2, *x.shape, dtype=torch.float64, device="cuda")
    for step in range(n // layers):
        for layer in range(layers):
            hats = rounded(step * layers + layer)
            for i in range(2):
                mean[i] += hats[i].double() / n
    # a rounding's deviation is at most half an interval, 0.2 (and its values' rounding of
    # 2^-10): six deviations of a mean of n
    assert torch.all((mean - x.double()).abs() <= 6 * (0.2 + 2.0 ** -10) / n ** 0.5)
