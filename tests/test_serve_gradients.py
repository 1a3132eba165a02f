"""The serving operators have no gradients: tensors that require one are refused, and are
taken where torch records none."""
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2608_18147_amd import ecasq

CPU = torch.device("cpu")  # every call below that runs here is refused before any device work


def test_inputs_that_require_a_gradient_refused():
    w = types.SimpleNamespace(dtype=torch.float16, device=CPU, n_in=8, n_out=4)
    with pytest.raises(ValueError, match="x requires a gradient"):
        ecasq.ecasq_matvec(w, torch.zeros(2, 8, dtype=torch.float16, requires_grad=True))
    kv = types.SimpleNamespace(dtype=torch.float16, device=CPU, batch=2, heads=1, head_dim=64)
    rows = torch.zeros(2, 1, 64, dtype=torch.float16)
    learnt = rows.clone().requires_grad_()
    with pytest.raises(ValueError, match="q requires a gradient"):
        ecasq.ecasq_kv_attention(kv, learnt * 2)
    for name, k, v in (("k", learnt, rows), ("v", rows, learnt)):
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            ecasq.ecasq_kv_write(kv, k, v, torch.zeros(3, dtype=torch.int32))


@pytest.mark.gpu
def test_gradients_on_the_device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sym = torch.randint(0, 16, (20, 64), dtype=torch.uint8, device="cuda")
    cb = torch.linspace(-1, 1, 16, dtype=torch.float64, device="cuda")
    sc = torch.ones(20, 2, dtype=torch.float16, device="cuda")
    for name, args in (("codebook", (cb.clone().requires_grad_(), sc)),
                       ("scales", (cb, sc.clone().requires_grad_()))):
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            ecasq.ecasq_weights_pack(sym, *args, 32)
    w = ecasq.ecasq_weights_pack(sym, cb, sc, 32)
    x = torch.randn(3, 64, device="cuda").half().requires_grad_()
    with pytest.raises(ValueError, match="x requires a gradient"):
        ecasq.ecasq_matvec(w, x)
    with torch.no_grad():
        y = ecasq.ecasq_matvec(w, x)
    assert not y.requires_grad and torch.equal(y, ecasq.ecasq_matvec(w, x.detach()))

    rows = torch.randn(4, 1, 16, 64, device="cuda").half()
    table = torch.arange(4, dtype=torch.int32, device="cuda").reshape(2, 2)
    lens = torch.tensor([20, 3], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="v requires a gradient"):
        ecasq.ecasq_kv_cache(rows, rows.clone().requires_grad_(), table, lens)
    kv = ecasq.ecasq_kv_cache(rows, rows.clone(), table, lens)
    q = torch.randn(2, 3, 64, device="cuda").half().requires_grad_()
    with pytest.raises(ValueError, match="q requires a gradient"):
        ecasq.ecasq_kv_attention(kv, q)
    with torch.inference_mode():
        out = ecasq.ecasq_kv_attention(kv, q)
    assert torch.equal(out, ecasq.ecasq_kv_attention(kv, q.detach()))
