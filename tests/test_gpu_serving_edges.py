"""Serving calls that have to be refused, natively and through ctypes alike, and rows to the bit."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import paper_2505_22857_amd as ng  # noqa: E402
from paper_2505_22857_amd import serving  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


@pytest.fixture(params=["native", "ctypes"])
def path(request, monkeypatch):
    """The serving calls by one of their two ways."""
    assert serving._native()
    if request.param == "ctypes":
        monkeypatch.setattr(serving, "_native_module", False)
    return request.param


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def test_gradients_are_refused(path):
    """Nothing here has a backward pass: a result without its graph would train nothing, in silence."""
    def new(*shape):
        return torch.randn(shape, device="cuda").half()
    q, kc, vc, k, v = new(2, 3, 4, 32), new(6, 8, 2, 32), new(6, 8, 2, 32), new(2, 3, 2, 32), new(2, 3, 2, 32)
    cos, sin = ng.rope_table(16, 16)
    pages, start = ints([[0, 1], [2, 3]]), ints([0, 5])

    def attend(**kw):
        return ng.attend(**{**dict(q=q, k_cache=kc, v_cache=vc, pages=pages, lengths=start + 3), **kw})

    def append(**kw):
        return ng.kv_append(**{**dict(k=k, v=v, k_cache=kc, v_cache=vc, pages=pages, start=start, cos=cos, sin=sin, q=q),
                               **kw})

    def leaf(x):
        return x.clone().requires_grad_()

    for call, names in ((attend, dict(q=q, k_cache=kc, v_cache=vc)),
                        (append, dict(k=k, v=v, q=q, k_cache=kc, v_cache=vc, cos=cos, sin=sin))):
        for name, x in names.items():
            before = kc.clone()
            for tracked in (leaf(x), leaf(x) * 1.0):
                with pytest.raises(TypeError, match="gradient"):
                    call(**{name: tracked})
            assert torch.equal(kc, before)
        want = call()
        for name, x in names.items():
            with torch.no_grad():
                assert torch.equal(call(**{name: leaf(x)}), want)
            assert torch.equal(call(**{name: leaf(x).detach()}), want)


@pytest.mark.parametrize("temperature", [1e-50, -1e-50, 5e-324, 1e-40, -1e-7])
def test_temperatures_that_round_to_zero(path, temperature):
    """Not greedy: refused, as the library's least temperature says."""
    from synth import make_model
    lm = ng.NgpuLM.from_model(make_model("trigram_v128")).upload("cuda")
    if path == "ctypes":
        lm._fast = None
    g = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn(2, 3, 128, generator=g, device="cuda")
    noise = torch.ones(2, 2, 128, device="cuda")
    with pytest.raises(ng.NgpuError, match="temperature"):
        ng.verify(logits, ints(np.zeros((2, 2))), uniforms=torch.rand(2, 2, device="cuda"), noise=noise[:, 0].contiguous(),
                  temperature=temperature)
    with pytest.raises(ng.NgpuError, match="temperature"):
        lm.draft(ints([0, 0]), 2, noise=noise, temperature=temperature)
