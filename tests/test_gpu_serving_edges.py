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


@pytest.mark.parametrize("V", [100, 300, 1000, 1024, 2000, 3000, 8192])
@pytest.mark.parametrize("temperature", [1.0, 0.8, 1.3])
def test_rows_have_the_formulas_roundings(V, temperature):
    """Draft rows are (x - max x) / temperature - log sum to the bit, each operation rounded once in fp32 and the division
    as a product with the rounded inverse: at the row's maximum that is the logarithm itself, negative.  That is off by
    an ulp of log2 of at most 13 bits (1e-6), and by the sum's relative error: exponents of size 20 rounded twice (2e-6)
    and up to 40 additions in a row that hardly ever err alike."""
    from synth import generate_model, uniform_states
    m = generate_model(V, [V, 3 * V, 2 * V], 1.0, seed=V)
    lm = ng.NgpuLM.from_model(m).upload("cuda:0")
    states = torch.from_numpy(uniform_states(m, 9, seed=2)).cuda()
    noise = torch.empty(9, 3, V, device="cuda").exponential_()
    _, after, rows = lm.draft(states, 3, noise=noise, temperature=temperature)
    inverse = np.float32(1) / np.float32(temperature)
    for k in range(3):
        x = lm.advance(after[:, k].contiguous())[0].cpu().numpy()
        row = rows[:, k].cpu().numpy()
        top = x.max(1, keepdims=True)
        log_sum = -row[x == top].reshape(9, -1)[:, :1]
        assert np.array_equal(row, (x - top) * inverse - log_sum)
        z = (x.astype(np.float64) - top) / np.float32(temperature)
        assert np.all(np.abs(log_sum[:, 0] - np.log(np.exp(z).sum(1))) <= 4e-6)
