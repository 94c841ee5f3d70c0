"""Whole numbers that the C calls take in 32 or 64 bits: what does not fit is refused, not cut to its lower bits."""

import pytest

torch = pytest.importorskip("torch")

import paper_2505_22857_amd as ng  # noqa: E402
from paper_2505_22857_amd import serving  # noqa: E402


def test_the_check():
    for x in (0, -1, 2 ** 31 - 1, -2 ** 31, 16.0, True):
        assert serving._whole(x, "x") == x
    assert serving._whole(2 ** 63 - 1, "x", 64) == 2 ** 63 - 1
    for x in (2 ** 31, -2 ** 31 - 1, 2 ** 32 + 16, 16.5):
        with pytest.raises(ValueError, match="x must be"):
            serving._whole(x, "x")
    with pytest.raises(ValueError):
        serving._whole(2 ** 64 + 1, "x", 64)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_calls(monkeypatch, native):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    if not native:
        monkeypatch.setattr(serving, "_native_module", False)
    refs = ints([1, 0, 1, 0])
    fork = (ints([[0, 2]]), ints([20]), ints([[0]]), refs)
    for page_size in (2 ** 32 + 16, 2 ** 31, 16.5):
        with pytest.raises(ValueError, match="page_size"):
            ng.kv_fork(*fork, page_size, tokens=1)
        with pytest.raises(ValueError, match="page_size"):
            ng.kv_compact(refs, page_size)
    for tokens in (2 ** 64 + 1, 2 ** 63, 0.5):
        with pytest.raises(ValueError, match="tokens"):
            ng.kv_fork(*fork, 16, tokens=tokens)
    assert refs.tolist() == [1, 0, 1, 0]
    # pages of 2^32 + 16 tokens, all the same one
    n = 2 ** 32 + 16
    c = torch.zeros(1, 1, 1, 16, dtype=torch.float16, device="cuda").expand(1, n, 1, 16)
    e = torch.zeros(1, 1, 1, 16, device="cuda").to(torch.float8_e4m3fn).expand(1, n, 1, 16)
    s = torch.ones(1, 1, 1, device="cuda").expand(1, n // 16, 1)
    q = torch.zeros(1, 1, 1, 16, dtype=torch.float16, device="cuda")
    for cache, scales in ((c, {}), (e, dict(k_scale=s, v_scale=s))):
        with pytest.raises(ValueError, match="dimension"):
            ng.attend(q, cache, cache, pages=ints([[0]]), lengths=ints([20]), **scales)
    kc = torch.zeros(2, 8, 1, 16, dtype=torch.float16, device="cuda")
    with pytest.raises(ValueError, match="layout"):
        ng.kv_append(q, q, kc, kc.clone(), ints([[0]]), ints([0]), layout=2 ** 32)


@pytest.mark.gpu
def test_modes_of_a_beam_step():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    from synth import make_model
    lm = ng.NgpuLM.from_model(make_model("trigram_v128")).upload("cuda")
    asr, states, scores = torch.zeros(1, 2, 129, device="cuda"), ints([[0, 0]]), torch.zeros(1, 2, device="cuda")
    for kw in (dict(mode=2 ** 32), dict(mode=2 ** 32 + 2), dict(k=1.5)):
        with pytest.raises(ValueError, match="whole"):
            lm.beam_step(asr, 0.5, states, scores, **kw)
    assert lm.beam_step(asr, 0.5, states, scores, k=2, mode=ng.NGPU_FUSION_TRANSDUCER)[0].shape == (1, 2)
