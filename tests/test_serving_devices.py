"""Tensors and streams of different devices, without a GPU: refused before anything is enqueued."""

from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

from paper_2505_22857_amd import serving  # noqa: E402


def test_a_stream_of_another_device_is_refused():
    """Its kernels would run on that device, with addresses of the tensors' one."""
    other = SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0)
    with pytest.raises(ValueError, match="stream"):
        with serving._on(torch.device("cuda", 0), other):
            pass


@pytest.mark.gpu
def test_states_of_another_device_are_refused():
    """The current device's kernels must not be given the other's addresses."""
    if torch.cuda.device_count() < 2:
        pytest.skip("needs two GPUs")
    import paper_2505_22857_amd as ng
    from synth import make_model
    lm = ng.NgpuLM.from_model(make_model("trigram_v128")).upload("cuda:0")
    with torch.cuda.device(0), pytest.raises(ng.NgpuError):
        lm.draft(torch.zeros(2, dtype=torch.int32, device="cuda:1"), 2, temperature=0.0)
