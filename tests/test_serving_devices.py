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
