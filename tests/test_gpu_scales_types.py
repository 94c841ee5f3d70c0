"""Scales that are no device tensors are refused by what they are, on every path."""

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import paper_2505_22857_amd as ng  # noqa: E402
from paper_2505_22857_amd import serving  # noqa: E402


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("bad", [0.5, "list", "host", "half"])
def test_types(monkeypatch, native, bad):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    if not native:
        monkeypatch.setattr(serving, "_native_module", False)
    s = torch.ones(2, 1, 1, device="cuda")
    bad = {"list": [0.5], "host": s.cpu(), "half": s.half()}.get(bad, bad)
    c = torch.zeros(2, 8, 1, 16, device="cuda").to(torch.float8_e4m3fn)
    q = torch.zeros(1, 1, 1, 16, dtype=torch.float16, device="cuda")
    table, one = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    for scales in (dict(k_scale=bad, v_scale=s), dict(k_scale=s, v_scale=bad)):
        with pytest.raises(TypeError, match="_scale must be"):
            ng.attend(q, c, c, pages=table, lengths=one, **scales)
        with pytest.raises(TypeError, match="_scale must be"):
            ng.kv_append(q, q, c, c, table, one, **scales)
        with pytest.raises(TypeError, match="_scale must be"):
            ng.kv_copy(c, c, torch.zeros(1, 3, dtype=torch.int32, device="cuda"), **scales)
