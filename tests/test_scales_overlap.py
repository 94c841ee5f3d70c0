"""Scales that share elements.  A call that writes scales gives each block and head its own, so two that share an element
would leave one of them wrong: such calls are refused.  Reading them is sound, and so is copying where all copies of an
element carry one value."""

import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2505_22857_amd as ng  # noqa: E402
from paper_2505_22857_amd import pages, serving  # noqa: E402

INVALID, P, BLOCKS, H = -1, 10, 2, 2
FAR = 1 << 20


def cache8(k=(4, 2, 1), v=(4, 2, 1), between=FAR, heads=H):
    c = serving._Cache(1, heads, 64, 16, P, 64, 1 << 30, 2048, 128, 64, 2048, 128, 64)
    return serving._Cache8(c, 16 // BLOCKS, FAR, FAR + between, *k, *v)


APART = [dict(), dict(k=(1, 10, 20), v=(1, 10, 20)), dict(k=(1, 10, 20)), dict(between=160, v=(1, 10, 20)),
         dict(k=(8, 4, 1), v=(8, 4, 1), between=8), dict(k=(8, 4, 2), v=(8, 4, 2), between=4), dict(k=(5, 3, 1), v=(9, 3, 1)),
         dict(k=(4, 2, 0), v=(2, 1, 9), heads=1), dict(between=160, k=(4, 2, 1))]
OVERLAP = [dict(k=(0, 2, 1)), dict(k=(4, 0, 1)), dict(k=(4, 2, 0)), dict(v=(0, 0, 0)), dict(v=(2, 1, 0)), dict(between=0),
           dict(k=(1, 1, 20)), dict(v=(3, 2, 1)), dict(between=156), dict(between=4), dict(between=2, k=(8, 4, 2), v=(8, 4, 2)),
           dict(between=8, v=(1, 10, 20)), dict(between=-156)]
ONE_VALUE = [dict(k=(0, 2, 1)), dict(k=(4, 0, 1)), dict(k=(4, 2, 0)), dict(v=(0, 0, 0)), dict(k=(0, 0, 0), v=(0, 0, 0)),
             dict(between=0), dict(k=(0, 0, 0), v=(0, 0, 0), between=0), dict(k=(0, 0, 0), v=(0, 0, 0), between=4)]


def refused(call, *args):
    """Whether the call names the scales; without a GPU what is not refused fails at its launch."""
    return call(*args) == INVALID and "overlap" in ng.load_library().ngpu_lm_last_error().decode()


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up: calls that are not refused would be launched")
def test_refusals_by_strides():
    from test_serving_host import ok_append
    append, copy = serving._library().ngpu_lm_kv_append8, pages._library().ngpu_lm_kv_copy8
    for kw in APART:
        assert not refused(append, ctypes.byref(cache8(**kw)), ctypes.byref(ok_append()), None), kw
        assert not refused(copy, ctypes.byref(cache8(**kw)), 64, 1, None), kw
    for kw in OVERLAP:
        assert refused(append, ctypes.byref(cache8(**kw)), ctypes.byref(ok_append()), None), kw
        assert refused(copy, ctypes.byref(cache8(**kw)), 64, 1, None) == (kw not in ONE_VALUE and kw != dict(v=(2, 1, 0))), kw
    for kw in ONE_VALUE:
        assert not refused(copy, ctypes.byref(cache8(**kw)), 64, 1, None), kw


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_tensors(monkeypatch, native):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    if not native:
        monkeypatch.setattr(serving, "_native_module", False)
    k = torch.randn(2, 3, 2, 64, device="cuda").half()
    kc, vc = (torch.zeros(4, 8, 2, 64, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    start = torch.zeros(2, dtype=torch.int32, device="cuda")
    own, other = torch.full((4, 2, 2), 0.25, device="cuda"), torch.full((4, 2, 2), 0.25, device="cuda")
    one = torch.full((), 0.25, device="cuda").expand(4, 2, 2)
    by_head = torch.full((2,), 0.25, device="cuda").expand(4, 2, 2)
    for ks, vs in ((one, other), (own, one), (own, by_head), (own[:, :1].expand(4, 2, 2), other), (own, own)):
        with pytest.raises(ng.NgpuError, match="overlap"):
            ng.kv_append(k, k, kc, vc, table, start, k_scale=ks, v_scale=vs)
    assert not kc.view(torch.uint8).any() and bool((own == 0.25).all()) and float(one[0, 0, 0]) == 0.25
    both = torch.ones(4, 2, 2, 2, device="cuda")   # keys' and values' side by side
    ng.kv_append(k, k, kc, vc, table, start, k_scale=both[:, :, 0], v_scale=both[:, :, 1])
    assert torch.equal(kc.view(torch.uint8), vc.view(torch.uint8)) and torch.equal(both[:, :, 0], both[:, :, 1])
    # one calibrated scale for all: read, and copied
    copies = torch.tensor([[0, 1, 3], [2, 3, 8]], dtype=torch.int32, device="cuda")
    was = kc.view(torch.uint8).clone()
    ng.kv_copy(kc, vc, copies, k_scale=one, v_scale=one)
    want = was.clone()
    want[1, :3], want[3] = was[0, :3], was[2]
    assert torch.equal(kc.view(torch.uint8), want) and torch.equal(vc.view(torch.uint8), want) and float(one[0, 0, 0]) == 0.25
    q = torch.randn(2, 1, 2, 64, device="cuda").half()
    lengths = torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    got = ng.attend(q, kc, vc, pages=table, lengths=lengths, k_scale=one, v_scale=one)
    want = ng.attend(q, kc, vc, pages=table, lengths=lengths, k_scale=own, v_scale=other)
    assert torch.equal(got, want)
    assert np.isfinite(got.float().cpu().numpy()).all()
