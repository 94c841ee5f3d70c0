"""Blocks whose scale is a number far below those that an append writes, as a program's own calibration may leave them."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import beam_reference as ref  # noqa: E402
import paper_2505_22857_amd as ng  # noqa: E402

VALUES = ref.e4m3_values()


@pytest.mark.parametrize("D", [64, 33])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("size", [0.0, 1e-33, 1e-29, 1.0])
@pytest.mark.parametrize("had", [2.0 ** -98, 2.0 ** -100, 2.0 ** -101, 2.0 ** -105, 1e-31, 3e-33, 2.0 ** -126, 2.0 ** -149])
def test_entries_before_keep_their_values(had, size, dtype, D):
    """From the definition: the block's scale stays where it is 2^-100 at least and holds the new tokens, else it is the least
    power of two from 2^-100 on that does, and the entries before stand for what they stood for, rounded to it."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    rng = np.random.default_rng(D)
    page, lead, H = 8, 5, 2
    bits = [rng.integers(0, 127, (3, page, H, D), dtype=np.uint8) for _ in range(2)]
    caches = [torch.from_numpy(b).cuda() for b in bits]
    scales = [torch.full((3, 1, H), had, device="cuda") for _ in range(2)]
    x = (torch.from_numpy(rng.uniform(0.5, 1.0, (1, 2, H, D))) * size).float().cuda().to(dtype)
    ng.kv_append(x, -x, *(c.view(torch.float8_e4m3fn) for c in caches), torch.tensor([[1]], dtype=torch.int32, device="cuda"),
                 torch.tensor([lead], dtype=torch.int32, device="cuda"), k_scale=scales[0], v_scale=scales[1])
    new = x[0].double().cpu().numpy()
    had = float(np.float32(had))
    for sign, was, cache, scale in zip((1, -1), bits, caches, scales):
        got, scale = VALUES[cache.cpu().numpy()], scale.double().cpu().numpy()
        for h in range(H):
            most = abs(new[:, h]).max()
            now = had
            if had < 2.0 ** -100 or most > 448 * had:
                now = 2.0 ** -100
                while most > 448 * now:
                    now *= 2
            assert scale[1, 0, h] == now
            before = VALUES[was[1, :lead, h]] * (had / now)   # (64 bits hold every quotient and product here)
            assert np.array_equal(got[1, :lead, h], before if now == had else ref.to_e4m3(before))
            assert np.array_equal(got[1, lead:lead + 2, h], ref.to_e4m3(sign * new[:, h] / now))
        assert np.array_equal(got[[0, 2]], VALUES[was[[0, 2]]]) and (scale[[0, 2]] == had).all()
