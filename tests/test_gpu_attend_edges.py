"""Attention where its inputs do not say all: what ran before a call, and scores far apart.

The bounds are those of test_gpu_attend.py, tighter ones are derived at the tests that have them.
"""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import paper_2505_22857_amd as ng  # noqa: E402
from test_gpu_attend import BF16, F16, check, ints, randn  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


def fill_lds(value):
    """Runs attention whose cache holds `value` everywhere, by workgroups that leave it in every CU's LDS."""
    kc = torch.full((64, 64, 8, 128), value, dtype=BF16, device="cuda")
    q = torch.zeros(16, 64, 32, 128, dtype=BF16, device="cuda")
    table = torch.arange(64, dtype=torch.int32, device="cuda").view(16, 4)
    ng.attend(q, kc, kc, pages=table, lengths=ints([256] * 16))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [72, 96, 128])
@pytest.mark.parametrize("T,rep", [(40, 2), (9, 1), (20, 2)])
def test_what_ran_before_does_not_matter(D, T, rep, dtype):
    """Drafts on whole tiles, by four wavefronts a block, one and two: equal bits after a call that leaves zeros in the
    chip's LDS and after one that leaves NaN there."""
    print(f"[case] attend after others D={D} T={T} x {rep} {dtype}", flush=True)
    rng = np.random.default_rng(D)
    q, kc, vc = (randn(rng, dtype, *s) for s in ((8, T, 2 * rep, D), (40, 64, 2, D), (40, 64, 2, D)))
    args = (q, kc, vc, ints(rng.permutation(40).reshape(8, 5)), ints([320, 256, 192, 128, 320, 64, 256, 320]))
    fill_lds(0.0)
    want = ng.attend(*args)
    for value in (float("nan"), 0.0, float("inf")):
        fill_lds(value)
        assert torch.equal(ng.attend(*args), want), value


@pytest.mark.parametrize("ragged", [False, True])
def test_prompts_of_96_dimensions(ragged):
    """Many blocks of rows that see each other, on whole tiles and in part."""
    n = np.array([300, 151]) if ragged else None
    check(G=0, beam=2, T=300, H=2, rep=4, D=96, page=16, own=(320, 411), q_lengths=n, seed=1)
    check(G=1, beam=2, T=300, H=2, rep=4, D=96, page=64, prefix=(70,), own=(320, 384), q_lengths=n, seed=2)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("above", [12.0, 17.2, 20.0, 40.0])
@pytest.mark.parametrize("where", [0, 3000, 8191])
def test_many_keys_far_below_one(dtype, D, above, where):
    """One key's score is far above 8191 others, which together still count.

    A half weight is off by at most half a step of 2^-24, its largest weight is at least 2^7: 2^-32 of the row's
    largest a key (bfloat16 has fp32's range).  So |out - exact| <= (2 u + 5e-4) A + 2^-32 keys max |v|, as in
    test_gpu_attend.py otherwise, and half a step of the result's own, 2^-25."""
    keys, page, S = 8192, 64, 128   # sequences enough that one workgroup takes all keys of a head
    rng = np.random.default_rng(where)
    print(f"[case] attend one key {above} above D={D} at {where} {dtype}", flush=True)
    q, kc, vc = torch.zeros(1, 1, 8, D), torch.zeros(keys, 8, D), torch.from_numpy(rng.random((keys, 8, D)))
    q[..., 0], q[..., 1] = 4.0, 1.0
    kc[:, :, 1] = torch.from_numpy(rng.random((keys, 8)))
    kc[where, :, 0], kc[where, :, 1] = above / 4, 0.5
    vc[where] = 0.0
    q, kc, vc = (x.to(dtype).cuda() for x in (q, kc, vc))
    cache = [x.view(-1, page, 8, D) for x in (kc, vc)]
    table = torch.arange(keys // page, dtype=torch.int32, device="cuda").expand(S, -1)
    out, lse = ng.attend(q.expand(S, 1, 8, D), *cache, table, ints([keys] * S), scale=1.0, return_lse=True)
    kx, vx = kc.double().cpu(), vc.double().cpu()
    x = torch.einsum("d,khd->hk", q[0, 0, 0].double().cpu(), kx)
    w = torch.softmax(x, -1)
    want = torch.einsum("hk,khd->hd", w, vx)
    u = 2.0 ** -11 if dtype == F16 else 2.0 ** -8
    bound = (2 * u + 5e-4) * want + (2.0 ** -32 * keys if dtype == F16 else 0) + 2.0 ** -25
    off = (out[:, 0].double().cpu() - want).abs()
    assert (off <= bound).all(), f"worst {float((off / bound).max())} of the bound"
    assert ((lse[:, 0].double().cpu() - torch.logsumexp(x, -1)).abs() <= 1e-3).all()
