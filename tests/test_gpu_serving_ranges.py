"""Sizes between and beyond those of the operators' own tests: many drafted sequences, vocabularies on both sides of
one launch and two, prompts of thousands of tokens, rows alone and in a batch."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import paper_2505_22857_amd as ng  # noqa: E402
import test_gpu_draft as draft  # noqa: E402
import test_gpu_verify as verify  # noqa: E402
from test_gpu_attend import BF16, F16, UNIT, ints, randn  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


@pytest.mark.parametrize("temperature", [0.0, 1.0])
def test_thousands_of_drafts(temperature):
    draft.check(*draft.model(128), 5000, 2, temperature, True)


@pytest.mark.parametrize("V", [8191, 8192, 8193])
@pytest.mark.parametrize("B,K", [(1, 4), (63, 2), (64, 2), (130, 5)])
@pytest.mark.parametrize("temperature", [0.0, 1.3])
def test_one_launch_and_two(B, K, V, temperature):
    """The largest rows that one workgroup takes, and the smallest that are cut."""
    verify.check(verify.inputs(B, K, V, verify.F32, B + V), temperature)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("past", [0, 777])
def test_long_prompts(D, past, dtype):
    """2049 tokens that see each other, and 777 before them; the bound is that of test_gpu_attend.py, with half weights
    down to 2^-32 of the largest."""
    T, H, rep, page = 2049, 1, 3, 64
    n = past + T
    rng = np.random.default_rng(D + past)
    print(f"[case] attend prompt of {T} after {past} D={D} {dtype}", flush=True)
    width = -(-n // page)
    table = rng.permutation(width)
    q, kc, vc = (randn(rng, dtype, *s) for s in ((1, T, H * rep, D), (width, page, H, D), (width, page, H, D)))
    out, lse = ng.attend(q, kc, vc, ints([table]), ints([n]), return_lse=True)
    k, v = (x[torch.from_numpy(table).cuda()].reshape(-1, D)[:n].double().cpu() for x in (kc, vc))
    hidden = torch.arange(n) > past + torch.arange(T)[:, None]
    u = UNIT[dtype]
    for h in range(H * rep):
        x = (q[0, :, h].double().cpu() @ k.T.contiguous()) / D ** 0.5
        x.masked_fill_(hidden, -np.inf)
        w = torch.softmax(x, -1)
        bound = (2 * u + 5e-4) * (w @ v.abs()) + 2.0 ** -25 + (2.0 ** -32 * n * float(v.abs().max()) if dtype == F16 else 0)
        assert ((out[0, :, h].double().cpu() - w @ v).abs() <= bound).all()
        assert ((lse[0, :, h].double().cpu() - torch.logsumexp(x, -1)).abs() <= 1e-3).all()


def test_rows_alone_and_in_a_batch():
    """A sequence by itself is cut differently: within both results' bounds of each other."""
    rng = np.random.default_rng(8)
    S, T, D = 16, 3, 128
    q, kc, vc = (randn(rng, BF16, *s) for s in ((S, T, 8, D), (300, 16, 2, D), (300, 16, 2, D)))
    pages, prefix = rng.permutation(300)[:64].reshape(S, 4), rng.permutation(300)[:200].reshape(2, 100)
    lengths, prefix_lengths = rng.integers(T, 64, S), np.array([1600, 900])
    all_rows = ng.attend(q, kc, vc, ints(pages), ints(lengths), ints(prefix), ints(prefix_lengths)).double()
    most = ng.attend(q, kc, vc.abs(), ints(pages), ints(lengths), ints(prefix), ints(prefix_lengths)).double()
    for s in range(S):
        g = s // (S // 2)
        one = ng.attend(q[s:s + 1], kc, vc, ints(pages[s:s + 1]), ints(lengths[s:s + 1]), ints(prefix[g:g + 1]),
                        ints(prefix_lengths[g:g + 1])).double()
        # (`most` is the softmax's sum of |v|, rounded as much itself)
        assert ((one[0] - all_rows[s]).abs() <= 2 * (2 * 2.0 ** -8 + 5e-4) * 1.02 * most[s]).all(), s
