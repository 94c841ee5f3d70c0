"""Drafting from the n-gram model against the oracle's scores and a softmax in 64 bits.

Tokens and states have to be equal.  The log-probabilities are (x - m) / T -
log(sum): two fp32 roundings of the first term (2^-23 of its size, doubled
below for the oracle's own), and a sum whose terms are off by an ulp or two of
the exponential, by 2^-24 of their exponent's size and by at most 40 additions
in a row: below 1e-5 for the sizes here.
"""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import paper_2505_22857_amd as ng  # noqa: E402
import serving_reference as ref  # noqa: E402
from oracle import Oracle  # noqa: E402
from synth import generate_model, tiny_model, uniform_states  # noqa: E402

_MODELS = {}


def model(V, order=3, bos_eos=False):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    key = V, order, bos_eos
    if key not in _MODELS:
        m = generate_model(V, [V, 3 * V, 2 * V, 2 * V, V][:order], 1.0, seed=V, bos_eos=bos_eos)
        _MODELS[key] = (m, ng.NgpuLM.from_model(m).upload("cuda:0"), Oracle.from_model(m))
    return _MODELS[key]


def dev(x):
    return None if x is None else torch.from_numpy(x).cuda()


def check(m, lm, o, B, k, temperature, last, seed=0, noise=None):
    rng = np.random.default_rng(seed)
    V = m.vocab_size
    states = uniform_states(m, B, seed=seed + 1)
    before = rng.integers(-1, V, B).astype(np.int32) if last else None
    if temperature and noise is None:
        noise = rng.standard_exponential((B, k, V)).astype(np.float32)
    print(f"[case] draft V={V} B={B} k={k} T={temperature} last={last}", flush=True)
    st = dev(states)
    tok, after, rows = lm.draft(st, k, noise=dev(noise), temperature=temperature, last=dev(before))
    wt, wa, wr = ref.draft(o, states, k, noise, temperature, before)
    assert np.array_equal(tok.cpu().numpy(), wt)
    assert np.array_equal(after.cpu().numpy(), wa)
    assert np.array_equal(st.cpu().numpy(), states)      # read only
    if temperature:
        got = rows.cpu().numpy()
        assert np.all(np.abs(got - wr) <= 1e-5 + 2.0 ** -22 * np.abs(wr))
    else:
        assert rows is None
    assert lm.check_states() == 0


@pytest.mark.parametrize("V,B,k", [
    (1, 3, 2), (5, 4, 3), (63, 3, 5), (64, 3, 4), (65, 3, 4), (256, 17, 5), (257, 9, 4), (512, 5, 3), (513, 5, 4),
    (1000, 33, 5), (1024, 40, 8), (1025, 7, 3), (2047, 5, 4), (2048, 5, 3), (2049, 5, 3), (4096, 5, 3), (4097, 3, 3),
    (8000, 3, 3), (8192, 3, 2), (128, 2, 63)])
@pytest.mark.parametrize("temperature", [0.0, 1.0, 0.6])
def test_draft(V, B, k, temperature):
    check(*model(V), B, k, temperature, last=V % 2 == 0, seed=V)


@pytest.mark.parametrize("order", [1, 2, 5])
@pytest.mark.parametrize("V", [40, 700, 1500])
def test_orders_and_forced_tokens(V, order):
    for last in (False, True):
        check(*model(V, order), 50, 4, 0.9, last, seed=order)


def test_markers_and_unlisted_unigrams():
    check(*model(300, 3, True), 20, 4, 1.0, True)
    m = tiny_model(9, 3, seed=21, n_unigrams=6)
    check(m, ng.NgpuLM.from_model(m).upload("cuda:0"), Oracle.from_model(m), 30, 6, 1.0, True)


@pytest.mark.parametrize("V", [50, 1024, 3000])
def test_odd_noise(V):
    """Zero noise wins (the lowest of several), infinite and NaN noise lose, rows and
    sequences may have any stride."""
    m, lm, o = model(V)
    rng = np.random.default_rng(V)
    B, k = 6, 3
    noise = rng.standard_exponential((B, k, V)).astype(np.float32)
    noise[0, :, [7, 11, V - 1]] = 0.0
    noise[1, :, 1:] = np.nan
    noise[2, :, :V - 1] = np.inf
    noise[3] = np.nan
    check(m, lm, o, B, k, 1.0, True, noise=noise)
    wide = torch.empty(B, k + 1, V + 3, device="cuda")
    wide[:, :k, 1:V + 1] = dev(noise)
    states = uniform_states(m, B, seed=1)
    a = lm.draft(dev(states), k, noise=wide[:, :k, 1:V + 1])
    b = lm.draft(dev(states), k, noise=dev(noise))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    one = dev(noise[4, 0]).expand(B, k, V)               # one row for all (strides of 0)
    a = lm.draft(dev(states), k, noise=one)
    b = lm.draft(dev(states), k, noise=one.contiguous())
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_temperatures_far_from_one():
    m, lm, o = model(700)
    check(m, lm, o, 8, 3, 50.0, False)
    states = uniform_states(m, 8, seed=2)
    cold = lm.draft(dev(states), 4, noise=torch.ones(8, 4, 700, device="cuda"), temperature=1e-6)
    greedy = lm.draft(dev(states), 4, temperature=0.0)
    assert torch.equal(cold[0], greedy[0]) and torch.equal(cold[1], greedy[1])


@pytest.mark.parametrize("V", [100, 2000])
def test_bad_states_and_tokens_are_counted(V):
    m, lm, _ = model(V)
    states = torch.tensor([0, -1, m.num_states, 0, 0], dtype=torch.int32, device="cuda")
    last = torch.tensor([-1, 0, 0, V, -2], dtype=torch.int32, device="cuda")
    tok, after, rows = lm.draft(states, 3, noise=torch.ones(5, 3, V, device="cuda"), last=last)
    assert (tok[1:] == -1).all() and (after[1:] == -1).all() and torch.isnan(rows[1:]).all()
    assert (tok[0] >= 0).all() and not torch.isnan(rows[0]).any()
    assert lm.check_states() == 4


def test_draft_follows_the_distribution():
    """20000 drafts of one token from one state: frequencies within five standard deviations."""
    m, lm, o = model(40)
    n = 20000
    g = torch.Generator(device="cuda").manual_seed(5)
    noise = torch.empty(n, 1, 40, device="cuda").exponential_(generator=g)
    tok, _, rows = lm.draft(torch.full((n,), 3, dtype=torch.int32, device="cuda"), 1, noise=noise, temperature=1.3)
    p = rows[0, 0].double().exp().cpu().numpy()
    assert abs(p.sum() - 1) < 1e-5
    count = np.bincount(tok[:, 0].cpu().numpy(), minlength=40)
    assert np.all(np.abs(count - n * p) <= 5 * np.sqrt(n * p * (1 - p)) + 1)


def test_many_sequences():
    m, lm, o = model(128)
    check(m, lm, o, 5000, 2, 1.0, True)


def test_other_stream():
    m, lm, _ = model(1024)
    states = dev(uniform_states(m, 30, seed=3))
    noise = torch.empty(30, 4, 1024, device="cuda").exponential_()
    want = lm.draft(states, 4, noise=noise)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = lm.draft(states, 4, noise=noise, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    m, lm, _ = model(40)
    states = torch.zeros(4, dtype=torch.int32, device="cuda")
    noise = torch.ones(4, 2, 40, device="cuda")
    for k in (0, -1, 64):
        with pytest.raises(ValueError):
            lm.draft(states, k, temperature=0.0)
    with pytest.raises(ValueError):
        lm.draft(states, 2)
    with pytest.raises(ValueError):
        lm.draft(states, 3, noise=noise)
    with pytest.raises(TypeError):
        lm.draft(states.long(), 2, noise=noise)
    with pytest.raises(TypeError):
        lm.draft(states, 2, noise=noise.double())
    with pytest.raises(TypeError):
        lm.draft(states, 2, noise=noise.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(ValueError):
        lm.draft(states, 2, noise=noise, last=states[:3])
    for t in (-1.0, float("nan"), float("inf"), 1e-9):
        with pytest.raises(ng.NgpuError):
            lm.draft(states, 2, noise=noise, temperature=t)
    tok, after, rows = lm.draft(states[:0], 2, noise=noise[:0])
    assert tok.shape == (0, 2) and after.shape == (0, 3) and rows.shape == (0, 2, 40)


def test_rows_past_the_caches():
    """So many rows that they are written past the caches."""
    check(*model(2048), 700, 6, 1.0, True)


@pytest.mark.parametrize("V", [1100, 2048])
@pytest.mark.parametrize("B", [512, 513])
def test_many_sequences(V, B):
    """Both sides of the batch from which fewer wavefronts take a sequence."""
    check(*model(V), B, 2, 1.0, True)
    check(*model(V), B, 2, 0.0, False)
