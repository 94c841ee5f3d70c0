"""The beam step against the oracle's scores and a stable sort.

Sums are rounded as the operator's definition says, so classes, parents, states and sums have to be equal."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import beam_reference as ref  # noqa: E402
import paper_2505_22857_amd as ng  # noqa: E402
from oracle import Oracle  # noqa: E402
from synth import generate_model, tiny_model, uniform_states  # noqa: E402

_MODELS = {}
MODES = {"plain": ng.NGPU_FUSION_PLAIN, "transducer": ng.NGPU_FUSION_TRANSDUCER, "aed": ng.NGPU_FUSION_AED}


def model(V, order=3, bos_eos=False):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    key = V, order, bos_eos
    if key not in _MODELS:
        m = generate_model(V, [V, 3 * V, 2 * V, 2 * V, V][:order], 1.0, seed=V + 1, bos_eos=bos_eos)
        _MODELS[key] = (m, ng.NgpuLM.from_model(m).upload("cuda:0"), Oracle.from_model(m))
    return _MODELS[key]


def dev(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def inputs(m, B, W, mode, seed, ended=0.0, empty=0.0, coarse=False):
    rng = np.random.default_rng(seed)
    C = m.vocab_size + (mode != "plain")
    asr = rng.standard_normal((B, W, C)) * 3
    asr = (asr - np.log(np.exp(asr).sum(-1, keepdims=True))).astype(np.float32)
    scores = (-rng.random((B, W)) * 8 - 20).astype(np.float32)
    if coarse:   # many equal sums
        asr, scores = np.round(asr), np.round(scores / 4) * 4
    scores[rng.random((B, W)) < empty] = -np.inf
    states = uniform_states(m, B * W, seed=seed).reshape(B, W)
    last = np.where(rng.random((B, W)) < ended, m.vocab_size, rng.integers(0, m.vocab_size, (B, W))).astype(np.int32)
    return asr, states, scores, last if mode == "aed" and ended else None


def check(m, lm, o, asr, states, scores, last, k, mode, lam=0.7, on=None, bad=0):
    print(f"[case] beam V={m.vocab_size} B={states.shape[0]} W={states.shape[1]} k={k} {mode}", flush=True)
    want = ref.beam_step(o, m.vocab_size, asr, lam, states, scores, k, mode, last)
    got = lm.beam_step(dev(asr) if on is None else on, lam, dev(states), dev(scores), k=k, last=dev(last), mode=MODES[mode])
    for name, x, y in zip(("classes", "parents", "scores", "states"), got, want):
        assert np.array_equal(x.cpu().numpy(), y), name
    assert lm.check_states() == want[4] == bad
    return got


@pytest.mark.parametrize("V,B,W,k", [
    (1, 3, 2, 2), (2, 2, 3, 5), (5, 4, 3, 3), (63, 3, 4, 4), (64, 3, 5, 8), (65, 2, 2, 3), (200, 9, 64, 64), (256, 5, 4, 4),
    (257, 3, 16, 16), (400, 20, 64, 40), (400, 7, 8, 8), (512, 3, 8, 33), (513, 5, 4, 4), (700, 130, 8, 8), (1000, 4, 8, 8),
    (1024, 6, 8, 8), (1024, 150, 8, 8), (1025, 3, 4, 4), (1200, 100, 8, 5), (1500, 100, 8, 4), (2000, 2, 10, 10),
    (2049, 4, 4, 4), (4000, 20, 8, 8), (5000, 2, 4, 4), (6144, 2, 3, 3), (8000, 1, 1, 1), (8192, 3, 16, 16), (8192, 1, 1, 64)])
@pytest.mark.parametrize("mode", ["plain", "transducer", "aed"])
def test_steps(V, B, W, k, mode):
    m = model(V, 3, mode == "aed")
    check(*m, *inputs(m[0], B, W, mode, seed=V + k, ended=0.2, empty=0.1), k, mode)


@pytest.mark.parametrize("order", [1, 2, 5])
@pytest.mark.parametrize("V", [40, 700, 1500])
def test_orders(V, order):
    m = model(V, order, True)
    for mode in MODES:
        check(*m, *inputs(m[0], 8, 6, mode, seed=order, ended=0.3), 6, mode, lam=1.3)


@pytest.mark.parametrize("V", [3, 100, 1000, 3000])
@pytest.mark.parametrize("W,k", [(1, 1), (1, 64), (64, 1), (64, 64), (7, 31)])
def test_widths_and_ties(V, W, k):
    """Without the model, sums of whole numbers: most are shared by many continuations."""
    m = model(V, 3, True)
    for mode in ("plain", "aed"):
        check(*m, *inputs(m[0], 3, W, mode, seed=k, ended=0.2, empty=0.2, coarse=True), k, mode, lam=0.0)


def test_all_alike():
    """Every sum the same: the lowest places, in order; and signed zeros, which are equal."""
    for V in (90, 1024, 2500):
        m = model(V, 2, True)
        for value in (-1.0, 0.0, -0.0):
            asr = np.full((2, 5, V + 1), value, np.float32)
            asr[:, :, ::2] = -value if value == 0 else value
            scores, states = np.full((2, 5), value, np.float32), uniform_states(m[0], 10, seed=1).reshape(2, 5)
            got = check(*m, asr, states, scores, np.zeros((2, 5), np.int32), 64, "aed", lam=0.0)
            assert got[0][0].tolist() == list(range(64)) and not got[1].any()


@pytest.mark.parametrize("V,W", [(256, 16), (250, 9), (512, 8), (300, 5), (1024, 4), (1000, 3), (2048, 2), (1900, 1),
                                 (1024, 8), (900, 7), (1000, 5)])
def test_one_launch(V, W):
    """All that one launch takes, up to its most wavefronts: sums that differ, that are few, and that are one."""
    m = model(V, 3, True)
    for k in (1, W, 64):
        check(*m, *inputs(m[0], 5, W, "aed", seed=k, ended=0.15, empty=0.1), k, "aed")
    check(*m, *inputs(m[0], 4, W, "aed", seed=3, ended=0.1, coarse=True), 40, "aed", lam=0.0)
    asr, states = np.full((2, W, V + 1), -2.0, np.float32), uniform_states(m[0], 2 * W, seed=1).reshape(2, W)
    scores, last = np.full((2, W), -7.0, np.float32), np.zeros((2, W), np.int32)
    check(*m, asr, states, scores, last, 64, "aed", lam=0.0)
    scores[:, 0], asr[0, W - 1, 17:19], asr[1, 0, V] = -9.0, -1.5, 3.0   # a few above those that are alike
    check(*m, asr, states, scores, last, 64, "aed", lam=0.0)
    last[0] = V                                                         # nothing but ended ones
    check(*m, asr, states, scores, last, 64, "aed", lam=0.0)


@pytest.mark.parametrize("V,W", [(200, 8), (200, 9), (500, 4), (500, 5), (1000, 2), (1000, 3), (1000, 8), (1500, 1),
                                 (1500, 2)])
def test_more_utterances_than_compute_units(V, W):
    m = model(V)
    for B in (256, 257):
        check(*m, *inputs(m[0], B, W, "transducer", seed=B), W, "transducer")


def test_infinities_and_nan():
    m = model(300, 3, True)
    asr, states, scores, last = inputs(m[0], 6, 4, "aed", seed=2, ended=0.2)
    asr[0, :, 5:] = -np.inf                      # a few classes left
    asr[1] = -np.inf                             # nothing
    asr[2, 0, 7], asr[2, 1, 8] = np.inf, np.nan
    asr[3] = np.nan
    asr[3, 2, 299], asr[3, 3, 300] = -4.0, np.inf
    scores[4] = [-np.inf, np.nan, np.inf, -1e30]
    asr[4, 2, 3] = -np.inf                       # inf - inf
    scores[5] = -np.inf
    for mode, k in (("aed", 4), ("aed", 64), ("transducer", 9), ("plain", 9)):
        check(*m, asr, states, scores, last if mode == "aed" else None, k, mode)


def test_no_continuation_and_left_over_places():
    m = model(2, 1, True)
    asr = np.array([[[-1, -np.inf, -2.0]]], np.float32)
    got = check(*m, asr, np.zeros((1, 1), np.int32), np.zeros((1, 1), np.float32), None, 5, "aed", lam=0.0)
    assert got[0].tolist() == [[0, 2, -1, -1, -1]] and got[3].tolist()[0][2:] == [0, 0, 0]
    ended = np.full((1, 2), 2, np.int32)         # all ended, one of them empty: the other goes on alone
    got = check(*m, np.zeros((1, 2, 3), np.float32), np.array([[7, -9]], np.int32), np.array([[-3.5, -np.inf]], np.float32),
                ended, 2, "aed")
    assert got[2].tolist() == [[-3.5, -np.inf]] and got[3].tolist() == [[7, 0]]   # its state is not looked at


def test_states_outside():
    """Those of live hypotheses are counted and give nothing."""
    m = model(100)
    asr, states, scores, _ = inputs(m[0], 3, 4, "plain", seed=4)
    states[0, 1], states[1, 2], states[2] = -1, m[2].num_states, 2 ** 31 - 1
    scores[2, :3] = -np.inf
    check(*m, asr, states, scores, None, 4, "plain", bad=3)


def test_unlisted_unigrams():
    m = tiny_model(9, 3, seed=21, n_unigrams=6)
    check(m, ng.NgpuLM.from_model(m).upload("cuda:0"), Oracle.from_model(m), *inputs(m, 5, 4, "plain", seed=5), 4, "plain")


def test_strides():
    """One frame for all hypotheses or utterances, rows of a longer one, and a row that begins anywhere."""
    m = model(130, 3, True)
    asr, states, scores, last = inputs(m[0], 5, 6, "aed", seed=6, ended=0.1)
    frame = asr[:, :1].repeat(6, 1)
    check(*m, frame, states, scores, last, 6, "aed", on=dev(asr[:, :1]).expand(5, 6, 131))
    check(*m, asr[:1].repeat(5, 0), states, scores, last, 6, "aed", on=dev(asr[:1]).expand(5, 6, 131))
    wide = np.concatenate([asr, np.full((5, 6, 10), 9.0, np.float32)], -1)     # classes past V + 1 are not looked at
    check(*m, asr, states, scores, last, 6, "aed", on=dev(wide))
    check(*m, asr, states, scores, last, 6, "aed", on=dev(wide)[:, :, :131])
    check(*m, asr, states, scores, last, 6, "aed", on=dev(wide.transpose(1, 0, 2)).transpose(0, 1))
    odd = torch.empty(asr.size + 1, device="cuda")
    odd[1:] = dev(asr).flatten()
    check(*m, asr, states, scores, last, 6, "aed", on=odd[1:].view(5, 6, 131))


def test_many_hypotheses():
    """More than one launch's shapes: every rule on the number of hypotheses."""
    for V, B, W in ((300, 40, 32), (600, 300, 4), (900, 300, 4), (1100, 200, 4), (1400, 200, 4), (3000, 33, 4)):
        m = model(V)
        check(*m, *inputs(m[0], B, W, "plain", seed=V), min(W, 8), "plain")


def test_empty_batch_and_refusals():
    m, lm, _ = model(100)
    z = torch.zeros
    out = lm.beam_step(z(0, 3, 100, device="cuda"), 0.5, z(0, 3, dtype=torch.int32, device="cuda"), z(0, 3, device="cuda"))
    assert [tuple(x.shape) for x in out] == [(0, 3)] * 4
    asr, st, sc = z(2, 3, 101, device="cuda"), z(2, 3, dtype=torch.int32, device="cuda"), z(2, 3, device="cuda")
    with pytest.raises(ng.NgpuError, match="beam step"):
        lm.beam_step(asr, 0.5, st, sc, mode=ng.NGPU_FUSION_CTC)
    with pytest.raises(ng.NgpuError, match="</s>"):
        lm.beam_step(asr, 0.5, st, sc, mode=ng.NGPU_FUSION_AED)
    with pytest.raises(ng.NgpuError, match="AED"):
        lm.beam_step(asr, 0.5, st, sc, last=st)
    with pytest.raises(ng.NgpuError, match="finite"):
        lm.beam_step(asr, float("nan"), st, sc)
    for bad in (dict(k=0), dict(k=65)):
        with pytest.raises(ValueError):
            lm.beam_step(asr, 0.5, st, sc, **bad)
    with pytest.raises(ValueError, match="classes"):
        lm.beam_step(asr[:, :, :100], 0.5, st, sc, mode=ng.NGPU_FUSION_TRANSDUCER)
    with pytest.raises(ValueError, match="shape"):
        lm.beam_step(asr, 0.5, st[:1], sc)
    with pytest.raises(TypeError):
        lm.beam_step(asr, 0.5, st.long(), sc)
    with pytest.raises(TypeError):
        lm.beam_step(asr.half(), 0.5, st, sc)
    for tracked in ((asr.clone().requires_grad_(), sc), (asr, sc.clone().requires_grad_())):
        for stream in (None, torch.cuda.current_stream()):
            with pytest.raises(TypeError, match="gradient"):
                lm.beam_step(tracked[0], 0.5, st, tracked[1], stream=stream)
        with torch.no_grad():
            lm.beam_step(tracked[0], 0.5, st, tracked[1])
    with pytest.raises(TypeError, match="stride"):
        lm.beam_step(z(2, 3, 202, device="cuda")[:, :, ::2], 0.5, st, sc)
    with pytest.raises(TypeError):
        lm.beam_step(asr.cpu(), 0.5, st, sc)
    assert lm.check_states() == 0


def test_on_a_stream_of_its_own_and_in_a_graph():
    m = model(500, 3, True)
    asr, states, scores, last = inputs(m[0], 7, 8, "aed", seed=8, ended=0.1)
    a, st, sc, la = (dev(x) for x in (asr, states, scores, last))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = m[1].beam_step(a, 0.7, st, sc, last=la, mode=ng.NGPU_FUSION_AED, stream=side)
    side.synchronize()
    want = ref.beam_step(m[2], 500, asr, 0.7, states, scores, 8, "aed", last)
    for x, y in zip(got, want):
        assert np.array_equal(x.cpu().numpy(), y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):   # two steps, one after the other
        first = m[1].beam_step(a, 0.7, st, sc, last=la, mode=ng.NGPU_FUSION_AED)
        second = m[1].beam_step(a, 0.7, first[3], first[2], last=first[0], mode=ng.NGPU_FUSION_AED)
    for seed in range(3):
        asr, states, scores, last = inputs(m[0], 7, 8, "aed", seed=20 + seed, ended=0.1)
        for x, y in ((a, asr), (st, states), (sc, scores), (la, last)):
            x.copy_(dev(y))
        graph.replay()
        m[1].beam_step(a, 0.7, st, sc)   # eager work between
        torch.cuda.synchronize()
        one = ref.beam_step(m[2], 500, asr, 0.7, states, scores, 8, "aed", last)
        two = ref.beam_step(m[2], 500, asr, 0.7, one[3], one[2], 8, "aed", one[0])
        for got, want in ((first, one), (second, two)):
            for x, y in zip(got, want):
                assert np.array_equal(x.cpu().numpy(), y)
