"""A beam search whose pool has too few pages: hypotheses that find none end, and no other is the worse for it."""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import beam_search as ex  # noqa: E402
import paper_2505_22857_amd as ng  # noqa: E402
from synth import generate_model  # noqa: E402

V, BEAM, TOKENS = 128, 4, 40


@pytest.mark.parametrize("pool", [0, 1, 3, 7])
def test_search(monkeypatch, pool):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    lm = ng.NgpuLM.from_model(generate_model(V, [V, 4 * V, 4 * V], 1.0, seed=5, bos_eos=True)).upload("cuda:0")
    net = ex.Network8(ex.Shape())
    frames = torch.randn(2, 20, net.shape.width, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").half()
    lengths = torch.tensor([20, 11], dtype=torch.int32, device="cuda")
    dropped, step, steps, fork, attend, beam_step = [], 0, [], ng.kv_fork, ng.attend, lm.beam_step

    def watched_fork(pages, n, parents, *a, **kw):
        got = fork(pages, n, parents, *a, **kw)
        if parents.shape == (2, BEAM):
            dropped.append((got[1] < 0).view(2, BEAM))
        return got

    def watched_attend(q, *a, **kw):
        if q.shape[1] == 1:   # a step: who goes on has all tokens that it was given
            goes_on = kw["q_lengths"] > 0
            assert bool((kw["lengths"][goes_on] == len(dropped)).all()) and not bool((goes_on.view(2, BEAM) & dropped[-1]).any())
        got = attend(q, *a, **kw)
        assert bool(torch.isfinite(got).all())
        return got

    def watched_step(asr, weight, states, scores, **kw):
        assert bool((scores[dropped[-1]] == -torch.inf).all())
        steps.append(int((scores > -torch.inf).sum()))
        return beam_step(asr, weight, states, scores, **kw)

    monkeypatch.setattr(ng, "kv_fork", watched_fork)
    monkeypatch.setattr(ng, "attend", watched_attend)
    monkeypatch.setattr(lm, "beam_step", watched_step)
    out, scores, most = ex.search(net, lm, frames, lengths, BEAM, TOKENS, first=3, compact_every=5, pool=pool)
    assert len(steps) == TOKENS and any(bool(d.any()) for d in dropped)
    assert most <= pool + 2 * -(-20 // net.shape.page)
    assert ((out[:, :, 0] >= 0) == (scores > -torch.inf)).all()
    if pool == 0:   # the second utterance's frames leave one page over: room for one of the two first hypotheses
        assert steps[0] == 1 and (out[1] == -1).all()
