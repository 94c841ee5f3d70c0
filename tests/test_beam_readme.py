"""The beam search's snippet of README.md, run step after step with stand-ins for the network and the operators: each step
goes on from the one before, and a hypothesis that finds no pages ends."""

import os
import re
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_steps_follow_each_other():
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    code, = [b for b in blocks if "beam_step" in b]
    appended, ordered = [], []
    drops = iter([None, 1, None])   # the row that finds no pages, of each step

    def beam_step(log_p, lam, st, scores, last, mode):
        ordered.append(scores.clone())
        return last, torch.arange(3, dtype=torch.int32)[None], scores, st

    def kv_fork(pages, lengths, parents, refs, page_size, tokens):
        after, row = lengths.clamp(min=0), next(drops)
        if row is not None:
            after[row] = -1
        return pages, after, None

    def kv_append(k, v, kc, vc, pages, start, q, lengths, **kw):
        appended.append((start.tolist(), lengths.tolist()))
        return q

    def attend(q, *a, lengths, q_lengths, **kw):
        assert (lengths >= q_lengths).all()

    ng = SimpleNamespace(kv_fork=kv_fork, kv_append=kv_append, attend=attend, kv_copy=lambda *a, **kw: None,
                         NGPU_FUSION_AED=3)
    names = dict.fromkeys("log_p st parents pages refs page_size k_cache v_cache k_scale v_scale k v q cos sin prefix "
                          "prefix_lengths".split())
    names |= dict(torch=torch, ng=ng, lm=SimpleNamespace(beam_step=beam_step, vocab_size=9), scores=torch.zeros(1, 3),
                  classes=torch.tensor([[4, 5, 9]], dtype=torch.int32), lengths=torch.tensor([7, 7, 7], dtype=torch.int32))
    for _ in range(3):
        exec(code, names)
    # the third has ended (class 9); the second is dropped in the second step
    assert appended == [([7, 7, 7], [1, 1, 0]), ([8, 0, 7], [1, 0, 0]), ([9, 0, 7], [1, 1, 0])]
    assert [s[0].tolist() for s in ordered] == [[0, 0, 0], [0, 0, 0], [0, -torch.inf, 0]]
