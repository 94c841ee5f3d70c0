"""A beam search's operators together, as a network's search calls them: every call against its reference, and each
hypothesis's cached values against those that its own tokens had."""

import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import beam_reference as ref  # noqa: E402
import beam_search as ex  # noqa: E402
import paper_2505_22857_amd as ng  # noqa: E402
import serving_reference  # noqa: E402
from oracle import Oracle  # noqa: E402
from synth import generate_model  # noqa: E402

VALUES = ref.e4m3_values()
V = 128


def host(x):
    return x.detach().cpu().numpy()


def elements(x):
    return VALUES[host(x.view(torch.uint8))]


class Watch:
    """Stands between the search and the operators."""

    def __init__(self, monkeypatch, lm, oracle, beam, layers, block):
        self.oracle, self.beam, self.layers, self.block = oracle, beam, layers, block
        self.values = [{} for _ in range(layers)]    # of the hypotheses' tokens, by layer and row
        self.calls, self.shared, self.layer = {}, 0, 0
        self.own = {}
        for name in ("kv_fork", "kv_copy", "kv_compact", "kv_append", "attend"):
            self.own[name] = getattr(ng, name)
            monkeypatch.setattr(ng, name, self.counted(name))
        self.own["beam_step"] = lm.beam_step
        monkeypatch.setattr(lm, "beam_step", self.counted("beam_step"))

    def counted(self, name):
        def call(*a, **kw):
            self.calls[name] = self.calls.get(name, 0) + 1
            return getattr(self, name)(*a, **kw)
        return call

    def beam_step(self, asr, weight, states, scores, last=None, mode=None):
        got = self.own["beam_step"](asr, weight, states, scores, last=last, mode=mode)
        want = ref.beam_step(self.oracle, V, host(asr), weight, host(states), host(scores), scores.shape[1], "aed", host(last))
        for x, y in zip(got, want):
            assert np.array_equal(host(x), y)
        return got

    def kv_fork(self, pages, lengths, parents, refs, page, tokens=0):
        K = parents.shape[1]
        wanted = host(tokens) if hasattr(tokens, "dim") else np.full(parents.shape, tokens)
        want = ref.fork(host(pages), host(lengths), host(parents), host(refs), page, wanted)
        got = self.own["kv_fork"](pages, lengths, parents, refs, page, tokens=tokens)
        for x, y in zip((*got, refs), want):
            assert np.array_equal(host(x), y)
        if K == self.beam:   # the hypotheses
            self.shared += int((want[2][:, 0] >= 0).sum())
            rows = [(i // K * self.beam + p) if p >= 0 else None for i, p in enumerate(host(parents).ravel().tolist())]
            self.values = [{i: list(v.get(r, [])) for i, r in enumerate(rows) if r is not None} for v in self.values]
        return got

    def kv_copy(self, kc, vc, copies, k_scale=None, v_scale=None):
        caches = (kc.view(torch.uint8), vc.view(torch.uint8), k_scale, v_scale)
        want = []
        for x in caches:
            c = host(copies).copy()
            if x.dim() == 3:   # all scales of a page
                c[:, 2] = x.shape[1]
            want.append(ref.copy(host(x), c))
        self.own["kv_copy"](kc, vc, copies, k_scale=k_scale, v_scale=v_scale)
        for x, y in zip(caches, want):
            assert np.array_equal(host(x), y)

    def kv_compact(self, refs, page, tables=()):
        want = ref.compact(host(refs), page, [host(t) for t in tables])
        got = self.own["kv_compact"](refs, page, tables=tables)
        for x, y in zip((*got, refs, *tables), (*want[:3], *want[3])):
            assert np.array_equal(host(x), y)
        return got

    def kv_append(self, k, v, kc, vc, pages, start, q=None, lengths=None, k_scale=None, v_scale=None, **kw):
        tables, at, counts = host(pages), host(start), host(lengths)
        was = elements(vc), host(v_scale)
        out = self.own["kv_append"](k, v, kc, vc, pages, start, q=q, lengths=lengths, k_scale=k_scale, v_scale=v_scale, **kw)
        want, scale, known = ref.append8(host(v.float()), *was, tables, at, counts)
        got = elements(vc)
        assert np.array_equal(got, want, equal_nan=True) and np.array_equal(host(v_scale), scale)
        if k.shape[1] == 1:   # a step's tokens, not the frames
            page, mine = vc.shape[1], self.values[self.layer]
            for s in range(len(v)):
                if counts[s] == 0:
                    assert not out[s].any()
                    continue
                mine[s].append(host(v[s, 0].double()))
                assert len(mine[s]) == at[s] + 1
                # A value is rounded once at its block's scale (2^-4 of it, or half a step 2^-9 of the smallest) and, as
                # the scale grows by powers of two, once more a growth, which only rounds what is below the least normal
                # one: half a step each time, the sum of which is below twice the last, 2^-9 of the scale in all.
                n = len(mine[s])
                p, e = tables[s, np.arange(n) // page], np.arange(n) % page
                of = scale[p, e // self.block][..., None]
                assert (abs(got[p, e] * of - np.array(mine[s])) <= 2.0 ** -4 * abs(np.array(mine[s])) + 2.0 ** -9 * of).all()
        return out

    def attend(self, q, kc, vc, pages=None, lengths=None, prefix_pages=None, prefix_lengths=None, q_lengths=None, k_scale=None,
               v_scale=None):
        got = self.own["attend"](q, kc, vc, pages=pages, lengths=lengths, prefix_pages=prefix_pages,
                                 prefix_lengths=prefix_lengths, q_lengths=q_lengths, k_scale=k_scale, v_scale=v_scale)
        meant = [elements(x) * host(s.double()).repeat(self.block, 1)[..., None] for x, s in ((kc, k_scale), (vc, v_scale))]
        last = None if prefix_pages is None else (host(prefix_pages), host(prefix_lengths))
        want, _, size = serving_reference.attend(host(q.double()), *meant, host(pages), host(lengths), *(last or (None, None)),
                                                 host(q_lengths))
        # half precision: one rounding of the output (2^-11), weights of two bfloat16 parts (2^-16), scores of fp32 whose
        # errors move a weight by less than 5e-4 of its size
        assert (abs(host(got.double()) - want) <= (2.0 ** -11 + 2.0 ** -16 + 5e-4) * size + 2.0 ** -25).all()
        self.layer = (self.layer + 1) % self.layers
        return got


@pytest.mark.parametrize("beam,compact_every", [(5, 0), (4, 3), (1, 2)])
def test_search(monkeypatch, beam, compact_every):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    m = generate_model(V, [V, 4 * V, 4 * V], 1.0, seed=5, bos_eos=True)
    lm = ng.NgpuLM.from_model(m).upload("cuda:0")
    net = ex.Network8(ex.Shape())
    g = torch.Generator(device="cuda").manual_seed(1)
    frames = torch.randn(2, 40, net.shape.width, generator=g, device="cuda").half()
    lengths = torch.tensor([40, 21], dtype=torch.int32, device="cuda")
    alone = ex.search(net, lm, frames, lengths, beam, 20, first=3)
    watch = Watch(monkeypatch, lm, Oracle.from_model(m), beam, len(net.layers), net.block)
    out, scores, most = ex.search(net, lm, frames, lengths, beam, 20, first=3, compact_every=compact_every)
    assert lm.check_states() == 0
    # where pages lie changes no result
    assert torch.equal(out, alone[0]) and torch.equal(scores, alone[1]) and most == alone[2]
    assert watch.calls["beam_step"] == 20 and watch.calls["attend"] == 21 * len(net.layers)
    assert watch.calls.get("kv_compact", 0) == (20 // compact_every if compact_every else 0)
    if beam > 1:
        assert watch.shared > 0   # pages that were filled in part went their own ways
    assert (out[:, :, 0] >= 0).all() and (scores > -torch.inf).all()
