"""Beam search with an n-gram model fused in, over a paged cache in 8 bits.

A small decoder network (random weights) reads an utterance's frames as a
prefix of cached keys and values, which all hypotheses of the utterance share,
and writes tokens after it.  Hypotheses share the pages of the tokens that they
have in common, and a page is copied only when one of them writes into it.  Each step

  1. the best continuations over all hypotheses and classes      (NgpuLM.beam_step),
  2. the chosen ones take over their parents' pages              (kv_fork, kv_copy),
  3. now and then the pool's pages move together                 (kv_compact, kv_copy),
  4. the network runs over the new tokens                        (kv_append, attend).

    python examples/beam_search.py --utterances 4 --beam 6 --tokens 48
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2505_22857_amd as ng  # noqa: E402
from speculative_decode import Network, Shape  # noqa: E402


class Network8(Network):
    """The decoder over caches in 8 bits, with a class more than there are tokens: the end."""

    def __init__(self, shape: Shape, block: int = 8, **kw):
        super().__init__(shape, **kw)
        self.block = block
        end = torch.randn(shape.width, 1, generator=torch.Generator().manual_seed(1)) * 4 / shape.width ** 0.5
        self.head = torch.cat([self.head, end.to(self.device, self.dtype)], 1)

    def make_cache(self, pages):
        s = self.shape
        elements, scales = (pages, s.page, s.kv_heads, s.dim), (pages, s.page // self.block, s.kv_heads)
        return [tuple(torch.zeros(elements, device=self.device).to(torch.float8_e4m3fn) for _ in range(2)) +
                tuple(torch.ones(scales, device=self.device) for _ in range(2)) for _ in self.layers]

    def run(self, x, cache, tables, pages, start, new, positions, prefix=None):
        """Hidden states of x [S, T, width], of which the first new[s] are appended at ``start``."""
        s = self.shape
        for layer, (kc, vc, ks, vs) in zip(self.layers, cache):
            qkv = (self.norm(x) @ layer["qkv"]).unflatten(-1, (-1, s.dim))
            q, k, v = qkv.split((s.q_heads, s.kv_heads, s.kv_heads), 2)
            q = ng.kv_append(k, v, kc, vc, pages, start, positions=positions, cos=tables[0], sin=tables[1], q=q,
                             lengths=new, k_scale=ks, v_scale=vs)
            y = ng.attend(q, kc, vc, pages=pages, lengths=start + new, prefix_pages=prefix and prefix[0],
                          prefix_lengths=prefix and prefix[1], q_lengths=new, k_scale=ks, v_scale=vs)
            x = x + y.flatten(2) @ layer["out"]
            x = x + torch.nn.functional.silu(self.norm(x) @ layer["up"]) @ layer["down"]
        return x


def search(net: Network8, lm: "ng.NgpuLM", frames, frame_lengths, beam: int, tokens: int, weight: float = 0.3,
           first: int = 0, compact_every: int = 0, pool: int = None):
    """At most ``tokens`` classes for the ``beam`` best hypotheses of each utterance of ``frames`` [G, L, width].

    ``pool``: pages for the hypotheses' tokens, as many as they could need unless given; one that finds none is given up.
    Returns the classes [G, beam, tokens] (the vocabulary's size: ended; -1 behind it, or no hypothesis), the sums [G, beam]
    and the most pages that were in use."""
    s, dev = net.shape, net.device
    G, L = frames.shape[:2]
    i32 = torch.int32
    prefix_width, width = -(-L // s.page), -(-tokens // s.page)
    if pool is None:
        pool = G * beam * width   # enough where hypotheses share nothing
    P = G * prefix_width + pool
    refs = torch.zeros(P, dtype=i32, device=dev)
    cache = net.make_cache(P)
    tables = ng.rope_table(L + tokens, s.rotary, device=dev)

    # the utterances' frames, once for all their hypotheses
    own = torch.zeros(G, 1, dtype=i32, device=dev)
    prefix, start, _ = ng.kv_fork(torch.full((G, prefix_width), -1, dtype=i32, device=dev), own[:, 0], own, refs, s.page,
                                  tokens=frame_lengths[:, None])
    at = torch.arange(L, dtype=i32, device=dev).expand(G, L).contiguous()
    net.run(frames, cache, tables, prefix, start, frame_lengths, at)

    # one hypothesis an utterance, which the first token is appended to
    scores = torch.full((G, beam), -torch.inf, device=dev)
    scores[:, 0] = 0
    states = torch.full((G, beam), lm.start_state, dtype=i32, device=dev)
    classes = torch.where(scores > -torch.inf, first, -1).to(i32)
    pages = torch.full((G * beam, width), -1, dtype=i32, device=dev)
    lengths = torch.zeros(G * beam, dtype=i32, device=dev)
    parents = torch.where(classes >= 0, torch.arange(beam, dtype=i32, device=dev), -1).to(i32)
    out = torch.full((G, beam, tokens), -1, dtype=i32, device=dev)
    most = torch.zeros((), dtype=torch.int64, device=dev)
    for t in range(tokens):
        new = ((classes >= 0) & (classes < s.vocab)).to(i32)
        pages, lengths, copies = ng.kv_fork(pages, lengths, parents, refs, s.page, tokens=new)
        gone = (lengths < 0).view(G, beam)   # dropped for want of pages
        scores, new = scores.masked_fill(gone, -torch.inf), new.masked_fill(gone, 0)
        for kc, vc, ks, vs in cache:
            ng.kv_copy(kc, vc, copies, k_scale=ks, v_scale=vs)
        most = torch.maximum(most, (refs > 0).sum())
        if compact_every and t % compact_every == compact_every - 1:
            copies, _ = ng.kv_compact(refs, s.page, tables=(prefix, pages))
            for kc, vc, ks, vs in cache:
                ng.kv_copy(kc, vc, copies, k_scale=ks, v_scale=vs)
        start, new = lengths.clamp(min=0), new.view(-1)
        x = net.embed[classes.clamp(0, s.vocab - 1).long()].view(G * beam, 1, -1)
        positions = (frame_lengths.repeat_interleave(beam) + start)[:, None]
        x = net.run(x, cache, tables, pages, start, new, positions, (prefix, frame_lengths))
        lengths = start + new
        log_p = torch.log_softmax((net.norm(x) @ net.head).float(), -1).view(G, beam, -1)
        classes, parents, scores, states = lm.beam_step(log_p, weight, states, scores, last=classes,
                                                        mode=ng.NGPU_FUSION_AED)
        kept = parents.clamp(min=0).long()
        out = out.gather(1, kept[..., None].expand(-1, -1, tokens))
        over = (out == s.vocab).any(-1)   # an ended hypothesis stays as it is
        out[:, :, t] = torch.where(over, -1, classes)
        out[parents < 0] = -1
    for table, n in ((pages, lengths), (prefix, frame_lengths)):   # all is given up
        ng.kv_fork(table, n, torch.full((G, 1), -1, dtype=i32, device=dev), refs, s.page)
    assert not refs.any()
    return out, scores, int(most)


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--utterances", type=int, default=4)
    p.add_argument("--beam", type=int, default=6)
    p.add_argument("--frames", type=int, default=200)
    p.add_argument("--tokens", type=int, default=48)
    p.add_argument("--weight", type=float, default=0.3)
    a = p.parse_args()
    from synth import generate_model
    V = Shape().vocab
    lm = ng.NgpuLM.from_model(generate_model(V, [V, 8 * V, 8 * V], 1.0, seed=1, bos_eos=True)).upload("cuda")
    net = Network8(Shape())
    frames = torch.randn(a.utterances, a.frames, net.shape.width, device="cuda").half()
    lengths = torch.randint(a.frames // 2, a.frames + 1, (a.utterances,), dtype=torch.int32, device="cuda")
    classes, scores, most = search(net, lm, frames, lengths, a.beam, a.tokens, a.weight, compact_every=8)
    print(f"{a.utterances} utterances, {a.beam} hypotheses each, at most {most} pages in use")
    print(round(float(scores[0, 0]), 3), classes[0, 0].tolist())


if __name__ == "__main__":
    main()
