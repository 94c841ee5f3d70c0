"""Speculative decoding with an n-gram model as the drafter.

A small decoder network (random weights) stands in for the target: it reads an
utterance's frames as a prefix of cached keys and values, which all hypotheses
of the utterance share, and writes tokens after it.  Each round

  1. the n-gram model drafts K tokens a hypothesis          (NgpuLM.draft),
  2. the network runs once over the last token and the draft, appending its
     rotated keys and values to the paged cache              (kv_append)
     and attending to the shared prefix and its own tokens   (attend),
  3. its logits keep a part of the draft and add one token   (verify).

    python examples/speculative_decode.py --utterances 4 --beam 2 --draft 4 --tokens 48
"""

from __future__ import annotations

import argparse
import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2505_22857_amd as ng  # noqa: E402


@dataclass
class Shape:
    vocab: int = 128
    layers: int = 2
    q_heads: int = 4
    kv_heads: int = 2
    dim: int = 64          # of a head
    rotary: int = 32
    page: int = 16

    @property
    def width(self):
        return self.q_heads * self.dim


class Network:
    """Pre-norm decoder layers over a paged cache; the products are torch's."""

    def __init__(self, shape: Shape, seed: int = 0, device="cuda", dtype=torch.float16):
        g = torch.Generator().manual_seed(seed)
        w, heads = shape.width, shape.q_heads + 2 * shape.kv_heads

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=g) / rows ** 0.5).to(device, dtype)
        self.shape, self.dtype, self.device = shape, dtype, device
        self.embed = torch.randn(shape.vocab, w, generator=g).to(device, dtype)
        self.head = matrix(w, shape.vocab) * 4
        self.layers = [{"qkv": matrix(w, heads * shape.dim), "out": matrix(w, w), "up": matrix(w, 2 * w),
                        "down": matrix(2 * w, w)} for _ in range(shape.layers)]

    def make_cache(self, pages):
        s = self.shape
        return [tuple(torch.zeros(pages, s.page, s.kv_heads, s.dim, dtype=self.dtype, device=self.device)
                      for _ in range(2)) for _ in self.layers]

    @staticmethod
    def norm(x):
        return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def run(self, x, cache, tables, pages, start, lengths, positions, prefix=None):
        """Hidden states of x [S, T, width], whose keys and values are appended at ``start``."""
        s = self.shape
        for layer, (kc, vc) in zip(self.layers, cache):
            qkv = (self.norm(x) @ layer["qkv"]).unflatten(-1, (-1, s.dim))
            q, k, v = qkv.split((s.q_heads, s.kv_heads, s.kv_heads), 2)
            q = ng.kv_append(k, v, kc, vc, pages, start, positions=positions, cos=tables[0], sin=tables[1], q=q)
            y = ng.attend(q, kc, vc, pages=pages, lengths=lengths, prefix_pages=prefix and prefix[0],
                          prefix_lengths=prefix and prefix[1])
            x = x + y.flatten(2) @ layer["out"]
            x = x + torch.nn.functional.silu(self.norm(x) @ layer["up"]) @ layer["down"]
        return x


def decode(net: Network, lm: "ng.NgpuLM", frames, frame_lengths, beam: int, draft: int, tokens: int, first: int = 0,
           temperature: float = 0.0, seed: int = 0):
    """Decode ``tokens`` tokens for ``beam`` hypotheses of each utterance of ``frames`` [G, L, width].

    Returns the tokens [G * beam, tokens], and the drafted tokens that were kept and all drafted ones."""
    s, dev = net.shape, net.device
    G, L = frames.shape[:2]
    S, T = G * beam, draft + 1
    prefix_width, own_width = -(-L // s.page), -(-(tokens + T) // s.page)
    cache = net.make_cache(G * prefix_width + S * own_width)
    every = torch.arange(G * prefix_width + S * own_width, dtype=torch.int32, device=dev)
    prefix_pages, pages = every[:G * prefix_width].view(G, -1), every[G * prefix_width:].view(S, -1)
    tables = ng.rope_table(L + tokens + T, s.rotary, device=dev)

    # the utterances' frames, once for all their hypotheses
    zero = torch.zeros(G, dtype=torch.int32, device=dev)
    at = torch.arange(L, dtype=torch.int32, device=dev).expand(G, L).contiguous()
    net.run(frames, cache, tables, prefix_pages, zero, torch.full_like(zero, L), at)

    g = torch.Generator(device=dev).manual_seed(seed)
    sample = temperature > 0

    def noise(*shape):
        return torch.empty(shape, device=dev).exponential_(generator=g) if sample else None

    lengths_of = frame_lengths.repeat_interleave(beam)
    states = torch.full((S,), lm.start_state, dtype=torch.int32, device=dev)
    last = torch.full((S,), first, dtype=torch.int32, device=dev)
    start = torch.zeros(S, dtype=torch.int32, device=dev)
    out = torch.full((S, tokens + T), -1, dtype=torch.int32, device=dev)
    step, kept, rounds = torch.arange(T, device=dev), 0, 0
    while int(start.min()) < tokens:
        # a hypothesis that has its tokens goes on in place, so that all rounds have one shape
        start.clamp_(max=tokens)
        drafted, after, logprobs = lm.draft(states, draft, noise=noise(S, draft, s.vocab), temperature=temperature,
                                            last=last)
        x = net.embed[torch.cat([last[:, None], drafted], 1).long()]
        positions = (lengths_of + start)[:, None] + step.to(torch.int32)
        x = net.run(x, cache, tables, pages, start, start + T, positions, (prefix_pages, frame_lengths))
        logits = net.norm(x) @ net.head
        uniforms = torch.rand(S, draft, generator=g, device=dev) if sample else None
        new, accepted, states = ng.verify(logits, drafted, logprobs, uniforms, noise(S, s.vocab), temperature,
                                          draft_states=after)
        out.scatter_(1, start.long()[:, None] + step, new)   # places past the kept ones are written again next round
        last = new.gather(1, accepted.long()[:, None])[:, 0]
        kept, rounds = kept + int(accepted.sum()), rounds + 1
        start = start + accepted + 1
    return out[:, :tokens], kept, rounds * S * draft


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--utterances", type=int, default=4)
    p.add_argument("--beam", type=int, default=2)
    p.add_argument("--frames", type=int, default=200)
    p.add_argument("--draft", type=int, default=4)
    p.add_argument("--tokens", type=int, default=48)
    p.add_argument("--temperature", type=float, default=0.0)
    a = p.parse_args()
    from synth import make_model
    lm = ng.NgpuLM.from_model(make_model("trigram_v128")).upload("cuda")
    net = Network(Shape())
    frames = torch.randn(a.utterances, a.frames, net.shape.width, device="cuda").half()
    lengths = torch.randint(a.frames // 2, a.frames + 1, (a.utterances,), dtype=torch.int32, device="cuda")
    tokens, kept, drafted = decode(net, lm, frames, lengths, a.beam, a.draft, a.tokens, temperature=a.temperature)
    print(f"{tokens.shape[0]} hypotheses, {tokens.shape[1]} tokens each; {kept} of {drafted} drafted tokens kept")
    print(tokens[0].tolist())


if __name__ == "__main__":
    main()
