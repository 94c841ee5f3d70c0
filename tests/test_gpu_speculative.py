"""The four serving operators together: greedy speculative decoding writes the
tokens that the network itself would, whatever was drafted."""

import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import paper_2505_22857_amd as ng  # noqa: E402
import speculative_decode as ex  # noqa: E402
from synth import make_model  # noqa: E402


def full_logits(net, frames, length, tokens):
    """The network over one utterance's frames and a hypothesis' tokens, densely and in 64 bits."""
    s = net.shape

    def norm(x):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6)

    def host(x):
        return x.double().cpu().numpy()

    def layers(x, positions, past):
        out = []
        freq = 10000.0 ** (-np.arange(0, s.rotary, 2) / s.rotary)
        angle = positions[:, None] * freq
        cos, sin, half = np.cos(angle)[:, None], np.sin(angle)[:, None], s.rotary // 2
        for n, w in enumerate(net.layers):
            qkv = (norm(x) @ host(w["qkv"])).reshape(len(x), -1, s.dim)
            q, k, v = np.split(qkv, [s.q_heads, s.q_heads + s.kv_heads], 1)

            def turn(z):
                a, b = z[..., :half], z[..., half:2 * half]
                return np.concatenate([a * cos - b * sin, a * sin + b * cos, z[..., 2 * half:]], -1)
            q, k = turn(q), turn(k)
            out.append((k, v))
            if past:
                k, v = np.concatenate([past[n][0][:length], k]), np.concatenate([past[n][1][:length], v])
            y = np.zeros_like(q)
            before = len(k) - len(x)
            for t in range(len(x)):
                for h in range(s.q_heads):
                    kv = h // (s.q_heads // s.kv_heads)
                    z = k[:before + t + 1, kv] @ q[t, h] / np.sqrt(s.dim)
                    z = np.exp(z - z.max())
                    y[t, h] = z @ v[:before + t + 1, kv] / z.sum()
            x = x + y.reshape(len(x), -1) @ host(w["out"])
            u = norm(x) @ host(w["up"])
            x = x + (u / (1 + np.exp(-u))) @ host(w["down"])
        return x, out

    _, past = layers(host(frames), np.arange(len(frames)), None)
    x, _ = layers(host(net.embed)[tokens], length + np.arange(len(tokens)), past)
    return norm(x) @ host(net.head)


@pytest.mark.parametrize("draft", [1, 4])
def test_greedy_speculation_writes_the_networks_tokens(draft):
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    lm = ng.NgpuLM.from_model(make_model("trigram_v128")).upload("cuda")
    net = ex.Network(ex.Shape())
    g = torch.Generator(device="cuda").manual_seed(1)
    frames = torch.randn(2, 50, net.shape.width, generator=g, device="cuda").half()
    lengths = torch.tensor([50, 33], dtype=torch.int32, device="cuda")
    tokens, kept, drafted = ex.decode(net, lm, frames, lengths, beam=2, draft=draft, tokens=24, first=3)
    assert lm.check_states() == 0 and 0 <= kept <= drafted
    tokens = tokens.cpu().numpy()
    assert ((tokens >= 0) & (tokens < 128)).all()
    assert np.array_equal(tokens[0], tokens[1]) and np.array_equal(tokens[2], tokens[3])   # same utterance, no noise
    for n in (0, 2):
        logits = full_logits(net, frames[n // 2], int(lengths[n // 2]), np.concatenate([[3], tokens[n, :-1]]))
        chosen = logits[np.arange(24), tokens[n]]
        # half-precision activations: 2^-11 of values of size 4 through a few layers, far below the logits' spread
        assert np.all(chosen >= logits.max(1) - 0.1)
        assert logits.std() > 2


def test_sampled_speculation_runs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    lm = ng.NgpuLM.from_model(make_model("trigram_v128")).upload("cuda")
    net = ex.Network(ex.Shape(), seed=2)
    frames = torch.randn(3, 40, net.shape.width, device="cuda").half()
    lengths = torch.full((3,), 40, dtype=torch.int32, device="cuda")
    tokens, kept, drafted = ex.decode(net, lm, frames, lengths, beam=3, draft=3, tokens=20, temperature=1.5)
    assert ((tokens >= 0) & (tokens < 128)).all() and lm.check_states() == 0 and 0 < kept < drafted
