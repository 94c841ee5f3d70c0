"""Verification of drafted tokens against its definition in 64 bits: kept
lengths and tokens have to be equal."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import paper_2505_22857_amd as ng  # noqa: E402
import serving_reference as ref  # noqa: E402

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


def dev(x, dtype=None):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to("cuda", dtype)


def inputs(B, K, V, dtype, seed, agree=0.5):
    """Logits and a draft that agree in part; the logits as the type holds them."""
    rng = np.random.default_rng(seed)
    z = 2.5 * rng.standard_normal((B, K + 1, V))
    logits = dev(z + agree * rng.standard_normal(z.shape)).to(dtype)
    z = z[:, :K] + agree * rng.standard_normal((B, K, V))
    m = z.max(-1, keepdims=True)
    lp = (z - m - np.log(np.exp(z - m).sum(-1, keepdims=True))).astype(np.float32)
    tokens = (lp - np.log(rng.standard_exponential(lp.shape))).argmax(-1).astype(np.int32)
    return dict(logits=logits, tokens=tokens, logprobs=lp, uniforms=rng.random((B, K), dtype=np.float32),
                noise=rng.standard_exponential((B, V)).astype(np.float32))


def check(x, temperature=1.0, lengths=None, one_hot=False, states=True, **kw):
    logits, tokens = x["logits"], x["tokens"]
    B, K = tokens.shape
    lp = None if one_hot or temperature == 0 else x["logprobs"]
    follow = np.arange(B * (K + 1), dtype=np.int32).reshape(B, K + 1) if states else None
    print(f"[case] verify {tuple(logits.shape)} {logits.dtype} T={temperature} one_hot={one_hot}", flush=True)
    got = ng.verify(logits, dev(tokens), logprobs=dev(lp), uniforms=dev(x["uniforms"]), noise=dev(x["noise"]),
                    temperature=temperature, lengths=dev(lengths), draft_states=dev(follow), **kw)
    out, kept = ref.verify(logits.double().cpu().numpy(), tokens, lp, x["uniforms"], x["noise"], temperature, lengths)
    assert np.array_equal(got[1].cpu().numpy(), kept)
    assert np.array_equal(got[0].cpu().numpy(), out)
    if states:
        assert np.array_equal(got[2].cpu().numpy(), follow[np.arange(B), kept])
    else:
        assert got[2] is None
    return kept


@pytest.mark.parametrize("B,K,V", [
    (1, 1, 1), (2, 3, 2), (1, 4, 5), (3, 0, 17), (5, 2, 63), (2, 7, 64), (1, 4, 1024), (40, 5, 1000), (3, 63, 65),
    (2, 5, 8192), (2, 3, 8193), (3, 4, 16391), (2, 2, 128001), (1, 1, 600000), (300, 1, 129), (9, 8, 4097)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("temperature", [0.0, 1.0, 0.7])
def test_verify(B, K, V, dtype, temperature):
    x = inputs(B, K, V, dtype, seed=B + K + V)
    if temperature == 0 and K:   # drafts that are partly right
        best = x["logits"].double().cpu().numpy().argmax(-1)[:, :K]
        x["tokens"] = np.where(x["uniforms"] < 0.7, best, x["tokens"]).astype(np.int32)
    kept = check(x, temperature)
    if B >= 40 and K:
        assert 0 < kept.mean() < K
    check(x, temperature, one_hot=True, states=False)


@pytest.mark.parametrize("V", [50, 9000])
@pytest.mark.parametrize("temperature", [0.0, 0.8])
def test_lengths_and_tokens_outside(V, temperature):
    """Lengths of zero, negative and too large ones, and tokens outside the vocabulary, which end a draft."""
    x = inputs(12, 4, V, F32, seed=V, agree=0.02)
    lengths = np.array([0, 1, 2, 3, 4, -3, 99, 4, 4, 4, 3, 4], np.int32)
    x["tokens"][7, 0] = -1
    x["tokens"][8, 2] = V
    x["tokens"][9, 3] = 2 ** 31 - 1
    x["tokens"][10, 1] = -(2 ** 31)
    kept = check(x, temperature, lengths)
    assert kept[0] == 0 and kept[7] == 0 and kept[8] <= 2
    check(x, temperature, lengths, one_hot=True)


@pytest.mark.parametrize("V", [40, 8500])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_odd_logits(V, dtype):
    """Masked logits (-inf, the type's lowest value), NaN, +inf, rows that hold nothing."""
    rng = np.random.default_rng(V)
    x = inputs(10, 3, V, dtype, seed=V)
    g, lowest = x["logits"], torch.finfo(dtype).min
    hide = dev(rng.random((10, 4, V)) < 0.9)
    for row, value in ((0, -np.inf), (1, lowest), (2, np.nan)):
        g[row][hide[row]] = value
    g[3, :, 5] = np.inf
    g[4, :, [5, V - 1]] = np.inf
    g[5] = -np.inf
    g[6, 1] = np.nan
    g[7] = lowest
    g[8, :, :-1] = -np.inf
    g[9, 0] = np.inf
    x["tokens"][3:5, 0] = 5
    x["tokens"][8] = V - 1
    for temperature in (0.0, 1.0, 0.7):
        check(x, temperature)
        check(x, temperature, one_hot=True)


def test_odd_drafts_and_numbers():
    """Draft rows that equal the network's (nothing is left to draw from), drafted tokens that the draft
    gave no mass, noise of zero, infinity and NaN, uniforms at their ends."""
    V = 300
    x = inputs(8, 2, V, F32, seed=1)
    z = x["logits"].double().cpu().numpy()
    z -= z.max(-1, keepdims=True)
    same = z - np.log(np.exp(z).sum(-1, keepdims=True))
    x["logprobs"][0] = same[0, :2].astype(np.float32) + 0.001      # p < q everywhere
    x["uniforms"][0] = 1 - 2.0 ** -24
    x["logprobs"][1] = -np.inf
    x["logprobs"][2, :, :100] = np.nan
    x["noise"][3, [9, 4, 200]] = 0.0
    x["noise"][4, 1:] = np.nan
    x["noise"][5, :-1] = np.inf
    x["noise"][6] = np.nan
    x["uniforms"][7] = 0.0
    check(x)
    check(x, one_hot=True)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("V", [70, 8197])
def test_strides(dtype, V):
    """Rows at any offset and stride, rows shared between places."""
    x = inputs(3, 2, V, dtype, seed=V)
    for pad, off in ((1, 0), (3, 1), (8, 5), (64, 7)):
        wide = torch.full((3, 5, V + pad + off), float("nan"), dtype=dtype, device="cuda")
        view = wide[:, 1:4, off:off + V]
        view.copy_(x["logits"])
        check(dict(x, logits=view))
        check(dict(x, logits=view), 0.0)
    one = x["logits"][:, :1].expand(3, 3, V)
    check(dict(x, logits=one))
    lp = torch.full((3, 2, V + 5), float("nan"), device="cuda")[:, :, 3:V + 3]
    lp.copy_(dev(x["logprobs"]))
    noise = torch.full((3, V + 1), float("nan"), device="cuda")[:, 1:]
    noise.copy_(dev(x["noise"]))
    a = ng.verify(x["logits"], dev(x["tokens"]), lp, dev(x["uniforms"]), noise)
    b = ng.verify(x["logits"], dev(x["tokens"]), dev(x["logprobs"]), dev(x["uniforms"]), dev(x["noise"]))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_ties_take_the_lowest_token():
    for V in (100, 20000):
        logits = torch.zeros(4, 3, V, device="cuda")
        logits[1, :, [V // 2, V - 1]] = 1.0
        tokens = np.zeros((4, 2), np.int32)
        tokens[1] = V // 2
        tokens[2, 1] = 1
        x = dict(logits=logits, tokens=tokens, uniforms=np.full((4, 2), 0.5, np.float32),
                 noise=np.ones((4, V), np.float32))
        check(x, 0.0)
        check(x, 1.0, one_hot=True)


def test_tokens_follow_the_target_distribution():
    """Drafts from q, verified against p: the first token is distributed as p.  20000 rounds of one
    drafted token, frequencies within five standard deviations."""
    V, n = 12, 20000
    g = torch.Generator(device="cuda").manual_seed(3)
    logits = torch.randn(1, 2, V, generator=g, device="cuda") * 1.5
    lq = torch.log_softmax(torch.randn(V, generator=g, device="cuda"), -1)

    def exponential(*shape):
        return torch.empty(shape, device="cuda").exponential_(generator=g)

    tokens = (lq.exp() / exponential(n, V)).argmax(-1).int()[:, None]
    out, kept, _ = ng.verify(logits.expand(n, 2, V), tokens, lq.expand(n, 1, V),
                             torch.rand(n, 1, generator=g, device="cuda"), exponential(n, V), temperature=0.8)
    p = ref.probabilities(logits[0, 0].cpu().numpy(), 0.8)
    count = np.bincount(out[:, 0].cpu().numpy(), minlength=V)
    assert np.all(np.abs(count - n * p) <= 5 * np.sqrt(n * p * (1 - p)) + 1)
    assert 0.2 * n < int(kept.sum()) < 0.95 * n


def test_other_stream_and_graph():
    x = inputs(6, 4, 9000, BF16, seed=9)
    args = (x["logits"], dev(x["tokens"]), dev(x["logprobs"]), dev(x["uniforms"]), dev(x["noise"]))
    want = ng.verify(*args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = ng.verify(*args, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ng.verify(*args)
    for i in range(4):   # each replay against the eager result, with eager work between
        args[3].uniform_()
        x["logits"].copy_(x["logits"].flip(1))
        graph.replay()
        torch.cuda.synchronize()
        want = ng.verify(*args)
        assert torch.equal(held[0], want[0]) and torch.equal(held[1], want[1]), i


def test_rows_past_2_31_elements():
    """Rows whose offset passes 32 bits."""
    V, stride = 1000, (1 << 31) + 64
    x = inputs(2, 1, V, F16, seed=4)
    far = torch.empty(stride + 2 * V, dtype=F16, device="cuda").as_strided((2, 2, V), (stride, V, 1))
    far.copy_(x["logits"])
    check(dict(x, logits=far))
    check(dict(x, logits=far), 0.0)


def test_refusals():
    x = inputs(3, 2, 50, F32, seed=2)
    args = (x["logits"], dev(x["tokens"]), dev(x["logprobs"]), dev(x["uniforms"]), dev(x["noise"]))
    ng.verify(*args)

    def bad(error, i=None, value=None, **kw):
        a = list(args)
        if i is not None:
            a[i] = value
        with pytest.raises(error):
            ng.verify(*a, **kw)

    bad(TypeError, 0, args[0].double())
    bad(TypeError, 0, args[0].cpu())
    bad(ValueError, 0, args[0][:, :2])
    bad(ValueError, 0, args[0][0])
    bad(TypeError, 0, args[0].transpose(1, 2).contiguous().transpose(1, 2))
    bad(TypeError, 1, args[1].long())
    bad(ValueError, 1, args[1][:2])
    bad(ValueError, 2, args[2][:, :, :49])
    bad(TypeError, 2, args[2].half())
    bad(ValueError, 3, None)
    bad(ValueError, 4, None)
    bad(ValueError, lengths=args[1][:, 0][:2].contiguous())
    bad(ValueError, draft_states=args[1])
    for t in (-1.0, float("nan"), float("inf"), 1e-8):
        bad(ng.NgpuError, temperature=t)
    with pytest.raises(ng.NgpuError):   # more than 63 drafted tokens
        ng.verify(torch.zeros(1, 65, 4, device="cuda"), torch.zeros(1, 64, dtype=torch.int32, device="cuda"),
                  temperature=0.0)
    out, kept, states = ng.verify(args[0][:0], args[1][:0], temperature=0.0)
    assert out.shape == (0, 3) and kept.shape == (0,) and states is None


@pytest.mark.parametrize("B,K,V", [
    (63, 1, 4097), (64, 1, 4097), (63, 2, 8192), (64, 2, 8192), (60, 5, 10001), (90, 5, 10001), (256, 3, 9000)])
@pytest.mark.parametrize("temperature", [0.0, 1.3])
def test_either_side_of_the_cuts(B, K, V, temperature):
    """Batches on both sides of one launch and two, and of each size of chunk."""
    check(inputs(B, K, V, F32, B + V), temperature)
