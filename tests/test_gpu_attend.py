"""Shared-prefix attention over the paged cache against its definition in 64 bits.

With u half an ulp of the type (2^-8 bfloat16, 2^-11 half) and A = sum of
softmax |v|: the weights are rounded to the type before they multiply v (at
most u A, and with half, below its normal range, 2^-25 of the largest |v| a
key), the output once more (u A), and scores and sums are fp32: a score is off
by at most 2^-24 (D + 4) sum |q k| scale, which is below 2e-4 here and moves a
weight by as much of its size.  So |out - exact| <= (2 u + 5e-4) A + 2^-25 (1 +
keys max |v|), and the log of the sum is off by at most 1e-3.
"""

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import paper_2505_22857_amd as ng  # noqa: E402
import serving_reference as ref  # noqa: E402

F16, BF16 = torch.float16, torch.bfloat16
UNIT = {F16: 2.0 ** -11, BF16: 2.0 ** -8}


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


def ints(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def host(x):
    return x.double().cpu().numpy()


def randn(rng, dtype, *shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda().to(dtype)


def compare(q, kc, vc, pages, lengths, prefix_pages, prefix_lengths, q_lengths=None, scale=None):
    out, lse = ng.attend(q, kc, vc, ints(pages), ints(lengths), ints(prefix_pages), ints(prefix_lengths),
                         ints(q_lengths), scale=scale, return_lse=True)
    want, want_lse, size = ref.attend(host(q), host(kc), host(vc), pages, lengths, prefix_pages, prefix_lengths,
                                      q_lengths, scale)
    got, got_lse = host(out), host(lse)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    u, keys = UNIT[q.dtype], max(1, (0 if pages is None else np.size(pages[0]) * kc.shape[1]) +
                                 (0 if prefix_pages is None else np.size(prefix_pages[0]) * kc.shape[1]))
    finite = host(vc)[np.isfinite(host(vc))]
    small = 2.0 ** -25 * (1 + (keys * np.abs(finite).max(initial=0) if q.dtype == F16 else 0))
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want) - ((2 * u + 5e-4) * size + small)
        assert not (off > 0).any(), f"worst {np.nanmax(off)}"
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got_lse), empty)
        assert not (np.abs(got_lse - want_lse)[~empty] > 1e-3).any()
    assert not got[empty].any()
    assert torch.equal(ng.attend(q, kc, vc, ints(pages), ints(lengths), ints(prefix_pages), ints(prefix_lengths),
                                 ints(q_lengths), scale=scale).nan_to_num(9), out.nan_to_num(9))
    return out


def check(G=2, beam=2, T=1, H=2, rep=2, D=64, page=16, prefix=(33, 20), own=(5, 9, 1, 30), q_lengths=None, dtype=BF16,
          seed=0, change=None, scale=None, spare=3):
    """``change(q, k_cache, v_cache, pages, prefix_pages)`` alters the inputs before the call."""
    rng = np.random.default_rng(seed)
    S = max(G, 1) * beam
    prefix, own = np.resize(prefix, max(G, 1)), np.resize(own, S)
    wp, wo = -(-max(int(prefix.max()), 1) // page), -(-max(int(own.max()), 1) // page)
    P = G * wp + S * wo + spare
    perm = rng.permutation(P)
    prefix_pages = perm[:G * wp].reshape(G, wp) if G else None
    pages = perm[G * wp:G * wp + S * wo].reshape(S, wo)
    q, kc, vc = randn(rng, dtype, S, T, H * rep, D), randn(rng, dtype, P, page, H, D), randn(rng, dtype, P, page, H, D)
    print(f"[case] attend G={G} beam={beam} T={T} H={H}x{rep} D={D} page={page} prefix={list(prefix)} own={list(own)} "
          f"{dtype}", flush=True)
    if change:
        q, kc, vc, pages, prefix_pages = change(q, kc, vc, pages, prefix_pages)
    return compare(q, kc, vc, pages, own, prefix_pages, prefix if G else None, q_lengths, scale)


@pytest.mark.parametrize("D", [1, 8, 17, 40, 64, 80, 96, 128, 136, 192, 200, 256])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_dimensions(D, dtype):
    check(D=D, dtype=dtype, T=1, seed=D)
    check(D=D, dtype=dtype, T=3, rep=3, own=(5, 9, 3, 40), seed=D)


@pytest.mark.parametrize("H,rep", [(1, 1), (1, 8), (8, 1), (3, 3), (2, 16), (1, 40)])
@pytest.mark.parametrize("T", [1, 2, 5])
def test_heads_and_tokens(H, rep, T):
    check(H=H, rep=rep, T=T, own=(5, 9, 7, 30), seed=T)


@pytest.mark.parametrize("page", [1, 3, 16, 64, 100])
@pytest.mark.parametrize("prefix", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000])
def test_prefix_lengths(page, prefix):
    check(page=page, prefix=(prefix, max(0, prefix - 1)), seed=prefix)


@pytest.mark.parametrize("own", [0, 1, 2, 31, 32, 33, 64, 65, 300])
@pytest.mark.parametrize("G", [0, 1])
def test_own_lengths(own, G):
    check(G=G, beam=3, T=2, own=(own, own + 1, max(0, own - 1)), page=8, seed=own)


@pytest.mark.parametrize("G,beam,T,rep", [(1, 1, 1, 1), (1, 4, 1, 2), (1, 16, 1, 1), (1, 17, 1, 1), (1, 8, 4, 1),
                                          (1, 11, 3, 1), (1, 16, 6, 1), (2, 16, 4, 2), (1, 16, 5, 4), (1, 50, 9, 1),
                                          (3, 2, 2, 5), (1, 1, 200, 1), (1, 3, 40, 2)])
def test_rows_sharing_a_prefix(G, beam, T, rep):
    """From one row a key to hundreds."""
    check(G=G, beam=beam, T=T, rep=rep, H=1, prefix=(200, 77, 150), own=(T + 3, T, T + 40, T + 100), D=64, seed=beam)


def test_long_prefix():
    check(G=2, beam=2, T=2, prefix=(9000, 4097), own=(700, 2, 350, 33), D=128, page=64)
    check(G=1, beam=1, T=1, H=1, rep=4, prefix=(20011,), own=(1,), D=128, page=32)


def test_prefix_only_and_own_only():
    rng = np.random.default_rng(3)
    q, kc, vc = (randn(rng, F16, *s) for s in ((6, 2, 4, 64), (9, 8, 2, 64), (9, 8, 2, 64)))
    table = rng.permutation(9)
    compare(q, kc, vc, None, None, table[:6].reshape(3, 2), [16, 0, 5])
    compare(q, kc, vc, table[:6].reshape(6, 1), [8, 0, 1, 2, 7, 3], None, None)
    out, lse = ng.attend(q, kc, vc, return_lse=True)
    assert not out.any() and torch.isneginf(lse).all()
    out, lse = ng.attend(q, kc[:0], vc[:0], ints(table[:6].reshape(6, 1)), ints([8] * 6), return_lse=True)
    assert not out.any() and torch.isneginf(lse).all()


@pytest.mark.parametrize("T", [1, 4, 20])
def test_ragged_queries(T):
    """Sequences with fewer query tokens, none, or more than they have own tokens."""
    q_lengths = np.array([T, 0, 1, -3, 99, (T + 1) // 2])
    check(G=2, beam=3, T=T, q_lengths=q_lengths, own=(T, 5, 1, 3, T - 1, T + 50), prefix=(40, 0), seed=T)
    check(G=0, beam=6, T=T, q_lengths=q_lengths, own=(0, 5, 0, 3, T - 1, T // 2), seed=T)


def test_lengths_past_the_tables():
    rng = np.random.default_rng(1)
    q, kc, vc = (randn(rng, BF16, *s) for s in ((4, 3, 2, 64), (12, 4, 1, 64), (12, 4, 1, 64)))
    table = rng.permutation(12)
    compare(q, kc, vc, table[:8].reshape(4, 2), [99, -5, 8, 2 ** 31 - 1], table[8:].reshape(2, 2), [9, -(2 ** 31)])


def test_pages_outside_the_cache():
    """Their keys take no part, at any place of a tile."""
    def holes(q, kc, vc, pages, prefix_pages):
        prefix_pages = prefix_pages.copy()
        prefix_pages[0, ::3], prefix_pages[0, 1::3], prefix_pages[1, :] = -1, len(kc), 2 ** 31 - 1
        pages = pages.copy()
        pages[0, 0], pages[1, -1], pages[3, :] = -7, len(kc) + 1, -(2 ** 31)
        return q, kc, vc, pages, prefix_pages
    for page in (4, 16, 64):
        check(T=3, page=page, prefix=(200, 100), own=(30, 70, 20, 9), change=holes)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("T,beam", [(1, 2), (6, 3), (30, 2)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_that_no_row_sees(dtype, T, beam, bad):
    """Whatever the cache holds past the lengths, in other pages and at tokens later than a query (NaN,
    infinities) does not reach its row; a value that a row does see does."""
    def spoil(q, kc, vc, pages, prefix_pages):
        keep_k, keep_v = torch.full_like(kc, bad), torch.full_like(vc, bad)
        for tables, lengths in ((prefix_pages, prefix), (pages, own)):
            for row, n in zip(tables, lengths):
                for j in range(n):
                    at = int(row[j // page]), j % page
                    keep_k[at], keep_v[at] = kc[at], vc[at]
        # the last tokens of sequence 0 are seen by its last queries only
        for j in range(own[0] - (T + 1) // 2, own[0]):
            at = int(pages[0][j // page]), j % page
            keep_v[at][0, 5] = bad
            keep_v[at][1, 40:] = bad
            if j == own[0] - 1:
                keep_k[at][1, 3] = bad
        return q, keep_k, keep_v, pages, prefix_pages

    page = 16
    prefix, own = np.array([37, 50]), np.resize([T + 11, T, T + 33, T + 2], 2 * beam)
    out = check(G=2, beam=beam, T=T, prefix=prefix, own=own, page=page, dtype=dtype, change=spoil)
    assert torch.isfinite(out[1:]).all()
    if T > 1:
        assert torch.isfinite(out[0, 0]).all() and not torch.isfinite(out[0, -1]).all()


def test_large_scores():
    """Scores far apart: one key takes a row's whole mass; equal scores share it; and with a scale of 0."""
    def loud(q, kc, vc, pages, prefix_pages):
        return q * 4, kc * 4, vc, pages, prefix_pages
    rng = np.random.default_rng(5)
    q, kc, vc = (randn(rng, F16, *s) for s in ((2, 2, 2, 64), (8, 16, 2, 64), (8, 16, 2, 64)))
    kc[3, 5] = q[0, 0, 0] * 30
    q[0, 0, 1] = q[0, 0, 0]
    pages, own = np.array([[0, 1, 2], [4, 5, 6]]), [40, 48]
    out = ng.attend(q, kc, vc, ints(pages), ints(own), ints([[3]]), ints([16]))
    assert (out[0, 0] - vc[3, 5]).abs().max() < 2e-3
    check(scale=0.0)
    check(scale=1.0, D=8)
    check(scale=-0.3, D=16)
    check(change=loud, D=32, scale=0.05)


@pytest.mark.parametrize("off", [0, 1, 4, 8])
def test_strides(off):
    """Queries split from a projection, caches with heads first, keys and values in one tensor, any offset."""
    def split(q, kc, vc, pages, prefix_pages):
        S, T, Hq, D = q.shape
        view = torch.zeros(S, T, Hq * D + 5 + off, dtype=q.dtype, device="cuda")[..., off:off + Hq * D].unflatten(
            -1, (Hq, D))
        view.copy_(q)
        return view, kc, vc, pages, prefix_pages

    def heads_first(q, kc, vc, pages, prefix_pages):
        return (q.transpose(0, 1).contiguous().transpose(0, 1),
                *[x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kc, vc)], pages, prefix_pages)

    def together(q, kc, vc, pages, prefix_pages):
        D = q.shape[-1]
        wide = torch.full((*kc.shape[:3], 2 * D + off), float("nan"), dtype=q.dtype, device="cuda")
        wide[..., off:off + D], wide[..., off + D:] = kc, vc
        return q, wide[..., off:off + D], wide[..., off + D:], pages, prefix_pages

    def one_head_for_all(q, kc, vc, pages, prefix_pages):
        return (q[:, :, :1].expand(q.shape), kc[:, :, :1].expand(kc.shape), vc[:, :, :1].expand(vc.shape), pages,
                prefix_pages)

    for change in (split, heads_first, together, one_head_for_all):
        for T in (1, 5):
            check(T=T, own=(5, 9, 7, 30), change=change, D=64)


def test_offsets_past_32_bits():
    """Pages past 2^31 elements, tables whose rows are apart."""
    pages, page, H, D = 3, 32, 2, 64
    stride = (1 << 30) + 128
    kc, vc = (torch.zeros(2 * stride + page * H * D, dtype=F16, device="cuda").as_strided(
        (pages, page, H, D), (stride, H * D, D, 1)) for _ in range(2))
    rng = np.random.default_rng(2)
    small_k, small_v = randn(rng, F16, pages, page, H, D), randn(rng, F16, pages, page, H, D)
    kc.copy_(small_k), vc.copy_(small_v)
    q = randn(rng, F16, 2, 3, 4, D)
    wide = torch.full((2, 7), -1, dtype=torch.int32, device="cuda")
    wide[:, :2] = ints([[2, 0], [1, 2]])
    args = dict(pages=wide[:, :2], lengths=ints([60, 33]), prefix_pages=ints([[2]]), prefix_lengths=ints([30]))
    got, want = ng.attend(q, kc, vc, **args), ng.attend(q, small_k, small_v, **args)
    assert torch.equal(got, want) and want.any()


def test_rows_do_not_depend_on_the_batch():
    """Repeated calls agree bit for bit."""
    rng = np.random.default_rng(8)
    q, kc, vc = (randn(rng, BF16, *s) for s in ((16, 3, 8, 128), (300, 16, 2, 128), (300, 16, 2, 128)))
    pages, prefix_pages = ints(rng.permutation(300)[:64].reshape(16, 4)), ints(rng.permutation(300)[:200].reshape(2, 100))
    args = (pages, ints(rng.integers(3, 64, 16)), prefix_pages, ints([1600, 900]))
    first = ng.attend(q, kc, vc, *args)
    for _ in range(20):
        assert torch.equal(ng.attend(q, kc, vc, *args), first)


def test_other_stream_and_graph():
    rng = np.random.default_rng(4)
    q, kc, vc = (randn(rng, F16, *s) for s in ((4, 2, 4, 64), (60, 16, 2, 64), (60, 16, 2, 64)))
    args = (ints(np.arange(8).reshape(4, 2)), ints([20, 5, 32, 9]), ints(np.arange(8, 58).reshape(1, 50)), ints([800]))
    want = ng.attend(q, kc, vc, *args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = ng.attend(q, kc, vc, *args, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ng.attend(q, kc, vc, *args)
    for i in range(4):
        q.mul_(-0.7)
        args[3].sub_(150)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, ng.attend(q, kc, vc, *args)), i


def test_refusals():
    kc, vc = (torch.zeros(6, 8, 2, 16, dtype=F16, device="cuda") for _ in range(2))
    q = torch.zeros(4, 3, 4, 16, dtype=F16, device="cuda")
    ok = dict(q=q, k_cache=kc, v_cache=vc, pages=ints([[0]] * 4), lengths=ints([3] * 4), prefix_pages=ints([[1], [2]]),
              prefix_lengths=ints([3, 4]))
    ng.attend(**ok)

    def bad(error, **kw):
        with pytest.raises(error):
            ng.attend(**{**ok, **kw})

    bad(TypeError, q=q.float())
    bad(TypeError, q=q.cpu())
    bad(ValueError, q=q[0])
    bad(ValueError, q=q[..., :8])
    bad(TypeError, q=q.transpose(2, 3).contiguous().transpose(2, 3))
    bad(ng.NgpuError, q=q[:, :, :3])                         # no multiple of the cache's heads
    bad(ng.NgpuError, prefix_pages=ints([[1]] * 3), prefix_lengths=ints([1] * 3))   # 4 sequences in 3 groups
    bad(TypeError, k_cache=kc.float(), v_cache=vc.float())
    bad(ValueError, v_cache=vc[:5])
    bad(ValueError, k_cache=kc[0])
    bad(TypeError, pages=ok["pages"].long())
    bad(ValueError, pages=ok["pages"][:3])
    bad(ValueError, lengths=None)
    bad(ValueError, lengths=ok["lengths"][:3])
    bad(ValueError, prefix_lengths=None)
    bad(ValueError, prefix_lengths=ok["lengths"])
    bad(ValueError, q_lengths=ok["prefix_lengths"])
    bad(ng.NgpuError, scale=float("nan"))
    bad(ng.NgpuError, scale=float("inf"))
    wide = torch.zeros(6, 8, 2, 300, dtype=F16, device="cuda")
    bad(ng.NgpuError, q=torch.zeros(4, 3, 4, 300, dtype=F16, device="cuda"), k_cache=wide, v_cache=wide)
    for shape in ((4, 0, 4, 16), (0, 3, 4, 16)):
        got = ng.attend(torch.zeros(shape, dtype=F16, device="cuda"), kc, vc)
        assert got.shape == shape
    assert math.isfinite(float(ng.attend(**ok).float().sum()))


@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("page", [2, 4, 8, 16, 24, 32, 48])
@pytest.mark.parametrize("beam", [1, 40])
def test_pages_and_tiles(D, page, beam):
    """Pages that hold a part of a load, one load or many, with one wavefront a tile and with four."""
    check(G=2, beam=beam, T=2, H=1, rep=2, D=D, page=page, prefix=(333, 96), own=(40, 2, 7, 33), seed=page, dtype=F16)


def test_more_tiles_than_lanes():
    """More groups than a wavefront's lanes, each prefix in one piece of more than 64 tiles."""
    prefix = np.random.default_rng(0).integers(0, 2600, 100)
    prefix[:3] = 2600, 2049, 2048
    check(G=100, beam=1, T=1, H=8, rep=1, D=16, page=64, prefix=prefix, own=(1, 2), seed=1)


@pytest.mark.parametrize("G,beam", [(2, 2), (5, 3), (5, 40), (64, 1), (65, 1)])
def test_ragged_prefixes(G, beam):
    """Prefixes of very different lengths, empty ones among them: the splits follow the lengths."""
    prefix = np.resize([3000, 0, 1, 64, 1500, 65], G)
    check(G=G, beam=beam, T=1, H=2, rep=2, D=32, page=32, prefix=prefix, own=(3, 40, 1), seed=G)
    check(G=G, beam=beam, T=1, H=2, rep=2, D=32, page=32, prefix=np.zeros(G, int) if G > 2 else (700, 0),
          own=(3, 40, 1), seed=G)


@pytest.mark.parametrize("T", [20, 80])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_late_values_in_long_drafts(T, bad):
    """The same as for short ones where several wavefronts, or blocks of rows, share the own tokens."""
    def spoil(q, kc, vc, pages, prefix_pages):
        vc, kc = vc.clone(), kc.clone()
        at = int(pages[0][(own[0] - 2) // 16]), (own[0] - 2) % 16
        vc[at][0, 5:9] = bad
        kc[at][1, 3] = bad
        return q, kc, vc, pages, prefix_pages
    own = np.array([T + 70, T])
    out = check(G=1, beam=2, T=T, rep=3, prefix=(40,), own=own, page=16, D=128, change=spoil)
    assert torch.isfinite(out[0, :T - 2]).all() and torch.isfinite(out[1]).all()
    assert not torch.isfinite(out[0, T - 2:, :3, 5:9]).any()
    if bad != bad:          # (an infinite key's score is -inf, a weight of zero, where the query's value is negative)
        assert not torch.isfinite(out[0, T - 2:, 3:]).any()


def test_one_part_is_written_directly():
    """A single piece of own tokens and no prefix: no join; with rows that do not count."""
    check(G=0, beam=5, T=4, own=(10, 4, 0, 63, 2), q_lengths=np.array([4, 0, 2, 3, 4]), page=64, D=128)
    check(G=0, beam=2, T=40, rep=4, H=1, own=(40, 60), page=64, D=256, q_lengths=np.array([40, 11]))


@pytest.mark.parametrize("D", [16, 17])
def test_more_than_2_23_rows(D):
    """Rows past 2^23, by both kernels: the first, the last and some between against the formula."""
    T, rep, n = (1 << 20) + 3, 8, 5
    g = torch.Generator(device="cuda").manual_seed(D)
    q = torch.randn(1, T, rep, D, generator=g, device="cuda").half()
    kc, vc = (torch.randn(2, 4, 1, D, generator=g, device="cuda").half() for _ in range(2))
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    print(f"[case] attend {T} x {rep} rows D={D}", flush=True)
    out = ng.attend(q, kc, vc, prefix_pages=ints([[1, 0]]), prefix_lengths=ints([n]))
    at = torch.cat([torch.arange(1000), torch.arange(T // 2, T // 2 + 1000), torch.arange(T - 1000, T)])
    keys, values = (x[[1, 0]].reshape(8, D)[:n].double().cpu() for x in (kc, vc))
    x = (q[0, at.cuda()].double().cpu() @ keys.T) / D ** 0.5
    w = torch.softmax(x, -1)
    # the weights are rounded to half before the sum, and the result once
    u = 2.0 ** -11
    bound = 4 * u * (w @ values.abs()) + u * (w @ values).abs() + 2.0 ** -24
    assert ((out[0, at.cuda()].double().cpu() - w @ values).abs() <= bound).all()


@pytest.mark.parametrize("D,T,own", [(64, 300, (300, 411)), (128, 300, (300, 411)), (256, 90, (90, 3)), (40, 1000, (1000, 1063))])
@pytest.mark.parametrize("ragged", [False, True])
def test_prompts(D, T, own, ragged):
    """Many blocks of rows, each of which sees other keys; some tokens do not count, some see nothing."""
    n = np.array([T, T // 2 + 1]) if ragged else None
    check(G=0, beam=2, T=T, H=2, rep=4, D=D, page=16, own=own, q_lengths=n, seed=D)
    check(G=1, beam=2, T=T, H=2, rep=4, D=D, page=16, prefix=(70,), own=own, q_lengths=n, seed=D + 1)
