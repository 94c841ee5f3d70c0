"""Attention over a cache in 8 bits against its definition in 64 bits, from the values that elements and scales stand for.

With u half an ulp of the output's type (2^-8 bfloat16, 2^-11 half) and A = sum of softmax |v|: the output is rounded once
(u A) and the weights, times their values' scales, to a sum of two bfloat16 (2^-16 A); scores and sums are fp32: a score is
off by at most 2^-24 (D + 4) sum |q k| scale, which is below 2e-4 here and moves a weight by as much of its size.  So
|out - exact| <= (u + 2^-16 + 5e-4) A + 2^-25, and the log of the sum is off by at most 1e-3.
"""

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import beam_reference  # noqa: E402
import paper_2505_22857_amd as ng  # noqa: E402
import serving_reference as ref  # noqa: E402

F16, BF16, E4M3 = torch.float16, torch.bfloat16, torch.float8_e4m3fn
BOUND = {F16: 2.0 ** -11 + 2.0 ** -16 + 5e-4, BF16: 2.0 ** -8 + 2.0 ** -16 + 5e-4}
VALUES = beam_reference.e4m3_values()


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


def cache(rng, P, page, blocks, H, D, any_scale=False):
    """Elements and scales whose products are about normal."""
    x = rng.standard_normal((P, blocks, page // blocks, H, D)) * np.exp2(rng.integers(-3, 2, (P, blocks, 1, H, 1)))
    s = np.abs(x).max((2, 4)) / 448
    s = s.astype(np.float32) if any_scale else np.exp2(np.ceil(np.log2(s))).astype(np.float32)
    x = torch.from_numpy((x / s[:, :, None, :, None]).clip(-448, 448).astype(np.float32).reshape(P, page, H, D))
    return x.cuda().to(E4M3), torch.from_numpy(s).cuda()


def meant(x, s):
    """What a cache's elements stand for."""
    block = x.shape[1] // s.shape[1]
    return VALUES[x.contiguous().view(torch.uint8).cpu().numpy()] * host(s).repeat(block, 1)[..., None]


def compare(q, kc, ks, vc, vs, pages, lengths, prefix_pages, prefix_lengths, q_lengths=None, scale=None):
    args = (ints(pages), ints(lengths), ints(prefix_pages), ints(prefix_lengths), ints(q_lengths))
    out, lse = ng.attend(q, kc, vc, *args, scale=scale, return_lse=True, k_scale=ks, v_scale=vs)
    want, want_lse, size = ref.attend(host(q), meant(kc, ks), meant(vc, vs), pages, lengths, prefix_pages, prefix_lengths,
                                      q_lengths, scale)
    got, got_lse = host(out), host(lse)
    assert out.dtype is q.dtype and np.array_equal(np.isnan(got), np.isnan(want))
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want) - (BOUND[q.dtype] * size + 2.0 ** -25)
        assert not (off > 0).any(), f"worst {np.nanmax(off)}"
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got_lse), empty)
        assert not (np.abs(got_lse - want_lse)[~empty] > 1e-3).any()
    assert not got[empty].any()
    again = ng.attend(q, kc, vc, *args, scale=scale, k_scale=ks, v_scale=vs)
    assert torch.equal(again.nan_to_num(9), out.nan_to_num(9))
    return out


def check(G=2, beam=2, T=1, H=2, rep=2, D=64, page=16, blocks=1, prefix=(33, 20), own=(5, 9, 1, 30), q_lengths=None,
          dtype=BF16, seed=0, change=None, scale=None, spare=3, any_scale=False):
    """``change(q, kc, ks, vc, vs, pages, prefix_pages)`` alters the inputs before the call."""
    rng = np.random.default_rng(seed)
    S = max(G, 1) * beam
    prefix, own = np.resize(prefix, max(G, 1)), np.resize(own, S)
    wp, wo = -(-max(int(prefix.max()), 1) // page), -(-max(int(own.max()), 1) // page)
    P = G * wp + S * wo + spare
    perm = rng.permutation(P)
    prefix_pages = perm[:G * wp].reshape(G, wp) if G else None
    pages = perm[G * wp:G * wp + S * wo].reshape(S, wo)
    q, (kc, ks), (vc, vs) = randn(rng, dtype, S, T, H * rep, D), *(cache(rng, P, page, blocks, H, D, any_scale) for _ in "kv")
    print(f"[case] attend8 G={G} beam={beam} T={T} H={H}x{rep} D={D} page={page}/{blocks} prefix={list(prefix)} "
          f"own={list(own)} {dtype}", flush=True)
    if change:
        q, kc, ks, vc, vs, pages, prefix_pages = change(q, kc, ks, vc, vs, pages, prefix_pages)
    return compare(q, kc, ks, vc, vs, pages, own, prefix_pages, prefix if G else None, q_lengths, scale)


@pytest.mark.parametrize("D", [1, 8, 16, 17, 32, 48, 64, 72, 80, 96, 112, 128, 144, 192, 200, 256])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_dimensions(D, dtype):
    check(D=D, dtype=dtype, T=1, seed=D, any_scale=True)
    check(D=D, dtype=dtype, T=3, rep=3, own=(5, 9, 3, 40), seed=D)
    check(D=D, dtype=dtype, T=9, rep=4, beam=3, prefix=(100, 64), own=(9, 29, 33, 40, 12), page=32, seed=D)


@pytest.mark.parametrize("H,rep", [(1, 1), (1, 8), (8, 1), (3, 3), (2, 16), (1, 40)])
@pytest.mark.parametrize("T", [1, 2, 5])
def test_heads_and_tokens(H, rep, T):
    check(H=H, rep=rep, T=T, own=(5, 9, 7, 30), seed=T)


@pytest.mark.parametrize("page,blocks", [(1, 1), (3, 3), (16, 1), (16, 4), (64, 2), (64, 64), (100, 4), (48, 3), (128, 1)])
@pytest.mark.parametrize("prefix", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000])
def test_prefix_lengths(page, blocks, prefix):
    check(page=page, blocks=blocks, prefix=(prefix, max(0, prefix - 1)), seed=prefix, any_scale=prefix % 2 == 0)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("beam", [5, 9])
@pytest.mark.parametrize("own", [511, 513, 1300])
def test_long_own_tokens_beside_prefixes_of_many_rows(D, beam, own):
    """In one launch with prefixes of two and four wavefronts."""
    check(G=2, beam=beam, T=2, H=1, rep=4, D=D, prefix=(200, 37), own=(own, 3, 0, own - 70, 512, 40, 1), seed=own, dtype=F16)
    check(G=1, beam=beam, T=1, H=3, rep=8, D=D, prefix=(0,), own=(7, own), seed=own + 1)


@pytest.mark.parametrize("own", [0, 1, 2, 31, 32, 33, 64, 65, 300])
@pytest.mark.parametrize("G", [0, 1])
def test_own_lengths(own, G):
    check(G=G, beam=3, T=2, own=(own, own + 1, max(0, own - 1)), page=8, blocks=2, seed=own)


@pytest.mark.parametrize("G,beam,T,rep", [(1, 1, 1, 1), (1, 4, 1, 2), (1, 16, 1, 1), (1, 17, 1, 1), (1, 8, 4, 1),
                                          (1, 11, 3, 1), (1, 16, 6, 1), (2, 16, 4, 2), (1, 16, 5, 4), (1, 50, 9, 1),
                                          (3, 2, 2, 5), (1, 1, 200, 1), (1, 3, 40, 2)])
@pytest.mark.parametrize("dtype,D", [(BF16, 64), (F16, 64), (F16, 128), (BF16, 112), (F16, 256)])
def test_rows_sharing_a_prefix(G, beam, T, rep, dtype, D):
    """From one row a key to hundreds."""
    check(G=G, beam=beam, T=T, rep=rep, H=1, prefix=(200, 77, 150), own=(T + 3, T, T + 40, T + 100), D=D, blocks=2,
          dtype=dtype, seed=beam)


def test_long_prefix():
    check(G=2, beam=2, T=2, prefix=(9000, 4097), own=(700, 2, 350, 33), D=128, page=64)
    check(G=1, beam=1, T=1, H=1, rep=4, prefix=(20011,), own=(1,), D=128, page=32, dtype=F16)


@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("page", [2, 4, 8, 16, 24, 32, 48])
@pytest.mark.parametrize("beam", [1, 40])
def test_pages_and_tiles(D, page, beam):
    """Pages smaller than a load's keys, than a tile, and neither."""
    check(G=1, beam=beam, T=2, H=1, rep=1, D=D, page=page, blocks=2, prefix=(301,), own=(40, 3, 77), seed=page)


@pytest.mark.parametrize("T", [1, 4, 20])
def test_ragged_queries(T):
    """Sequences with fewer query tokens, none, or more than they have own tokens."""
    q_lengths = np.array([T, 0, 1, -3, 99, (T + 1) // 2])
    check(G=2, beam=3, T=T, q_lengths=q_lengths, own=(T, 5, 1, 3, T - 1, T + 50), prefix=(40, 0), seed=T)
    check(G=0, beam=6, T=T, q_lengths=q_lengths, own=(0, 5, 0, 3, T - 1, T // 2), dtype=F16, seed=T)


def test_prompts():
    """Many blocks of rows that see each other."""
    n = np.array([300, 151])
    for D, dtype in ((96, F16), (128, BF16), (64, F16)):
        check(G=0, beam=2, T=300, H=2, rep=4, D=D, page=16, own=(320, 411), dtype=dtype, seed=1)
        check(G=1, beam=2, T=300, H=2, rep=4, D=D, page=64, blocks=2, prefix=(70,), own=(320, 384), q_lengths=n, seed=2)


def test_prefix_only_and_own_only():
    rng = np.random.default_rng(3)
    q, (kc, ks), (vc, vs) = randn(rng, F16, 6, 2, 4, 64), *(cache(rng, 9, 8, 2, 2, 64) for _ in "kv")
    table = rng.permutation(9)
    compare(q, kc, ks, vc, vs, None, None, table[:6].reshape(3, 2), [16, 0, 5])
    compare(q, kc, ks, vc, vs, table[:6].reshape(6, 1), [8, 0, 1, 2, 7, 3], None, None)
    out, lse = ng.attend(q, kc, vc, return_lse=True, k_scale=ks, v_scale=vs)
    assert not out.any() and torch.isneginf(lse).all()
    out, lse = ng.attend(q, kc[:0], vc[:0], ints(table[:6].reshape(6, 1)), ints([8] * 6), return_lse=True, k_scale=ks[:0],
                         v_scale=vs[:0])
    assert not out.any() and torch.isneginf(lse).all()


def test_lengths_past_the_tables():
    rng = np.random.default_rng(1)
    q, (kc, ks), (vc, vs) = randn(rng, BF16, 4, 3, 2, 64), *(cache(rng, 12, 4, 1, 1, 64) for _ in "kv")
    table = rng.permutation(12)
    compare(q, kc, ks, vc, vs, table[:8].reshape(4, 2), [99, -5, 8, 2 ** 31 - 1], table[8:].reshape(2, 2), [9, -(2 ** 31)])


def test_pages_outside_the_cache():
    """Their keys take no part, at any place of a tile."""
    def holes(q, kc, ks, vc, vs, pages, prefix_pages):
        prefix_pages = prefix_pages.copy()
        prefix_pages[0, ::3], prefix_pages[0, 1::3], prefix_pages[1, :] = -1, len(kc), 2 ** 31 - 1
        pages = pages.copy()
        pages[0, 0], pages[1, -1], pages[3, :] = -7, len(kc) + 1, -(2 ** 31)
        return q, kc, ks, vc, vs, pages, prefix_pages
    for page in (4, 16, 64):
        for D in (64, 80):
            check(T=3, page=page, D=D, prefix=(200, 100), own=(30, 70, 20, 9), change=holes)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("T,beam", [(1, 2), (6, 3), (30, 2)])
@pytest.mark.parametrize("D", [64, 112, 256])
def test_values_that_no_row_sees(dtype, T, beam, D):
    """Whatever the cache holds past the lengths, in other pages, scales among it, and at tokens later than a query does not
    reach its row; a value that a row does see does."""
    def spoil(q, kc, ks, vc, vs, pages, prefix_pages):
        kb, vb = torch.full_like(kc.view(torch.uint8), 0x7f), torch.full_like(vc.view(torch.uint8), 0xff)
        bad = [torch.full_like(ks, float("nan")), torch.full_like(vs, float("inf"))]
        for tables, lengths in ((prefix_pages, prefix), (pages, own)):
            for row, n in zip(tables, lengths):
                for j in range(n):
                    at = int(row[j // page]), j % page
                    kb[at], vb[at] = kc.view(torch.uint8)[at], vc.view(torch.uint8)[at]
                    bad[0][at], bad[1][at] = ks[at], vs[at]
        # the last tokens of sequence 0 are seen by its last queries only
        for j in range(own[0] - (T + 1) // 2, own[0]):
            at = int(pages[0][j // page]), j % page
            vb[at][0, 5] = 0x7f
            if j % 2:
                bad[1][at][1] = float("nan")
            if j == own[0] - 1:
                kb[at][1, 3] = 0xff
                bad[0][at][0] = float("nan")
        return q, kb.view(E4M3), bad[0], vb.view(E4M3), bad[1], pages, prefix_pages

    page = 16
    prefix, own = np.array([37, 50]), np.resize([T + 11, T, T + 33, T + 2], 2 * beam)
    out = check(G=2, beam=beam, T=T, D=D, prefix=prefix, own=own, page=page, blocks=page, dtype=dtype, change=spoil)
    assert torch.isfinite(out[1:]).all()
    if T > 1:
        assert torch.isfinite(out[0, 0]).all() and not torch.isfinite(out[0, -1]).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_scales_far_apart(dtype):
    """Blocks whose scales lie 2^60 apart: the small ones count where the large ones have zeros or no weight."""
    def apart(q, kc, ks, vc, vs, pages, prefix_pages):
        vb = vc.view(torch.uint8).clone()
        vs = vs.clone()
        vs[::2] *= 2.0 ** -30
        vs[1::2] *= 2.0 ** 6 if q.dtype == F16 else 2.0 ** 30
        vb[1::2, :, :, :20] = 0
        return q, kc, ks, vb.view(E4M3), vs, pages, prefix_pages
    for T, rep in ((1, 2), (9, 4)):
        check(T=T, rep=rep, prefix=(300, 100), own=(T + 30, T + 9), dtype=dtype, change=apart)

    def loud(q, kc, ks, vc, vs, pages, prefix_pages):   # keys of one block far above the others
        ks = ks.clone()
        ks[::3] *= 8
        return q, kc, ks, vc, vs, pages, prefix_pages
    check(T=2, prefix=(300, 100), own=(30, 9), dtype=dtype, D=32, change=loud)
    check(scale=0.0, dtype=dtype)
    check(scale=-0.3, D=16, dtype=dtype)


@pytest.mark.parametrize("off", [0, 1, 8, 16])
def test_strides(off):
    """Queries split from a projection, caches with heads first, keys and values in one tensor, any offset."""
    def split(q, kc, ks, vc, vs, pages, prefix_pages):
        S, T, Hq, D = q.shape
        view = torch.zeros(S, T, Hq * D + 5 + off, dtype=q.dtype, device="cuda")[..., off:off + Hq * D].unflatten(
            -1, (Hq, D))
        view.copy_(q)
        return view, kc, ks, vc, vs, pages, prefix_pages

    def heads_first(q, kc, ks, vc, vs, pages, prefix_pages):
        turn = [x.view(torch.uint8).transpose(1, 2).contiguous().transpose(1, 2).view(E4M3) for x in (kc, vc)]
        scales = [x.permute(2, 1, 0).contiguous().permute(2, 1, 0) for x in (ks, vs)]
        return q.transpose(0, 1).contiguous().transpose(0, 1), turn[0], scales[0], turn[1], scales[1], pages, prefix_pages

    def together(q, kc, ks, vc, vs, pages, prefix_pages):
        D = q.shape[-1]
        wide = torch.full((*kc.shape[:3], 2 * D + off), 0x7f, dtype=torch.uint8, device="cuda")
        wide[..., off:off + D], wide[..., off + D:] = kc.view(torch.uint8), vc.view(torch.uint8)
        wide, both = wide.view(E4M3), torch.stack([ks, vs], -1)
        return q, wide[..., off:off + D], both[..., 0], wide[..., off + D:], both[..., 1], pages, prefix_pages

    def one_for_all(q, kc, ks, vc, vs, pages, prefix_pages):
        kc, vc = (x.view(torch.uint8)[:, :, :1].expand(x.shape).view(E4M3) for x in (kc, vc))
        return (q[:, :, :1].expand(q.shape), kc, ks[:1, :1, :1].expand(ks.shape), vc, vs[:1, :1, :1].expand(vs.shape), pages,
                prefix_pages)

    for change in (split, heads_first, together, one_for_all):
        for T in (1, 5):
            check(T=T, own=(5, 9, 7, 30), change=change, D=64, blocks=2)


def test_offsets_past_32_bits():
    """Pages further apart than 2^31 elements, tables whose rows are apart."""
    pages, page, H, D = 3, 32, 2, 64
    stride = (1 << 31) + 128
    rng = np.random.default_rng(2)
    (small_k, ks), (small_v, vs) = (cache(rng, pages, page, 1, H, D) for _ in "kv")
    kc, vc = (torch.zeros(2 * stride + page * H * D, dtype=torch.uint8, device="cuda").as_strided(
        (pages, page, H, D), (stride, H * D, D, 1)) for _ in range(2))
    kc.copy_(small_k.view(torch.uint8)), vc.copy_(small_v.view(torch.uint8))
    q = randn(rng, F16, 2, 3, 4, D)
    wide = torch.full((2, 7), -1, dtype=torch.int32, device="cuda")
    wide[:, :2] = ints([[2, 0], [1, 2]])
    args = dict(pages=wide[:, :2], lengths=ints([60, 33]), prefix_pages=ints([[2]]), prefix_lengths=ints([30]), k_scale=ks,
                v_scale=vs)
    got, want = ng.attend(q, kc.view(E4M3), vc.view(E4M3), **args), ng.attend(q, small_k, small_v, **args)
    assert torch.equal(got, want) and want.any()


@pytest.mark.parametrize("D", [48, 96, 112, 128])
@pytest.mark.parametrize("T,rep", [(40, 2), (9, 1), (20, 2), (1, 4)])
def test_what_ran_before_does_not_matter(D, T, rep):
    """Equal bits after calls that leave zeros, NaN and infinities in the chip's LDS."""
    from test_gpu_attend_edges import fill_lds
    rng = np.random.default_rng(D)
    q, (kc, ks), (vc, vs) = randn(rng, BF16, 8, T, 2 * rep, D), *(cache(rng, 40, 64, 2, 2, D) for _ in "kv")
    args = (q, kc, vc, ints(rng.permutation(40).reshape(8, 5)), ints([320, 256, 190, 128, 320, 64, 250, 320]))
    fill_lds(0.0)
    want = ng.attend(*args, k_scale=ks, v_scale=vs)
    assert want.isfinite().all()
    for value in (float("nan"), 0.0, float("inf")):
        fill_lds(value)
        assert torch.equal(ng.attend(*args, k_scale=ks, v_scale=vs), want), value


def test_other_stream_and_graph():
    rng = np.random.default_rng(4)
    q, (kc, ks), (vc, vs) = randn(rng, F16, 4, 2, 4, 64), *(cache(rng, 60, 16, 1, 2, 64) for _ in "kv")
    args = (ints(np.arange(8).reshape(4, 2)), ints([20, 5, 32, 9]), ints(np.arange(8, 58).reshape(1, 50)), ints([800]))
    want = ng.attend(q, kc, vc, *args, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = ng.attend(q, kc, vc, *args, k_scale=ks, v_scale=vs, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ng.attend(q, kc, vc, *args, k_scale=ks, v_scale=vs)
    for i in range(4):
        q.mul_(-0.7)
        vs.mul_(2)
        args[3].sub_(150)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, ng.attend(q, kc, vc, *args, k_scale=ks, v_scale=vs)), i


def test_what_append_writes():
    """Tokens appended one by one and at once are attended to as what the cache then holds."""
    rng = np.random.default_rng(6)
    S, page, H, D = 3, 16, 2, 64
    tables = rng.permutation(12).reshape(S, 4)
    kc, vc = (torch.zeros(12, page, H, D, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    ks, vs = torch.zeros(12, 2, H, device="cuda"), torch.zeros(12, 2, H, device="cuda")
    cos, sin = ng.rope_table(64, 32)
    start = np.array([0, 3, 10])
    for i, T in enumerate((20, 1, 1, 7, 1)):
        k, v, q = (randn(rng, F16, S, T, h, D) * 2.0 ** i for h in (H, H, 4))
        q = ng.kv_append(k, v, kc, vc, ints(tables), ints(start), cos=cos, sin=sin, q=q, k_scale=ks, v_scale=vs) / 2 ** i
        start = start + T
        live = [x.clone() for x in (ks, vs)]
        for s in live:
            s[s == 0] = 1   # (blocks that hold nothing yet)
        compare(q, kc, live[0], vc, live[1], tables, start, None, None, scale=0.01)


def test_refusals():
    kc, vc = (torch.zeros(6, 8, 2, 16, dtype=E4M3, device="cuda") for _ in range(2))
    s = torch.ones(6, 2, 2, device="cuda")
    q = torch.zeros(4, 3, 4, 16, dtype=F16, device="cuda")
    ok = dict(q=q, k_cache=kc, v_cache=vc, pages=ints([[0]] * 4), lengths=ints([3] * 4), prefix_pages=ints([[1], [2]]),
              prefix_lengths=ints([3, 4]), k_scale=s, v_scale=s)
    assert math.isfinite(float(ng.attend(**ok).float().sum()))

    def bad(error, **kw):
        with pytest.raises(error):
            ng.attend(**{**ok, **kw})

    bad(ValueError, k_scale=None)
    bad(ValueError, v_scale=None)
    bad(TypeError, k_scale=None, v_scale=None)
    bad(TypeError, k_cache=kc.half(), v_cache=vc.half())
    bad(TypeError, v_cache=vc.half())
    bad(TypeError, q=q.float())
    bad(TypeError, q=q.to(E4M3))
    bad(TypeError, q=q.cpu())
    bad(ValueError, q=q[0])
    bad(ng.NgpuError, q=q[:, :, :3])
    bad(ValueError, v_cache=vc[:5])
    bad(ValueError, k_scale=s[:5])
    bad(ValueError, k_scale=torch.ones(6, 3, 2, device="cuda"), v_scale=torch.ones(6, 3, 2, device="cuda"))
    bad(TypeError, k_scale=s.half())
    bad(TypeError, k_scale=s.cpu())
    bad(TypeError, v_scale=s.clone().requires_grad_())
    bad(ng.NgpuError, scale=float("inf"))
    wide = torch.zeros(6, 8, 2, 300, dtype=E4M3, device="cuda")
    bad(ng.NgpuError, q=torch.zeros(4, 3, 4, 300, dtype=F16, device="cuda"), k_cache=wide, v_cache=wide)
    for shape in ((4, 0, 4, 16), (0, 3, 4, 16)):
        got = ng.attend(torch.zeros(shape, dtype=F16, device="cuda"), kc, vc, k_scale=s, v_scale=s)
        assert got.shape == shape
