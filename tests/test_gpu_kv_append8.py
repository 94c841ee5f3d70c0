"""Appending to a cache in 8 bits against its definition.

Values are copied and keys rotated in fp32 by two products and a sum, each rounded, which the reference does alike:
the bytes and scales have to be equal, with keys that were rotated by numpy in fp32.  Queries are rounded once to the
type and have to be equal too."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import beam_reference as ref  # noqa: E402
import paper_2505_22857_amd as ng  # noqa: E402

F16, BF16, E4M3 = torch.float16, torch.bfloat16, torch.float8_e4m3fn
HALF, INTER = ng.NGPU_ROPE_HALF, ng.NGPU_ROPE_INTERLEAVED
VALUES = ref.e4m3_values()


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def host(x):
    return x.float().cpu().numpy()


def values(bits):
    return VALUES[bits.cpu().numpy()]


def turned(x, cos, sin, pos, layout):
    """x [S, T, H, D] fp32 with the first dimensions rotated, products and sums rounded to fp32 each."""
    y, R = x.copy(), 2 * cos.shape[1]
    i = np.arange(R // 2)
    a, b = (i, i + R // 2) if layout == HALF else (2 * i, 2 * i + 1)
    ok = (pos >= 0) & (pos < len(cos))
    c, s = cos[np.where(ok, pos, 0)][:, :, None], sin[np.where(ok, pos, 0)][:, :, None]
    with np.errstate(over="ignore", invalid="ignore"):
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    y[~ok] = np.where(np.arange(x.shape[-1]) < R, np.nan, y[~ok]) if (~ok).any() else y[~ok]
    return y


def check(S=3, T=5, H=2, Hq=4, D=64, rotary=64, layout=HALF, page=8, block=8, dtype=BF16, start=None, lengths=None,
          positions=None, tables=None, size=1.0, change=None, rows=64, wide=0, times=1, scales=None, seed=0):
    rng = np.random.default_rng(seed)
    print(f"[case] append8 S={S} T={T} H={H}/{Hq} D={D} R={rotary} {layout} page={page}/{block} {dtype}", flush=True)
    width = 6
    P = S * width + 2
    k, v, q = (torch.from_numpy((rng.standard_normal((S, T, h, D)) * size).astype(np.float32)).cuda().to(dtype)
               for h in (H, H, Hq))
    if change is not None:
        change(k, v)
    bits = [torch.from_numpy(rng.integers(0, 256, (P, page, H, D + wide), dtype=np.uint8)).cuda() for _ in range(2)]
    caches = [b.view(E4M3)[..., :D] for b in bits]
    if scales is None:
        scales = [np.exp2(rng.integers(-9, 3, (P, page // block, H))).astype(np.float32) for _ in range(2)]
    on = [torch.from_numpy(s).cuda() for s in scales]
    tables = rng.permutation(P)[:S * width].reshape(S, width) if tables is None else np.asarray(tables)
    start = rng.integers(0, width * page - T, S) if start is None else np.asarray(start)
    cos, sin = ng.rope_table(rows, rotary) if rotary else (None, None)
    pos = start[:, None] + np.arange(T) if positions is None else np.asarray(positions)
    counts = [T if lengths is None else min(max(int(lengths[s]), 0), T) for s in range(S)]
    x = [host(k), host(v), host(q)]
    if rotary:
        x[0], x[2] = (turned(y, host(cos), host(sin), pos, layout) for y in (x[0], x[2]))
    kw = {} if rotary == 0 else dict(cos=cos, sin=sin, layout=layout, positions=None if positions is None else ints(pos))
    before = [values(b) for b in bits]
    for _ in range(times):
        out = ng.kv_append(k, v, *caches, ints(tables), ints(start), q=q, k_scale=on[0], v_scale=on[1],
                           lengths=None if lengths is None else ints(lengths), **kw)
    for i, (b, was) in enumerate(zip(bits, before)):
        want, scale, known = ref.append8(x[i], was[..., :D], scales[i], tables, start, counts)
        got = values(b)
        assert np.array_equal(host(on[i]), scale, equal_nan=True), "scales"   # (of blocks that are not written to)
        assert np.array_equal(got[..., :D], want, equal_nan=True), "elements"   # also those that are not meant
        assert np.array_equal(got[..., D:], was[..., D:], equal_nan=True)
    want = torch.from_numpy(x[2]).to(dtype).float().numpy()
    for s in range(S):
        want[s, counts[s]:] = 0
    assert np.array_equal(host(out), want, equal_nan=True)
    return caches, on


@pytest.mark.parametrize("D,rotary", [(64, 64), (64, 32), (128, 128), (128, 64), (80, 80), (80, 32), (96, 48), (256, 256),
                                      (256, 32), (2, 2), (10, 6), (24, 16), (33, 32), (1, 0), (72, 8), (64, 0), (40, 24)])
@pytest.mark.parametrize("layout", [HALF, INTER])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_dimensions(D, rotary, layout, dtype):
    check(D=D, rotary=rotary, layout=layout, dtype=dtype, seed=D + rotary)
    check(D=D, rotary=rotary, layout=layout, dtype=dtype, S=1, T=1, H=1, Hq=1, page=1, block=1, seed=D)


@pytest.mark.parametrize("page,block", [(1, 1), (8, 2), (16, 16), (64, 32), (6, 3), (7, 7), (48, 1), (128, 128)])
@pytest.mark.parametrize("T", [1, 2, 9, 33, 100])
def test_blocks(page, block, T):
    if T > 6 * page:
        T = 6 * page - 1 or 1
    check(page=page, block=block, T=T, D=128, H=3, Hq=3, rotary=64, start=[0, 0, 1] if T >= 6 * page - 1 else None, rows=800, seed=T)
    check(page=page, block=block, T=T, D=40, H=1, Hq=1, rotary=0, wide=3, start=[0, 0, 0] if T >= 6 * page - 1 else None, seed=T)


@pytest.mark.parametrize("times", [1, 2])
def test_growing_scales(times):
    """Large tokens behind small ones: what is there is rounded again, once."""
    for size in (1e-3, 1.0, 300.0, 3e4):
        check(size=size, page=16, block=16, start=[3, 15, 7], T=4, times=times, seed=int(size))
    old = [np.full((20, 1, 2), s, np.float32) for s in (0.3, 1.7)]   # scales that are no powers of two
    check(page=8, block=8, start=[1, 2, 3], T=2, size=2.0, scales=old)
    check(page=8, block=8, start=[1, 2, 3], T=2, size=500.0, scales=old)


def test_scales_that_are_none():
    """A block's earlier entries with a scale of 0, less, NaN or infinity, as in memory that was never written."""
    bad = np.array([0.0, -1.0, np.nan, np.inf, 1e-38, 2.0 ** -100, 2.0 ** 120, 3.4e38], np.float32)
    for shift in range(4):
        s = np.resize(np.roll(bad, shift), (20, 1, 2)).astype(np.float32)
        check(page=8, block=8, start=[1, 7, 3], T=2, size=1.0, scales=[s, s[::-1].copy()], seed=shift)
        check(page=8, block=8, start=[0, 8, 16], T=2, size=1.0, scales=[s, s[::-1].copy()], seed=shift)


def test_borders_of_the_scale():
    """Largest elements around 448 * 2^e, zeros, the smallest and the largest numbers of the types."""
    for dtype, points in ((BF16, [1.75, 1.765625, 1.7421875, 1.0, 2.0, 0.0, 1e-38, 1e-45, 3e38, 2.0 ** -100, 448.0, 450.0]),
                          (F16, [1.75, 1.751, 1.7490234375, 448.0, 448.25, 65504.0, 6e-8, 0.0, 2.0 ** -14])):
        for p in points:
            def change(k, v, p=p):
                for x in (k, v):
                    x.mul_(0)
                    x[..., 3] = p
                    x[0, 0, :, 1] = -p / 3
            check(dtype=dtype, change=change, rotary=0, start=[0, 8, 5], T=3)


@pytest.mark.parametrize("D", [64, 33])
def test_numbers_that_are_not_finite(D):
    """Infinities and NaN become NaN where they stand, and the scale goes by the others."""
    def change(k, v):
        for x in (k, v):
            x[0, 1, 0, 5], x[0, 2, 1, 7], x[1, 0, 0, 0], x[1, 1, :, 2] = float("inf"), -float("inf"), float("nan"), 9.0
            x[2] = float("nan")
    check(D=D, rotary=32, change=change)
    check(D=D, rotary=0, change=change, page=16, block=4)


def test_every_value_and_every_tie():
    """Elements at, between and halfway between the 8-bit values, with both signs, scaled by 1."""
    levels = np.unique(np.abs(VALUES[~np.isnan(VALUES)]))
    mid = (levels[1:] + levels[:-1]) / 2
    x = np.concatenate([levels, mid, mid * (1 + 2.0 ** -7), mid * (1 - 2.0 ** -7)])
    x = np.concatenate([x, -x, np.full(-2 * len(x) % 63, 3.0)]).reshape(-1, 63)
    x = np.concatenate([np.full((len(x), 1), 448.0), x], 1)

    def change(k, v):
        for y in (k, v):
            y.copy_(torch.from_numpy(x.astype(np.float32))[None, :, None].expand(y.shape).to(y))
    for dtype in (F16, BF16):
        check(S=1, T=len(x), H=2, D=64, rotary=0, page=4, block=1, change=change, dtype=dtype, start=[1]) if len(x) <= 22 else \
            check(S=1, T=len(x), H=2, D=64, rotary=0, page=64, block=1, change=change, dtype=dtype, start=[1])


def test_ragged_and_outside():
    """Padding, places before 0 and behind the table, pages outside the cache, positions outside the tables."""
    check(lengths=[0, 3, 9])
    check(lengths=[-4, 5, 1], page=4, block=2)
    check(start=[-3, 46, 44], T=5)
    check(start=[-9, 100, 2 ** 31 - 3], T=5, rotary=0)
    tables = np.arange(18).reshape(3, 6)
    tables[0, 0], tables[1, 1], tables[2] = -1, 400, -5
    check(tables=tables, start=[5, 5, 0], T=12)
    check(positions=np.array([[0, 1, 2, 3, 4], [-1, 63, 64, 5, 5], [9, 8, 7, -2 ** 31, 2 ** 31 - 1]]))


def test_strides():
    """Queries, keys and values of one projection, and odd places."""
    rng = np.random.default_rng(0)
    tables, start = np.arange(12).reshape(2, 6), np.array([3, 9])
    for odd in (0, 1):
        buf = torch.from_numpy(rng.standard_normal(2 * 4 * 6 * 64 + odd).astype(np.float32)).cuda().half()
        q, k, v = buf[odd:].view(2, 4, 6, 64).split((2, 2, 2), 2)
        kc, vc = (torch.zeros(14, 8, 2, 64, dtype=torch.uint8, device="cuda").transpose(1, 2).contiguous().transpose(1, 2)
                  .view(E4M3) for _ in range(2))
        whole = torch.zeros(2, 2, 2, 14, device="cuda")   # [k or v, heads, blocks, pages]
        ks, vs = whole.permute(0, 3, 2, 1).unbind(0)
        out = ng.kv_append(k, v, kc, vc, ints(tables), ints(start), q=q, k_scale=ks, v_scale=vs)
        for x, c, s in ((k, kc, ks), (v, vc, vs)):
            want, scale, known = ref.append8(host(x), np.zeros((14, 8, 2, 64)), np.zeros((14, 2, 2), np.float32), tables,
                                             start, [4, 4])
            assert np.array_equal(host(s), scale)
            assert np.array_equal(values(c.view(torch.uint8))[known], want[known])
        assert torch.equal(out, q)


def test_empty_calls():
    check(S=1, T=3, lengths=[0], start=[0])
    c = torch.zeros(4, 8, 2, 64, dtype=E4M3, device="cuda")
    s = torch.ones(4, 1, 2, device="cuda")
    for S, T in ((0, 3), (3, 0)):
        k = torch.zeros(S, T, 2, 64, dtype=F16, device="cuda")
        ng.kv_append(k, k, c, c.clone(), ints(np.zeros((S, 2))), ints(np.zeros(S)), k_scale=s, v_scale=s.clone())
    assert not c.view(torch.uint8).any() and bool((s == 1).all())


def test_refusals():
    k = torch.zeros(2, 3, 2, 64, dtype=F16, device="cuda")
    c, s = torch.zeros(4, 8, 2, 64, dtype=E4M3, device="cuda"), torch.ones(4, 2, 2, device="cuda")
    t, st = ints(np.zeros((2, 2))), ints([0, 8])
    with pytest.raises(ValueError, match="together"):
        ng.kv_append(k, k, c, c, t, st, k_scale=s)
    with pytest.raises(TypeError, match="float8"):
        ng.kv_append(k, k, c, c, t, st)
    with pytest.raises(TypeError, match="float8"):
        ng.kv_append(k, k, c.half(), c.half(), t, st, k_scale=s, v_scale=s)
    with pytest.raises(TypeError, match="float16 or bfloat16"):
        ng.kv_append(k.float(), k.float(), c, c, t, st, k_scale=s, v_scale=s)
    with pytest.raises(TypeError, match="v must be"):
        ng.kv_append(k, k.bfloat16(), c, c, t, st, k_scale=s, v_scale=s)
    for bad in (s[:3], s[:, :, :1], torch.ones(4, 3, 2, device="cuda"), s[0], torch.ones(4, 0, 2, device="cuda")):
        with pytest.raises(ValueError):
            ng.kv_append(k, k, c, c, t, st, k_scale=bad, v_scale=bad)
    with pytest.raises(TypeError):
        ng.kv_append(k, k, c, c, t, st, k_scale=s.double(), v_scale=s)
    with pytest.raises(TypeError, match="gradient"):
        ng.kv_append(k.clone().requires_grad_(), k, c, c, t, st, k_scale=s, v_scale=s)


def test_copies_take_the_scales_along():
    rng = np.random.default_rng(2)
    for D, page, blocks in ((64, 16, 2), (33, 6, 3), (128, 8, 1)):
        bits = [torch.from_numpy(rng.integers(0, 256, (9, page, 2, D), dtype=np.uint8)).cuda() for _ in range(2)]
        scales = [torch.rand(9, blocks, 2, device="cuda") for _ in range(2)]
        before = [x.cpu().numpy() for x in bits + scales]
        copies = np.array([[0, 5, 3], [8, 1, page], [-1, 2, 4], [3, 9, 4], [4, 6, 0], [7, 2, 1]])
        ng.kv_copy(*(b.view(E4M3) for b in bits), ints(copies), k_scale=scales[0], v_scale=scales[1])
        for x, was in zip(bits, before):
            assert np.array_equal(x.cpu().numpy(), ref.copy(was, copies))
        whole = copies.copy()
        whole[:, 2] = np.where(copies[:, 2] > 0, blocks, 0)
        for x, was in zip(scales, before[2:]):
            assert np.array_equal(x.cpu().numpy(), ref.copy(was, whole))


def test_in_a_graph():
    k = torch.randn(3, 2, 2, 64, device="cuda").half()
    c = [torch.zeros(6, 8, 2, 64, dtype=torch.uint8, device="cuda") for _ in range(2)]
    s = [torch.ones(6, 1, 2, device="cuda") for _ in range(2)]
    tables, start = ints(np.arange(6).reshape(3, 2)), ints([0, 0, 0])

    def call():
        ng.kv_append(k, k, c[0].view(E4M3), c[1].view(E4M3), tables, start, k_scale=s[0], v_scale=s[1])
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for x in c:
        x.zero_()
    for step in range(4):
        k.normal_(std=3.0 ** step)
        was = [values(x) for x in c], [host(x) for x in s]
        graph.replay()
        torch.cuda.synchronize()
        for i in range(2):
            want, scale, _ = ref.append8(host(k), was[0][i], was[1][i], tables.cpu().numpy(), start.cpu().numpy(), [2] * 3)
            assert np.array_equal(values(c[i]), want) and np.array_equal(host(s[i]), scale)
        start += 2
