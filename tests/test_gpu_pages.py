"""Forking, compacting and copying pages against their definitions, one after the other.  Integers and bytes:
everything has to be equal, also what is not to be written."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import beam_reference as ref  # noqa: E402
import paper_2505_22857_amd as ng  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def host(x):
    return x.cpu().numpy()


def tables(rng, G, W, page, trunk, past, spare, width=None):
    """Consistent tables: a group's rows share whole pages of a trunk, some also a page filled in part."""
    width = width or trunk // page + past // page + 3
    P = G * (trunk // page + W * (past // page + 1)) + spare
    numbers = rng.permutation(P)
    pages, lengths, at = np.full((G * W, width), -1, np.int32), np.zeros(G * W, np.int32), 0
    for g in range(G):
        shared = numbers[at:at + trunk // page]
        at += len(shared)
        for w in range(W):
            n = trunk // page * page + int(rng.integers(0, past + 1))
            if w > 0 and rng.random() < 0.3:   # a fork that has not been appended to
                pages[g * W + w], lengths[g * W + w] = pages[g * W + w - 1], lengths[g * W + w - 1]
                continue
            more = -(-n // page) - len(shared)
            pages[g * W + w, :len(shared)] = shared
            pages[g * W + w, len(shared):len(shared) + more] = numbers[at:at + more]
            lengths[g * W + w] = n
            at += more
    refs = np.bincount(pages[pages >= 0], minlength=P).astype(np.int32)
    return pages, lengths, refs


def check_fork(pages, lengths, parents, refs, page, tokens, wide=0):
    G, K = parents.shape
    print(f"[case] fork G={G} rows={len(pages)} K={K} width={pages.shape[1]} page={page} pool={len(refs)}", flush=True)
    per_row = np.broadcast_to(np.asarray(tokens), (G, K))
    want = ref.fork(pages, lengths, parents, refs, page, per_row)
    table = torch.full((len(pages), pages.shape[1] + wide), 77, dtype=torch.int32, device="cuda")
    table[:, :pages.shape[1]] = ints(pages)
    counts = ints(refs)
    got = ng.kv_fork(table[:, :pages.shape[1]], ints(lengths), ints(parents), counts, page,
                     tokens=int(tokens) if np.ndim(tokens) == 0 else ints(per_row))
    for name, x, y in zip(("pages", "lengths", "copies", "refs"), (*got, counts), want):
        assert np.array_equal(host(x), y), name
    assert np.array_equal(host(table[:, :pages.shape[1]]), pages)
    return want


@pytest.mark.parametrize("G,W,K", [(1, 1, 1), (1, 4, 4), (3, 5, 2), (2, 1, 7), (16, 8, 8), (5, 64, 64), (300, 2, 3),
                                   (1, 300, 300), (70, 1, 1), (4, 3, 0)])
@pytest.mark.parametrize("page,tokens", [(16, 1), (1, 1), (8, 0), (4, 9), (7, 3), (64, 1)])
def test_forks(G, W, K, page, tokens):
    rng = np.random.default_rng(G * 1000 + W * 10 + page)
    pages, lengths, refs = tables(rng, G, W, page, trunk=5 * page + 3, past=3 * page, spare=G * K * (tokens // page + 2))
    parents = rng.integers(-1, W + 1, (G, K)).astype(np.int32)   # W: outside, so none
    after = check_fork(pages, lengths, parents, refs, page, tokens)
    counted = np.bincount(after[0][after[0] >= 0], minlength=len(refs))
    assert np.array_equal(counted, after[3])   # refs are the entries that hold a page


@pytest.mark.parametrize("spare", [0, 1, 5, 20])
def test_too_few_pages_drop_rows(spare):
    rng = np.random.default_rng(spare)
    pages, lengths, refs = tables(rng, 6, 4, 8, trunk=24, past=16, spare=spare, width=9)
    tokens = rng.integers(0, 30, (6, 5))
    parents = rng.integers(0, 4, (6, 5)).astype(np.int32)
    after = check_fork(pages, lengths, parents, refs, 8, tokens)
    assert (after[1] == -1).any() == (spare < 20)   # by the definition alone: 20 are enough
    assert np.array_equal(np.bincount(after[0][after[0] >= 0], minlength=len(refs)), after[3])


def test_the_last_holder_keeps_the_page():
    """Three children of one parent with 5 of 8 entries: two copies; with a holder elsewhere, three."""
    pages, lengths = np.array([[3, 1, -1]]), np.array([13])
    refs = np.array([0, 1, 0, 1, 0, 0])
    after = check_fork(pages, lengths, np.zeros((1, 3), np.int32), refs, 8, 1)
    assert after[2].tolist() == [[1, 0, 5], [1, 2, 5], [-1, -1, 0]] and after[3].tolist() == [1, 1, 1, 3, 0, 0]
    refs[1] = 2
    assert check_fork(pages, lengths, np.zeros((1, 3), np.int32), refs, 8, 1)[2][:, 0].tolist() == [1, 1, 1]


def test_a_page_shared_by_two_groups():
    """Each group counts its own rows: both copy, and nobody holds the page then."""
    pages, lengths = np.array([[2, -1], [2, -1]]), np.array([3, 3])
    after = check_fork(pages, lengths, np.zeros((2, 1), np.int32), np.array([0, 0, 2, 0]), 4, 1)
    assert after[3].tolist() == [1, 1, 0, 0]


def test_a_new_sequence_and_its_end():
    """Prompts of ragged lengths from nothing, then all of it freed."""
    pages, zero = np.full((3, 6), -1, np.int32), np.zeros(3, np.int32)
    parents, tokens = np.zeros((3, 1), np.int32), np.array([[17], [0], [24]])
    after = check_fork(pages, zero, parents, np.zeros(9, np.int32), 4, tokens)
    assert (after[0] >= 0).sum(1).tolist() == [5, 0, 0] and after[1].tolist() == [0, 0, -1]
    after = check_fork(pages, zero, parents, np.zeros(11, np.int32), 4, tokens)
    assert (after[0] >= 0).sum(1).tolist() == [5, 0, 6]
    for empty in (np.zeros((3, 0), np.int32), np.full((3, 2), -1, np.int32)):
        assert not check_fork(after[0], tokens[:, 0], empty, after[3], 4, 0)[3].any()


def test_rejected_tokens_are_given_up():
    pages, refs = np.array([[0, 1, 2, 3], [0, 4, 5, -1]]), np.array([2, 1, 1, 1, 1, 1])
    after = check_fork(pages, np.array([9, 17]), np.array([[0], [0]]), refs, 8, 0)
    assert after[0].tolist() == [[0, 1, -1, -1], [0, 4, 5, -1]] and after[3].tolist() == [2, 1, 0, 0, 1, 1]


@pytest.mark.parametrize("wide", [0, 1, 3])
def test_tables_with_entries_outside_the_pool_and_strides(wide):
    """Entries outside [0, pages) hold nothing and go on as they are; lengths past the table are cut."""
    pages = np.array([[5, -7, 900, 2], [1, 0, -1, 3]])
    refs = np.bincount([5, 2, 1, 0, 3], minlength=8)
    for lengths in ([99, 6], [-5, 12], [12, 16], [15, 0]):
        check_fork(pages, np.array(lengths), np.array([[0, 1, 0, 1]]), refs, 4, 1, wide)
        check_fork(pages, np.array(lengths), np.array([[1, 1, 1]]), refs, 4, 0, wide)


def test_the_largest_numbers():
    """Tokens and lengths near 2^31 do not fit and are dropped; negative tokens count as none."""
    pages, refs = np.array([[0, 1]]), np.array([1, 1, 0])
    check_fork(pages, np.array([2 ** 31 - 1]), np.zeros((1, 3), np.int32), refs, 4,
               np.array([[2 ** 31 - 1, -2 ** 31, 1]]))
    check_fork(pages, np.array([5]), np.zeros((1, 2), np.int32), refs, 2 ** 31 - 1, 2 ** 31 - 1)


@pytest.mark.parametrize("P", [4095, 4096, 4097, 70000, 4096 * 1024 + 5])
def test_large_pools(P):
    """Free pages are found behind many blocks of used ones."""
    rng = np.random.default_rng(P)
    refs = np.where(rng.random(P) < 0.999, 1, 0).astype(np.int32)
    refs[:min(P // 2, 20000)] = 1
    refs[-3:] = 0
    free = np.flatnonzero(refs == 0)
    pages = np.full((5, 300), -1, np.int32)
    tokens = np.array([[2], [0], [min(300, len(free) - 2)], [1], [0]])
    after = check_fork(pages, np.zeros(5, np.int32), np.zeros((5, 1), np.int32), refs, 1, tokens)
    assert after[1].tolist() == [0, 0, 0, -1 if len(free) <= 302 else 0, 0]


def test_tables_without_entries():
    pages, lengths, refs = np.zeros((6400, 0), np.int32), np.arange(6400, dtype=np.int32), np.zeros(9, np.int32)
    parents = np.arange(40, dtype=np.int32).repeat(100).reshape(100, 40)
    for tokens in (0, 1):
        after = check_fork(pages, lengths, parents, refs, 4, tokens)
        assert (after[1] == -tokens).all()


def test_many_rows():
    """More rows than a block of them, in groups that span two."""
    rng = np.random.default_rng(5)
    pages, lengths, refs = tables(rng, 37, 30, 4, trunk=9, past=30, spare=3000)
    check_fork(pages, lengths, rng.integers(0, 30, (37, 30)).astype(np.int32), refs, 4, 3)
    pages, lengths, refs = tables(rng, 3, 700, 4, trunk=9, past=30, spare=1500)
    check_fork(pages, lengths, rng.integers(0, 700, (3, 500)).astype(np.int32), refs, 4, 3)


def check_compact(refs, page, *held):
    print(f"[case] compact pool={len(refs)} used={np.count_nonzero(refs)}", flush=True)
    copies, moved, after, new = ref.compact(refs, page, held)
    counts, on = ints(refs), [ints(t) for t in held]
    got = ng.kv_compact(counts, page, tables=on)
    assert np.array_equal(host(got[0]), copies) and np.array_equal(host(got[1]), moved)
    assert np.array_equal(host(counts), after)
    for x, y in zip(on, new):
        assert np.array_equal(host(x), y)


@pytest.mark.parametrize("P", [0, 1, 2, 3, 64, 65, 1000, 4096, 4097, 8192, 50001, 4096 * 1024 + 7])
@pytest.mark.parametrize("used", [0.0, 0.03, 0.5, 0.97, 1.0])
def test_compactions(P, used):
    rng = np.random.default_rng(P)
    refs = np.where(rng.random(P) < used, rng.integers(1, 9, P), 0).astype(np.int32)
    check_compact(refs, 16, rng.integers(-2, P + 2, (7, 13)).astype(np.int32), rng.integers(-1, max(P, 1), (1, 300)).astype(np.int32))


def test_compactions_of_one_side():
    """All used pages low, all high, alternating, and negative counts, which are not free."""
    for refs in ([1] * 5 + [0] * 9, [0] * 9 + [1] * 5, [0, 1] * 20, [1, 0] * 20, [0, -3, 0, 5]):
        check_compact(np.array(refs, np.int32), 1, np.arange(len(refs))[None].astype(np.int32))


def test_tables_of_a_compaction():
    refs = ints([0, 1, 0, 1])
    wide = ints([[3, 1, 3], [1, 3, -1]])
    ng.kv_compact(refs, 4, tables=(wide[:, :2],))   # behind its rows nothing is touched
    assert wide.tolist() == [[0, 1, 3], [1, 0, -1]]
    with pytest.raises(ValueError, match="twice"):
        ng.kv_compact(refs, 4, tables=(wide, wide))
    with pytest.raises(ValueError, match="overlap"):
        ng.kv_compact(refs, 4, tables=(wide[:1].expand(2, 3),))


def caches(rng, P, page, H, D, dtype, wide=0):
    bits = [torch.from_numpy(rng.integers(-30000, 30000, (P, page, H, D + wide), dtype=np.int16)).cuda() for _ in range(2)]
    return [b.view(dtype)[..., :D] for b in bits], bits


@pytest.mark.parametrize("D,H,page", [(64, 2, 16), (128, 8, 64), (256, 1, 1), (80, 3, 7), (33, 2, 5), (1, 1, 3), (8, 5, 130)])
@pytest.mark.parametrize("wide", [0, 8, 3])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_copies(D, H, page, wide, dtype):
    rng = np.random.default_rng(D + page)
    P = 23
    (kc, vc), bits = caches(rng, P, page, H, D, dtype, wide)
    before = [host(b) for b in bits]
    at = rng.permutation(P)
    copies = np.array([[at[0], at[1], page], [at[2], at[3], 1], [-1, at[4], page], [at[5], P, page], [at[6], at[6], page],
                       [at[0], at[7], (page + 1) // 2], [at[8], at[9], 0], [at[8], at[10], -5], [at[8], at[11], 10 ** 9],
                       [P + 3, at[12], page], [at[13], -1, page]])
    print(f"[case] copy D={D} H={H} page={page} wide={wide}", flush=True)
    assert ng.kv_copy(kc, vc, ints(copies)) is None
    for b, x in zip(bits, before):
        want = x.copy()
        want[..., :D] = ref.copy(x[..., :D], copies)
        assert np.array_equal(host(b), want)


def test_copies_of_other_layouts():
    """Heads before tokens, keys and values in one buffer, an odd first element, and no rows at all."""
    rng = np.random.default_rng(1)
    copies = np.array([[0, 5, 3], [2, 1, 4], [4, 3, 9]])
    both = torch.from_numpy(rng.integers(-30000, 30000, (6, 2, 3, 4, 64), dtype=np.int16)).cuda()
    odd = torch.from_numpy(rng.integers(-30000, 30000, 2 * 6 * 4 * 3 * 64 + 1, dtype=np.int16)).cuda()
    for bits in (both.transpose(2, 3).unbind(1), odd[1:].view(2, 6, 4, 3, 64).unbind(0)):
        before = [host(b) for b in bits]
        ng.kv_copy(*(b.view(torch.float16) for b in bits), ints(copies))
        for b, x in zip(bits, before):
            assert np.array_equal(host(b), ref.copy(x, copies))
        ng.kv_copy(*(b.view(torch.float16) for b in bits), ints(np.zeros((0, 3))))


def test_a_cache_whose_offsets_pass_32_bits():
    """Pages further apart than 2^31 elements."""
    buf = torch.zeros((1 << 31) + (1 << 30), dtype=torch.int16, device="cuda")
    kc = torch.as_strided(buf, (3, 2, 1, 64), (5 << 28, 64, 64, 1))
    kc[0] = 7
    half = kc.view(torch.float16)
    vc = torch.zeros(3, 2, 1, 64, dtype=torch.float16, device="cuda")
    ng.kv_copy(half, vc, ints([[0, 2, 2]]))
    assert int(kc[2].sum()) == 7 * 128 and int(kc[1].sum()) == 0


def test_a_step_of_forks_copies_and_appends():
    """Hypotheses fork, copy and append for a while: every hypothesis's tokens are those of its history."""
    rng = np.random.default_rng(3)
    G, W, page, width, P, H, D = 3, 4, 4, 8, 60, 2, 64
    kc, vc = (torch.zeros(P, page, H, D, dtype=torch.float16, device="cuda") for _ in range(2))
    refs = torch.zeros(P, dtype=torch.int32, device="cuda")
    pages, lengths = ints(np.full((G * W, width), -1)), ints(np.zeros(G * W))
    history = [[] for _ in range(G * W)]
    for step in range(25):
        parents = np.tile(np.arange(W), (G, 1)) if step == 0 else np.sort(rng.integers(0, W, (G, W)), 1)
        T = int(rng.integers(1, 3)) if step < 12 else 1
        pages, lengths, copies = ng.kv_fork(pages, lengths, ints(parents), refs, page, tokens=T)
        ng.kv_copy(kc, vc, copies)
        x = rng.integers(1, 1000, (G * W, T))
        k = ints(x).half()[..., None, None].expand(G * W, T, H, D).contiguous()
        ng.kv_append(k, -k, kc, vc, pages, lengths)
        lengths = lengths + T
        history = [history[g * W + parents[g, j]] + x[g * W + j].tolist() for g in range(G) for j in range(W)]
        if step % 7 == 6:
            moves, _ = ng.kv_compact(refs, page, tables=(pages,))
            ng.kv_copy(kc, vc, moves)
        if step == 15:   # the later half is given up
            lengths = lengths // 2
            history = [h[:len(h) // 2] for h in history]
        table, n = host(pages), host(lengths)
        assert np.array_equal(np.bincount(table[table >= 0], minlength=P), host(refs))
        for r in range(G * W):
            assert n[r] == len(history[r])
            at = [(table[r, i // page], i % page) for i in range(n[r])]
            assert [float(kc[p, e, 1, 5]) for p, e in at] == history[r]
            assert [-float(vc[p, e, 0, 9]) for p, e in at] == history[r]


def test_on_a_stream_of_its_own_and_in_a_graph():
    rng = np.random.default_rng(9)
    pages, lengths, refs = tables(rng, 4, 4, 8, trunk=20, past=20, spare=50)
    parents = rng.integers(0, 4, (4, 4)).astype(np.int32)
    want = ref.fork(pages, lengths, parents, refs, 8, np.ones((4, 4)))
    p, n, a, start = ints(pages), ints(lengths), ints(parents), ints(refs)
    counts = start.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ng.kv_fork(p, n, a, counts, 8, tokens=1, stream=side)
    side.synchronize()
    for x, y in zip((*got, counts), want):
        assert np.array_equal(host(x), y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        counts.copy_(start)
        got = ng.kv_fork(p, n, a, counts, 8, tokens=1)
        moved = counts.clone()
        packed = ng.kv_compact(moved, 8, tables=(got[0].clone(),))
    for seed in range(3):
        a.copy_(ints(np.random.default_rng(seed).integers(0, 4, (4, 4))))
        graph.replay()
        torch.cuda.synchronize()
        want = ref.fork(pages, lengths, host(a), refs, 8, np.ones((4, 4)))
        for x, y in zip((*got, counts), want):
            assert np.array_equal(host(x), y)
        assert np.array_equal(host(packed[0]), ref.compact(want[3], 8, ())[0])
        (refs_twice := start.clone(), ng.kv_fork(p, n, a, refs_twice, 8, tokens=1))   # eager work between
