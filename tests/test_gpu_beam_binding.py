"""The beam search's calls through the native per-call module and through ctypes: the same results, and the same
refusals."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import paper_2505_22857_amd as ng  # noqa: E402
from paper_2505_22857_amd import serving  # noqa: E402

E4M3 = torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def both(monkeypatch, name, call, *changed):
    """The call natively, which has to answer it, and through ctypes: equal results and equal changed tensors."""
    native, answers = serving._native(), []
    start = [t.clone() for t in changed]

    class Spy:
        def __getattr__(self, f):
            def run(*a):
                answers.append((f, getattr(native, f)(*a)))
                return answers[-1][1]
            return run

    def once(module):
        for t, s in zip(changed, start):
            t.copy_(s)
        monkeypatch.setattr(serving, "_native_module", module)
        out = call()
        out = out if isinstance(out, (tuple, list)) else [out]
        return [None if x is None else x.clone() for x in (*out, *changed)]

    got = once(Spy())
    assert [f for f, r in answers if r is not None] == [name]
    want = once(False)
    monkeypatch.setattr(serving, "_native_module", native)
    for x, y in zip(got, want):
        assert (x is None and y is None) or (x.dtype is y.dtype and torch.equal(x.view(torch.uint8) if x.dtype is E4M3 else x,
                                                                             y.view(torch.uint8) if y.dtype is E4M3 else y))


def test_pages(monkeypatch):
    pages, lengths, refs = ints([[0, 1, -1], [0, 2, -1]]), ints([9, 12]), ints([2, 1, 1, 0, 0, 0, 0])
    for tokens in (1, 0, ints([[1, 2, 3]])):
        both(monkeypatch, "kv_fork", lambda: ng.kv_fork(pages, lengths, ints([[0, 0, 1]]), refs, 8, tokens=tokens), refs)
    both(monkeypatch, "kv_fork", lambda: ng.kv_fork(pages, lengths, ints(np.zeros((1, 0))), refs, 8), refs)
    wide = ints([[6, 2, 9], [0, -1, 9]])
    both(monkeypatch, "kv_compact", lambda: ng.kv_compact(ints([1, 0, 1, 0, 0, 0, 2]), 8, tables=[wide[:, :2]]), wide)
    both(monkeypatch, "kv_compact", lambda: ng.kv_compact(refs, 8), refs)


def test_copies(monkeypatch):
    c = [torch.randn(5, 4, 2, 64, device="cuda").half() for _ in range(2)]
    copies = ints([[0, 3, 4], [1, 2, 1], [-1, -1, 0]])
    both(monkeypatch, "kv_copy", lambda: ng.kv_copy(*c, copies), *c)
    bits = [torch.randint(0, 255, (5, 4, 2, 64), dtype=torch.uint8, device="cuda") for _ in range(2)]
    s = [torch.rand(5, 2, 2, device="cuda") for _ in range(2)]
    both(monkeypatch, "kv_copy", lambda: ng.kv_copy(*(b.view(E4M3) for b in bits), copies, k_scale=s[0], v_scale=s[1]), *bits, *s)


def test_append_and_attend(monkeypatch):
    k, q = torch.randn(3, 2, 2, 64, device="cuda").half(), torch.randn(3, 2, 4, 64, device="cuda").half()
    bits = [torch.zeros(9, 8, 2, 64, dtype=torch.uint8, device="cuda") for _ in range(2)]
    s = [torch.ones(9, 2, 2, device="cuda") for _ in range(2)]
    table, start = ints(np.arange(6).reshape(3, 2)), ints([0, 3, 9])
    cos, sin = ng.rope_table(20, 32)
    kw = dict(k_scale=s[0], v_scale=s[1])
    both(monkeypatch, "kv_append", lambda: ng.kv_append(k, k, *(b.view(E4M3) for b in bits), table, start, cos=cos, sin=sin,
                                                        q=q, **kw), *bits, *s)
    both(monkeypatch, "kv_append", lambda: ng.kv_append(k, k, *(b.view(E4M3) for b in bits), table, start, **kw), *bits, *s)
    both(monkeypatch, "attend", lambda: ng.attend(q, *(b.view(E4M3) for b in bits), pages=table, lengths=start + 2,
                                                  prefix_pages=ints([[7, 8]]), prefix_lengths=ints([13]), **kw))


def test_beam_step():
    from synth import generate_model, uniform_states
    m = generate_model(200, [200, 900, 500], 1.0, seed=5, bos_eos=True)
    lm = ng.NgpuLM.from_model(m).upload("cuda:0")
    st = torch.from_numpy(uniform_states(m, 12, seed=1).reshape(3, 4)).cuda()
    sc, last = -torch.rand(3, 4, device="cuda"), ints([[200, 1, 2, 3]] * 3)
    fast = lm._fast
    assert fast
    for C, mode, l, k in ((200, ng.NGPU_FUSION_PLAIN, None, None), (201, ng.NGPU_FUSION_AED, last, 7),
                          (201, ng.NGPU_FUSION_TRANSDUCER, None, 2)):
        asr = torch.randn(3, 4, C, device="cuda")
        assert fast.beam_step(lm._h.value, 200, asr, 0.5, st, sc, k, l, mode) is not None
        for x in (asr, asr[:, :1].expand(3, 4, C)):
            got = lm.beam_step(x, 0.5, st, sc, k=k, last=l, mode=mode)
            lm._fast = None
            want = lm.beam_step(x, 0.5, st, sc, k=k, last=l, mode=mode)
            lm._fast = fast
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    for bad in (dict(mode=ng.NGPU_FUSION_CTC), dict(last=last), dict(k=65), dict(mode=ng.NGPU_FUSION_AED, last=last.long())):
        for module in (fast, None):
            lm._fast = module
            with pytest.raises((ng.NgpuError, ValueError, TypeError)):
                lm.beam_step(torch.randn(3, 4, 201, device="cuda"), 0.5, st, sc, **bad)
    lm._fast = fast


@pytest.mark.parametrize("native", [True, False])
def test_refusals(monkeypatch, native):
    if not native:
        monkeypatch.setattr(serving, "_native_module", False)
    pages, lengths, parents, refs = ints([[0, 1]] * 4), ints([3] * 4), ints([[0, 1], [0, 0]]), ints([4, 4, 0, 0])
    ok = dict(pages=pages, lengths=lengths, parents=parents, refs=refs, page_size=8)

    def bad(error, **kw):
        with pytest.raises(error):
            ng.kv_fork(**{**ok, **kw})
    bad(ValueError, pages=pages[:3])
    bad(ValueError, pages=pages[0])
    bad(TypeError, pages=pages.long())
    bad(TypeError, pages=ints([[0, 1, 2, 3]] * 4)[:, ::2])
    bad(ValueError, lengths=lengths[:3])
    bad(TypeError, lengths=lengths.cpu())
    bad(ValueError, parents=parents[0])
    bad(TypeError, parents=parents.t())
    bad(ValueError, refs=refs[None])
    bad(TypeError, refs=refs.cpu())
    bad(TypeError, refs=ints(np.zeros(8))[::2])
    bad(ng.NgpuError, page_size=0)
    bad(ng.NgpuError, tokens=-1)
    bad(ValueError, tokens=ints([1, 2]))
    bad(TypeError, tokens=torch.ones(2, 2, device="cuda"))
    bad(ValueError, parents=ints(np.zeros((0, 2))))
    assert refs.tolist() == [4, 4, 0, 0]
    out = ng.kv_fork(pages[:0], lengths[:0], ints(np.zeros((0, 2))), refs, 8)
    assert [tuple(x.shape) for x in out] == [(0, 2), (0,), (0, 3)]
    c = torch.zeros(4, 8, 2, 16, dtype=torch.float16, device="cuda")
    for copies in (ints([[0, 1]]), ints([0, 1, 2]), torch.zeros(1, 3, device="cuda"), ints(np.zeros((3, 1))).t()[:, :2]):
        with pytest.raises((TypeError, ValueError)):
            ng.kv_copy(c, c, copies)
    with pytest.raises(TypeError, match="gradient"):
        ng.kv_copy(c.clone().requires_grad_(), c, ints([[0, 1, 2]]))
    with pytest.raises(ValueError, match="together"):
        ng.kv_copy(c, c, ints([[0, 1, 2]]), k_scale=torch.ones(4, 1, 2, device="cuda"))
    table = ints([[0, 1], [2, 3]])
    for tables in ((table, table), (table[:1].expand(3, 2),), (table.long(),), (table.cpu(),), (table[0],), (table.t(),)):
        with pytest.raises((TypeError, ValueError)):
            ng.kv_compact(refs, 8, tables=tables)
    with pytest.raises(ng.NgpuError):
        ng.kv_compact(refs, 0)
    assert refs.tolist() == [4, 4, 0, 0] and table.tolist() == [[0, 1], [2, 3]]
