"""The pages' C ABI and binding without a GPU: refusals come before any device call, and the binding's structures
match the header's."""

import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2505_22857_amd as ng
from paper_2505_22857_amd import pages, serving

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID = -1


@pytest.fixture(scope="module")
def lib():
    return pages._library()


def error():
    return ng.load_library().ngpu_lm_last_error().decode()


def test_structures_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc is not available")
    names = {"ngpu_beam_step_t": ng._BeamStep, "ngpu_kv_fork_t": pages._Fork, "ngpu_kv_cache8_t": serving._Cache8}
    lines = ["#include <stdio.h>", '#include "ngpu_lm.h"', "int main(void) {"]
    for name, cls in names.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {"lambda" if f == "lam" else f}));' for f, _ in cls._fields_]
    lines.append('printf("fork %d\\npages %lld\\n", NGPU_LM_MAX_FORK, (long long)NGPU_LM_MAX_PAGES);')
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = dict(x.split() for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for name, cls in names.items():
        assert int(got[name]) == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)
    assert int(got["fork"]) == ng.MAX_FORK and int(got["pages"]) == ng.MAX_PAGES


def ok_fork(**kw):
    a = dict(G=2, W=3, K=3, pages=64, width=5, pages_stride=5, lengths=64, parents=64, T=1, page_size=16, num_pages=100,
             refs=64, out_pages=128, out_lengths=64, copies=64)
    return pages._Fork(**{**a, **kw})


@pytest.mark.parametrize("change", [
    dict(G=-1), dict(G=(1 << 20) + 1), dict(W=-1), dict(W=4097), dict(K=-1), dict(K=4097), dict(G=1 << 19, W=3),
    dict(G=1 << 19, K=3), dict(pages=None), dict(width=-1), dict(width=1 << 31), dict(pages_stride=-1), dict(lengths=None),
    dict(parents=None), dict(T=-1), dict(T=1 << 31), dict(page_size=0), dict(page_size=-3), dict(num_pages=-1),
    dict(num_pages=(1 << 28) + 1), dict(refs=None), dict(out_pages=None), dict(out_lengths=None), dict(copies=None),
    dict(out_pages=64), dict(G=1 << 10, W=1 << 10, K=1 << 10, width=1 << 30)])
def test_fork_refuses(lib, change):
    assert lib.ngpu_lm_kv_fork(ctypes.byref(ok_fork(**change)), 64, 1 << 40, None) == INVALID and error()


def test_fork_workspace(lib):
    need = lib.ngpu_lm_kv_fork_workspace(2, 3, 100)
    assert need >= 4 * 100 + 6 * 20
    assert lib.ngpu_lm_kv_fork(ctypes.byref(ok_fork()), 64, need - 1, None) == INVALID and str(need) in error()
    assert lib.ngpu_lm_kv_fork(ctypes.byref(ok_fork()), 68, need, None) == INVALID and "aligned" in error()
    assert lib.ngpu_lm_kv_fork(None, 64, need, None) == INVALID
    for none in ((0, 3, 100), (2, 0, 100), (-1, 3, 100), (2, 5000, 100), (2, 3, -1), (2, 3, 1 << 29)):
        assert lib.ngpu_lm_kv_fork_workspace(*none) == 0
    assert lib.ngpu_lm_kv_fork(ctypes.byref(ok_fork(G=0)), None, 0, None) == 0 and not error()
    assert lib.ngpu_lm_kv_fork(ctypes.byref(ok_fork(W=0, K=0)), None, 0, None) == 0


def test_copy_refuses(lib):
    cache = serving._Cache(1, 2, 64, 16, 10, 64, 64, 2048, 128, 64, 2048, 128, 64)
    assert lib.ngpu_lm_kv_copy(None, 64, 1, None) == INVALID
    assert lib.ngpu_lm_kv_copy(ctypes.byref(cache), None, 1, None) == INVALID
    assert lib.ngpu_lm_kv_copy(ctypes.byref(cache), 64, -1, None) == INVALID
    assert lib.ngpu_lm_kv_copy(ctypes.byref(cache), None, 0, None) == 0
    cache.dtype = 0
    assert lib.ngpu_lm_kv_copy(ctypes.byref(cache), 64, 1, None) == INVALID


def ok_cache8(**kw):
    a = dict(cache=serving._Cache(1, 2, 64, 16, 10, 64, 64, 2048, 128, 64, 2048, 128, 64), block=8, k_scale=64, v_scale=64,
             k_scale_stride_page=4, k_scale_stride_block=2, k_scale_stride_head=1, v_scale_stride_page=4,
             v_scale_stride_block=2, v_scale_stride_head=1)
    return serving._Cache8(**{**a, **kw})


@pytest.mark.parametrize("change", [
    dict(block=0), dict(block=-8), dict(block=5), dict(block=32), dict(k_scale=None), dict(v_scale=None),
    dict(k_scale_stride_page=-1), dict(k_scale_stride_block=-1), dict(k_scale_stride_head=-1), dict(v_scale_stride_page=-1),
    dict(v_scale_stride_block=-1), dict(v_scale_stride_head=-1),
    dict(cache=serving._Cache(0, 2, 64, 16, 10, 64, 64, 2048, 128, 64, 2048, 128, 64)),
    dict(cache=serving._Cache(1, 2, 257, 16, 10, 64, 64, 2048, 128, 64, 2048, 128, 64)),
    dict(cache=serving._Cache(1, 1, 1, 1 << 20, 1, 64, 64, 1, 1, 1, 1, 1, 1), block=1 << 20)])
def test_bad_caches_of_8_bits_are_refused(lib, change):
    from test_serving_host import ok_append
    c = ok_cache8(**change)
    lib8 = serving._library()
    assert lib8.ngpu_lm_kv_append8(ctypes.byref(c), ctypes.byref(ok_append()), None) == INVALID and error()
    assert lib.ngpu_lm_kv_copy8(ctypes.byref(c), 64, 1, None) == INVALID and error()
    from test_serving_host import ok_attend
    assert lib8.ngpu_lm_attend8(ctypes.byref(c), ctypes.byref(ok_attend()), 64, 1 << 30, None) == INVALID and error()
    assert lib8.ngpu_lm_attend8_workspace(ctypes.byref(c), ctypes.byref(ok_attend())) == 0


def test_attend8_refuses(lib):
    from test_serving_host import ok_attend
    lib8, c = serving._library(), ok_cache8()
    need = lib8.ngpu_lm_attend8_workspace(ctypes.byref(c), ctypes.byref(ok_attend()))
    assert need >= 2 * 4 * 2 * 4 * (64 * 4 + 8)
    assert lib8.ngpu_lm_attend8(ctypes.byref(c), ctypes.byref(ok_attend()), 64, need - 1, None) == INVALID
    assert lib8.ngpu_lm_attend8(None, ctypes.byref(ok_attend()), 64, need, None) == INVALID
    assert lib8.ngpu_lm_attend8(ctypes.byref(c), None, 64, need, None) == INVALID
    assert lib8.ngpu_lm_attend8_workspace(None, ctypes.byref(ok_attend())) == 0
    for change in (dict(S=-1), dict(T=1 << 31), dict(q_heads=3), dict(G=3), dict(q=None), dict(out=None), dict(lengths=None),
                   dict(prefix_lengths=None), dict(q_stride_seq=-1), dict(scale=float("nan"))):
        assert lib8.ngpu_lm_attend8(ctypes.byref(c), ctypes.byref(ok_attend(**change)), 64, 1 << 30, None) == INVALID
    assert lib8.ngpu_lm_attend8(ctypes.byref(c), ctypes.byref(ok_attend(S=0, G=1)), None, 0, None) == 0


def test_append8_and_copy8_refuse(lib):
    from test_serving_host import ok_append
    lib8, c = serving._library(), ok_cache8()
    assert lib8.ngpu_lm_kv_append8(None, ctypes.byref(ok_append()), None) == INVALID
    assert lib8.ngpu_lm_kv_append8(ctypes.byref(c), None, None) == INVALID
    for change in (dict(k=None), dict(start=None), dict(rotary=66), dict(layout=2), dict(q=64, q_heads=2, q_out=64)):
        assert lib8.ngpu_lm_kv_append8(ctypes.byref(c), ctypes.byref(ok_append(**change)), None) == INVALID
    assert lib8.ngpu_lm_kv_append8(ctypes.byref(c), ctypes.byref(ok_append(T=0)), None) == 0
    assert lib.ngpu_lm_kv_copy8(None, 64, 1, None) == INVALID
    assert lib.ngpu_lm_kv_copy8(ctypes.byref(c), None, 1, None) == INVALID
    assert lib.ngpu_lm_kv_copy8(ctypes.byref(c), None, 0, None) == 0


def test_compact_refuses(lib):
    need = lib.ngpu_lm_kv_compact_workspace(100)
    assert need >= 4 and lib.ngpu_lm_kv_compact_workspace(0) == 0 and lib.ngpu_lm_kv_compact_workspace(1 << 29) == 0
    good = [64, 100, 16, 64, 64, 64, need, None]
    for i, bad in ((0, None), (1, -1), (1, 1 << 29), (2, 0), (3, None), (4, None), (5, None), (5, 72), (6, need - 1)):
        args = list(good)
        args[i] = bad
        assert lib.ngpu_lm_kv_compact(*args) == INVALID and error()
    assert lib.ngpu_lm_kv_compact(None, 0, 16, None, None, None, 0, None) == 0
    good = [64, 2, 5, 5, 64, 100, None]
    for i, bad in ((0, None), (1, -1), (2, -1), (2, 1 << 31), (3, 4), (4, None), (5, -1), (1, 1 << 40)):
        args = list(good)
        args[i] = bad
        assert lib.ngpu_lm_kv_move(*args) == INVALID and error()
    assert lib.ngpu_lm_kv_move(None, 0, 5, 5, None, 100, None) == 0


def test_device_tensors_are_asked_for():
    torch = pytest.importorskip("torch")
    x, c = torch.zeros(4, 4, dtype=torch.int32), torch.zeros(1, 1, 1, 8, dtype=torch.float16)
    with pytest.raises(TypeError):
        ng.kv_fork(x, x[0], x, x[0], 16)
    with pytest.raises(TypeError):
        ng.kv_compact(x[0], 16)
    with pytest.raises(TypeError):
        ng.kv_copy(c, c, x[:, :3])


def test_a_beam_step_needs_an_uploaded_model():
    from synth import make_model
    lib, m = ng.load_library(), ng.NgpuLM.from_model(make_model("trigram_v128"))
    a = ng._BeamStep(1, 2, 2, 0, 0.5, 64, 256, 128, 64, 64, None, 64, 64, 64, 64)
    assert lib.ngpu_lm_beam_step(None, ctypes.byref(a), 64, 1 << 20, None) == INVALID
    assert lib.ngpu_lm_beam_step(m._h, None, 64, 1 << 20, None) == INVALID
    assert lib.ngpu_lm_beam_step(m._h, ctypes.byref(a), 64, 1 << 20, None) == -8
    assert lib.ngpu_lm_beam_step_workspace(4, 8, 8) >= 4 * 8 * 9 * 12
    for none in ((0, 8, 8), (-1, 8, 8), (4, 0, 8), (4, 65, 8), (4, 8, 0), (4, 8, 65), (1 << 26, 8, 8)):
        assert lib.ngpu_lm_beam_step_workspace(*none) == 0
