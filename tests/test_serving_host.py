"""The serving operators' C ABI without a GPU: refusals come before any device
call, workspace sizes, and the binding's structures match the header's."""

import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2505_22857_amd as ng
from paper_2505_22857_amd import serving

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID = -1


@pytest.fixture(scope="module")
def lib():
    return serving._library()


def error():
    return ng.load_library().ngpu_lm_last_error().decode()


def test_structures_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc is not available")
    names = {"ngpu_verify_t": serving._Verify, "ngpu_kv_cache_t": serving._Cache, "ngpu_kv_append_t": serving._Append,
             "ngpu_attend_t": serving._Attend}
    lines = ["#include <stdio.h>", '#include "ngpu_lm.h"', "int main(void) {"]
    for name, cls in names.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = dict(x.split() for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for name, cls in names.items():
        assert int(got[name]) == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)


def ok_verify(**kw):
    a = dict(B=2, K=3, V=50, dtype=0, logits=64, logits_stride_b=200, logits_stride_k=50, tokens=64, uniforms=64,
             noise=64, noise_stride_b=50, temperature=1.0, out_tokens=64, accepted=64)
    return serving._Verify(**{**a, **kw})


@pytest.mark.parametrize("change", [
    dict(B=-1), dict(B=(1 << 20) + 1), dict(K=-1), dict(K=64), dict(V=0), dict(V=1 << 31), dict(dtype=3), dict(dtype=-1),
    dict(temperature=-0.5), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-7),
    dict(logits=None), dict(tokens=None), dict(uniforms=None), dict(noise=None), dict(out_tokens=None),
    dict(accepted=None), dict(states=64), dict(logits_stride_b=-1), dict(logits_stride_k=-1), dict(noise_stride_b=-1),
    dict(logprobs=64, logprobs_stride_b=-1)])
def test_verify_refuses(lib, change):
    assert lib.ngpu_lm_verify(ctypes.byref(ok_verify(**change)), None, 0, None) == INVALID and error()


def test_verify_workspace(lib):
    assert lib.ngpu_lm_verify(None, None, 0, None) == INVALID
    assert lib.ngpu_lm_verify_workspace(4, 3, 8192) == 0          # one launch
    need = lib.ngpu_lm_verify_workspace(4, 3, 8193)
    assert need >= 4 * 4 * 2 * 8
    assert lib.ngpu_lm_verify_workspace(-1, 3, 100) == 0 and lib.ngpu_lm_verify_workspace(1, 3, 0) == 0
    big = ok_verify(V=8193)
    assert lib.ngpu_lm_verify(ctypes.byref(big), None, 0, None) == INVALID and str(need // 2) in error()
    assert lib.ngpu_lm_verify(ctypes.byref(big), 64, need // 2 - 1, None) == INVALID
    assert lib.ngpu_lm_verify(ctypes.byref(big), 68, need, None) == INVALID and "aligned" in error()
    assert lib.ngpu_lm_verify(ctypes.byref(ok_verify(B=0)), None, 0, None) == 0 and not error()


def ok_cache(**kw):
    a = dict(dtype=1, heads=2, dim=64, page_size=16, num_pages=10, k=64, v=64, k_stride_page=2048, k_stride_token=128,
             k_stride_head=64, v_stride_page=2048, v_stride_token=128, v_stride_head=64)
    return serving._Cache(**{**a, **kw})


BAD_CACHES = [dict(dtype=0), dict(dtype=7), dict(heads=0), dict(heads=70000), dict(dim=0), dict(dim=257),
              dict(page_size=0), dict(num_pages=-1), dict(num_pages=1 << 31), dict(k=None), dict(v=None),
              dict(k_stride_page=-1), dict(k_stride_token=-1), dict(k_stride_head=-1), dict(v_stride_page=-1),
              dict(v_stride_token=-1), dict(v_stride_head=-1)]


def ok_append(**kw):
    a = dict(S=2, T=3, k=64, v=64, k_stride_seq=384, k_stride_token=128, k_stride_head=64, v_stride_seq=384,
             v_stride_token=128, v_stride_head=64, pages=64, pages_width=2, pages_stride=2, start=64, rotary=32,
             cos=64, sin=64, positions_count=99, layout=0)
    return serving._Append(**{**a, **kw})


@pytest.mark.parametrize("change", [
    dict(S=-1), dict(S=(1 << 20) + 1), dict(T=-1), dict(T=1 << 31), dict(S=1 << 20, T=1 << 30), dict(k=None), dict(v=None),
    dict(start=None), dict(pages=None), dict(pages_width=-1), dict(pages_stride=-1), dict(rotary=-2), dict(rotary=3),
    dict(rotary=66), dict(layout=2), dict(layout=-1), dict(cos=None), dict(sin=None), dict(k_stride_seq=-1),
    dict(v_stride_head=-1), dict(q=64, q_heads=0, q_out=128), dict(q=64, q_heads=2), dict(q=64, q_heads=2, q_out=64),
    dict(q=64, q_heads=2, q_out=128, q_stride_token=-1)])
def test_append_refuses(lib, change):
    c = ok_cache()
    assert lib.ngpu_lm_kv_append(ctypes.byref(c), ctypes.byref(ok_append(**change)), None) == INVALID and error()


@pytest.mark.parametrize("change", BAD_CACHES)
def test_bad_caches_are_refused(lib, change):
    c = ok_cache(**change)
    assert lib.ngpu_lm_kv_append(ctypes.byref(c), ctypes.byref(ok_append()), None) == INVALID and error()
    assert lib.ngpu_lm_attend(ctypes.byref(c), ctypes.byref(ok_attend()), None, 0, None) == INVALID and error()
    assert lib.ngpu_lm_attend_workspace(ctypes.byref(c), ctypes.byref(ok_attend())) == 0


def ok_attend(**kw):
    a = dict(S=4, T=2, q_heads=4, q=64, q_stride_seq=512, q_stride_token=256, q_stride_head=64, G=2, prefix_pages=64,
             prefix_width=3, prefix_stride=3, prefix_lengths=64, pages=64, pages_width=2, pages_stride=2, lengths=64,
             scale=0.125, out=64)
    return serving._Attend(**{**a, **kw})


@pytest.mark.parametrize("change", [
    dict(S=-1), dict(S=(1 << 20) + 4), dict(T=-1), dict(T=1 << 31), dict(q_heads=0), dict(q_heads=3), dict(q_heads=70000),
    dict(G=-1), dict(G=3), dict(q=None), dict(out=None), dict(prefix_lengths=None), dict(prefix_pages=None),
    dict(lengths=None), dict(prefix_width=-1), dict(prefix_stride=-1), dict(pages_width=-1), dict(pages_stride=-1),
    dict(q_stride_seq=-1), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_attend_refuses(lib, change):
    c = ok_cache()
    assert lib.ngpu_lm_attend(ctypes.byref(c), ctypes.byref(ok_attend(**change)), 64, 1 << 30, None) == INVALID and error()


def test_attend_workspace(lib):
    c = ok_cache()
    need = lib.ngpu_lm_attend_workspace(ctypes.byref(c), ctypes.byref(ok_attend()))
    rows = 4 * 2 * 4
    assert need >= 2 * rows * (64 * 4 + 8)                        # at least one part of each kind
    assert lib.ngpu_lm_attend(ctypes.byref(c), ctypes.byref(ok_attend()), 64, need - 1, None) == INVALID
    assert lib.ngpu_lm_attend(None, ctypes.byref(ok_attend()), 64, need, None) == INVALID
    assert lib.ngpu_lm_attend(ctypes.byref(c), None, 64, need, None) == INVALID
    assert lib.ngpu_lm_attend(ctypes.byref(c), ctypes.byref(ok_attend(S=0, G=1)), None, 0, None) == 0
    odd = ok_cache(dim=63)                                        # by the kernel that needs none
    assert lib.ngpu_lm_attend_workspace(ctypes.byref(odd), ctypes.byref(ok_attend())) == 0


def test_draft_needs_an_uploaded_model(lib):
    from synth import make_model
    m = ng.NgpuLM.from_model(make_model("trigram_v128"))
    assert lib.ngpu_lm_draft(None, 64, None, 1, 1, 0.0, None, 0, 0, 64, 64, None, None) == INVALID
    assert lib.ngpu_lm_draft(m._h, 64, None, 1, 1, 0.0, None, 0, 0, 64, 64, None, None) == -8


def test_device_tensors_are_asked_for():
    torch = pytest.importorskip("torch")
    x = torch.zeros(1, 1, 1, 8, dtype=torch.float16)
    with pytest.raises(TypeError):
        ng.attend(x, x, x)
    with pytest.raises(TypeError):
        ng.kv_append(x, x, x, x, None, None)
    with pytest.raises(TypeError):
        ng.verify(torch.zeros(1, 2, 8), None, temperature=0.0)
