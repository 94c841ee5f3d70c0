"""Arguments of the serving calls by their places: what a program passed before the calls took more stays where it was."""

import inspect

import pytest

torch = pytest.importorskip("torch")

import paper_2505_22857_amd as ng  # noqa: E402

PLACES = {
    "kv_append": ["k", "v", "k_cache", "v_cache", "pages", "start", "positions", "cos", "sin", "layout", "q", "lengths",
                  "stream"],
    "attend": ["q", "k_cache", "v_cache", "pages", "lengths", "prefix_pages", "prefix_lengths", "q_lengths", "scale",
               "return_lse", "stream"],
}


@pytest.mark.parametrize("name", PLACES)
def test_places(name):
    places = list(inspect.signature(getattr(ng, name)).parameters)
    assert places[:len(PLACES[name])] == PLACES[name]


@pytest.mark.gpu
def test_a_stream_by_its_place():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(2, 3, 2, 64, generator=g, device="cuda").half() for _ in range(2))
    kc, vc = (torch.zeros(4, 8, 2, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    pages = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    start = torch.zeros(2, dtype=torch.int32, device="cuda")
    lengths = start + 3
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q = ng.kv_append(k, v, kc, vc, pages, start, None, None, None, ng.NGPU_ROPE_HALF, k, None, side)
    got, lse = ng.attend(q, kc, vc, pages, lengths, None, None, None, None, True, side)
    side.synchronize()
    assert torch.equal(kc[0, :3], k[0]) and torch.equal(vc[2, :3], v[1]) and torch.equal(q, k)
    want, to = ng.attend(q, kc, vc, pages=pages, lengths=lengths, return_lse=True)
    assert torch.equal(got, want) and torch.equal(lse, to)
