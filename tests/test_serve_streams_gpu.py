"""Calls on a stream that is not the current one: what they make, and the workspace they use, belong to that stream."""
import pytest

pytestmark = pytest.mark.gpu

import paper_2410_21271_b200 as eora
from helpers import make_case
from test_serve_gpu import DEV, bank_case, gen, ints, normal


def pool_of(t):
    """The stream whose pool of torch's allocator a tensor's memory is from."""
    import torch
    at = t.data_ptr()
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= at < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not torch's memory")


def calls():
    """name -> a function of a stream that makes all of its results and returns them."""
    import torch
    g, a, b, rk, sc = bank_case(900, 3, 512, 256, 16, "f16")
    bank = eora.AdapterBank(a, b, scales=sc)
    x, ids = normal(g, 5, 512), ints([0, 1, 2, -1, 0])
    rope = eora.QKNormRope(4, 2, 64, None, dtype="f16")
    q, k, v = normal(g, 5, 256), normal(g, 5, 128), normal(g, 5, 128)
    kc, vc = normal(g, 6, 2, 16, 64), normal(g, 6, 2, 16, 64)
    cache, pages = eora.PagedCache(kc, vc), ints([[0], [1], [2], [3], [4]])
    attn = eora.PagedAttention(4, 2, 64, page_size=16, max_batch=5, max_pages=1, dtype="f16")
    zeros, lengths = ints([0] * 5), ints([3, 1, 16, 7, 0])
    layer, fused = eora.Layer(*make_case(901, 512, 256, 32), max_m=8), eora.FusedLayers([make_case(902, 512, 256, 32), make_case(903, 512, 128, 32)], max_m=8)
    cases = [make_case(904, 512, 256, 32)] + [make_case(905, 512, 256, 32)]
    multi = eora.MultiAdapterLayer(cases[0][0], [c[1:] for c in cases], max_m=8)
    w, wh, xt = (torch.randn(s, device=DEV) for s in ((128, 192), (128, 192), (192, 320)))
    return {"adapters": lambda s: [bank.forward(x, ids, stream=s)],
            "rotation": lambda s: list(rope.forward(q, k, None, zeros, stream=s)),
            "attention": lambda s: [attn.forward(q, cache, pages, lengths, stream=s)],
            "layer": lambda s: [layer.forward(x, stream=s)],
            "layer with adapters": lambda s: [layer.forward(x, stream=s, adapters=(bank, ids))],
            "fused layers": lambda s: fused.forward(x, stream=s),
            "layer of adapters": lambda s: [multi.forward(x, [0, 1, -1, 0, 1], stream=s)],
            "solve": lambda s: list(eora.solve(w, wh, xt, 16, stream=s))}


@pytest.mark.parametrize("how", ["object", "handle", "outer"])
def test_results_belong_to_the_stream_of_the_call(how):
    import torch
    side, outer = torch.cuda.Stream(), torch.cuda.Stream()
    for name, call in calls().items():
        want = call(None)
        torch.cuda.synchronize()
        if how == "outer":                                   # the call's stream is not the current one, which is not the default one
            with torch.cuda.stream(outer):
                torch.cuda.synchronize()
                got = call(side)
        else:
            got = call(side if how == "object" else side.cuda_stream)
        assert {pool_of(t) for t in got} == {side.cuda_stream}, name
        torch.cuda.synchronize()
        if name not in ("layer", "layer with adapters", "fused layers", "layer of adapters", "solve"):      # (the order of those sums may change)
            assert all(torch.equal(a, b) for a, b in zip(got, want)), name
    for legacy in (0, 1):                                    # two names of the default stream
        assert {pool_of(t) for c in calls().values() for t in c(legacy)} == {0}
    torch.cuda.synchronize()


def test_layers_results_without_the_native_module(monkeypatch):
    """As in a build without torch: torch makes them, on the stream of the call all the same."""
    import torch
    side, todo = torch.cuda.Stream(), {n: c for n, c in calls().items() if "layer" in n}
    monkeypatch.setattr(eora, "_native_module", None)
    for stream, pool in ((side, side.cuda_stream), (side.cuda_stream, side.cuda_stream), (None, 0), (0, 0), (1, 0)):
        for name, call in todo.items():
            assert {pool_of(t) for t in call(stream)} == {pool}, (name, stream)
            torch.cuda.synchronize()


def test_results_do_not_take_memory_that_the_current_stream_still_reads():
    """A block that the current stream has given back with work on it still to come."""
    import torch
    side = torch.cuda.Stream()
    g, a, b, rk, sc = bank_case(906, 1, 128, 4096, 8, "f16")
    bank, x, ids = eora.AdapterBank(a, b), normal(g, 64, 128), ints([0] * 64)
    bank.forward(x, ids, stream=side)
    u = torch.empty(64, 4096, dtype=torch.float16, device=DEV)
    torch.cuda.synchronize()
    t = normal(g, 64, 4096)
    want = t.clone()
    torch.cuda._sleep(20_000_000)
    u.copy_(t)
    del t
    y = bank.forward(x, ids, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(u, want) and y.data_ptr() != u.data_ptr()


@pytest.mark.parametrize("how", ["object", "current", "handle"])
def test_a_workspace_outlives_the_object_while_a_call_runs(how):
    import torch
    g = gen(907)
    kc, vc = normal(g, 40, 2, 16, 64), normal(g, 40, 2, 16, 64)
    cache, pages = eora.PagedCache(kc, vc), torch.randperm(40, device=DEV).int().view(1, 40)
    q, n, out = normal(g, 1, 256), ints([640]), torch.empty(1, 256, dtype=torch.float16, device=DEV)
    make = lambda: eora.PagedAttention(4, 2, 64, page_size=16, max_batch=1, max_pages=40, dtype="f16")
    side, attn = torch.cuda.Stream(), make()
    want = attn.forward(q, cache, pages, n).clone()
    torch.cuda.synchronize()
    at, size = attn.workspace.data_ptr(), attn.workspace.numel()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
        if how == "current":
            attn.forward(q, cache, pages, n, out=out)
    if how != "current":
        attn.forward(q, cache, pages, n, out=out, stream=side if how == "object" else side.cuda_stream)
    assert not side.query()
    del attn
    if how == "handle":                                      # the allocator cannot ask such a stream: dropping the object waits
        assert side.query()
    else:
        other = [torch.empty(size, dtype=torch.uint8, device=DEV).fill_(255) for _ in range(3)]
        assert not side.query() and at not in [t.data_ptr() for t in other]
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_a_stream_of_no_gpu_is_refused():
    import torch
    for call in (c for n, c in calls().items() if n in ("adapters", "rotation", "attention")):
        with pytest.raises((AttributeError, TypeError, eora.EoraError)):
            call("side")
    torch.cuda.synchronize()
