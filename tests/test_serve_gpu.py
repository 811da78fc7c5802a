"""The serving operators against their float64 oracle, at the sizes, masks, strides and contents where they can go wrong.
Tolerances are the oracle's bounds, derived from the roundings of the formulas."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import paper_2410_21271_b200 as eora
from oracle import serve_oracle as orc

DEV = "cuda:0"


def tt(name):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[name]


def gen(seed):
    import torch
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype="f16", std=1.0):
    import torch
    return (torch.randn(shape, device=DEV, generator=g) * std).to(tt(dtype))


def ints(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def f64(t):
    return t.double().cpu().numpy()


def within(got, ref, bound, what=""):
    got = f64(got).reshape(ref.shape)
    fine = np.isfinite(ref)
    assert np.array_equal(got[~fine], ref[~fine]), what
    over = np.abs(got[fine] - ref[fine]) - bound[fine]
    assert np.isfinite(got[fine]).all() and over.max(initial=-1.0) <= 0, f"{what}: {np.abs(got[fine] - ref[fine]).max():.3e} off, {over.max():.3e} over the bound"


# ------------------------------------------------------------------------------------------------------------ adapters
def bank_case(seed, n, K, N, R, x_type, ranks=None, scales=True):
    """Adapters whose unused columns and rows hold NaN."""
    import torch
    g = gen(seed)
    a, b = normal(g, n, K, R, dtype=x_type, std=0.02), normal(g, n, R, N, dtype=x_type, std=0.02)
    rk = None
    if ranks is not None:
        rk = ints(ranks)
        for j, r in enumerate(ranks):
            r = min(max(r, 0), R)
            a[j, :, r:] = float("nan")
            b[j, r:] = float("nan")
    sc = 0.5 + torch.rand(n, device=DEV, generator=g) if scales else None
    return g, a, b, rk, sc


def adapters_ref(x, a, b, ids, rk, sc, base, x_type, y_type):
    return orc.adapters(f64(x), np.nan_to_num(f64(a)), np.nan_to_num(f64(b)), ids, None if rk is None else rk.tolist(), None if sc is None else sc.tolist(),
                        None if base is None else f64(base), x_type, y_type)


ADAPTERS = [
    # m, n, K, N, max_rank, ids (function of i), ranks, x type, y type
    (1, 1, 128, 32, 8, lambda i: 0, None, "f16", "f16"),
    (1, 3, 4096, 1024, 16, lambda i: 2, None, "bf16", "bf16"),
    (1, 2, 256, 64, 16, lambda i: -1, None, "f16", "f16"),
    (2, 2, 384, 96, 24, lambda i: 1 - i, [24, 7], "f16", "f32"),
    (7, 4, 640, 160, 64, lambda i: (i * 3) % 5 - 1, [64, 1, 33, 0], "bf16", "f32"),
    (16, 1, 512, 256, 256, lambda i: 0, None, "f16", "f16"),
    (17, 1, 512, 256, 256, lambda i: 0, [200], "bf16", "bf16"),
    (33, 48, 1024, 416, 64, lambda i: (i * 29) % 48, [(j * 13) % 70 - 2 for j in range(48)], "f16", "f16"),
    (61, 5, 4096, 1312, 128, lambda i: i % 6, None, "f16", "f32"),                       # id 5: outside the bank
    (64, 3, 14336, 256, 40, lambda i: i // 30, None, "bf16", "bf16"),
    (65, 2, 128, 4096, 128, lambda i: [0, 1, -7, 2**31 - 1][i % 4], [128, 100], "bf16", "f16"),
    (130, 64, 256, 128, 16, lambda i: (i * i) % 67 - 2, None, "f16", "bf16"),
    (257, 1, 896, 224, 32, lambda i: 0 if i % 17 else -1, None, "f16", "f16"),
    (300, 7, 512, 544, 256, lambda i: i // 50, [256, 255, 17, 8, 129, 64, 1], "bf16", "f32"),
    (520, 300, 128, 96, 8, lambda i: (i * 7) % 300, None, "f16", "f32"),
]


@pytest.mark.parametrize("case", range(len(ADAPTERS)))
def test_adapters_match_the_oracle(case):
    import torch
    m, n, K, N, R, of, ranks, xt, yt = ADAPTERS[case]
    g, a, b, rk, sc = bank_case(100 + case, n, K, N, R, xt, ranks, scales=case % 3 != 1)
    x, base = normal(g, m, K, dtype=xt), normal(g, m, N, dtype=yt)
    ids = [of(i) for i in range(m)]
    bank = eora.AdapterBank(a, b, ranks=rk, scales=sc, y_dtype=yt)
    ref, bound = adapters_ref(x, a, b, ids, rk, sc, base, xt, yt)
    y = bank.forward(x, ints(ids), base=base)
    assert y.dtype == tt(yt)
    within(y, ref, bound, "out of place")
    off = [i for i, j in enumerate(ids) if not 0 <= j < n]
    assert torch.equal(y[off], base[off])
    ref0, bound0 = adapters_ref(x, a, b, ids, rk, sc, None, xt, yt)
    within(bank.forward(x, ints(ids)), ref0, bound0, "without a base")
    same = bank.forward(x, ints(ids), base=base)
    inplace = base.clone()
    assert bank.forward(x, ints(ids), base=inplace, y=inplace) is inplace
    torch.cuda.synchronize()
    assert torch.equal(same, y) and torch.equal(inplace, y)                # the same bits every time


@pytest.mark.parametrize("m", [3, 80])
def test_adapters_strides_and_rows_behind(m):
    """Rows of x, base and y inside wider buffers; what lies around them stays as it is."""
    import torch
    n, K, N, R = 3, 256, 96, 16
    g, a, b, rk, sc = bank_case(7, n, K, N, R, "f16")
    wide_x, wide_b = normal(g, m + 2, K + 24), normal(g, m + 2, N + 8)
    wide_y = torch.full((m + 2, N + 16), 7.0, dtype=torch.float16, device=DEV)
    ids = [i % 4 - 1 for i in range(m)]
    eora.AdapterBank(a, b, scales=sc).forward(wide_x[:m, 8:K + 8], ints(ids), base=wide_b[:m, :N], y=wide_y[:m, 8:N + 8])
    ref, bound = adapters_ref(wide_x[:m, 8:K + 8], a, b, ids, rk, sc, wide_b[:m, :N], "f16", "f16")
    within(wide_y[:m, 8:N + 8], ref, bound)
    assert (wide_y[m:] == 7).all() and (wide_y[:, :8] == 7).all() and (wide_y[:, N + 8:] == 7).all()


@pytest.mark.parametrize("m", [4, 100])
def test_adapters_beyond_the_range_of_fp16(m):
    """t = x . A of 10^6 and of 10^-6 (out of fp16's range on both sides) with B's that bring the result back."""
    import torch
    g, a, b, rk, sc = bank_case(8, 2, 512, 64, 16, "f16", scales=False)
    x = normal(g, m, 512).abs() * 100
    a[0] = a[0].abs() * 1000
    b[0] *= 1e-3
    a[1] *= 2.0**-10
    x[1::2] *= 2.0**-8
    ids = [i % 2 for i in range(m)]
    y = eora.AdapterBank(a, b, y_dtype="f32").forward(x, ints(ids))
    ref, bound = adapters_ref(x, a, b, ids, None, None, None, "f16", "f32")
    bound = bound - 2.0**-25 + 2.0**-24 * np.abs(ref)          # (an fp32 output has no step of 2^-24 at small values)
    assert np.abs(ref[::2]).max() > 1 and np.isfinite(ref).all()
    within(y, ref, bound)


@pytest.mark.parametrize("m", [5, 90])
def test_adapters_infinities_stay_in_their_rows(m):
    import torch
    g, a, b, rk, sc = bank_case(9, 2, 256, 64, 16, "bf16", scales=False)
    x, base = normal(g, m, 256, dtype="bf16"), normal(g, m, 64, dtype="bf16")
    ids = [i % 2 for i in range(m)]
    bank = eora.AdapterBank(a, b)
    good = bank.forward(x, ints(ids), base=base)
    x[2, 5] = float("inf")
    x[3, 7] = float("nan")
    y = bank.forward(x, ints(ids), base=base)
    assert not torch.isfinite(y[2]).any() and torch.isnan(y[3]).all()
    keep = [i for i in range(m) if i not in (2, 3)]
    assert torch.equal(y[keep], good[keep])


@pytest.mark.parametrize("m", [6, 70, 300])
def test_adapters_tokens_do_not_depend_on_each_other(m):
    """The same token with the same adapter in calls of the same size, among other tokens with other adapters, at another place."""
    import torch
    g, a, b, rk, sc = bank_case(14, 4, 1024, 96, 64, "bf16", [64, 40, 16, 64])
    bank = eora.AdapterBank(a, b, ranks=rk, scales=sc, y_dtype="f32")
    x = normal(g, m, 1024, dtype="bf16")
    first = bank.forward(x, ints([1] + [i % 5 - 1 for i in range(m - 1)]))
    x2 = normal(g, m, 1024, dtype="bf16")
    x2[m - 2] = x[0]
    second = bank.forward(x2, ints([2] * (m - 2) + [1, 0]))
    assert torch.equal(first[0], second[m - 2])


def test_adapters_in_a_graph_with_ids_and_weights_that_change():
    import torch
    m, n, K, N, R = 6, 4, 512, 128, 16
    g, a, b, rk, sc = bank_case(10, n, K, N, R, "f16")
    x, base, ids = normal(g, m, K), normal(g, m, N), ints([0, 1, 2, 3, -1, 0])
    y = torch.empty_like(base)
    bank = eora.AdapterBank(a, b, scales=sc)
    bank.forward(x, ids, base=base, y=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bank.forward(x, ids, base=base, y=y)
    for step in range(3):
        want = [(i * step + 1) % 5 - 1 for i in range(m)]
        ids.copy_(ints(want))
        a[step] = normal(g, K, R, std=0.02)
        x.copy_(normal(g, m, K))
        graph.replay()
        ref, bound = adapters_ref(x, a, b, want, rk, sc, base, "f16", "f16")
        within(y, ref, bound, f"replay {step}")


def test_adapters_offsets_beyond_32_bits():
    """The last adapter of a bank of more than 2^32 bytes in A and in B."""
    import torch
    n, K, N, R = 1100, 8192, 8192, 256
    a, b = (torch.empty((n, *s), dtype=torch.bfloat16, device=DEV) for s in ((K, R), (R, N)))
    g = gen(11)
    a[-1], b[-1] = normal(g, K, R, dtype="bf16", std=0.02), normal(g, R, N, dtype="bf16", std=0.02)
    x = normal(g, 2, K, dtype="bf16")
    y = eora.AdapterBank(a, b).forward(x, ints([n - 1, -1]))
    ref, bound = adapters_ref(x[:1], a[-1:], b[-1:], [0], None, None, None, "bf16", "bf16")
    within(y[:1], ref, bound)
    assert not y[1].any()


def test_adapters_more_tokens_than_a_launch_takes():
    import torch
    m, n, K, N, R = 17000, 5, 128, 32, 8
    g, a, b, rk, sc = bank_case(13, n, K, N, R, "f16", [8, 3, 8, 0, 5])
    x, base = normal(g, m, K), normal(g, m, N)
    ids = torch.randint(-1, n + 1, (m,), device=DEV, generator=g).int()
    ids[2000:9000] = 1
    y = eora.AdapterBank(a, b, ranks=rk, scales=sc).forward(x, ids, base=base)
    ref, bound = adapters_ref(x, a, b, ids.tolist(), rk, sc, base, "f16", "f16")
    within(y, ref, bound)


def test_adapters_wrapper_refusals():
    import torch
    g, a, b, rk, sc = bank_case(12, 2, 256, 64, 16, "f16")
    bank = eora.AdapterBank(a, b)
    x, ids, y = normal(g, 3, 256), ints([0, 1, 0]), normal(g, 3, 64)
    for bad in (dict(x=x.bfloat16()), dict(x=x[:, :128]), dict(x=x.t().contiguous().t()), dict(ids=ids.long()), dict(ids=ids[:2]), dict(ids=ids.cpu()), dict(y=y.float()), dict(y=y[:2]),
                dict(base=y[:2]), dict(base=y.float()), dict(x=x.cpu())):
        with pytest.raises(eora.EoraError):
            bank.forward(**{**dict(x=x, ids=ids, base=None, y=y.clone()), **bad})
    for bad in ((a, b[:1]), (a, b.bfloat16()), (a[:, :, :8], b[:, :8]), (a.float(), b.float())):
        with pytest.raises(eora.EoraError):
            eora.AdapterBank(*bad)
    assert bank.forward(x[:0], ids[:0]).shape == (0, 64)


@pytest.mark.parametrize("m", [3, 200])
def test_adapters_beside_a_compensated_layer(m):
    """Layer.forward with the requests' adapters: the layer's own result and the bank's, one rounding each."""
    import torch
    from helpers import make_case
    K, N = 512, 256
    layer = eora.Layer(*make_case(90, K, N, 64), max_m=m, y_dtype="f32")
    g, a, b, rk, sc = bank_case(91, 3, K, N, 16, "f16", [16, 5, 9])
    bank = eora.AdapterBank(a, b, ranks=rk, scales=sc, y_dtype="f32")
    x, ids = normal(g, m, K), [i % 4 - 1 for i in range(m)]
    plain = layer.forward(x)
    y = layer.forward(x, adapters=(bank, ints(ids)))
    ref, bound = adapters_ref(x, a, b, ids, rk, sc, None, "f16", "f32")
    # (the layer's own sums, whose order may change from call to call, are the same within 2^-19 of their size; one more rounding of the sum)
    slack = 2.0**-19 * plain.abs().max().item() + 2.0**-23 * np.abs(f64(plain) + ref)
    assert (np.abs(f64(y) - f64(plain) - ref) <= bound + slack).all()
    assert layer.device_status() == 0


# ---------------------------------------------------------------------------------------------- norms, rotation, cache
def table_of(far, rot, base=10000.0):
    import torch
    ang = torch.arange(far, device=DEV, dtype=torch.float64)[:, None] * base ** -(torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    return torch.cat([ang.cos(), ang.sin()], 1).float()


ROTATE = [
    # m, heads, kv heads, dim, rot, pairs, norm, page, layout, type, fused
    (1, 32, 8, 128, 128, "half", False, 16, "hnd", "f16", False),
    (1, 1, 1, 16, 16, "half", True, 1, "hnd", "bf16", False),
    (5, 4, 2, 64, 32, "adjacent", True, 4, "nhd", "f16", True),
    (9, 6, 2, 80, 48, "half", True, 16, "hnd", "bf16", True),
    (33, 14, 2, 96, 96, "adjacent", True, 32, "nhd", "bf16", False),
    (40, 8, 1, 256, 64, "half", True, 64, "hnd", "f16", False),
    (7, 5, 5, 128, 0, "half", True, 8, "hnd", "f16", False),
    (64, 3, 3, 32, 16, "half", False, 16, "hnd", "bf16", True),
    (1030, 8, 2, 64, 64, "half", True, 128, "nhd", "bf16", True),
    # many tokens
    (6500, 8, 2, 128, 128, "half", True, 16, "hnd", "bf16", False),
    (13000, 4, 1, 64, 32, "adjacent", False, 64, "nhd", "f16", True),
    (4100, 8, 1, 256, 128, "half", True, 32, "hnd", "f16", True),
    (12500, 2, 1, 96, 96, "half", True, 16, "nhd", "bf16", False),
    (12100, 1, 1, 80, 0, "half", True, 16, "hnd", "f16", False),
]


@pytest.mark.parametrize("case", range(len(ROTATE)))
def test_norm_rotation_and_cache(case):
    import torch
    m, H, KV, D, rot, pairs, norm, page, layout, ty, fused = ROTATE[case]
    g, far = gen(200 + case), 700
    if fused:
        q, k, v = normal(g, m, (H + 2 * KV) * D, dtype=ty).split([H * D, KV * D, KV * D], 1)
    else:
        q, k, v = normal(g, m, H * D, dtype=ty), normal(g, m, KV * D, dtype=ty), normal(g, m, KV * D, dtype=ty)
    qw, kw = ((1 + 0.2 * normal(g, D, dtype="f32")).to(tt(ty)) if norm else None for _ in range(2))
    table = table_of(far, rot) if rot else None
    pages = -(-m // page) + 2
    shape = (pages, KV, page, D) if layout == "hnd" else (pages, page, KV, D)
    kc, vc = (torch.full(shape, 3.0, dtype=tt(ty), device=DEV) for _ in range(2))
    pos = torch.randint(0, far, (m,), device=DEV, generator=g).int()
    slots = torch.randperm(pages * page, device=DEV, generator=g)[:m].int()
    if m > 4:
        slots[1], slots[2] = -1, pages * page                  # kept nowhere
        if rot:
            pos[3], pos[4] = -1, far                           # skipped altogether
    rope = eora.QKNormRope(H, KV, D, table, q_weight=qw, k_weight=kw, eps=1e-5, pairs=pairs, dtype=ty)
    cache = eora.PagedCache(kc, vc, layout=layout)
    q_out = torch.full((m, H * D), 9.0, dtype=tt(ty), device=DEV)
    k_out = torch.full((m, KV * D), 9.0, dtype=tt(ty), device=DEV)
    rope.forward(q, k, v, pos, slots=slots, cache=cache, q_out=q_out, k_out=k_out)
    skip = [i for i in range(m) if rot and not 0 <= int(pos[i]) < far]
    did = [i for i in range(m) if i not in skip]
    w64 = lambda w: None if w is None else f64(w)
    t64, p64 = (np.zeros((far, 0)) if table is None else f64(table)), pos.cpu().numpy()[did]
    rq, bq = orc.qk_norm_rope(f64(q)[did], w64(qw), t64, p64, H, rot, pairs, 1e-5, ty)
    rk, bk = orc.qk_norm_rope(f64(k)[did], w64(kw), t64, p64, KV, rot, pairs, 1e-5, ty)
    within(q_out[did], rq, bq, "q")
    within(k_out[did], rk, bk, "k")
    assert (q_out[skip] == 9).all() and (k_out[skip] == 9).all()
    kv_rows = lambda c: (c if layout == "nhd" else c.transpose(1, 2)).reshape(pages * page, KV * D)
    kept = [i for i in did if 0 <= int(slots[i]) < pages * page]
    at = slots[kept].long()
    assert torch.equal(kv_rows(kc)[at], k_out[kept]) and torch.equal(kv_rows(vc)[at], v[kept])
    rest = torch.ones(pages * page, dtype=torch.bool, device=DEV)
    rest[at] = False
    assert (kv_rows(kc)[rest] == 3).all() and (kv_rows(vc)[rest] == 3).all()
    # without a cache, and in place
    want = q_out.clone(), k_out.clone()
    q2, k2 = rope.forward(q, k, None, pos)
    assert torch.equal(q2[did], want[0][did]) and torch.equal(k2[did], want[1][did])
    qi, ki = q.clone(), k.clone()
    rope.forward(qi, ki, None, pos, q_out=qi, k_out=ki)
    assert torch.equal(qi[did], want[0][did]) and torch.equal(ki[did], want[1][did])
    assert torch.equal(qi[skip], q[skip])


def test_rotation_parts_of_a_token_agree():
    """A token's result does not depend on how many tokens the call has."""
    import torch
    g = gen(33)
    q, k, v = normal(g, 7000, 8 * 128), normal(g, 7000, 2 * 128), normal(g, 7000, 2 * 128)
    pos = torch.arange(7000, device=DEV).int()
    rope = eora.QKNormRope(8, 2, 128, table_of(7000, 128), dtype="f16", q_weight=normal(g, 128), k_weight=normal(g, 128))
    a = rope.forward(q, k, None, pos)
    for lo, hi in ((0, 1), (1, 4), (1000, 1100), (6999, 7000), (500, 2500)):
        b = rope.forward(q[lo:hi], k[lo:hi], None, pos[lo:hi])
        assert torch.equal(a[0][lo:hi], b[0]) and torch.equal(a[1][lo:hi], b[1])


def test_rotation_wrapper_refusals():
    import torch
    g = gen(34)
    rope = eora.QKNormRope(4, 2, 64, table_of(50, 64), dtype="f16")
    q, k, v, pos = normal(g, 3, 256), normal(g, 3, 128), normal(g, 3, 128), ints([0, 1, 2])
    kc = torch.zeros(2, 2, 16, 64, dtype=torch.float16, device=DEV)
    cache = eora.PagedCache(kc, kc.clone())
    good = dict(q=q, k=k, v=v, positions=pos, slots=pos, cache=cache)
    rope.forward(**good)
    for bad in (dict(v=None), dict(slots=None), dict(cache=None), dict(q=q.bfloat16()), dict(q=q[:, :128]), dict(k=k[:2]), dict(positions=pos.long()), dict(positions=pos[:2]),
                dict(slots=pos[:2]), dict(q=q.cpu()), dict(cache=eora.PagedCache(kc.bfloat16(), kc.bfloat16())), dict(cache=eora.PagedCache(kc[:, :1], kc[:, :1])),
                dict(q_out=q[:2].clone())):
        with pytest.raises(eora.EoraError):
            rope.forward(**{**good, **bad})
    assert rope.forward(q[:0], k[:0], None, pos[:0])[0].shape == (0, 256)
    assert rope.forward(q.view(3, 4, 64), k.view(3, 2, 64), None, pos)[0].shape == (3, 256)


# ----------------------------------------------------------------------------------------------------------- attention
def filled_cache(g, lengths, KV, D, page, layout, ty, window=0, extra=3, std=1.0, max_pages=None):
    """A cache that holds NaN in every row that no sequence sees, its page table (entries behind a sequence's pages point nowhere)."""
    import torch
    per = max_pages or max(1, max(-(-max(n, 0) // page) for n in lengths))
    need = [-(-max(n, 0) // page) for n in lengths]
    pages = sum(need) + extra
    order = torch.randperm(pages, device=DEV, generator=g).tolist()
    table = np.full((len(lengths), per), -1, np.int32)
    kc, vc = (torch.full((pages, KV, page, D), float("nan"), dtype=tt(ty), device=DEV) for _ in range(2))
    at, keys, values = 0, [], []
    for i, n in enumerate(lengths):
        n = max(n, 0)
        mine = order[at:at + need[i]]
        at += need[i]
        table[i, :need[i]] = mine
        first = max(0, n - window) if window else 0
        k, v = normal(g, KV, n, D, dtype=ty, std=std), normal(g, KV, n, D, dtype=ty)
        if first:
            k[:, :first], v[:, :first] = float("nan"), float("nan")
        keys.append(k[:, first:])
        values.append(v[:, first:])
        for j, pg in enumerate(mine):
            rows = slice(j * page, min(n, (j + 1) * page))
            kc[pg, :, :rows.stop - rows.start], vc[pg, :, :rows.stop - rows.start] = k[:, rows], v[:, rows]
    if layout == "nhd":
        kc, vc = kc.transpose(1, 2).contiguous(), vc.transpose(1, 2).contiguous()
    return kc, vc, torch.from_numpy(table).to(DEV), keys, values


def attention_ref(q, keys, values, H, scale, ty):
    B, D = q.shape[0], q.shape[1] // H
    outs = [np.zeros((B, H, D)), np.zeros((B, H)), np.zeros((B, H, D)), np.zeros((B, H))]
    q64 = f64(q).reshape(B, H, D)
    for i in range(B):
        KV = keys[i].shape[0]
        G = H // KV
        for h in range(KV):
            r = orc.attention(q64[i, h * G:(h + 1) * G], f64(keys[i][h]), f64(values[i][h]), scale, ty)
            for o, x in zip(outs, r):
                o[i, h * G:(h + 1) * G] = x
    return outs[0].reshape(B, -1), outs[1], outs[2].reshape(B, -1), outs[3]


ATTEND = [
    # lengths, heads, kv heads, dim, page, layout, type, window
    ([1], 1, 1, 64, 16, "hnd", "f16", 0),
    ([0], 4, 2, 128, 16, "hnd", "bf16", 0),
    ([1, 0, 2, 17, 16, 15], 8, 2, 128, 16, "hnd", "f16", 0),
    ([1000], 32, 8, 128, 16, "hnd", "f16", 0),
    ([333, 1, 64, 65, 127, 128, 129, 700], 14, 2, 64, 16, "nhd", "bf16", 0),
    ([500, 77], 12, 1, 96, 8, "hnd", "bf16", 0),
    ([200, 31, 450], 16, 1, 96, 32, "nhd", "f16", 0),
    ([130, 5, 0, 260], 20, 1, 128, 1, "hnd", "f16", 0),                # pages of one token, a group of twenty
    ([140, 90], 40, 1, 64, 2, "nhd", "bf16", 0),                       # a group in two parts
    ([260, 100], 35, 1, 128, 128, "hnd", "bf16", 0),
    ([300, 0, 65], 24, 3, 256, 16, "hnd", "f16", 0),
    ([100, 513], 32, 1, 256, 64, "nhd", "bf16", 0),
    ([900, 100, 101, 99, 50, 0, 1], 10, 2, 128, 16, "hnd", "bf16", 100),
    ([1000, 64], 8, 8, 64, 32, "nhd", "f16", 1),
    ([5000, 3000], 8, 4, 128, 64, "hnd", "bf16", 1111),
    ([9000], 2, 1, 64, 64, "hnd", "f16", 0),
    ([4000, -5, 1], 4, 1, 256, 32, "hnd", "bf16", 0),
    ([(i * 37) % 290 for i in range(70)], 4, 2, 64, 16, "hnd", "bf16", 0),        # three chunks of the scan, empty sequences among them
    ([(i * 53) % 41 for i in range(300)], 2, 2, 64, 16, "nhd", "f16", 24),
]


@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attention_matches_the_oracle(case):
    import torch
    lengths, H, KV, D, page, layout, ty, window = ATTEND[case]
    g = gen(300 + case)
    B = len(lengths)
    kc, vc, table, keys, values = filled_cache(g, lengths, KV, D, page, layout, ty, window)
    q = normal(g, B, H * D, dtype=ty, std=2.0)
    attn = eora.PagedAttention(H, KV, D, page_size=page, max_batch=B + 3, max_pages=table.shape[1], dtype=ty, window=window)
    cache = eora.PagedCache(kc, vc, layout=layout)
    lse = torch.full((B, H), 5.0, device=DEV)
    wide = torch.full((B + 2, H * D + 8), 7.0, dtype=tt(ty), device=DEV)
    out = wide[:B, :H * D]
    attn.forward(q, cache, table, ints(lengths), out=out, lse=lse)
    ref, rl, bo, bl = attention_ref(q, keys, values, H, D**-0.5, ty)
    within(out, ref, bo, "out")
    within(lse, rl, bl, "lse")
    assert (wide[B:] == 7).all() and (wide[:, H * D:] == 7).all()
    again = attn.forward(q, cache, table, ints(lengths))                     # the scratch is as it was; the same bits
    assert torch.equal(again, out)
    if B > 2:                                                                # fewer sequences through the same workspace
        part = attn.forward(q[:2], cache, table[:2], ints(lengths[:2]))
        within(part, ref[:2], bo[:2], "two of them")


def test_attention_of_peaked_and_flat_scores():
    """Scores over +-200 (one token takes all), and 40000 tokens of equal score with one 17 above them: what they weigh together (e^-17 each) counts."""
    import torch
    g = gen(40)
    n, D = 40000, 64
    for ty in ("f16", "bf16"):
        kc, vc, table, keys, values = filled_cache(g, [n, 500], 1, D, 64, "hnd", ty)
        q = normal(g, 2, D, dtype=ty)
        # sequence 0: keys 0 except one token along q
        q[0] = 0
        q[0, 0] = 17
        page_of = lambda t: (int(table[0, t // 64]), t % 64)
        keys[0].zero_()
        values[0].copy_(values[0].abs())
        keys[0][0, 12345, 0] = 1
        for t0 in range(0, n, 64):
            pg, rows = int(table[0, t0 // 64]), min(64, n - t0)
            kc[pg, 0, :rows], vc[pg, 0, :rows] = keys[0][0, t0:t0 + rows], values[0][0, t0:t0 + rows]
        q[1] *= 12
        attn = eora.PagedAttention(1, 1, D, page_size=64, max_batch=2, max_pages=table.shape[1], dtype=ty, scale=1.0)
        out, lse = torch.empty_like(q), torch.empty((2, 1), device=DEV)
        attn.forward(q, eora.PagedCache(kc, vc), table, ints([n, 500]), out=out, lse=lse)
        ref, rl, bo, bl = attention_ref(q, keys, values, 1, 1.0, ty)
        within(out, ref, bo)
        within(lse, rl, bl)


def test_attention_leaves_out_pages_that_are_none_and_clamps_lengths():
    import torch
    g = gen(41)
    kc, vc, table, keys, values = filled_cache(g, [160, 64], 2, 128, 16, "hnd", "bf16", max_pages=10)
    pages = kc.shape[0]
    table[0, 3], table[0, 7] = pages, -1
    table[1, 0] = 2**31 - 1
    table[1, 1:4] = -3
    q = normal(g, 2, 8 * 128, dtype="bf16")
    attn = eora.PagedAttention(8, 2, 128, page_size=16, max_batch=2, max_pages=10, dtype="bf16")
    out, lse = torch.empty_like(q), torch.empty((2, 8), device=DEV)
    attn.forward(q, eora.PagedCache(kc, vc), table, ints([2**31 - 1, 64]), out=out, lse=lse)     # the first: all ten pages
    seen = [t for t in range(160) if t // 16 not in (3, 7)]
    keys[0], values[0], keys[1], values[1] = keys[0][:, seen], values[0][:, seen], keys[1][:, :0], values[1][:, :0]
    ref, rl, bo, bl = attention_ref(q, keys, values, 8, 128**-0.5, "bf16")
    within(out, ref, bo)
    within(lse, rl, bl)
    assert not out[1].any() and torch.isneginf(lse[1]).all()


def test_attention_offsets_beyond_32_bits():
    """Pages at the far end of a cache of more than 2^32 elements."""
    import torch
    g = gen(42)
    pages, KV, page, D = 2200, 8, 1024, 256
    kc, vc = (torch.empty((pages, KV, page, D), dtype=torch.float16, device=DEV) for _ in range(2))
    n = 1500
    k, v = normal(g, KV, n, D), normal(g, KV, n, D)
    kc[pages - 1], vc[pages - 1] = k[:, :page], v[:, :page]
    kc[pages - 3, :, :n - page], vc[pages - 3, :, :n - page] = k[:, page:], v[:, page:]
    assert (pages - 3) * KV * page * D > 2**32
    q = normal(g, 1, KV * D)
    attn = eora.PagedAttention(KV, KV, D, page_size=page, max_batch=1, max_pages=2, dtype="f16")
    out = attn.forward(q, eora.PagedCache(kc, vc), ints([[pages - 1, pages - 3]]), ints([n]))
    ref, _, bo, _ = attention_ref(q, [k], [v], KV, D**-0.5, "f16")
    within(out, ref, bo)
    rope = eora.QKNormRope(KV, KV, D, None, dtype="f16")                     # and the write into them
    slots = ints([(pages - 1) * page + 5])
    rope.forward(q, q, q, ints([0]), slots=slots, cache=eora.PagedCache(kc, vc))
    assert torch.equal(kc[pages - 1, :, 5].reshape(-1), q[0]) and torch.equal(vc[pages - 1, :, 5].reshape(-1), q[0])


def test_attention_in_a_graph_while_sequences_grow():
    import torch
    g = gen(43)
    H, KV, D, page, ty = 8, 2, 128, 16, "bf16"
    final = [40, 3, 700]
    kc, vc, table, keys, values = filled_cache(g, final, KV, D, page, "hnd", ty)
    cache = eora.PagedCache(kc, vc)
    attn = eora.PagedAttention(H, KV, D, page_size=page, max_batch=3, max_pages=table.shape[1], dtype=ty)
    q, lens = normal(g, 3, H * D, dtype=ty), ints([1, 0, 1])
    out = torch.empty_like(q)
    attn.forward(q, cache, table, lens, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attn.forward(q, cache, table, lens, out=out)
    for now in ([5, 1, 16], [39, 0, 600], final, [1, 3, 0]):
        lens.copy_(ints(now))
        q.copy_(normal(g, 3, H * D, dtype=ty))
        graph.replay()
        ref, _, bo, _ = attention_ref(q, [k[:, :n] for k, n in zip(keys, now)], [v[:, :n] for v, n in zip(values, now)], H, D**-0.5, ty)
        within(out, ref, bo, str(now))


def test_attention_on_two_streams_with_two_workspaces():
    import torch
    g = gen(44)
    jobs = []
    for i in range(2):
        kc, vc, table, keys, values = filled_cache(g, [3000 + i, 20], 2, 128, 16, "hnd", "f16")
        q = normal(g, 2, 4 * 128)
        jobs.append((eora.PagedAttention(4, 2, 128, page_size=16, max_batch=2, max_pages=table.shape[1], dtype="f16"), eora.PagedCache(kc, vc), table, ints([3000 + i, 20]), q,
                     torch.empty_like(q), keys, values, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for a, c, t, n, q, o, _, _, s in jobs:
            a.forward(q, c, t, n, out=o, stream=s)
    torch.cuda.synchronize()
    for a, c, t, n, q, o, keys, values, s in jobs:
        ref, _, bo, _ = attention_ref(q, keys, values, 4, 128**-0.5, "f16")
        within(o, ref, bo)


def test_attention_interleaved_keys_and_values_and_a_view_of_heads():
    """K and V of a page in one buffer, and a cache object over some heads of a wider one."""
    import torch
    g = gen(45)
    kc, vc, table, keys, values = filled_cache(g, [90, 33], 4, 64, 16, "hnd", "f16")
    both = torch.stack([kc, vc], 1)                                          # [page][2][head][row][channel]
    q = normal(g, 2, 4 * 64)
    attn = eora.PagedAttention(4, 2, 64, page_size=16, max_batch=2, max_pages=table.shape[1], dtype="f16")
    out = attn.forward(q, eora.PagedCache(both[:, 0, 1:3], both[:, 1, 1:3]), table, ints([90, 33]))
    ref, _, bo, _ = attention_ref(q, [k[1:3] for k in keys], [v[1:3] for v in values], 4, 0.125, "f16")
    within(out, ref, bo)


def test_attention_strided_queries_and_tables():
    """q as columns of a wider product, [batch][heads][dim] views, a page table that is wider than a sequence can be, with rows further apart still."""
    import torch
    g = gen(47)
    kc, vc, table, keys, values = filled_cache(g, [150, 3, 77], 2, 128, 16, "nhd", "bf16")
    wide_q = normal(g, 3, 6 * 128 + 24, dtype="bf16")
    q = wide_q[:, 8:8 + 6 * 128]
    wide_t = torch.full((3, table.shape[1] + 9), -7, dtype=torch.int32, device=DEV)
    wide_t[:, 1:1 + table.shape[1]] = table
    attn = eora.PagedAttention(6, 2, 128, page_size=16, max_batch=3, max_pages=table.shape[1], dtype="bf16")
    cache, lens = eora.PagedCache(kc, vc, layout="nhd"), ints([150, 3, 77])
    out = attn.forward(q, cache, wide_t[:, 1:], lens)
    ref, _, bo, _ = attention_ref(q.contiguous(), keys, values, 6, 128**-0.5, "bf16")
    within(out, ref, bo)
    out3 = torch.empty(3, 6, 128, dtype=torch.bfloat16, device=DEV)
    assert attn.forward(q.unflatten(1, (6, 128)), cache, table, lens, out=out3) is out3
    assert torch.equal(out3.flatten(1), out)


def test_calls_on_a_side_stream():
    """All three on a stream that is not the current one, behind work that it has to wait for."""
    import torch
    g = gen(48)
    side = torch.cuda.Stream()
    n, K, N, R = 3, 512, 4 * 64, 16
    gb, a, b, rk, sc = bank_case(49, n, K, N, R, "f16")
    x0 = normal(g, 5, K)
    kc, vc = (torch.zeros(6, 2, 16, 64, dtype=torch.float16, device=DEV) for _ in range(2))
    cache, pages = eora.PagedCache(kc, vc), ints([[0], [1], [2], [3], [4]])
    bank, rope = eora.AdapterBank(a, b, scales=sc), eora.QKNormRope(4, 2, 64, table_of(32, 64), dtype="f16")
    attn = eora.PagedAttention(4, 2, 64, page_size=16, max_batch=5, max_pages=1, dtype="f16")
    k, v, ids, pos, slots, one = normal(g, 5, 128), normal(g, 5, 128), ints([0, 1, 2, -1, 0]), ints([0] * 5), ints([0, 16, 32, 48, 64]), ints([1] * 5)
    x, y, q, o = (torch.zeros_like(t) for t in (x0, normal(g, 5, N), normal(g, 5, N), normal(g, 5, N)))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        x.copy_(x0)
    bank.forward(x, ids, y=y, stream=side)
    rope.forward(y, k, v, pos, slots=slots, cache=cache, q_out=q, stream=side)
    attn.forward(q, cache, pages, one, out=o, stream=side.cuda_stream)
    side.synchronize()
    ref, bound = adapters_ref(x0, a, b, [0, 1, 2, -1, 0], rk, sc, None, "f16", "f16")
    within(y, ref, bound)
    assert torch.equal(q, y)                                                 # position 0 turns nothing
    assert torch.equal(o.view(5, 2, 2, 64), v.view(5, 2, 1, 64).expand(5, 2, 2, 64))       # one token: its value


def test_attention_wrapper_refusals():
    import torch
    g = gen(46)
    kc, vc, table, _, _ = filled_cache(g, [40, 33], 2, 64, 16, "hnd", "f16")
    attn, cache = eora.PagedAttention(4, 2, 64, page_size=16, max_batch=2, max_pages=3, dtype="f16"), eora.PagedCache(kc, vc)
    q, lens = normal(g, 2, 256), ints([40, 33])
    out = torch.empty_like(q)
    good = dict(q=q, cache=cache, page_table=table, lengths=lens)
    for bad in (dict(q=q.bfloat16()), dict(q=q[:, :128]), dict(page_table=table.long()), dict(page_table=table[:1]), dict(page_table=table[:, :2]), dict(lengths=lens[:1]), dict(lengths=lens.long()),
                dict(out=out[:1]), dict(lse=torch.empty(2, 3, device=DEV)), dict(q=q.cpu()), dict(q=torch.cat([q, q])), dict(cache=eora.PagedCache(kc.bfloat16(), vc.bfloat16())),
                dict(cache=eora.PagedCache(kc[:, :, :8], vc[:, :, :8])), dict(lengths=None)):
        with pytest.raises(eora.EoraError):
            attn.forward(**{**good, **bad})
    assert attn.forward(q[:0], cache, table[:0], lens[:0]).shape == (0, 256)
    with pytest.raises(eora.EoraError):
        eora.PagedAttention(4, 2, 80, page_size=16, max_batch=2, max_pages=3)
    assert torch.isfinite(attn.forward(**good)).all()


def test_first_calls_can_be_captured():
    """A fresh process whose first call of each operator is made while a graph is captured."""
    import subprocess
    import sys
    code = """
import torch, paper_2410_21271_b200 as E
d = "cuda:0"
h = dict(dtype=torch.float16, device=d)
x, a, b = torch.ones(3, 128, **h), torch.ones(2, 128, 8, **h), torch.ones(2, 8, 32, **h)
bank = E.AdapterBank(a, b)
kc = torch.zeros(4, 2, 16, 64, **h); vc = kc.clone()
cache = E.PagedCache(kc, vc)
rope = E.QKNormRope(4, 2, 64, None, dtype="f16")
attn = E.PagedAttention(4, 2, 64, page_size=16, max_batch=3, max_pages=1, dtype="f16")
i = torch.zeros(3, dtype=torch.int32, device=d); i1 = i + 1; slots = torch.tensor([0, 16, 32], dtype=torch.int32, device=d)
table = torch.tensor([[0], [1], [2]], dtype=torch.int32, device=d)
q, k = torch.ones(3, 256, **h), torch.ones(3, 128, **h)
y, qo, o = torch.zeros(3, 32, **h), torch.zeros(3, 256, **h), torch.zeros(3, 256, **h)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    bank.forward(x, i, y=y)
    rope.forward(q, k, 3 * k, i, slots=slots, cache=cache, q_out=qo)
    attn.forward(qo, cache, table, i1, out=o)
g.replay()
torch.cuda.synchronize()
assert (y == 1024).all() and (o == 3).all(), (y, o)
print("fine")
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]


# --------------------------------------------------------------------------------------------- together, as they are used
@pytest.mark.parametrize("fused", [True, False])
def test_attention_half_of_a_block_decoding_three_requests(fused):
    """q|k|v by the compensated layers with an adapter per request beside them, norms and rotation into the cache, attention over it, o: token by
    token, against the same in float64 with the whole sequence at hand."""
    import torch
    from helpers import make_case
    hid, H, KV, D, page, steps, B, n_ad, R = 512, 4, 2, 64, 16, 21, 3, 2, 16
    outs = (H * D, KV * D, KV * D)
    parts = [make_case(60 + i, hid, n, 64) for i, n in enumerate(outs)]
    o_parts = make_case(70, H * D, hid, 64)
    layer = [eora.Layer(*p, max_m=8) for p in parts]
    qkv = eora.FusedLayers(parts, max_m=8) if fused else None
    o = eora.Layer(*o_parts, max_m=8)
    dense = [f64(l.dump(1)) + f64(l.dump(2)) @ f64(l.dump(3)) for l in layer + [o]]
    g, a, b, rk, sc = bank_case(71, n_ad, hid, H * D, R, "f16", [16, 9])
    bank = eora.AdapterBank(a, b, ranks=rk, scales=sc)
    qw, kw = ((1 + 0.1 * normal(g, D, dtype="f32")).half() for _ in range(2))
    table = table_of(64, D)
    rope = eora.QKNormRope(H, KV, D, table, q_weight=qw, k_weight=kw, eps=1e-5, dtype="f16")
    per = -(-steps // page)
    kc, vc = (torch.full((B * per, KV, page, D), float("nan"), dtype=torch.float16, device=DEV) for _ in range(2))
    cache = eora.PagedCache(kc, vc)
    pages = ints(np.random.default_rng(72).permutation(B * per).reshape(B, per).tolist())
    attn = eora.PagedAttention(H, KV, D, page_size=page, max_batch=B, max_pages=per, dtype="f16")
    ids = [1, -1, 0]
    xs = normal(g, steps, B, hid)
    got = []
    for t in range(steps):
        with_bank = (bank, ints(ids))
        if fused:
            q, k, v = qkv.forward(xs[t], adapters=[with_bank, None, None])
        else:
            q, k, v = (l.forward(xs[t], adapters=with_bank if l is layer[0] else None) for l in layer)
        slots = pages[:, t // page] * page + t % page
        q, _ = rope.forward(q, k, v, ints([t] * B), slots=slots, cache=cache, q_out=q)
        got.append(o.forward(attn.forward(q, cache, pages, ints([t + 1] * B))))
    got = f64(torch.stack(got))
    x64 = f64(xs)
    ref = np.zeros((steps, B, hid))
    A, Bm = np.nan_to_num(f64(a)), np.nan_to_num(f64(b))
    for i in range(B):
        q = orc.adapters(x64[:, i], A, Bm, [ids[i]] * steps, rk.tolist(), sc.tolist(), base=x64[:, i] @ dense[0])[0]
        q = orc.qk_norm_rope(q, f64(qw), f64(table), np.arange(steps), H, D, "half", 1e-5)[0].reshape(steps, H, D)
        k = orc.qk_norm_rope(x64[:, i] @ dense[1], f64(kw), f64(table), np.arange(steps), KV, D, "half", 1e-5)[0].reshape(steps, KV, D)
        v = (x64[:, i] @ dense[2]).reshape(steps, KV, D)
        for t in range(steps):
            row = [orc.attention(q[t, h * 2:h * 2 + 2], k[:t + 1, h], v[:t + 1, h], D**-0.5)[0] for h in range(KV)]
            ref[t, i] = np.concatenate(row).reshape(-1) @ dense[3]
    # Two projections of the compensated layers (2e-3 each, the library's own tolerance), three fp16 roundings of what stands between them (2^-11
    # each, q and k after a norm), an error d of q or k moving a score of magnitude |q||k|/sqrt(D) <= sqrt(D) (1.1)^2 by that times d: twice
    # sqrt(64) 1.2 (2e-3 / sqrt(64) as the errors of a row's channels are independent, + 2^-11) of the weights; together below 2e-2.
    err = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    assert err <= 2e-2, err
    for l in layer + [o] + ([qkv] if qkv else []):
        assert l.device_status() == 0
