"""The serving kernels in their steady state: rings that are refilled many times, blocks with several pieces of work, several passes over the columns."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import paper_2410_21271_b200 as eora
from oracle import serve_oracle as orc
from test_serve_gpu import DEV, adapters_ref, bank_case, f64, filled_cache, gen, ints, normal, within

RAGGED = [100 + (i * 2417) % 3900 for i in range(40)]              # 100 .. 4000
RAGGED[3] = RAGGED[17] = RAGGED[18] = RAGGED[39] = 0
# A block of the chip has total / 148 units of 128 tokens (64 at head size 256): a serving batch has 35 and more, of two to five pairs that begin or
# end in it; few pairs have 10 and more each.
ATTEND = [
    # lengths, heads, kv heads, dim, page, layout, type, window, pairs that are looked at
    (RAGGED, 16, 8, 128, 64, "hnd", "bf16", 0, 2),
    (RAGGED, 8, 8, 64, 32, "nhd", "f16", 0, 3),
    (RAGGED, 16, 8, 96, 64, "nhd", "bf16", 1500, 2),
    (RAGGED, 8, 8, 256, 64, "hnd", "f16", 0, 1),
    (RAGGED, 40, 4, 128, 128, "hnd", "f16", 2000, 1),                # groups of ten
    (RAGGED, 60, 3, 64, 64, "nhd", "bf16", 0, 1),                    # groups of twenty; pairs of one sequence in several blocks
    ([50000, 47001], 8, 2, 128, 64, "hnd", "bf16", 0, 2),            # few pairs, 37 blocks each: joined in two rounds
    ([50000, 0, 3000, 170], 4, 2, 64, 128, "nhd", "f16", 0, 2),      # few pairs of very different length
    ([26000], 4, 2, 256, 64, "nhd", "bf16", 0, 2),
    ([30000, 29000, 31000], 6, 2, 96, 64, "hnd", "f16", 20000, 2),
    ([199000], 2, 1, 64, 64, "hnd", "bf16", 0, 1),                   # one pair for all blocks
]


@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attention_of_many_units_a_block(case):
    import torch
    lengths, H, KV, D, page, layout, ty, window, looks = ATTEND[case]
    g, rng, B, G = gen(830 + case), np.random.default_rng(case), len(lengths), H // KV
    kc, vc, table, keys, values = filled_cache(g, lengths, KV, D, page, layout, ty, window)
    q = normal(g, B, H * D, dtype=ty, std=2.0)
    attn = eora.PagedAttention(H, KV, D, page_size=page, max_batch=B, max_pages=table.shape[1], dtype=ty, window=window)
    cache, n = eora.PagedCache(kc, vc, layout=layout), ints(lengths)
    lse = torch.zeros(B, H, device=DEV)
    out = attn.forward(q, cache, table, n, lse=lse)
    for _ in range(3):                                               # the workspace as it was; the same bits
        assert torch.equal(attn.forward(q, cache, table, n), out)
    got, gl, q64 = f64(out).reshape(B, H, D), f64(lse), f64(q).reshape(B, H, D)
    assert np.isfinite(got).all()
    for i in range(B):
        for h in rng.choice(KV, looks, replace=False):
            mine = slice(h * G, (h + 1) * G)
            ref, rl, bo, bl = orc.attention(q64[i, mine], f64(keys[i][h]), f64(values[i][h]), D**-0.5, ty)
            assert (np.abs(got[i, mine] - ref) <= bo).all(), (i, h, np.abs(got[i, mine] - ref).max())
            assert np.array_equal(gl[i, mine], rl) if lengths[i] == 0 else (np.abs(gl[i, mine] - rl) <= bl).all(), (i, h)


ADAPTERS = [
    # m, n, K, N, max rank, ranks, x type, y type: clusters that are small against d_in and d_out, so that each warp goes round its ring of two stages
    # many times and takes several times 64 columns
    (2500, 60, 4096, 4096, 64, "mixed", "bf16", "bf16"),             # clusters of 4: 8 steps of A a warp, 4 times its columns
    (2500, 60, 4096, 4096, 64, "mixed", "f16", "f32"),
    (1500, 120, 2048, 2048, 136, "mixed", "f16", "f16"),
    (700, 3, 14336, 4096, 200, "equal", "bf16", "f32"),              # ranks above 128: one warp for 64 columns, 28 steps
    (61, 5, 4096, 14336, 128, "equal", "f16", "f32"),                # few tokens, two times the columns
    (200, 12, 8192, 8192, 256, "mixed", "bf16", "bf16"),
    (256, 200, 4096, 4096, 32, "mixed", "f16", "f16"),               # few tokens, clusters of one
]


@pytest.mark.parametrize("case", range(len(ADAPTERS)))
def test_adapters_of_many_steps_a_warp(case):
    import torch
    m, n, K, N, R, kind, xt, yt = ADAPTERS[case]
    ranks = None if kind == "equal" else [max(1, R >> (j % 3)) + (j % 5 == 4) for j in range(n)]
    g, a, b, rk, sc = bank_case(850 + case, n, K, N, R, xt, None if ranks is None else [min(r, R) for r in ranks])
    ids = torch.randint(-1, n, (m,), device=DEV, generator=g).int()
    ids[m // 3:m // 2] = n // 2                                      # a prompt among them
    x, base = normal(g, m, K, dtype=xt), normal(g, m, N, dtype=yt)
    bank = eora.AdapterBank(a, b, ranks=rk, scales=sc, y_dtype=yt)
    y = bank.forward(x, ids, base=base)
    bare = bank.forward(x, ids)
    inplace = base.clone()
    bank.forward(x, ids, base=inplace, y=inplace)
    assert torch.equal(inplace, y) and torch.equal(bank.forward(x, ids, base=base), y)
    some = np.unique(np.concatenate([np.random.default_rng(case).choice(m, min(m, 160), replace=False), [0, m - 1]]))
    named = sorted({int(ids[i]) for i in some} - {-1})
    at = {j: k for k, j in enumerate(named)}
    pick = lambda base: adapters_ref(x[some], a[named], b[named], [at.get(int(ids[i]), -1) for i in some], None if rk is None else rk[named], sc[named],
                                     None if base is None else base[some], xt, yt)
    within(y[some], *pick(base), "with a base")
    within(bare[some], *pick(None), "without")
    off = ids < 0
    assert torch.equal(y[off], base[off]) and not bare[off].any()
    # every token, to catch a row or a run of columns that the samples miss: half a step of the output (bf16), and for t's parts (2^-16 of it) and the
    # sums (below 2^-13 of their terms over 14336 products) 2^-10 of the largest result, which the terms of a sum do not exceed eight times
    ref = base.float()
    for j in range(n):
        rows = (ids == j).nonzero()[:, 0]
        r = R if rk is None else int(rk[j])
        t = x[rows].double() @ a[j, :, :r].double()
        ref[rows] += (float(sc[j]) * (t @ b[j, :r].double())).float()
    size = ref.abs().max()
    assert ((y.float() - ref).abs() <= 2.0**-8 * ref.abs() + 2.0**-10 * size).all()
