"""What the serving operators keep of their intermediate results, and infinities, against the float64 oracle.  Tolerances are derived beside the tests."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import paper_2410_21271_b200 as eora
from oracle import serve_oracle as orc
from test_serve_gpu import DEV, f64, filled_cache, gen, ints, normal, within


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("H,KV,D", [(8, 2, 128), (2, 2, 64), (9, 1, 96), (24, 1, 128), (12, 1, 256)])
def test_attention_weights_keep_more_than_their_type(ty, H, KV, D):
    """Two tokens of nearly the same weight and opposite values: the output is the difference of the weights, which one part of 16 bits each would lose.

    A weight in two parts: bf16 has eight bits in the high part, cut, so the low part is below 2^-7 of the weight and its half step 2^-8 of that: 2^-15.
    fp16 has eleven, cut after 2^-10 was taken off: the low part is below 2^-9, its half step 2^-11 of that: 2^-20.  Everything else is the oracle's bound."""
    step = {"bf16": 2.0**-15, "f16": 2.0**-20}[ty]
    B = 24
    g = gen(800)
    kc, vc, table, keys, values = filled_cache(g, [2] * B, KV, D, 16, "hnd", ty, std=0.1)
    for i in range(B):
        vc[int(table[i, 0]), :, 1] = -vc[int(table[i, 0]), :, 0]
        values[i][:, 1] = -values[i][:, 0]
    q = normal(g, B, H * D, dtype=ty, std=0.1)
    attn = eora.PagedAttention(H, KV, D, page_size=16, max_batch=B, max_pages=1, dtype=ty)
    out = f64(attn.forward(q, eora.PagedCache(kc, vc), table, ints([2] * B))).reshape(B, H, D)
    q64, G = f64(q).reshape(B, H, D), H // KV
    for i in range(B):
        for h in range(KV):
            mine = slice(h * G, (h + 1) * G)
            ref, _, bound, _ = orc.attention(q64[i, mine], f64(keys[i][h]), f64(values[i][h]), D**-0.5, ty, weight_step=step)
            over = np.abs(out[i, mine] - ref) - bound
            assert over.max() <= 0, (i, h, np.abs(out[i, mine] - ref).max(), over.max())


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("m", [6, 90, 300])
def test_adapters_infinities_are_those_of_the_formula(m, ty):
    """Rows of t that hold infinities: +-inf where all terms of a sum have one sign (ranks 1 and 16 with positive weights), NaN where two signs meet."""
    import torch
    n, K, R, N = 3, 256, 16, 64
    g = gen(810)
    a, b = normal(g, n, K, R, dtype=ty, std=0.02), normal(g, n, R, N, dtype=ty, std=0.02)
    a[0], b[0] = a[0].abs(), b[0].abs()
    a[a == 0], b[b == 0] = 0.01, 0.01
    x, base = normal(g, m, K, dtype=ty), normal(g, m, N, dtype=ty)
    inf = float("inf")
    x[0, 5], x[1, 5], x[2, 77], x[3, 200], x[4, 0], base[5, 3] = inf, -inf, inf, -inf, float("nan"), inf
    ids = [0, 0, 1, 2, 1, 2] + [i % 4 - 1 for i in range(m - 6)]
    bank = eora.AdapterBank(a, b, ranks=ints([16, 1, 16]), y_dtype="f32")
    y = f64(bank.forward(x, ints(ids), base=base.float()))
    for i in range(6):
        r, j = [16, 1, 16][ids[i]], ids[i]
        with np.errstate(invalid="ignore"):
            t = (f64(x[i])[:, None] * f64(a[j, :, :r])).sum(0)
            want = f64(base[i]) + (t[:, None] * f64(b[j, :r])).sum(0)
        assert np.array_equal(np.isnan(y[i]), np.isnan(want)), i
        assert np.array_equal(y[i][np.isinf(want)], want[np.isinf(want)]) and np.array_equal(np.isinf(y[i]), np.isinf(want)), i
    assert np.isposinf(y[0]).all() and np.isneginf(y[1]).all() and np.isinf(y[2]).all() and np.isnan(y[4]).all()
    assert np.isfinite(y[6:]).all()
