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


def plainly(q, k, v, scale):
    """Attention in float64 as the formula stands, infinities and all.  q [g][d], k, v [t][d]."""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        s = scale * (q[:, None, :] * k[None]).sum(-1)
        e = np.exp(s - s.max(1, keepdims=True))
        lse = np.where(np.isposinf(s).any(1) & ~np.isnan(s).any(1), np.inf, np.logaddexp.reduce(s, axis=1))
        return s, ((e / e.sum(1, keepdims=True))[:, :, None] * v[None]).sum(1), lse


@pytest.mark.parametrize("ty", ["f16", "bf16"])
@pytest.mark.parametrize("n", [1, 3, 40, 3000])
@pytest.mark.parametrize("H,KV,D", [(4, 2, 64), (9, 1, 128), (2, 2, 256)])
def test_attention_infinities_are_those_of_the_formula(H, KV, D, n, ty):
    import torch
    g, inf, G = gen(820), float("inf"), H // KV
    what = ["all scores -inf", "all +inf", "one +inf", "some -inf", "one NaN", "all -inf but one", "an infinite value", "two infinite values", "nothing"]
    B = len(what)
    kc, vc, table, keys, values = filled_cache(g, [n] * B, KV, D, 16, "hnd", ty)
    q = normal(g, B, H * D, dtype=ty)
    q3 = q.view(B, H, D)
    q3[:, :, 1] = q3[:, :, 1].abs() + 0.25
    at = n * 2 // 3
    for i in range(B):
        k, v = keys[i], values[i]
        if i in (0, 1, 2):                                   # the first head of each group has an infinity in q
            q3[i, ::G, 0] = inf
            k[:, :, 0] = (k[:, :, 0].abs() + 0.1) * (1 if i == 1 else -1)
            if i == 2:
                k[:, at, 0] *= -1
        elif i == 3:
            k[:, : n // 2, 1] = -inf
            k[:, n // 2 + 1::3, 1] = -inf
        elif i == 4:
            k[:, at, 2] = float("nan")
        elif i == 5:
            k[:, :, 1] = -inf
            k[:, at, 1] = 0.5
        elif i in (6, 7):
            v[:, at, 3] = inf
            v[:, n // 3, 5] = -inf
            if i == 7:
                v[:, 0, 3] = -inf
        for t0 in range(0, n, 16):
            pg, rows = int(table[i, t0 // 16]), min(16, n - t0)
            kc[pg, :, :rows], vc[pg, :, :rows] = k[:, t0:t0 + rows], v[:, t0:t0 + rows]
    attn = eora.PagedAttention(H, KV, D, page_size=16, max_batch=B, max_pages=table.shape[1], dtype=ty)
    lse = torch.zeros(B, H, device=DEV)
    out = f64(attn.forward(q, eora.PagedCache(kc, vc), table, ints([n] * B), lse=lse)).reshape(B, H, D)
    lse, q64 = f64(lse), f64(q3)
    for i in range(B):
        for h in range(H):
            k, v = f64(keys[i][h // G]), f64(values[i][h // G])
            s, want, wl = (r[0] for r in plainly(q64[i, h:h + 1], k, v, D**-0.5))
            assert np.array_equal(np.isnan(out[i, h]), np.isnan(want)), (what[i], h)
            assert np.array_equal(out[i, h][np.isinf(want)], want[np.isinf(want)]) and np.array_equal(np.isinf(out[i, h]), np.isinf(want)), (what[i], h)
            fine = np.isfinite(want)
            if np.isfinite(wl):
                some = ~np.isneginf(s)
                ref, rl, bo, bl = orc.attention(q64[i, h:h + 1], k[some], np.where(np.isfinite(v[some]), v[some], 0), D**-0.5, ty)
                assert (np.abs(out[i, h] - ref[0])[fine] <= bo[0][fine]).all() and abs(lse[i, h] - rl[0]) <= bl[0], (what[i], h)
            else:
                assert lse[i, h] == wl or np.isnan(lse[i, h]) and np.isnan(wl), (what[i], h, lse[i, h], wl)
    assert np.isnan(out[0, 0]).all() and np.isneginf(lse[0, 0]) and np.isposinf(lse[1, 0]) and np.isfinite(out[8]).all()


@pytest.mark.parametrize("pairs", ["half", "adjacent"])
@pytest.mark.parametrize("m,D,rot", [(5, 64, 32), (7000, 64, 32), (3, 128, 0), (4200, 256, 64)])
def test_norm_weights_that_are_not_finite_stay_in_their_channels(m, D, rot, pairs):
    """Channels that are not rotated have no partner: an infinite weight of one is nothing to another."""
    import torch
    from test_serve_gpu import table_of
    g = gen(880)
    q, k = normal(g, m, 2 * D), normal(g, m, D)
    w = normal(g, D)
    bad = [rot + 3, D - 1, D - 9]
    w[bad[0]], w[bad[1]], w[bad[2]] = float("inf"), float("nan"), -float("inf")
    pos = (torch.arange(m, device=DEV) % 50).int()
    rope = eora.QKNormRope(2, 1, D, table_of(50, rot) if rot else None, q_weight=w, k_weight=w, pairs=pairs, dtype="f16")
    clean = w.clone()
    clean[bad] = 1.0
    sound = eora.QKNormRope(2, 1, D, table_of(50, rot) if rot else None, q_weight=clean, k_weight=clean, pairs=pairs, dtype="f16")
    keep = [c for c in range(D) if c not in bad]
    for got, want in zip(rope.forward(q, k, None, pos), sound.forward(q, k, None, pos)):
        got, want = got.view(m, -1, D), want.view(m, -1, D)
        assert torch.equal(got[..., keep], want[..., keep])
        assert not torch.isfinite(got[..., bad]).any()
