"""The serving operators at the largest counts that their calls take, against torch in float64 (or products of it), on the device."""
import pytest

pytestmark = pytest.mark.gpu

import paper_2410_21271_b200 as eora
from test_serve_gpu import DEV, bank_case, gen, ints, normal, table_of, tt


def test_attention_of_65536_sequences_and_more_than_2_to_24_units():
    """All sequences look at the same two pages: 65536 x 8 pairs of 33 units of 128 tokens, past the 32-bit form of the shares; lengths of zero, one and
    at the border of a unit among them."""
    import torch
    g, B, KV, D, page, ty = gen(900), 65536, 8, 64, 4096, "bf16"
    kc, vc = normal(g, 2, KV, page, D, dtype=ty), normal(g, 2, KV, page, D, dtype=ty)
    q = normal(g, B, KV * D, dtype=ty)
    full = 33 * 128
    kinds = [full, full, full, full - 1, full - 127, full, full, 0, 1] + [full] * 100
    lengths = torch.tensor(kinds, device=DEV).repeat(B // len(kinds) + 1)[:B]
    assert int(((lengths + 127) // 128).sum()) * KV > 2**24
    table = ints([[0, 1]]).repeat(B, 1)
    attn = eora.PagedAttention(KV, KV, D, page_size=page, max_batch=B, max_pages=2, dtype=ty)
    lse = torch.empty(B, KV, device=DEV)
    out = attn.forward(q, eora.PagedCache(kc, vc), table, lengths.int(), lse=lse).view(B, KV, D)
    k, v = (c.transpose(0, 1).reshape(KV, 2 * page, D)[:, :full].double() for c in (kc, vc))
    for n in sorted(set(kinds)):
        rows = (lengths == n).nonzero()[:, 0]
        if n == 0:
            assert not out[rows].any() and torch.isneginf(lse[rows]).all()
            continue
        for part in rows.split(8192):
            for h in range(KV):
                s = q.view(B, KV, D)[part, h].double() @ k[h, :n].t() * D**-0.5
                ref, rl = torch.softmax(s, 1) @ v[h, :n], torch.logsumexp(s, 1)
                # half a step of the output; scores of up to 8 in fp32 (64 products of up to 25: 2^-19), weights in two parts (2^-15), sums: below 2^-12 of values up to 6
                assert ((out[part, h].double() - ref).abs() <= 2.0**-8 * ref.abs() + 6 * 2.0**-12).all(), (n, h)
                assert ((lse[part, h].double() - rl).abs() <= 2.0**-16 * (1 + rl.abs())).all(), (n, h)


def test_adapters_and_rotation_of_2_to_20_tokens():
    import torch
    m, n, K, N, R = 1 << 20, 3, 128, 32, 8
    g, a, b, rk, sc = bank_case(901, n, K, N, R, "f16")
    x, base = normal(g, m, K), normal(g, m, N)
    ids = torch.randint(-1, n, (m,), device=DEV, generator=g).int()
    y = eora.AdapterBank(a, b, scales=sc).forward(x, ids, base=base)
    ref, reach = base.double(), torch.zeros(m, N, dtype=torch.float64, device=DEV)
    for j in range(n):
        mine = (ids == j)[:, None]
        t = x.double() @ a[j].double()
        ref += torch.where(mine, float(sc[j]) * (t @ b[j].double()), 0.0)
        reach += torch.where(mine, float(sc[j]) * ((x.double().abs() @ a[j].double().abs()) @ b[j].double().abs()), 0.0)
    # half a step of the output, and 2^-18 of the terms for sums of 128 and 8 products and t's two parts
    assert ((y.double() - ref).abs() <= 2.0**-11 * ref.abs() + 2.0**-18 * reach + 2.0**-25).all()
    q, k, w, table = normal(g, m, 2 * 32), normal(g, m, 32), normal(g, 32), table_of(100, 32)
    pos = torch.randint(0, 100, (m,), device=DEV, generator=g).int()
    rope = eora.QKNormRope(2, 1, 32, table, q_weight=w, k_weight=w, dtype="f16")
    for got, u in zip(rope.forward(q, k, None, pos), (q, k)):
        u = u.view(m, -1, 32).double()
        u = u / (u.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
        c, s = table[pos.long()].double().view(m, 1, 2, 16).unbind(2)
        ref = torch.cat([u[..., :16] * c - u[..., 16:] * s, u[..., 16:] * c + u[..., :16] * s], -1)
        reach = (u[..., :16].abs() + u[..., 16:].abs()).repeat(1, 1, 2)
        assert ((got.view(m, -1, 32).double() - ref).abs() <= 2.0**-11 * ref.abs() + 2.0**-18 * reach + 2.0**-25).all()


@pytest.mark.parametrize("ty", ["f16", "bf16"])
def test_1024_heads(ty):
    """The most heads that the calls take: one key head for all of them, and as many."""
    import torch
    g, H, D, n = gen(902), 1024, 64, 37
    for KV in (1, 1024):
        kc, vc = normal(g, 3, KV, 16, D, dtype=ty), normal(g, 3, KV, 16, D, dtype=ty)
        q, k, v = normal(g, 2, H * D, dtype=ty), normal(g, 2, KV * D, dtype=ty), normal(g, 2, KV * D, dtype=ty)
        cache = eora.PagedCache(kc, vc)
        rope = eora.QKNormRope(H, KV, D, None, dtype=ty)
        q2, _ = rope.forward(q, k, v, ints([0, 0]), slots=ints([2 * 16 + 4, -1]), cache=cache)
        assert torch.equal(q2, q) and torch.equal(kc[2, :, 4].reshape(-1), k[0]) and torch.equal(vc[2, :, 4].reshape(-1), v[0])
        attn = eora.PagedAttention(H, KV, D, page_size=16, max_batch=2, max_pages=3, dtype=ty)
        out = attn.forward(q, cache, ints([[0, 1, 2], [2, 0, 1]]), ints([n, 17])).view(2, H, D).double()
        for i, (pages, t) in enumerate((([0, 1, 2], n), ([2, 0, 1], 17))):
            kk, vv = (c[pages].transpose(0, 1).reshape(KV, 48, D)[:, :t].double().repeat_interleave(H // KV, 0) for c in (kc, vc))
            s = torch.einsum("hd,htd->ht", q.view(2, H, D)[i].double(), kk) * D**-0.5
            ref = torch.einsum("ht,htd->hd", torch.softmax(s, 1), vv)
            assert ((out[i] - ref).abs() <= torch.finfo(tt(ty)).eps / 2 * ref.abs() + 6 * 2.0**-12).all()
