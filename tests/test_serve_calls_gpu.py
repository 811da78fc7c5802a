"""The C calls by their Python names, which take pointers and strides as they are, beside the objects that check them: the same bits."""
import pytest

pytestmark = pytest.mark.gpu

import paper_2410_21271_b200 as eora
from test_serve_gpu import DEV, bank_case, filled_cache, gen, ints, normal, table_of


@pytest.mark.parametrize("how", ["current", "object", "handle"])
def test_calls_by_name_are_the_objects_calls(how):
    import torch
    side = torch.cuda.Stream()
    stream = {"current": None, "object": side, "handle": side.cuda_stream}[how]
    g, a, b, rk, sc = bank_case(870, 3, 512, 256, 16, "f16", [16, 5, 9])
    bank = eora.AdapterBank(a, b, ranks=rk, scales=sc)
    x, base, ids = normal(g, 5, 512), normal(g, 5, 256), ints([0, 1, 2, -1, 0])
    y = torch.empty_like(base)
    kc, vc, table, _, _ = filled_cache(g, [30, 9, 1, 17, 0], 2, 64, 16, "hnd", "bf16")
    cache = eora.PagedCache(kc, vc)
    q, k, v = (normal(g, 5, n * 64, dtype="bf16") for n in (4, 2, 2))
    w = normal(g, 64, dtype="bf16")
    rope = eora.QKNormRope(4, 2, 64, table_of(50, 64), q_weight=w, k_weight=w)
    pos, slots = ints([29, 8, 0, 16, 5]), ints([int(table[i, p // 16]) * 16 + p % 16 for i, p in enumerate([29, 8, 0, 16])] + [-1])
    attn = eora.PagedAttention(4, 2, 64, page_size=16, max_batch=5, max_pages=table.shape[1])
    lens = ints([30, 9, 1, 17, 0])
    qo, ko, out, lse, ws = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty(5, 4, device=DEV), torch.zeros_like(attn.workspace)
    torch.cuda.synchronize()
    assert eora.eora_adapters_forward(bank.cfg, bank.weights, x, 512, 5, ids, base, 256, y, 256, stream) == eora.EORA_OK
    assert eora.eora_qk_norm_rope(rope.cfg, q, 256, k, 128, v, 128, pos, 5, qo, 256, ko, 128, slots, cache.struct, stream) == eora.EORA_OK
    assert eora.eora_attention_workspace_bytes(attn.cfg) == ws.numel()
    assert eora.eora_attention_forward(attn.cfg, qo, 256, cache.struct, table, table.shape[1], lens, 5, out, 256, lse, ws, ws.numel(), stream) == eora.EORA_OK
    torch.cuda.synchronize()
    kept = kc.clone(), vc.clone()
    assert torch.equal(bank.forward(x, ids, base=base), y)
    q2, k2 = rope.forward(q, k, v, pos, slots=slots, cache=cache, k_out=torch.empty_like(k))
    assert torch.equal(q2, qo) and torch.equal(k2, ko)
    assert all(torch.equal(c.view(torch.int16), d.view(torch.int16)) for c, d in zip(kept, (kc, vc)))
    lse2 = torch.empty_like(lse)
    assert torch.equal(attn.forward(q2, cache, table, lens, lse=lse2), out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("lengths,H,KV,D", [([7, 0, 300, 64], 4, 2, 64), ([9000, 20], 24, 2, 128), ([(i * 571) % 2900 for i in range(40)], 16, 8, 128), ([700] * 3, 40, 1, 96)])
def test_attention_in_place(lengths, H, KV, D):
    """The queries' buffer takes the result: whole pairs, pairs in several blocks, pairs in several blocks joined in two rounds, groups in two parts."""
    import torch
    g, B = gen(890), len(lengths)
    kc, vc, table, _, _ = filled_cache(g, lengths, KV, D, 64, "hnd", "bf16")
    wide = normal(g, B, H * D + 16, dtype="bf16", std=2.0)
    attn, cache = eora.PagedAttention(H, KV, D, page_size=64, max_batch=B, max_pages=table.shape[1]), eora.PagedCache(kc, vc)
    want = attn.forward(wide[:, 8:8 + H * D], cache, table, ints(lengths))
    for _ in range(5):
        mine = wide.clone()
        q = mine[:, 8:8 + H * D]
        assert attn.forward(q, cache, table, ints(lengths), out=q) is q
        assert torch.equal(q, want) and torch.equal(mine[:, :8], wide[:, :8]) and torch.equal(mine[:, 8 + H * D:], wide[:, 8 + H * D:])
