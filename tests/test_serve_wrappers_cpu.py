"""What the Python objects refuse before anything is launched; needs no GPU."""
import pytest

import paper_2410_21271_b200 as eora
from paper_2410_21271_b200 import build as eora_build

P = 4096            # an aligned address that is never read: every call here is refused first


class Bank:
    def __init__(self):
        self.calls = []

    def forward(self, x, ids, base=None, y=None, stream=None):
        self.calls.append((ids, y))


@pytest.mark.parametrize("n", [0, 1, 2, 4])
def test_fused_layers_take_an_entry_of_adapters_for_each_layer(n, monkeypatch):
    import torch
    launched = []
    monkeypatch.setattr(eora, "eora_linear_forward_fused", lambda *a: launched.append(a))
    layers = object.__new__(eora.FusedLayers)
    layers.cfgs, layers.handle, layers.y_torch_dtype = [eora.eora_linear_config(d_out=d) for d in (64, 32, 32)], None, torch.float16
    x, bank = torch.zeros(2, 128, dtype=torch.float16), Bank()
    with pytest.raises(eora.EoraError) as e:
        layers.forward(x, adapters=[(bank, i) for i in range(n)])
    assert e.value.status == eora.EORA_ERR_BAD_SHAPE and not launched and not bank.calls
    ys = layers.forward(x, adapters=((bank, 7), None, (bank, 9)))
    assert len(launched) == 1 and [c[0] for c in bank.calls] == [7, 9] and bank.calls[0][1] is ys[0] and bank.calls[1][1] is ys[2]
    layers.forward(x)
    assert len(launched) == 2 and len(bank.calls) == 2
    layers.forward(x, adapters=(p for p in [None, (bank, 5), None]))
    assert [c[0] for c in bank.calls] == [7, 9, 5]


def test_calls_by_name_raise_or_return_the_status():
    eora_build.build()
    bank, weights = eora.eora_adapters_config(200, 64, 16, 4, 0, 0), eora.eora_adapters_weights(P, P, None, None)
    rope, attn = eora.eora_qk_config(4, 2, 72, 64, 0, 0, 100, 1e-6, None, None, P), eora.eora_attention_config(8, 2, 80, 0, 16, 10, 4, 0, 0.1)
    cache = eora.eora_kv_cache(P, P, 2 * 16 * 64, 16 * 64, 64, 5, 16, 2, 64, 0)
    calls = [lambda **kw: eora.eora_adapters_forward(bank, weights, P, 256, 3, P, P, 64, P, 64, 0, **kw),
             lambda **kw: eora.eora_qk_norm_rope(rope, P, 288, P, 144, P, 144, P, 3, P, 288, None, 0, P, cache, 0, **kw),
             lambda **kw: eora.eora_attention_forward(attn, P, 640, cache, P, 10, P, 2, P, 640, None, P, 1 << 30, 0, **kw)]
    for call, name in zip(calls, ("eora_adapters_forward", "eora_qk_norm_rope", "eora_attention_forward")):
        assert call(check=False) == eora.EORA_ERR_BAD_SHAPE
        with pytest.raises(eora.EoraError, match=name) as e:
            call()
        assert e.value.status == eora.EORA_ERR_BAD_SHAPE
    assert eora.eora_attention_workspace_bytes(attn) == 0


def test_attention_in_place_needs_one_stride():
    eora_build.build()
    attn = eora.eora_attention_config(8, 2, 64, 0, 16, 10, 4, 0, 0.1)
    cache = eora.eora_kv_cache(P, P, 2 * 16 * 64, 16 * 64, 64, 5, 16, 2, 64, 0)
    need = eora.eora_attention_workspace_bytes(attn)
    call = lambda qs, os: eora.eora_attention_forward(attn, P, qs, cache, P, 10, P, 2, P, os, None, P, need, 0, check=False)
    assert call(520, 512) == call(512, 520) == eora.EORA_ERR_BAD_SHAPE
