"""What the Python objects refuse before anything is launched; needs no GPU."""
import pytest

import paper_2410_21271_b200 as eora


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
