"""Serving operators, what needs no GPU: struct layouts, refusals before the device is touched, the oracle's own pins."""
import ctypes
import os
import re

import numpy as np
import pytest

import paper_2410_21271_b200 as eora
from oracle import serve_oracle as orc
from paper_2410_21271_b200 import build as eora_build

P = 4096            # an aligned address that is never read: every call here is refused first


@pytest.fixture(scope="module")
def lib():
    eora_build.build()
    return eora.lib()


@pytest.mark.parametrize("name", ["eora_adapters_config", "eora_adapters_weights", "eora_kv_cache", "eora_qk_config", "eora_attention_config"])
def test_structs_match_the_header(name):
    hdr = open(os.path.join(os.path.dirname(eora.HEADER_PATH), "eora_serve.h")).read()
    hdr = re.sub(r"/\*.*?\*/", "", hdr, flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", hdr).group(1)
    want = []
    for decl in body.split(";"):
        found = re.match(r"\s*(?:const )?(int32_t|int64_t|float|void|float|int32_t)\s*(\*?)\s*(.*)", decl.strip(), flags=re.S)
        if found and found.group(3):
            kind = ctypes.c_void_p if found.group(2) else {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float}[found.group(1)]
            want += [(n.strip(), kind) for n in found.group(3).split(",")]
    assert want == list(getattr(eora, name)._fields_)


def adapters_call(lib, cfg=None, w=None, **kw):
    c = eora.eora_adapters_config(256, 64, 16, 4, 0, 0)
    for k, v in (cfg or {}).items():
        setattr(c, k, v)
    wt = eora.eora_adapters_weights(P, P, None, None)
    for k, v in (w or {}).items():
        setattr(wt, k, v)
    a = {**dict(x=P, x_stride=c.d_in, m=3, ids=P, base=P, base_stride=c.d_out, y=P, y_stride=c.d_out), **kw}
    return lib.eora_adapters_forward(ctypes.addressof(c), ctypes.addressof(wt), a["x"], a["x_stride"], a["m"], a["ids"], a["base"], a["base_stride"], a["y"], a["y_stride"], None)


def test_adapters_refusals(lib):
    assert lib.eora_adapters_forward(None, None, P, 256, 1, P, P, 64, P, 64, None) == eora.EORA_ERR_NULL_ARG
    for cfg in (dict(d_in=200), dict(d_in=0), dict(d_out=40), dict(max_rank=0), dict(max_rank=12), dict(max_rank=264), dict(n_adapters=0), dict(n_adapters=4097)):
        assert adapters_call(lib, cfg) == eora.EORA_ERR_BAD_SHAPE, cfg
    for cfg in (dict(x_dtype=2), dict(x_dtype=-1), dict(y_dtype=3)):
        assert adapters_call(lib, cfg) == eora.EORA_ERR_UNSUPPORTED, cfg
    for kw in (dict(m=-1), dict(m=2**20 + 1), dict(x_stride=255), dict(y_stride=32), dict(base_stride=0), dict(base_stride=72)):
        assert adapters_call(lib, **kw) == eora.EORA_ERR_BAD_SHAPE, kw
    for kw in (dict(x=None), dict(ids=None), dict(y=None), dict(w=dict(a=None)), dict(w=dict(b=None))):
        assert adapters_call(lib, **kw) == eora.EORA_ERR_NULL_ARG, kw
    for kw in (dict(x=P + 8), dict(y=P + 2, base=None), dict(base=P + 4), dict(ids=P + 2), dict(x_stride=260), dict(y_stride=68, base=None), dict(w=dict(a=P + 8)),
               dict(w=dict(ranks=P + 1)), dict(w=dict(scales=P + 2))):
        assert adapters_call(lib, **kw) == eora.EORA_ERR_MISALIGNED, kw
    assert adapters_call(lib, m=0) == eora.EORA_OK


def cache_struct(**kw):
    c = eora.eora_kv_cache(P, P, 2 * 16 * 64, 16 * 64, 64, 5, 16, 2, 64, 0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rope_call(lib, cfg=None, cache=(), **kw):
    c = eora.eora_qk_config(4, 2, 64, 64, 0, 0, 100, 1e-6, None, None, P)
    for k, v in (cfg or {}).items():
        setattr(c, k, v)
    a = {**dict(q=P, qs=256, k=P, ks=128, v=P, vs=128, pos=P, m=3, qo=P, qos=256, ko=None, kos=0, slots=P), **kw}
    cs = cache_struct(**dict(cache)) if cache is not None else None
    return lib.eora_qk_norm_rope(ctypes.addressof(c), a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["pos"], a["m"], a["qo"], a["qos"], a["ko"], a["kos"],
                                 a["slots"], ctypes.addressof(cs) if cs is not None else None, None)


def test_norm_and_rotation_refusals(lib):
    assert lib.eora_qk_norm_rope(None, *([None, 0] * 3), None, 1, None, 0, None, 0, None, None, None) == eora.EORA_ERR_NULL_ARG
    for cfg in (dict(head_dim=72), dict(head_dim=272), dict(head_dim=0), dict(rot_dim=80), dict(rot_dim=24), dict(rot_dim=-16), dict(n_heads=0), dict(n_heads=5),
                dict(n_kv_heads=0), dict(n_positions=0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(n_heads=2048)):
        assert rope_call(lib, cfg) == eora.EORA_ERR_BAD_SHAPE, cfg
    for cfg in (dict(dtype=2), dict(pairs=2)):
        assert rope_call(lib, cfg) == eora.EORA_ERR_UNSUPPORTED, cfg
    for kw in (dict(q=None), dict(k=None), dict(qo=None), dict(pos=None), dict(slots=None), dict(v=None), dict(cfg=dict(cos_sin=None)), dict(cache=None)):
        assert rope_call(lib, **kw) == eora.EORA_ERR_NULL_ARG, kw
    for kw in (dict(m=-1), dict(qs=248), dict(ks=120), dict(vs=0), dict(qos=128), dict(ko=P, kos=64), dict(qos=264), dict(ko=P, kos=136)):
        assert rope_call(lib, **kw) == eora.EORA_ERR_BAD_SHAPE, kw
    for cache in (dict(n_kv_heads=1), dict(head_dim=32), dict(page_size=12), dict(page_size=0), dict(n_pages=0), dict(n_pages=2**28), dict(token_stride=32), dict(head_stride=-64),
                  dict(head_stride=0), dict(page_stride=0)):
        assert rope_call(lib, cache=cache) == eora.EORA_ERR_BAD_SHAPE, cache
    assert rope_call(lib, cache=dict(dtype=1)) == eora.EORA_ERR_UNSUPPORTED
    assert rope_call(lib, cache=dict(k=None)) == eora.EORA_ERR_NULL_ARG
    for kw in (dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(qo=P + 8), dict(ko=P + 8, kos=128), dict(pos=P + 2), dict(qs=260), dict(cfg=dict(cos_sin=P + 4)),
               dict(cfg=dict(q_weight=P + 2)), dict(cache=dict(v=P + 8)), dict(cache=dict(token_stride=68))):
        assert rope_call(lib, **kw) == eora.EORA_ERR_MISALIGNED, kw
    assert rope_call(lib, m=0) == eora.EORA_OK


def attention_call(lib, cfg=None, cache=(), **kw):
    c = eora.eora_attention_config(8, 2, 64, 0, 16, 10, 4, 0, 0.1)
    for k, v in (cfg or {}).items():
        setattr(c, k, v)
    need = lib.eora_attention_workspace_bytes(ctypes.addressof(c))
    a = {**dict(q=P, qs=512, t=P, ts=10, n=P, b=2, o=P, os=512, lse=None, ws=P, wsb=need), **kw}
    cs = cache_struct(**dict(cache)) if cache is not None else None
    return lib.eora_attention_forward(ctypes.addressof(c), a["q"], a["qs"], ctypes.addressof(cs) if cs is not None else None, a["t"], a["ts"], a["n"], a["b"], a["o"], a["os"],
                                      a["lse"], a["ws"], a["wsb"], None)


def test_attention_refusals(lib):
    for cfg in (dict(head_dim=80), dict(head_dim=0), dict(n_heads=7), dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=2048), dict(page_size=24), dict(page_size=0), dict(max_pages=0),
                dict(max_pages=2**28), dict(max_pages=2**26 + 1), dict(max_batch=0), dict(max_batch=65537), dict(window=-1), dict(scale=0.0), dict(scale=float("inf")), dict(scale=float("nan"))):
        assert attention_call(lib, cfg) == eora.EORA_ERR_BAD_SHAPE, cfg
        c = eora.eora_attention_config(8, 2, 64, 0, 16, 10, 4, 0, 0.1)
        for k, v in cfg.items():
            setattr(c, k, v)
        assert eora.eora_attention_workspace_bytes(c) == 0, cfg
    assert attention_call(lib, dict(dtype=2)) == eora.EORA_ERR_UNSUPPORTED
    assert attention_call(lib, b=0) == eora.EORA_OK
    assert attention_call(lib, b=5) == eora.EORA_ERR_M_TOO_LARGE and attention_call(lib, b=-1) == eora.EORA_ERR_BAD_SHAPE
    for kw in (dict(qs=504), dict(os=256), dict(ts=9), dict(wsb=100), dict(cache=dict(n_kv_heads=1)), dict(cache=dict(page_size=32)), dict(cache=dict(head_dim=32)), dict(cfg=dict(n_kv_heads=4)),
               dict(cfg=dict(head_dim=128), qs=1024, os=1024)):
        assert attention_call(lib, **kw) == eora.EORA_ERR_BAD_SHAPE, kw
    for kw in (dict(qs=516), dict(q=P + 2), dict(o=P + 8), dict(n=P + 1), dict(t=P + 2), dict(lse=P + 2), dict(ws=P + 8), dict(cache=dict(k=P + 2))):
        assert attention_call(lib, **kw) == eora.EORA_ERR_MISALIGNED, kw
    for kw in (dict(q=None), dict(cache=None), dict(t=None), dict(n=None), dict(o=None), dict(ws=None), dict(cache=dict(v=None))):
        assert attention_call(lib, **kw) == eora.EORA_ERR_NULL_ARG, kw
    assert attention_call(lib, cache=dict(dtype=1)) == eora.EORA_ERR_UNSUPPORTED
    assert lib.eora_attention_workspace_bytes(None) == 0
    assert lib.eora_attention_forward(None, P, 512, None, P, 10, P, 1, P, 512, None, P, 0, None) == eora.EORA_ERR_NULL_ARG


def test_wrappers_refuse_host_tensors():
    import torch
    with pytest.raises(eora.EoraError):
        eora.AdapterBank(torch.zeros(2, 128, 8, dtype=torch.float16), torch.zeros(2, 8, 32, dtype=torch.float16))
    with pytest.raises(eora.EoraError):
        eora.PagedCache(torch.zeros(2, 2, 16, 64, dtype=torch.float16), torch.zeros(2, 2, 16, 64, dtype=torch.float16))
    with pytest.raises(eora.EoraError):
        eora.QKNormRope(4, 2, 64, torch.zeros(8, 64), dtype="f16")
    with pytest.raises(eora.EoraError):
        eora.QKNormRope(4, 2, 64, None, dtype="f32")
    rope = eora.QKNormRope(4, 2, 64, None, dtype="f16")
    q, k, pos = torch.zeros(3, 256, dtype=torch.float16), torch.zeros(3, 128, dtype=torch.float16), torch.zeros(3, dtype=torch.int32)
    for bad in ((q, k, None, pos), (None, k, None, pos), (q, 3, None, pos), (q.float(), k, None, pos)):
        with pytest.raises(eora.EoraError):
            rope.forward(*bad)


# ---- the oracle against facts that hold whatever its code does
def test_oracle_adapters_by_hand():
    x, a, b = np.array([[1.0, 2.0]]), np.array([[[3.0], [4.0]]]), np.array([[[5.0, -1.0]]])
    y, off = orc.adapters(x, a, b, [0], scales=[2.0], base=np.array([[1.0, 1.0]]))
    assert np.array_equal(y, [[1 + 2 * 11 * 5, 1 - 2 * 11]]) and (off > 0).all()
    assert np.array_equal(orc.adapters(x, a, b, [1], base=np.array([[1.0, 1.0]]))[0], [[1.0, 1.0]])
    assert np.array_equal(orc.adapters(x, a, b, [0], ranks=[0])[0], [[0.0, 0.0]])


@pytest.mark.parametrize("pairs", ["half", "adjacent"])
def test_oracle_rotation_keeps_lengths_and_relative_angles(pairs):
    rng = np.random.default_rng(5)
    ang = np.arange(50)[:, None] * 100.0 ** -(np.arange(8) / 8)
    table = np.concatenate([np.cos(ang), np.sin(ang)], 1)
    q, k = rng.normal(size=(1, 24)), rng.normal(size=(1, 24))
    turn = lambda x, p: orc.qk_norm_rope(x, None, table, np.array([p]), 1, 16, pairs, 0.0)[0][0]
    assert np.isclose(np.linalg.norm(turn(q, 17)), np.linalg.norm(q))
    assert np.isclose(turn(q, 30) @ turn(k, 20), turn(q, 10) @ turn(k, 0)) and np.array_equal(turn(q, 9)[16:], q[0, 16:])
    y = orc.qk_norm_rope(3 * q, np.ones(24), table, np.array([0]), 1, 0, pairs, 0.0)[0]
    assert np.isclose((y * y).mean(), 1.0)


def test_oracle_attention_limits():
    rng = np.random.default_rng(6)
    q, k, v = rng.normal(size=(3, 8)), rng.normal(size=(7, 8)), rng.normal(size=(7, 8))
    assert np.allclose(orc.attention(0 * q, k, v, 1.0)[0], v.mean(0)) and np.allclose(orc.attention(0 * q, k, v, 1.0)[1], np.log(7))
    assert np.allclose(orc.attention(q, k[:1], v[:1], 1.0)[0], v[0])
    out, lse = orc.attention(q, k[:0], v[:0], 1.0)[:2]
    assert not out.any() and np.isneginf(lse).all()
    # joined from two parts by their log sums
    o1, l1 = orc.attention(q, k[:3], v[:3], 0.5)[:2]
    o2, l2 = orc.attention(q, k[3:], v[3:], 0.5)[:2]
    o, l = orc.attention(q, k, v, 0.5)[:2]
    w = np.exp(l1 - l)[:, None]
    assert np.allclose(w * o1 + (1 - w) * o2, o) and np.allclose(np.logaddexp(l1, l2), l)
