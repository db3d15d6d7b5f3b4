"""CPU tests of the operators that read the packed cache beside the decode:
sizes, and every refusal, before anything is enqueued (the pointers are never
dereferenced)."""
import ctypes

import numpy as np
import pytest

from paper_2606_24033_amd import blockgtq as bg

torch = pytest.importorskip("torch")
F = ctypes.c_void_p(256)
BIG = 1 << 40


def cfg_of(**kw):
    c = dict(n_layers=2, batch=3, n_kv_heads=2, group=4, capacity=1024, k_budget=128, v_bits=2)
    c.update(kw)
    return bg.Config(**c)


def cache_at(**kw):
    p = dict(k_codes=256, k_norms=256, v_codes=256, v_norms=256)
    p.update(kw)
    return bg._Cache(**p)


def err(rc, text=None):
    if text is not None:
        assert text in bg.lib().blockgtq_last_error().decode(), bg.lib().blockgtq_last_error()
    return rc


def test_dequantize_rows_refusals():
    L, cfg = bg.lib(), cfg_of()

    def call(c=None, layer=0, cache=None, n=10, pos=F, ctx=None, k=F, v=F, t=0, layout=F):
        return L.blockgtq_dequantize_rows(ctypes.byref((c or cfg).c()), layout, layer, ctypes.byref(cache or cache_at()), n,
                                          pos, ctx, k, v, t, None)
    assert L.blockgtq_dequantize_rows(None, F, 0, ctypes.byref(cache_at()), 1, F, None, F, F, 0, None) == -1
    assert L.blockgtq_dequantize_rows(ctypes.byref(cfg.c()), F, 0, None, 1, F, None, F, F, 0, None) == -1
    assert call(layer=2) == call(layer=-2) == -1
    assert call(n=-1) == -1
    assert err(call(n=1025), "capacity") == -3
    assert call(pos=None) == call(layout=None) == -1
    assert err(call(k=None, v=None), "both NULL") == -1
    assert err(call(t=2), "out_dtype") == call(t=-1) == -1
    assert err(call(k=ctypes.c_void_p(264)), "aligned") == -1
    assert err(call(v=ctypes.c_void_p(260)), "aligned") == -1
    assert err(call(cache=cache_at(v_norms=264)), "aligned") == -1
    assert call(cache=cache_at(k_codes=0)) == -1
    assert call(c=cfg_of(group=9)) == -5
    assert call(c=cfg_of(n_layers=1 << 20), layer=-1) == -5
    assert call(n=0) == 0  # nothing to read, nothing launched


def test_cross_sizes_and_refusals():
    L, cfg = bg.lib(), cfg_of()
    assert bg.cross_workspace_bytes(cfg, 1, 0, 0, 100) == 0
    assert bg.cross_workspace_bytes(cfg, 2, 5, 0, 1024) > 0
    for bad in [(3, 5, 0, 100), (1, -1, 0, 100), (1, 5, -1, 100), (1, 5, 5000, 100)]:
        with pytest.raises(bg.BlockGTQError) as e:
            bg.cross_workspace_bytes(cfg, *bad)
        assert e.value.code == -1, bad
    for ctx in (-1, 1025):
        with pytest.raises(bg.BlockGTQError) as e:
            bg.cross_workspace_bytes(cfg, 1, 5, 0, ctx)
        assert e.value.code == -3
    with pytest.raises(bg.BlockGTQError) as e:
        bg.cross_workspace_bytes(cfg, 2, 1 << 20, 0, 100)
    assert e.value.code == -5

    def call(c=None, layer=0, q=F, n_q=10, ctx=F, max_ctx=100, cache=None, out=F, t=1, ws=F, n=BIG, splits=0, layout=F):
        return L.blockgtq_cross_attn(ctypes.byref((c or cfg).c()), layout, layer, q, n_q, ctx, max_ctx,
                                     ctypes.byref(cache or cache_at()), out, t, ws, n, splits, None)
    assert L.blockgtq_cross_attn(ctypes.byref(cfg.c()), F, 0, F, 1, F, 10, None, F, 0, F, BIG, 0, None) == -1
    assert call(layer=2) == call(layer=-2) == -1
    assert call(n_q=-1) == -1
    assert call(max_ctx=1025) == call(max_ctx=-1) == -3
    assert call(splits=4097) == call(splits=-1) == -1
    assert call(t=2) == -1
    assert call(q=None) == call(ctx=None) == call(out=None) == call(ws=None) == call(layout=None) == -1
    for name in ("q", "out", "ws"):
        assert err(call(**{name: ctypes.c_void_p(264)}), "aligned") == -1
    assert err(call(cache=cache_at(k_norms=8)), "aligned") == -1
    need = bg.cross_workspace_bytes(cfg, 1, 10, 0, 100)
    assert need == 0 or err(call(n=need - 1), "workspace") == -4
    assert call(n_q=1 << 22) == -5
    assert call(c=cfg_of(head_dim=64)) == -5
    assert call(n_q=0) == 0


def test_shared_sizes_and_refusals():
    L, cfg, one = bg.lib(), cfg_of(), cfg_of(batch=1, capacity=4096)
    assert bg.shared_workspace_bytes(cfg, one, 2, 0, 4096, 1024) > 0
    for kw in (dict(batch=2), dict(n_layers=1), dict(n_kv_heads=1), dict(group=2), dict(k_budget=192), dict(v_bits=3),
               dict(in_dtype=bg.BGTQ_FP32)):
        with pytest.raises(bg.BlockGTQError) as e:
            bg.shared_workspace_bytes(cfg, cfg_of(**{**dict(batch=1), **kw}), 1, 0, 100, 100)
        assert e.value.code == -1, kw
    for a in ((4097, 100), (100, 1025), (-1, 100), (100, -1)):
        with pytest.raises(bg.BlockGTQError) as e:
            bg.shared_workspace_bytes(cfg, one, 1, 0, *a)
        assert e.value.code == -3, a

    def call(p=None, layer=0, q=F, prefix=None, plen=F, max_prefix=100, ctx=F, max_ctx=100, cache=None, out=F, t=0, ws=F,
             n=BIG, splits=0, layout=F):
        return L.blockgtq_decode_attn_shared(ctypes.byref(cfg.c()), layout, layer, q, ctypes.byref((p or one).c()),
                                             ctypes.byref(prefix or cache_at()), plen, max_prefix, ctx, max_ctx,
                                             ctypes.byref(cache or cache_at()), out, t, ws, n, splits, None)
    assert err(call(p=cfg), "prefix") == -1
    assert L.blockgtq_decode_attn_shared(ctypes.byref(cfg.c()), F, 0, F, None, ctypes.byref(cache_at()), F, 1, F, 1,
                                         ctypes.byref(cache_at()), F, 0, F, BIG, 0, None) == -1
    assert call(layer=2) == call(layer=-2) == -1
    assert call(max_prefix=4097) == call(max_ctx=1025) == -3
    assert call(splits=4097) == call(t=3) == -1
    for name in ("q", "plen", "ctx", "out", "ws", "layout"):
        assert call(**{name: None}) == -1, name
    for name in ("q", "out", "ws"):
        assert err(call(**{name: ctypes.c_void_p(8)}), "aligned") == -1
    assert err(call(prefix=cache_at(v_codes=24)), "aligned") == -1
    assert err(call(cache=cache_at(v_codes=24)), "aligned") == -1
    need = bg.shared_workspace_bytes(cfg, one, 1, 0, 100, 100)
    assert err(call(n=need - 1), "workspace") == -4


def test_binding_refuses_wrong_tensors():
    """Shapes, types, layout and devices, before the library is called (CPU tensors: never a GPU call)."""
    cfg = cfg_of(n_layers=1)
    one = cfg_of(n_layers=1, batch=1, capacity=64)
    cache, prefix = bg.Cache(cfg, device="cpu"), bg.Cache(one, device="cpu")

    class L:
        blob, k_bits, k_budget = torch.zeros(8, dtype=torch.uint8), np.zeros((2, 16), dtype=np.uint8), cfg.k_budget

    class Other(L):
        k_bits = np.zeros((4, 16), dtype=np.uint8)

    class Wide(L):
        k_budget = 2 * cfg.k_budget
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32)  # noqa: E731
    ctx, ws = i32(1, 2, 3), torch.zeros(1 << 20, dtype=torch.uint8)
    q = torch.zeros((3, 5, 8, 128), dtype=torch.bfloat16)

    def cross(q=q, ctx=ctx, cache=cache, **kw):
        return bg.blockgtq_cross_attn(cfg, L, 0, q, ctx, 100, cache, workspace=ws, **kw)
    with pytest.raises(ValueError, match="CUDA"):
        cross()
    for bad in (dict(q=q.float()), dict(q=q[:2]), dict(q=q[:, :, :4]), dict(q=q[:, 0]), dict(ctx=ctx.long()), dict(ctx=ctx[:2]),
                dict(out=torch.zeros((3, 5, 8, 64))), dict(out=torch.zeros((3, 5, 8, 128), dtype=torch.float16)),
                dict(out=torch.zeros((3, 5, 8, 128)), out_dtype=torch.bfloat16), dict(out_dtype=torch.float16),
                dict(cache=prefix)):
        with pytest.raises(ValueError):
            cross(**bad)

    def shared(q=q[:, 0].contiguous(), prefix=prefix, plen=i32(4), ctx=ctx, cache=cache, **kw):
        return bg.blockgtq_decode_attn_shared(cfg, L, 0, q, one, prefix, plen, 64, ctx, 100, cache, workspace=ws, **kw)
    with pytest.raises(ValueError, match="CUDA"):
        shared()
    for bad in (dict(q=q), dict(prefix=cache), dict(cache=prefix), dict(plen=i32(4, 5)), dict(plen=i32(4).long()),
                dict(ctx=ctx[:1]), dict(out_dtype=torch.float64)):
        with pytest.raises(ValueError):
            shared(**bad)

    for layout in (Other, Wide):
        with pytest.raises(ValueError, match="layout"):
            bg.blockgtq_dequantize_rows(cfg, layout, 0, cache, ctx, 7)
        with pytest.raises(ValueError, match="layout"):
            bg.blockgtq_cross_attn(cfg, layout, 0, q, ctx, 100, cache, workspace=ws)
        with pytest.raises(ValueError, match="layout"):
            bg.blockgtq_decode_attn_shared(cfg, layout, 0, q[:, 0].contiguous(), one, prefix, i32(4), 64, ctx, 100, cache,
                                           workspace=ws)

    def rows(pos=ctx, n=7, cache=cache, **kw):
        return bg.blockgtq_dequantize_rows(cfg, L, 0, cache, pos, n, **kw)
    with pytest.raises(ValueError, match="CUDA"):
        rows()
    shape = (3, 7, 2, 128)
    for bad in (dict(pos=ctx.long()), dict(pos=ctx[:2]), dict(ctx_len=ctx[:2]), dict(k_out=torch.zeros((3, 8, 2, 128))),
                dict(k_out=torch.zeros(shape), v_out=torch.zeros(shape, dtype=torch.bfloat16)),
                dict(k_out=torch.zeros(shape, dtype=torch.float16)), dict(k_out=torch.zeros(shape), out_dtype=torch.bfloat16),
                dict(cache=prefix)):
        with pytest.raises(ValueError):
            rows(**bad)
