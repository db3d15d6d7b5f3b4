"""CPU tests of a serving step over pages: sizes, and every refusal, before
anything is enqueued (the pointers are never dereferenced)."""
import ctypes

import numpy as np
import pytest

from paper_2606_24033_amd import blockgtq as bg

torch = pytest.importorskip("torch")
F = ctypes.c_void_p(256)
ODD = ctypes.c_void_p(264)
BIG = 1 << 40


def cfg_of(**kw):
    c = dict(n_layers=2, batch=30, n_kv_heads=2, group=4, capacity=128, k_budget=128, v_bits=2)
    c.update(kw)
    return bg.Config(**c)


def cache_at(**kw):
    p = dict(k_codes=256, k_norms=256, v_codes=256, v_norms=256)
    p.update(kw)
    return bg._Cache(**p)


def chunk_at(**kw):
    p = dict(cu_new=256, ctx_len=256, pages=256, n_seqs=3, n_tokens=100, max_pages=8, max_new=50, max_ctx=1000)
    p.update(kw)
    return bg._Chunk(**p)


def err(rc, text=None):
    if text is not None:
        assert text in bg.lib().blockgtq_last_error().decode(), bg.lib().blockgtq_last_error()
    return rc


THETA = [10000.0 ** (-2 * i / 128) for i in range(64)]


def test_norm_rope_refusals():
    L = bg.lib()

    def call(c=None, rope=None, n=5, q=F, qs=1024, k=F, ks=256, pos=F, qw=F, kw=F, eps=1e-6, qo=F, qos=1024, ko=F, kos=256, t=1):
        r = rope or bg.Rope(THETA)
        return L.blockgtq_norm_rope(ctypes.byref((c or cfg_of()).c()), ctypes.byref(r.c()), n, q, qs, k, ks, pos, qw, kw, eps,
                                    qo, qos, ko, kos, t, None)
    assert L.blockgtq_norm_rope(None, ctypes.byref(bg.Rope(THETA).c()), 0, F, 1024, F, 256, F, F, F, 0.0, F, 1024, F, 256, 1, None) == -1
    assert L.blockgtq_norm_rope(ctypes.byref(cfg_of().c()), None, 0, F, 1024, F, 256, F, F, F, 0.0, F, 1024, F, 256, 1, None) == -1
    assert call(n=-1) == -1
    assert call(n=0) == 0
    assert err(call(t=2), "out_dtype") == -1
    for axes in (0, 5):
        assert err(call(rope=bg.Rope(THETA, n_axes=axes)), "n_axes") == -1
    assert err(call(rope=bg.Rope(THETA, axis=[0] * 63 + [2], n_axes=2)), "axis 2 of 2") == -1
    assert err(call(rope=bg.Rope([float("nan")] + THETA[1:])), "finite") == -1
    for eps in (-1e-6, float("nan"), float("inf")):
        assert err(call(eps=eps), "eps") == -1
    assert call(pos=None) == -1
    assert call(q=None, k=None, qo=None, ko=None) == -1
    assert err(call(q=None), "without") == err(call(ko=None), "without") == -1
    assert err(call(qs=1016), "below") == err(call(kos=255), "below") == -1
    assert err(call(q=ODD), "aligned") == err(call(ko=ODD), "aligned") == err(call(qw=ODD), "aligned") == -1
    assert err(call(qs=1028), "aligned") == -1
    assert err(call(c=cfg_of(in_dtype=bg.BGTQ_FP32), qs=1030), "aligned") == -1
    assert err(call(n=1 << 30), "tokens") == -5
    assert call(c=cfg_of(group=9)) == -5


def test_rope_checks():
    with pytest.raises(ValueError):
        bg.Rope(THETA[:63])
    with pytest.raises(ValueError):
        bg.Rope(THETA, axis=[0] * 65)
    assert bg.Rope(THETA, axis=[0] * 32 + [2] * 32).n_axes == 3


def test_chunk_refusals():
    L = bg.lib()

    def append(c=None, layer=0, k=F, ks=256, v=F, vs=256, chunk=None, cache=None, layout=F):
        return L.blockgtq_paged_append(ctypes.byref((c or cfg_of()).c()), layout, layer, k, ks, v, vs,
                                       ctypes.byref(chunk or chunk_at()), ctypes.byref(cache or cache_at()), None)

    def attn(c=None, layer=0, q=F, chunk=None, scores=None, cache=None, out=F, t=1, ws=F, n=BIG, splits=0, layout=F):
        return L.blockgtq_paged_attn(ctypes.byref((c or cfg_of()).c()), layout, layer, q, ctypes.byref(chunk or chunk_at()),
                                     None if scores is None else ctypes.byref(scores), ctypes.byref(cache or cache_at()), out,
                                     t, ws, n, splits, None)
    for call in (append, attn):
        for bad in (dict(n_seqs=-1), dict(n_seqs=65536), dict(n_tokens=-1), dict(max_new=-1), dict(max_new=101),
                    dict(max_ctx=49), dict(max_pages=7), dict(max_pages=-1), dict(cu_new=0), dict(ctx_len=0), dict(pages=0)):
            assert call(chunk=chunk_at(**bad)) == -1, bad
        assert err(call(chunk=chunk_at(max_ctx=(1 << 30) + 1, max_pages=1 << 24)), "2^30") == -5
        assert err(call(chunk=chunk_at(n_tokens=(1 << 21) + 1)), "2^24") == -5
        for layer in (-1, 2):
            assert err(call(layer=layer), "layer") == -1
        assert call(layout=None) == -1
        assert call(cache=cache_at(k_norms=0)) == -1
        assert err(call(cache=cache_at(v_codes=264)), "aligned") == -1
        assert call(c=cfg_of(group=9)) == -5
        # nothing to do, nothing launched
        assert call(chunk=chunk_at(n_seqs=0)) == 0
        assert call(chunk=chunk_at(max_new=0, n_tokens=0)) == 0
    assert append(k=None) == append(v=None) == -1
    assert err(append(ks=255), "below") == err(append(vs=260), "aligned") == err(append(v=ODD), "aligned") == -1
    assert attn(q=None) == attn(out=None) == attn(ws=None) == -1
    assert err(attn(q=ODD), "aligned") == err(attn(out=ODD), "aligned") == err(attn(ws=ODD), "aligned") == -1
    assert err(attn(t=7), "out_dtype") == -1
    assert err(attn(splits=-1), "n_splits") == err(attn(splits=4097), "n_splits") == -1
    for cap in (-1.0, float("nan"), float("inf")):
        assert err(attn(scores=bg._Scores(cap, None, None)), "cap") == -1
    need = ctypes.c_size_t()
    for sizes in ((3, 100, 50, 1000), (3, 100, 1, 1000), (1, 100, 100, 100), (64, 2000, 1900, 100000)):
        assert L.blockgtq_paged_workspace_bytes(ctypes.byref(cfg_of().c()), *sizes, 0, ctypes.byref(need)) == 0
        c = chunk_at(n_seqs=sizes[0], n_tokens=sizes[1], max_new=sizes[2], max_ctx=sizes[3], max_pages=1000)
        assert err(attn(chunk=c, n=need.value - 1), "workspace") == -4


def test_workspace_sizes():
    cfg = cfg_of()
    z = torch.zeros

    def ws(n_seqs, n_tokens, max_new, max_ctx, splits=0):
        c = bg.Chunk(z(n_seqs + 1, dtype=torch.int32), z(n_seqs, dtype=torch.int32), z((n_seqs, 1), dtype=torch.int32), max_new, max_ctx)
        return bg.paged_workspace_bytes(cfg, c, n_tokens, splits)
    assert ws(0, 0, 0, 0) == 0
    assert ws(5, 0, 0, 100) == 0
    # partials of 132 floats for each split of the 4-row units, where there is more than one
    assert ws(5, 5, 1, 100, 1) == 256
    assert ws(5, 5, 1, 1000, 3) >= 5 * 2 * 4 * 3 * 132 * 4
    # the rotated query rows of a long chunk (a short one on a short context is taken 32 rows at a time)
    assert ws(1, 20000, 20000, 20000) >= 20000 * 8 * 128 * 4
    for bad in [(1, 5, 1, 100, 5000), (1, 5, 6, 100), (1, 5, 1, 0), (-1 % 70000, 5, 1, 10)]:
        with pytest.raises(bg.BlockGTQError):
            ws(*bad)


def test_too_many_splits_are_refused():
    L = bg.lib()
    cfg = cfg_of(n_kv_heads=256, group=1)
    c = chunk_at(n_seqs=65535, n_tokens=65535, max_new=1, max_ctx=1 << 20, max_pages=1 << 13)
    assert err(L.blockgtq_paged_attn(ctypes.byref(cfg.c()), F, 0, F, ctypes.byref(c), None, ctypes.byref(cache_at()), F, 1, F,
                                     1 << 62, 4096, None), "too many") == -5


def test_binding_checks():
    cfg = cfg_of()
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    for bad in ((i32(4), i32(4), i32(4, 2)), (i32(5), i32(4), i32(3, 2)), (i32(5), i32(4), i32(4)),
                (i32(5), i32(4).long(), i32(4, 2))):
        with pytest.raises(ValueError):
            bg.Chunk(*bad, 1, 10)
    q, k = torch.zeros((5, 8, 128), dtype=torch.bfloat16), torch.zeros((5, 2, 128), dtype=torch.bfloat16)
    rope = bg.Rope(THETA)
    for kw in (dict(q=None, k=None), dict(q=q.float(), k=k), dict(q=q, k=k[:4]), dict(q=q, k=k, pos=i32(5)),
               dict(q=q, k=k, pos=i32(5, 2)), dict(q=q, k=k, q_weight=torch.zeros(64)), dict(q=None, k=k, q_out=q),
               dict(q=q, k=k, q_out=q, k_out=k.float()), dict(q=q, k=k, q_out=q, out_dtype=torch.float32),
               dict(q=q, k=k, out_dtype=torch.float16), dict(q=q.transpose(0, 1).contiguous().transpose(0, 1), k=k)):
        with pytest.raises(ValueError):
            bg.blockgtq_norm_rope(cfg, rope, **{"pos": i32(5, 1), **kw})
    # rows on the CPU are refused, and views of wider rows give their stride
    with pytest.raises(ValueError):
        bg.blockgtq_norm_rope(cfg, rope, q, k, i32(5, 1))
    wide = torch.zeros((5, 12, 128), dtype=torch.bfloat16)
    assert bg._token_rows("q", wide[:, :8], 5, 8, torch.bfloat16) == 12 * 128
    assert bg._token_rows("q", wide[:1, :8], 1, 8, torch.bfloat16) == 8 * 128
