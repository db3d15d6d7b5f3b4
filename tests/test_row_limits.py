"""CPU tests of the limits of calls over very many rows: refused before anything is enqueued."""
import ctypes

from paper_2606_24033_amd import blockgtq as bg

F = ctypes.c_void_p(256)


def cfg_of(**kw):
    return bg.Config(**{**dict(n_layers=1, batch=1, n_kv_heads=1, group=4, capacity=64, k_budget=64, v_bits=1), **kw})


def test_rows_read_back():
    cache = bg._Cache(k_codes=256, k_norms=256, v_codes=256, v_norms=256)

    def read(layer, n_rows, **kw):
        return bg.lib().blockgtq_dequantize_rows(ctypes.byref(cfg_of(**kw).c()), F, layer, ctypes.byref(cache), n_rows, F, None, F,
                                                 F, 0, None)
    assert read(0, 1, n_kv_heads=1 << 21) == -5
    assert read(-1, 1, n_kv_heads=1 << 12, n_layers=(1 << 9) + 1) == -5
    assert read(0, 64, batch=1 << 29) == read(0, 1 << 20, batch=1 << 16, capacity=1 << 20) == -5
