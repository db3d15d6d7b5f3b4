"""CPU tests of the limits of the attention passes over packed rows: sizes at
which positions would leave 32 bits are refused before anything is enqueued."""
import ctypes

import pytest

from paper_2606_24033_amd import blockgtq as bg

F = ctypes.c_void_p(256)
TOP = 1 << 30  # rows that one call may attend


def cfg_of(capacity, **kw):
    return bg.Config(**{**dict(n_layers=1, batch=1, n_kv_heads=1, group=4, capacity=capacity, k_budget=64, v_bits=1), **kw})


@pytest.mark.parametrize("n_splits", [0, 1, 3])
@pytest.mark.parametrize("n_q", [1, 333])
def test_cross_rows_of_a_call(n_q, n_splits):
    """A split ends at its first row plus its length, and a wave steps up to 512 rows past its last tile: both below
    2^31 for 2^30 rows, not for 2^31 - 64."""
    big = cfg_of(2 ** 31 - 64)
    assert bg.cross_workspace_bytes(big, 1, n_q, n_splits, TOP) > 0
    cache = bg._Cache(k_codes=256, k_norms=256, v_codes=256, v_norms=256)
    for n in (TOP + 1, 2 ** 31 - 64):
        with pytest.raises(bg.BlockGTQError) as e:
            bg.cross_workspace_bytes(big, 1, n_q, n_splits, n)
        assert e.value.code == -5 and "2^30" in str(e.value)
        assert bg.lib().blockgtq_cross_attn(ctypes.byref(big.c()), F, 0, F, n_q, F, n, ctypes.byref(cache), F, 0, F, 1 << 60,
                                            n_splits, None) == -5


def test_shared_rows_of_a_call():
    big, small = cfg_of(2 ** 31 - 64), cfg_of(64)
    assert bg.shared_workspace_bytes(small, big, 1, 0, TOP, 64) > 0
    assert bg.shared_workspace_bytes(big, small, 1, 0, 64, TOP) > 0
    cache = bg._Cache(k_codes=256, k_norms=256, v_codes=256, v_norms=256)
    for cfg, prefix, n_prefix, n_own in ((small, big, TOP + 64, 64), (big, small, 64, 2 ** 31 - 64)):
        with pytest.raises(bg.BlockGTQError) as e:
            bg.shared_workspace_bytes(cfg, prefix, 1, 0, n_prefix, n_own)
        assert e.value.code == -5
        assert bg.lib().blockgtq_decode_attn_shared(
            ctypes.byref(cfg.c()), F, 0, F, ctypes.byref(prefix.c()), ctypes.byref(cache), F, n_prefix, F, n_own,
            ctypes.byref(cache), F, 0, F, 1 << 60, 0, None) == -5


@pytest.mark.parametrize("k_budget,wide", [(256, False), (512, True)])
def test_wide_key_rows_go_to_the_wide_passes_sooner(k_budget, wide):
    """A tile of a 32-word key row costs the 32-row pass twice what a 16-word one does, and the wide passes the same: 256
    query positions on 4096 rows take 104 us there and 78 us here.  (Their workspace holds the rotated queries, 512 bytes a
    row.)"""
    cfg = cfg_of(4096, n_kv_heads=8, k_budget=k_budget, v_bits=4)
    assert (bg.cross_workspace_bytes(cfg, 1, 256, 0, 4096) >= 256 * 32 * 512) == wide
