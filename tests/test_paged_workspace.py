"""CPU tests of what the attention over pages asks for: its workspace from above, and that the heuristic's own plan is
never refused where one split would serve (nothing is launched: the workspaces handed over are a byte too small)."""
import ctypes
import random

import pytest

from paper_2606_24033_amd import blockgtq as bg

F = ctypes.c_void_p(256)
MIB = 1 << 20


def needed(cfg, n_seqs, n_tokens, max_new, max_ctx, splits=0):
    n = ctypes.c_size_t()
    assert bg.lib().blockgtq_paged_workspace_bytes(ctypes.byref(cfg.c()), n_seqs, n_tokens, max_new, max_ctx, splits, ctypes.byref(n)) == 0
    return n.value


def refused(cfg, n_seqs, n_tokens, max_new, max_ctx, splits=0):
    """The error of a call whose workspace is a byte too small."""
    need = needed(cfg, n_seqs, n_tokens, max_new, max_ctx, splits)
    cache = bg._Cache(k_codes=256, k_norms=256, v_codes=256, v_norms=256)
    chunk = bg._Chunk(256, 256, 256, n_seqs, n_tokens, (max_ctx + cfg.capacity - 1) // cfg.capacity, max_new, max_ctx)
    assert need > 0
    return bg.lib().blockgtq_paged_attn(ctypes.byref(cfg.c()), F, 0, F, ctypes.byref(chunk), None, ctypes.byref(cache), F, 1, F,
                                        need - 1, splits, None)


def cfg_of(kv, group, **kw):
    return bg.Config(**{**dict(n_layers=1, batch=64, n_kv_heads=kv, group=group, capacity=256, k_budget=128, v_bits=2), **kw})


@pytest.mark.parametrize("kv,group,n_seqs,n_tokens,max_new,max_ctx,most", [
    (8, 4, 16, 315, 300, 4097, 60 * MIB),          # 15 generated tokens beside a chunk
    (8, 4, 257, 2304, 2048, 131072, 140 * MIB),    # 256 beside a long one on a long context: partials and rotated queries
    (8, 4, 513, 1024, 512, 131072, 145 * MIB),     # 512 beside one
    (32, 1, 65, 576, 512, 32768, 140 * MIB),
    (8, 4, 1, 1, 1, 131072, 8 * MIB),              # one token of one sequence
])
def test_workspace_of_serving_batches(kv, group, n_seqs, n_tokens, max_new, max_ctx, most):
    assert needed(cfg_of(kv, group), n_seqs, n_tokens, max_new, max_ctx) <= most


def draws(n):
    rng = random.Random(7)
    while n:
        kv, group = rng.choice([1, 2, 4, 8, 16, 32, 64]), rng.randint(1, 8)
        n_seqs = min(65535, int(2 ** rng.uniform(0, 16)))
        n_tokens = max(1, int(n_seqs * 2 ** rng.uniform(-1, 4)))
        if n_tokens * kv * group > 1 << 24:
            continue
        max_new = rng.choice([1, 2, min(n_tokens, 8), int(n_tokens ** rng.random()), n_tokens])
        max_new = max(1, min(max_new, n_tokens))
        max_ctx = max(max_new, int(2 ** rng.uniform(0, 20)))
        yield cfg_of(kv, group, k_budget=rng.choice([64, 128, 192, 512])), n_seqs, n_tokens, max_new, max_ctx
        n -= 1


def test_workspace_from_above():
    """Two passes' partials of 64 MiB each and the query rows, whatever the batch."""
    for cfg, *sizes in draws(4000):
        rows = sizes[1] * cfg.n_q_heads
        assert needed(cfg, *sizes) <= 2 * 64 * MIB + 512 * rows + 1024, (cfg, sizes)


def test_no_batch_is_refused_for_the_splits_that_it_did_not_ask_for():
    served = 0
    for cfg, *sizes in list(draws(4000)) + [(cfg_of(32, 1), 3021, 4475, 1455, 34321)]:
        one = refused(cfg, *sizes, 1)
        assert one in (-4, -5)
        if one == -4:
            assert refused(cfg, *sizes) == -4, (cfg, sizes)
            served += 1
    assert served > 3900


def test_a_requested_number_of_splits_is_kept():
    """528 bytes a query row and split, in a single pass of one sequence's tokens."""
    cfg = cfg_of(8, 4)
    for n in (1, 7, 500):
        sizes = [needed(cfg, 1, n, n, 1 << 16, s) for s in (2, 4, 8, 16)]
        step = n * 32 * 528
        assert [b - a for a, b in zip(sizes, sizes[1:])] == pytest.approx([2 * step, 4 * step, 8 * step], abs=512)
