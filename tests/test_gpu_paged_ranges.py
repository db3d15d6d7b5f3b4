"""GPU tests of the attention over pages whose rows have radii of very different sizes: a few rows or groups of 8 to 512
times the others' (early ones, ones that only later tokens of the same tile see), ordinary ones beside them.

Tolerances: element by element as in test_gpu_paged.py, and in the 2-norm, where an error in every logit shows that a
bound of single elements hides behind the outputs' own rounding.  Rounding alone, bf16(ref) - ref, is in the reference.
Weights in one fp16 part (bf16 outputs) are off by up to 2^-11, in rms, over a significand in [1, 2) of logarithmic
density, 2^-10 / sqrt(12) * sqrt(E[1 / m^2] = 0.541) = 2.07e-4 of each, which is as much of an output: value rows are
random, so that errors and terms add up alike.  Logits are off by 2^-20 of their terms at most: nothing beside that in
the mean.  With half as much again for the sample: 3e-4.
"""
import math

import numpy as np
import pytest

from oracle import blockgtq_oracle as o
from paper_2606_24033_amd import blockgtq as bg
from paper_2606_24033_amd import synth
from tests.test_gpu_cache_readers import Packed, check
from tests.test_gpu_paged import Batch, expect, slots_of, typed

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
WEIGHTS = 3e-4


@pytest.fixture(scope="module", autouse=True)
def _require_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bg.lib()


@pytest.fixture(scope="module")
def rotations():
    return synth.rotations(7)


def enlarge(pool, b, seq, t, keys=1.0, values=1.0, group=None):
    """Radii of row t of a sequence times powers of two: in the cache and in the rows it stands for."""
    page = pool.cfg.capacity
    p, i = int(b.table[seq, t // page]), t % page
    for h in range(pool.cfg.n_kv_heads):
        groups, S = o.groups(pool.bits[0, h]), slots_of(pool, 0, h)
        for g, (_, dims) in enumerate(groups):
            if group is None or g == group % len(groups):
                pool.cache.k_norms[0, p, h, i * S + g] *= keys
                pool.k[0, p, h, i, dims] *= keys
        pool.cache.v_norms[0, p, h, i] *= values
        pool.v[0, p, h, i] *= values


def paged(rotations, news, lens, kv=1, group=4, **kw):
    pool = Packed(rotations, 41, batch=sum((t + 63) // 64 for t in lens) + 1, kv=kv, group=group, cap=64, **kw)
    b = Batch(pool, news, lens, seed=6)
    return pool, b, *pool.queries((b.n,))


def near(what, b, q, dq, out, cap=0.0):
    got = bg.blockgtq_paged_attn(b.pool.cfg, b.pool.layout, 0, dq, b.chunk, b.pool.cache, out_dtype=typed(out), cap=cap)
    ref, bound = expect(b, q, typed(out), cap=cap)
    check(what, got, ref, bound)
    size = np.linalg.norm(ref)
    off = np.linalg.norm(got.double().cpu().numpy() - ref) / size
    if out == "fp32":
        print(f"{what}: {off:.3g} of the 2-norm", flush=True)
        return
    alone = np.linalg.norm(torch.from_numpy(ref).to(torch.bfloat16).double().numpy() - ref) / size
    print(f"{what}: {off:.5f} of the 2-norm, the rounding alone {alone:.5f}", flush=True)
    assert off <= math.hypot(alone, WEIGHTS)


CHUNKS = [([200], [700]), ([8, 5], [300, 140]), ([300], [300]), ([150, 1, 90], [400, 200, 90]),
          ([900], [2500]), ([2000], [2000])]


@pytest.mark.parametrize("news,lens", CHUNKS)
@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("times", [1, 8, 64, 512])
def test_rows_of_many_times_the_radii(rotations, times, out, news, lens):
    """One row in 50 and each sequence's first, as a row that all tokens attend would be."""
    pool, b, q, dq = paged(rotations, news, lens, k_budget=192, v_bits=3, kind="wide")
    for s, n in enumerate(lens):
        for t in range(0, n, 50):
            enlarge(pool, b, s, t, keys=times)
    near(f"{times} times", b, q, dq, out)


@pytest.mark.parametrize("news,lens", CHUNKS)
@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("times", [64, 512])
def test_groups_of_many_times_the_radii(rotations, times, out, news, lens):
    """A group of every seventh row, another group each time."""
    pool, b, q, dq = paged(rotations, news, lens, k_budget=192, v_bits=3, kind="wide")
    for s, n in enumerate(lens):
        for t in range(0, n, 7):
            enlarge(pool, b, s, t, keys=times, group=t // 7)
    near(f"{times} times", b, q, dq, out)


@pytest.mark.parametrize("news,lens", [([200], [700]), ([60], [60]), ([8], [300]), ([300], [301]), ([900], [2500])])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("times", [64, 512])
@pytest.mark.parametrize("which", ["keys", "values"])
def test_rows_that_only_later_tokens_see(rotations, which, times, out, news, lens):
    """The earlier tokens' outputs are as exact as without them."""
    pool, b, q, dq = paged(rotations, news, lens)
    first = lens[0] - news[0]
    for t in range(first + 5, lens[0], 40):
        enlarge(pool, b, 0, t, **{which: times})
    near(f"{which} {times} times", b, q, dq, out)


@pytest.mark.parametrize("times", [1, 64, 512])
def test_a_few_rows_of_a_long_context(rotations, times):
    """One row in 200 of 8000."""
    pool, b, q, dq = paged(rotations, [400], [8000])
    for t in range(7, 8000, 200):
        enlarge(pool, b, 0, t, keys=times)
    near(f"{times} times", b, q, dq, "bf16")


@pytest.mark.parametrize("times", [1, 64, 512])
@pytest.mark.parametrize("group", [1, 4, 7])
def test_single_tokens_and_narrow_groups_of_many_times_the_radii(rotations, group, times):
    """A group of 1 or 2 bits beside wider ones may carry the logits as well as any other."""
    pool, b, q, dq = paged(rotations, [1] * 6, [500, 64, 130, 700, 400, 333], kv=2, group=group, k_budget=192, v_bits=3, kind="wide")
    for s, n in enumerate(b.lens):
        for t in range(0, n, 7):
            for g in (0, 1):
                enlarge(pool, b, s, t, keys=times, group=g)
    near(f"{times} times", b, q, dq, "bf16")


@pytest.mark.parametrize("news,lens", [([1, 1], [300, 64]), ([8], [300]), ([200], [500])])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("cap", [1e-40, 1e-20, 1e-3, 1.0, 50.0, 1e3, 1e5, 1e7, 1e20, 3.2e38])
def test_caps_of_every_size(rotations, cap, out, news, lens):
    """From a cap that leaves no difference between the rows to one that changes nothing, as exact as without it."""
    pool, b, q, dq = paged(rotations, news, lens)
    near(f"cap {cap}", b, 4 * q, 4 * dq, out, cap=cap)
