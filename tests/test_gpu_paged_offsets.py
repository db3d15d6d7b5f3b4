"""GPU tests of a ragged batch whose offsets are at fault: what belongs to no such sequence is right, what does is not a
number or not appended, and nothing outside the buffers is touched."""
import numpy as np
import pytest

from paper_2606_24033_amd import blockgtq as bg
from paper_2606_24033_amd import synth
from tests.test_gpu_cache_readers import D, Packed, check, i32
from tests.test_gpu_paged import Batch, expect, raw, typed

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
LO, HI = -2 ** 31, 2 ** 31 - 1


@pytest.fixture(scope="module", autouse=True)
def _require_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bg.lib()


@pytest.fixture(scope="module")
def rotations():
    return synth.rotations(7)


def claims(cu, lens, n_tokens, max_new, max_ctx):
    """Of each sequence: the inputs' rows that its offsets name, and whether its numbers stand by themselves."""
    out = []
    for c0, c1, length in zip(cu[:-1], cu[1:], lens):
        a, z = (min(max(int(c), 0), n_tokens) for c in (c0, c1))
        fine = a == c0 and z == c1 and c0 <= c1 and z - a <= max_new and z - a <= length <= max_ctx
        out.append((range(a, z), fine))
    return out


def faults(first, n):
    """Offsets with one number that cannot be, and some with several."""
    for i in range(len(first)):
        for x in (LO, LO + 3, -1, n + 1, HI):
            cu = first.copy()
            cu[i] = x
            yield cu
    for pair in ((LO, HI), (HI, HI), (-1, -1), (HI, LO)):
        cu = first.copy()
        cu[1:3] = pair
        yield cu


BATCHES = [([1, 1, 1, 1], [70, 66, 90, 64]), ([3, 2, 1, 4], [70, 66, 90, 64]), ([1, 60, 1, 2], [70, 130, 90, 64]),
           ([60, 70, 80, 60], [70, 130, 90, 64])]


@pytest.mark.parametrize("news,lens", BATCHES)
def test_attention_of_a_batch_with_offsets_at_fault(rotations, news, lens):
    """Rows that only a sequence at fault claims are not numbers; those that it claims of another sequence may be; the
    others are right, and the rows around the outputs as they were."""
    pool = Packed(rotations, 6, batch=14, kv=2, group=4, cap=64)
    b = Batch(pool, news, lens, seed=3, pad=4)
    q, dq = pool.queries((b.n,))
    ref, bound = expect(b, q, torch.float32)
    around = 300
    for cu in faults(b.first, b.n):
        for splits in (0, 1, 2):
            print(f"offsets {cu.tolist()} of {b.n} rows, {splits} splits", flush=True)
            chunk = bg.Chunk(i32(cu), i32(lens), i32(b.table), max(news), max(lens))
            whole = torch.full((b.n + 2 * around, 8, D), 7.0, device="cuda")
            got = whole[around:around + b.n]
            bg.blockgtq_paged_attn(pool.cfg, pool.layout, 0, dq, chunk, pool.cache, out=got, n_splits=splits)
            assert (whole[:around] == 7.0).all() and (whole[around + b.n:] == 7.0).all()
            right, gone = set(), set()
            for rows, fine in claims(cu, lens, b.n, max(news), max(lens)):
                (right if fine else gone).update(rows)
            sure = sorted(right - gone)
            if sure:
                check(f"{cu}", got[sure], ref[sure], bound[sure])
            for i in right & gone:
                if not torch.isnan(got[i]).all():
                    fine = ~torch.isnan(got[i]).cpu().numpy()
                    assert (np.abs(got[i].double().cpu().numpy() - ref[i]) <= bound[i])[fine].all()
            assert torch.isnan(got[sorted(gone - right)]).all()
            assert (got[sorted(set(range(b.n)) - right - gone)] == 7.0).all()
