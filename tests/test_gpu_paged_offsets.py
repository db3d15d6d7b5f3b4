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
           ([60, 70, 80, 60], [70, 130, 90, 64]),
           ([1, 60, 1, 1, 1, 1], [70, 130, 90, 64, 70, 66])]  # (single tokens in a pass of their own)


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


def cache_tensors(cache):
    return cache.k_codes, cache.k_norms, cache.v_codes, cache.v_norms


class Appends:
    """Appends of a batch to the pages of a pool as it was."""

    def __init__(self, rotations, news, lens, dtype):
        self.pool = Packed(rotations, 8, batch=14, kv=2, cap=64, k_budget=192, v_bits=3, kind="wide", dtype=dtype)
        self.b, self.lens, self.most = Batch(self.pool, news, lens, seed=4, pad=4), lens, max(news)
        g = torch.Generator(device="cuda").manual_seed(1)
        self.kv = torch.randn((self.b.n, 2, 2, D), generator=g, device="cuda").to(typed(dtype))
        self.start = raw(self.pool.cache)

    def run(self, cu, lens=None):
        for x, y in zip(cache_tensors(self.pool.cache), self.start):
            x.copy_(y)
        chunk = bg.Chunk(i32(cu), i32(self.lens if lens is None else lens), i32(self.b.table), self.most, max(self.lens))
        bg.blockgtq_paged_append(self.pool.cfg, self.pool.layout, 0, self.kv[:, 0], self.kv[:, 1], chunk, self.pool.cache)
        return raw(self.pool.cache)

    def alone(self, cu, s):
        """Sequence s by itself: the others' lengths are none that a sequence has."""
        return self.run(cu, [n if i == s else -1 for i, n in enumerate(self.lens)])

    def pages_equal(self, x, y, pages):
        return all(torch.equal(a[0, p], c[0, p]) for p in pages for a, c in zip(x, y))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("news,lens", BATCHES + [([1, 1, 0, 1, 0, 1, 1], [70, 64, 3, 65, 0, 1, 2])])
def test_append_of_a_batch_with_offsets_at_fault(rotations, news, lens, dtype):
    """The other sequences' rows arrive, keys and values alike, and the pages of those at fault stay as they were."""
    a = Appends(rotations, news, lens, dtype)
    full = a.run(a.b.first)
    for cu in faults(a.b.first, a.b.n):
        print(f"offsets {cu.tolist()} of {a.b.n} rows", flush=True)
        got = a.run(cu)
        for s, (rows, fine) in enumerate(claims(cu, lens, a.b.n, max(news), max(lens))):
            pages = a.b.table[s, :a.b.per[s]]
            assert a.pages_equal(got, full if fine else a.start, pages), (cu, s)


def falls(first, n):
    """Offsets inside the inputs that fall."""
    for i in range(1, len(first) - 1):
        for x in (0, int(first[i - 1]) // 2, int(first[i + 1]) + 1, n):
            cu = first.copy()
            cu[i] = x
            yield cu
    yield np.concatenate([[0, first[1], 0, first[1]], first[4:]]).astype(np.int32)  # the same rows twice


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("news,lens", BATCHES)
def test_append_of_a_batch_whose_offsets_fall(rotations, news, lens, dtype):
    """A sequence's rows arrive all together or not at all, and surely where it claims rows of no earlier one."""
    a = Appends(rotations, news, lens, dtype)
    for cu in falls(a.b.first, a.b.n):
        print(f"offsets {cu.tolist()} of {a.b.n} rows", flush=True)
        got = a.run(cu)
        end = 0
        for s, (rows, fine) in enumerate(claims(cu, lens, a.b.n, max(news), max(lens))):
            pages = a.b.table[s, :a.b.per[s]]
            alone = a.alone(cu, s)
            if fine and rows.start >= end:
                assert a.pages_equal(got, alone, pages), (cu, s)
            else:
                assert a.pages_equal(got, a.start, pages) or (fine and a.pages_equal(got, alone, pages)), (cu, s)
            end = max(end, rows.stop if fine else 0)


@pytest.mark.parametrize("news,lens", BATCHES + [([300, 300, 300], [300, 340, 300])])
def test_attention_of_a_batch_whose_offsets_fall(rotations, news, lens):
    """Every row that a sequence claims is not a number or one of its claimants' outputs, and surely right where the only
    claimant starts behind the earlier ones."""
    pool = Packed(rotations, 6, batch=18, kv=2, group=4, cap=64)
    b = Batch(pool, news, lens, seed=3, pad=4)
    q, dq = pool.queries((b.n,))
    for cu in list(falls(b.first, b.n)):
        told = claims(cu, lens, b.n, max(news), max(lens))
        b.first, b.news = cu, [len(rows) if fine else 0 for rows, fine in told]
        refs = [expect(b, q, torch.float32, only=[s]) for s in range(len(news))]
        claimed, sure, end = {}, [], 0
        for s, (rows, fine) in enumerate(told):
            for i in rows:
                claimed.setdefault(i, []).append(s if fine and rows.start >= end else -1 - s)
            end = max(end, rows.stop if fine else 0)
        for splits in (0, 1, 2):
            print(f"offsets {cu.tolist()} of {b.n} rows, {splits} splits", flush=True)
            chunk = bg.Chunk(i32(cu), i32(lens), i32(b.table), max(news), max(lens))
            got = torch.full((b.n, 8, D), 7.0, device="cuda")
            bg.blockgtq_paged_attn(pool.cfg, pool.layout, 0, dq, chunk, pool.cache, out=got, n_splits=splits)
            x = got.double().cpu().numpy()
            for i in range(b.n):
                if i not in claimed:
                    assert (x[i] == 7.0).all(), i
                    continue
                near = np.isnan(x[i])
                if len(claimed[i]) == 1 and claimed[i][0] >= 0:
                    near[:] = False
                for s, (rows, fine) in enumerate(told):
                    if fine and i in rows:
                        near |= np.abs(x[i] - refs[s][0][i]) <= refs[s][1][i]
                assert near.all(), (cu, splits, i)


@pytest.mark.parametrize("splits", [0, 1, 3])
@pytest.mark.parametrize("news", [[1] * 200 + [300] + [1] * 130 + [0] * 70 + [2], [3] * 90 + [0] * 200 + [250, 1, 40] + [5] * 70,
                                  [4] * 150 + [0] * 90 + [1] * 10])
def test_hundreds_of_sequences(rotations, news, splits):
    """Chunks among single tokens and empty sequences, over several reads of 64: every row by the formula."""
    lens = [n + (13 * i) % 80 for i, n in enumerate(news)]
    pool = Packed(rotations, 9, batch=sum((t + 63) // 64 for t in lens) + 1, kv=2, group=3, cap=64)
    b = Batch(pool, news, lens, seed=5, pad=7)
    q, dq = pool.queries((b.n,))
    ref, bound = expect(b, q, torch.float32)
    got = torch.full((b.n, 6, D), 7.0, device="cuda")
    bg.blockgtq_paged_attn(pool.cfg, pool.layout, 0, dq, b.chunk, pool.cache, out=got, n_splits=splits)
    live = int(b.first[-1])
    check(f"{len(news)} sequences", got[:live], ref[:live], bound[:live])
    assert (got[live:] == 7.0).all()


@pytest.mark.parametrize("splits", [0, 1, 2])
def test_more_claims_than_blocks_of_rows(rotations, splits):
    """The same 40 rows claimed a hundred times, then five others: the first claimant's or not numbers, and the five right."""
    claimants = 100
    pool = Packed(rotations, 12, batch=5, kv=1, group=8, cap=64)
    b = Batch(pool, [40, 5], [90, 70], seed=2)
    q, dq = pool.queries((b.n,))
    ref, bound = expect(b, q, torch.float32)
    cu = np.array([0, 40] * claimants + [45], np.int32)
    lens = [90, 90] * (claimants - 1) + [90, 70]
    table = np.concatenate([np.repeat(b.table[:1], len(lens) - 1, 0), b.table[1:]])
    chunk = bg.Chunk(i32(cu), i32(lens), i32(table), 40, 90)
    got = torch.full((b.n, 8, D), 7.0, device="cuda")
    bg.blockgtq_paged_attn(pool.cfg, pool.layout, 0, dq, chunk, pool.cache, out=got, n_splits=splits)
    check("the five", got[40:], ref[40:], bound[40:])
    near = np.isnan(got[:40].cpu().numpy()) | (np.abs(got[:40].double().cpu().numpy() - ref[:40]) <= bound[:40])
    assert near.all()


@pytest.mark.parametrize("news,lens", [([3] * 5, [70, 66, 90, 64, 66]), ([9] * 5, [70, 66, 90, 64, 66]), ([9] * 5, [70, 128, 90, 64, 66]),
                                       ([1] * 5, [70, 65, 90, 64, 66])])
@pytest.mark.parametrize("bad", [14, -1, HI, LO])
def test_append_without_a_page(rotations, news, lens, bad):
    """Rows whose page the pool does not have are dropped; those on the sequence's other page arrive, and the others'."""
    a = Appends(rotations, news, lens, "bf16")
    full, table = a.run(a.b.first), a.b.table.copy()
    a.b.table[1, 1] = bad
    got = a.run(a.b.first)
    for s in range(len(lens)):
        for i, p in enumerate(table[s, :a.b.per[s]]):
            assert a.pages_equal(got, a.start if (s, i) == (1, 1) else full, [p]), (s, i)


@pytest.mark.parametrize("n_seqs", [3, 70, 700])
@pytest.mark.parametrize("max_new", [1, 3, 90])
@pytest.mark.parametrize("kind", ["any", "inside", "edges"])
def test_offsets_without_any_sense(rotations, kind, max_new, n_seqs):
    """Numbers of every size: rows that nobody claims stay as they were, rows that only refused sequences claim are not
    numbers, the others are or are finite; the pool's pages change only where a sequence's numbers stand."""
    rng = np.random.default_rng([n_seqs, max_new, len(kind)])
    pool = Packed(rotations, 15, batch=4, kv=2, group=4, cap=64)
    n, ctx, around = 90, 120, 50
    q = torch.from_numpy(synth.cast(rng.standard_normal((n, 8, D)), "bf16")).to(torch.bfloat16).cuda()
    for trial in range(6):
        cu = {"any": lambda: rng.integers(LO, HI, n_seqs + 1), "inside": lambda: rng.integers(0, n + 1, n_seqs + 1),
              "edges": lambda: rng.choice([LO, -1, 0, 1, 2, 3, 44, n - 1, n, n + 1, HI], n_seqs + 1)}[kind]().astype(np.int32)
        lens = rng.choice([ctx, ctx, ctx, ctx + 1, -1, 2], n_seqs).astype(np.int32)
        print(f"{kind} {n_seqs} sequences, at most {max_new} new, trial {trial}: {cu[:12].tolist()}", flush=True)
        chunk = bg.Chunk(i32(cu), i32(lens), i32(np.tile([[1, 3]], (n_seqs, 1))), max_new, ctx)
        told = claims(cu, lens, n, max_new, ctx)
        right, gone = np.zeros(n, bool), np.zeros(n, bool)
        for rows, fine in told:
            (right if fine else gone)[rows.start:rows.stop] = True
        for splits in (0, 2):
            whole = torch.full((n + 2 * around, 8, D), 7.0, device="cuda")
            bg.blockgtq_paged_attn(pool.cfg, pool.layout, 0, q, chunk, pool.cache, out=whole[around:around + n], n_splits=splits)
            x = whole.cpu().numpy()
            assert (x[:around] == 7.0).all() and (x[around + n:] == 7.0).all()
            x = x[around:around + n]
            assert (x[~right & ~gone] == 7.0).all()
            assert np.isnan(x[gone & ~right]).all()
            assert (x[right] != 7.0).all() and not np.isinf(x[right]).any()
    before = raw(pool.cache)
    kv = torch.randn((n, 2, 2, D), device="cuda").to(torch.bfloat16)
    chunk = bg.Chunk(i32(cu), i32(np.full(n_seqs, -1)), i32(np.tile([[1, 3]], (n_seqs, 1))), max_new, ctx)
    bg.blockgtq_paged_append(pool.cfg, pool.layout, 0, kv[:, 0], kv[:, 1], chunk, pool.cache)
    assert all(torch.equal(a, c) for a, c in zip(raw(pool.cache), before))
    # pages outside the pool: nothing to write, whatever the offsets
    chunk = bg.Chunk(i32(cu), i32(np.full(n_seqs, ctx)), i32(np.tile([[4, -1]], (n_seqs, 1))), max_new, ctx)
    bg.blockgtq_paged_append(pool.cfg, pool.layout, 0, kv[:, 0], kv[:, 1], chunk, pool.cache)
    assert all(torch.equal(a, c) for a, c in zip(raw(pool.cache), before))
