"""GPU tests of a serving step over pages: head norms with the rotation, the
append of a ragged batch's rows into pages, the attention of its new tokens,
and a run of them together.

Tolerances, element by element, from the arithmetic alone (u = 2^-24), as in
the tests of the other cache readers; the cap and the bias add their own terms
(attend below), the rotation those of its angle (rotated below).
Where a chunk's bf16 outputs come from 6-bit operands of the small products, a
logit could be off by 2^-12 of its terms; it is held to the same 2^-20 here.
"""
import math

import numpy as np
import pytest

from oracle import blockgtq_oracle as o
from paper_2606_24033_amd import blockgtq as bg
from paper_2606_24033_amd import synth
from tests import _parity as P
from tests.test_gpu_cache_readers import D, U, Packed, check, i32

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _require_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bg.lib()


@pytest.fixture(scope="module")
def rotations():
    return synth.rotations(7)


def typed(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


# ---------------------------------------------------------------- norms and rotation

def rotated(x, w, eps, pos, axis, theta, out_dtype):
    """The formula in 64 bits on the rows x [n, heads, 128], and how far the kernel may be off."""
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    turn = pos[:, axis].astype(np.float64) * np.array(theta)
    c, s = np.cos(turn)[:, None], np.sin(turn)[:, None]
    a, b = x[..., :64], x[..., 64:]
    ref = np.concatenate([a * c - b * s, a * s + b * c], -1)
    # norm: the sum of 128 squares in 16-term chains and 3 exchanges (20 u, half of it in the root), the root, three
    # products (6 u); angle: a fraction of a turn rounded to fp32 (pi u), the sine's 4 u; two products and a sum (3 u)
    size = np.abs(a) + np.abs(b)
    size = np.concatenate([size, size], -1)
    # (the angle itself, in 53 bits: three roundings of it)
    far = 2.0 ** -51 * np.abs(turn)[:, None]
    far = np.concatenate([far, far], -1)
    step = 2.0 ** -8 if out_dtype == torch.bfloat16 else U
    return ref, (28 * U + far) * size + step * np.abs(ref) + 1e-37


@pytest.mark.parametrize("n,kv,group,dtype,out,axes,norm,fused,scale", [
    (1, 8, 4, "bf16", "bf16", 1, "qk", True, 1.0),
    (1, 1, 1, "fp32", "fp32", 1, "", False, 1.0),
    (7, 2, 8, "fp32", "fp32", 3, "qk", False, 30.0),
    (33, 3, 5, "bf16", "fp32", 2, "q", True, 1e-3),
    (300, 2, 8, "bf16", "bf16", 4, "k", False, 1.0),
    (1025, 8, 4, "fp32", "bf16", 3, "qk", True, 1.0),
    (5000, 8, 4, "bf16", "bf16", 3, "", True, 1.0),
    (2, 20, 7, "bf16", "bf16", 1, "qk", True, 100.0),
    (4097, 1, 4, "fp32", "fp32", 1, "qk", True, 1.0),
])
def test_norm_rope(n, kv, group, dtype, out, axes, norm, fused, scale):
    rng = np.random.default_rng([n, kv, axes])
    hq = kv * group
    x = synth.cast(scale * rng.standard_normal((n, hq + 2 * kv, D)), dtype)
    x[n // 2, 0] = 0  # a row of zeros
    pos = rng.integers(-5, 10 ** 6, (n, axes)).astype(np.int32)
    pos[0] = 2 ** 31 - 1
    pos[-1] = 0 if n > 1 else pos[-1]
    axis = rng.integers(0, axes, 64)
    axis[-1] = axes - 1
    theta = [1e6 ** (-2 * i / 128) for i in range(64)]
    w = {c: 1 + 0.3 * rng.standard_normal(D).astype(np.float32) if c in norm else None for c in "qk"}
    cfg = bg.Config(n_layers=1, batch=1, n_kv_heads=kv, group=group, capacity=64, k_budget=128, v_bits=2,
                    in_dtype=bg.BGTQ_BF16 if dtype == "bf16" else bg.BGTQ_FP32)
    qkv = torch.from_numpy(x).to(typed(dtype)).cuda()
    part = {"q": (0, hq), "k": (hq, hq + kv)}
    dev = {c: qkv[:, a:b] if fused else qkv[:, a:b].contiguous() for c, (a, b) in part.items()}
    wd = {c: None if t is None else torch.from_numpy(t).cuda() for c, t in w.items()}
    got = dict(zip("qk", bg.blockgtq_norm_rope(cfg, bg.Rope(theta, axis), dev["q"], dev["k"], torch.from_numpy(pos).cuda(),
                                               q_weight=wd["q"], k_weight=wd["k"], eps=1e-5, out_dtype=typed(out))))
    one = dict(zip("qk", bg.blockgtq_norm_rope(cfg, bg.Rope(theta, axis), None, dev["k"], torch.from_numpy(pos).cuda(),
                                               k_weight=wd["k"], eps=1e-5, out_dtype=typed(out))))
    assert one["q"] is None and torch.equal(one["k"], got["k"])
    assert np.array_equal(qkv.float().cpu().numpy(), x.astype(np.float32))  # the inputs are left as they were
    for c, (a, b) in part.items():
        ref, bound = rotated(x[:, a:b].astype(np.float64), w[c], 1e-5, pos, axis, theta, typed(out))
        check(f"{c} n={n}", got[c], ref, bound)
    if dtype == out:  # each its own output, in the projection's rows
        bg.blockgtq_norm_rope(cfg, bg.Rope(theta, axis), qkv[:, :hq], qkv[:, hq:hq + kv], torch.from_numpy(pos).cuda(),
                              q_weight=wd["q"], k_weight=wd["k"], eps=1e-5, q_out=qkv[:, :hq], k_out=qkv[:, hq:hq + kv])
        assert torch.equal(qkv[:, :hq], got["q"]) and torch.equal(qkv[:, hq:hq + kv], got["k"])
        assert np.array_equal(qkv[:, hq + kv:].float().cpu().numpy(), x[:, hq + kv:].astype(np.float32))


def test_norm_rope_is_the_decode_steps_rotation():
    """Turning text's axis only, rows without a norm are those that the decode step forms."""
    rng = np.random.default_rng(3)
    cfg = bg.Config(n_layers=1, batch=1, n_kv_heads=1, group=1, capacity=64, k_budget=128, v_bits=2, in_dtype=bg.BGTQ_FP32)
    k = rng.standard_normal((50, 1, D)).astype(np.float32)
    theta = [10000.0 ** (-2 * i / 128) for i in range(64)]
    pos = np.arange(50, dtype=np.int32)[:, None] * 20000
    _, got = bg.blockgtq_norm_rope(cfg, bg.Rope(theta), None, torch.from_numpy(k).cuda(), torch.from_numpy(pos).cuda())
    ref, bound = rotated(k.astype(np.float64), None, 0, pos, np.zeros(64, int), theta, torch.float32)
    check("text", got, ref, bound)


def test_norm_rope_empty_and_odd_values():
    cfg = bg.Config(n_layers=1, batch=1, n_kv_heads=2, group=2, capacity=64, k_budget=128, v_bits=2)
    rope = bg.Rope([1.0] * 64)
    q, k = bg.blockgtq_norm_rope(cfg, rope, torch.zeros((0, 4, D), dtype=torch.bfloat16, device="cuda"),
                                 torch.zeros((0, 2, D), dtype=torch.bfloat16, device="cuda"),
                                 torch.zeros((0, 1), dtype=torch.int32, device="cuda"))
    assert q.shape == (0, 4, D) and k.shape == (0, 2, D)
    # not a number and infinite rows stay in their own head
    x = torch.ones((3, 4, D), dtype=torch.bfloat16, device="cuda")
    x[1, 1, 5], x[1, 2, 7] = math.nan, math.inf
    q, _ = bg.blockgtq_norm_rope(cfg, rope, x, None, torch.zeros((3, 1), dtype=torch.int32, device="cuda"),
                                 q_weight=torch.ones(D, device="cuda"))
    fine = torch.isfinite(q).all(-1).cpu()
    assert fine.tolist() == [[True] * 4, [True, False, False, True], [True] * 4]


# ---------------------------------------------------------------- pages

class Batch:
    """A ragged batch whose sequences' pages are spread over a pool."""

    def __init__(self, pool, news, lens, seed=0, pad=0, spare=0):
        rng = np.random.default_rng([seed, 3])
        P = pool.cfg.capacity
        per = [(t + P - 1) // P for t in lens]
        self.most = max(per + [1]) + spare
        self.table = rng.integers(-9, 10 ** 6, (len(lens), self.most)).astype(np.int32)  # entries that nobody needs
        places, at = rng.permutation(pool.cfg.batch), 0
        for b, n in enumerate(per):
            self.table[b, :n] = places[at:at + n]
            at += n
        self.per, self.news, self.lens = per, news, lens
        self.first = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        self.n = int(self.first[-1]) + pad
        self.max_new, self.max_ctx = max(news), max(lens)
        self.chunk = bg.Chunk(i32(self.first), i32(np.array(lens, np.int32)), i32(self.table), self.max_new, self.max_ctx)
        self.pool = pool

    def rows(self, b, h, which, layer=0):
        x = (self.pool.k if which == "k" else self.pool.v)[layer, :, h]
        return np.concatenate([x[p] for p in self.table[b, :self.per[b]]] or [np.zeros((0, D))])[:self.lens[b]]


def raw(cache):
    return [t.clone() for t in (cache.k_codes, cache.k_norms, cache.v_codes, cache.v_norms)]


def slots_of(pool, layer, h):
    return (len(o.groups(pool.bits[layer, h])) + 1) // 2 * 2


@pytest.mark.parametrize("layers,kv,k_budget,v_bits,kind,dtype,page,news,lens,pad,strided", [
    (1, 1, 128, 2, "mixed", "bf16", 64, [1], [1], 0, False),
    (2, 2, 192, 3, "wide", "fp32", 64, [1, 1, 1, 1], [65, 64, 100, 1], 0, True),     # the decode step's kernel
    (1, 2, 192, 5, "wide", "bf16", 64, [4, 1, 0, 3, 2], [66, 64, 70, 194, 130], 2, True),  # over page ends, none, padded
    (1, 2, 192, 3, "wide", "bf16", 64, [2, 4, 3, 4, 1, 4, 2], [34, 33, 64, 68, 40, 96, 2], 1, False),  # words that neighbours share
    (1, 2, 128, 2, "mixed", "bf16", 64, [1] * 9 + [0] * 70 + [1] * 13, None, 0, True),  # four tokens a workgroup
    (1, 2, 128, 2, "mixed", "bf16", 64, [5, 0, 1, 70, 64], [5, 10, 64, 150, 64], 0, False),
    (2, 3, 192, 3, "wide", "fp32", 128, [200, 33, 1], [301, 65, 129], 7, True),
    (1, 1, 512, 8, "uniform", "bf16", 192, [100, 31, 1, 1], [250, 31, 193, 33], 0, True),
    (1, 2, 256, 7, "wide", "fp32", 64, [1] * 3 + [0] * 130 + [9, 2] + [1] * 70, None, 5, False),  # many sequences, many empty
    (1, 8, 128, 2, "mixed", "bf16", 256, [9000, 333], [9100, 777], 0, True),         # 16-wave workgroups
    (1, 8, 64, 1, "uniform", "fp32", 64, [5000, 4000], [5000, 4031], 3, False),
])
def test_paged_append(rotations, layers, kv, k_budget, v_bits, kind, dtype, page, news, lens, pad, strided):
    if lens is None:
        lens = [n + (7 * i) % 90 for i, n in enumerate(news)]
    pages = sum((t + page - 1) // page for t in lens) + 2
    small = max(news) <= 4
    pool = Packed(rotations, 31, layers=layers, batch=pages, kv=kv, cap=page, k_budget=k_budget, v_bits=v_bits, kind=kind,
                  dtype=dtype) if pages * page * kv < 20000 else bare_pool(rotations, layers, pages, kv, page, k_budget, v_bits, kind, dtype)
    b = Batch(pool, news, lens, seed=len(news), pad=pad)
    cfg, layer = pool.cfg, layers - 1
    before = raw(pool.cache)
    t = typed(dtype)
    g = torch.Generator(device="cuda").manual_seed(5)
    kvs = torch.randn((b.n, 3 * kv, D), generator=g, device="cuda").to(t)
    k, v = (kvs[:, kv:2 * kv], kvs[:, 2 * kv:]) if strided else (kvs[:, :kv].contiguous(), kvs[:, kv:2 * kv].contiguous())
    bg.blockgtq_paged_append(cfg, pool.layout, layer, k, v, b.chunk, pool.cache)
    after = raw(pool.cache)
    # each sequence by the append of a cache of its own: its new rows (with some behind them, so that its kernel is the
    # batch's: rows do not depend on one another).  Bit for bit, but for bf16 rows of the ordinary widths, whose products
    # have another order of their sums: there a code may differ where 64 bits put the coordinate next to a threshold
    extra = 0 if small else 5
    exact = small or dtype == "fp32" or k_budget > 256 or v_bits > 4
    cap = (max(lens) + extra + 63) // 64 * 64
    cfg1 = bg.Config(n_layers=layers, batch=1, n_kv_heads=kv, group=pool.cfg.group, capacity=cap, k_budget=k_budget,
                     v_bits=v_bits, in_dtype=cfg.in_dtype)
    touched = np.zeros((pages, page), dtype=bool)
    for s, (n, total) in enumerate(zip(news, lens)):
        if n == 0:
            continue
        one = bg.Cache(cfg1)
        rows = slice(int(b.first[s]), int(b.first[s]) + n)
        more = lambda x: torch.cat([x[rows], torch.ones((extra,) + x.shape[1:], dtype=t, device="cuda")])[None].contiguous()  # noqa: E731
        pos = total - n
        bg.blockgtq_quantize_append(cfg1, pool.layout, layer, more(k), more(v), i32([pos]), one)
        for i in range(pos, total):
            touched[b.table[s, i // page], i % page] = True
        at = torch.arange(pos, total, device="cuda")
        pg, pl = torch.from_numpy(b.table[s].astype(np.int64)).cuda()[at // page], at % page
        for h in range(kv):
            same_codes(key_codes(after[0][layer, pg, h, pl], pool.bits[layer, h]), key_codes(one.k_codes[layer, 0, h, at], pool.bits[layer, h]),
                       *rotated_rows(k[rows, h], o.groups(pool.bits[layer, h]), pool.rot_k), exact)
            same_codes(value_codes(after[2][layer], v_bits)[pg, h, pl], value_codes(one.v_codes[layer], v_bits)[0, h, at],
                       *rotated_rows(v[rows, h], [(v_bits, list(range(D)))], {D: pool.rot_v}), exact)
        assert near_radii(after[3][layer, pg, :, pl], one.v_norms[layer, 0, :, at].transpose(0, 1), exact), s
        for h in range(kv):
            S = slots_of(pool, layer, h)
            ng = len(o.groups(pool.bits[layer, h]))
            mine = after[1][layer, :, h, :page * S].view(pages, page, S)[pg, pl]
            other = one.k_norms[layer, 0, h, :cap * S].view(cap, S)[at]
            assert near_radii(mine[:, :ng], other[:, :ng], exact), (s, h)
    # every other row of the touched pages, every other page and layer as before
    other = torch.from_numpy(~touched).cuda()
    for l2 in range(layers):
        keep = other if l2 == layer else torch.ones_like(other)
        assert torch.equal(after[0][l2].transpose(1, 2)[keep], before[0][l2].transpose(1, 2)[keep])
        assert torch.equal(after[3][l2].transpose(1, 2)[keep], before[3][l2].transpose(1, 2)[keep])
        assert torch.equal(value_codes(after[2][l2], v_bits).transpose(1, 2)[keep],
                           value_codes(before[2][l2], v_bits).transpose(1, 2)[keep])
        for h in range(kv):
            S = slots_of(pool, l2, h)
            a, c = (x[1][l2, :, h, :page * S].view(pages, page, S) for x in (after, before))
            assert torch.equal(a[keep], c[keep])
            assert torch.equal(after[1][l2, :, h, page * S:], before[1][l2, :, h, page * S:])


def key_codes(words, bits):
    """[n, words] key rows as [n, 128] codes in stream order."""
    w = torch.from_numpy(P.stream_widths(bits)).cuda()
    at = torch.cumsum(w, 0) - w
    x = torch.nn.functional.pad(words.to(torch.int64) & 0xFFFFFFFF, (0, 1))
    return ((x[:, at // 32] | x[:, at // 32 + 1] << 32) >> (at % 32)) & ((1 << w) - 1)


def rotated_rows(x, groups, rot):
    """Rows in units of the codebooks, in stream order and 64 bits, how far fp32 sums may be off, and the widths."""
    x = x.double()
    z, off, widths = [], [], []
    for width, dims in groups:
        m, y = torch.from_numpy(rot[len(dims)]).double().cuda(), x[:, torch.tensor(dims, device="cuda")]
        unit = math.sqrt(len(dims)) / y.norm(dim=1, keepdim=True).clamp_min(1e-300)
        z.append(y @ m.T * unit)
        # 128 terms in fp32, some in three parts; the radius and the scale 16 u more of the coordinate
        off.append(2 * (136 * U * (y.abs() @ m.abs().T) * unit + 16 * U * z[-1].abs()))
        widths += [width] * len(dims)
    return torch.cat(z, 1), torch.cat(off, 1), torch.tensor(widths, device="cuda")


def same_codes(got, ref, z, off, widths, exact):
    if exact:
        assert torch.equal(got, ref)
        return
    differ = got != ref
    assert ((got - ref).abs() <= 1).all()
    for i, p in differ.nonzero().tolist():
        _, thr = bg.blockgtq_codebook(int(widths[p]))
        near = float(np.abs(thr.astype(np.float64) - float(z[i, p])).min())
        assert near <= float(off[i, p]), (i, p, near, float(off[i, p]))


def near_radii(a, b, exact):
    """Equal, or (another order of the sum of squares) neighbouring fp16 numbers."""
    return torch.equal(a, b) if exact else bool(((a.view(torch.int16).int() - b.view(torch.int16).int()).abs() <= 1).all())


def value_codes(words, bits):
    """[..., tiles, 128, bits] words as [..., 32 tiles, 128] codes."""
    w = words.to(torch.int64) & 0xFFFFFFFF
    w = torch.nn.functional.pad(w, (0, 1))
    bit = torch.arange(32, device="cuda") * bits
    x = ((w[..., bit // 32] | w[..., bit // 32 + 1] << 32) >> (bit % 32)) & ((1 << bits) - 1)
    return x.transpose(-1, -2).flatten(-3, -2)


class bare_pool:
    """An empty pool with a layout (larger than Packed fills in a reasonable time)."""

    def __init__(self, rotations, layers, pages, kv, page, k_budget, v_bits, kind, dtype, group=4):
        few = Packed(rotations, 31, layers=layers, batch=1, kv=kv, group=group, cap=64, k_budget=k_budget, v_bits=v_bits, kind=kind, dtype=dtype)
        self.cfg = bg.Config(n_layers=layers, batch=pages, n_kv_heads=kv, group=group, capacity=page, k_budget=k_budget,
                             v_bits=v_bits, in_dtype=few.cfg.in_dtype)
        self.bits, self.layout, self.cache = few.bits, few.layout, bg.Cache(self.cfg)
        self.rot_k, self.rot_v = rotations


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_paged_append_of_single_tokens_among_many_rows(rotations, dtype):
    """Inputs padded on both sides to more rows than a grid's dimension holds workgroups of four."""
    pool = bare_pool(rotations, 1, 4, 1, 64, 192, 3, "wide", dtype)
    b = Batch(pool, [1, 1, 1], [64, 3, 40], seed=2)
    kv = torch.randn((3, 2, 1, D), generator=torch.Generator(device="cuda").manual_seed(9), device="cuda").to(typed(dtype))
    bg.blockgtq_paged_append(pool.cfg, pool.layout, 0, kv[:, 0], kv[:, 1], b.chunk, pool.cache)
    few = raw(pool.cache)
    for t in (pool.cache.k_codes, pool.cache.k_norms, pool.cache.v_codes, pool.cache.v_norms):
        t.zero_()
    n, at = 4 * 65536 + 7, 4 * 65535 + 2
    rows = torch.ones((n, 2, 1, D), device="cuda", dtype=typed(dtype))
    rows[at:at + 3] = kv
    chunk = bg.Chunk(i32(b.first + at), i32(b.lens), i32(b.table), 1, b.max_ctx)
    bg.blockgtq_paged_append(pool.cfg, pool.layout, 0, rows[:, 0], rows[:, 1], chunk, pool.cache)
    many = raw(pool.cache)
    # three rows of random numbers have no coordinate next to a threshold: the kernels agree in every code
    assert torch.equal(many[0], few[0]) and torch.equal(many[2], few[2])
    assert near_radii(many[1], few[1], False) and near_radii(many[3], few[3], False)


@pytest.mark.parametrize("small", [True, False])
def test_paged_append_refused_sequences_and_pages(rotations, small):
    """Sequences whose numbers make no sense, and rows without a page, are passed over; the others' rows arrive."""
    pool = Packed(rotations, 8, batch=12, kv=2, cap=64, k_budget=192, v_bits=3, kind="wide")
    n = 3 if small else 9
    news, lens = [n, n, n, n, n], [70, 66, 90, 64, 66]
    b = Batch(pool, news, lens, seed=4)
    kv = torch.randn((b.n, 2, 2, D), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    start = raw(pool.cache)

    def run(cu=None, ctx=None, table=None, max_new=n, max_ctx=90):
        for x, y in zip((pool.cache.k_codes, pool.cache.k_norms, pool.cache.v_codes, pool.cache.v_norms), start):
            x.copy_(y)
        c = bg.Chunk(i32(b.first if cu is None else cu), i32(lens if ctx is None else ctx),
                     i32(b.table if table is None else table), max_new, max_ctx)
        bg.blockgtq_paged_append(pool.cfg, pool.layout, 0, kv[:, 0], kv[:, 1], c, pool.cache)
        return raw(pool.cache)

    def pages_changed(x):
        return {p for p in range(12) if any(not torch.equal(a[0, p], c[0, p]) for a, c in zip(x, start))}

    def pages_of(seqs):
        return {int(b.table[s, i // 64]) for s in seqs for i in range(lens[s] - n, lens[s])}
    full = run()
    assert pages_changed(full) == pages_of(range(5))
    # longer than max_ctx, shorter than its new rows, a length below zero
    for ctx in ([70, 91, 90, 64, 66], [70, n - 1, 90, 64, 66], [70, -5, 90, 64, 66]):
        assert pages_changed(run(ctx=ctx)) == pages_of([0, 2, 3, 4])
    # more than max_new rows: every sequence
    assert pages_changed(run(max_new=n - 1)) == set()
    # offsets that fall: the sequence that falls, and whatever overlaps keeps its own rows
    cu = b.first.copy()
    cu[2] = cu[1] - 1
    x = run(cu=cu)
    assert not pages_changed(x) & (pages_of([1]) - pages_of([0, 2, 3, 4]))
    # offsets outside the inputs
    cu = b.first.copy()
    cu[5] = b.n + 1
    assert pages_changed(run(cu=cu)) == pages_of([0, 1, 2, 3])
    cu = b.first.copy()
    cu[0] = -1
    assert pages_changed(run(cu=cu)) == pages_of([1, 2, 3, 4])
    # a page that the pool does not have: its rows are dropped, the sequence's other page is written
    for bad in (12, -1, 2 ** 31 - 1, -2 ** 31):
        table = b.table.copy()
        table[1, 1] = bad
        x = run(table=table)
        assert pages_changed(x) == pages_of([0, 2, 3, 4]) | {int(b.table[1, 0])} if lens[1] - n < 64 else pages_of([0, 2, 3, 4])
        assert all(torch.equal(p[0, b.table[1, 0]], q[0, b.table[1, 0]]) for p, q in zip(x, full))


# ---------------------------------------------------------------- attention

def attend(q, k, v, see, pos, bits, rot_k, rot_v, out_dtype, cap=0.0, slope=None):
    """The rows q [n, 128] against rows k, v [T, 128], row i seeing those where see[i]; slope: of each row's head."""
    x0 = q @ k.T / math.sqrt(D)
    x = cap * np.tanh(x0 / cap) if cap else x0
    bias = np.zeros(x.shape) if slope is None else -slope[:, None] * np.abs(pos[:, None] - np.arange(len(k)))
    dcap = 0.0
    if cap:  # bf16: t, 1 - t, 1 + t, the quotient: 8 u of the cap; the product and what enters: 2 u more.  fp32, relative:
        # z 4 u (at most its own share of either polynomial), four steps of each, the quotient and two products; where
        # the argument is cut off, 1.5e-7
        dcap = 10 * U * cap if out_dtype == torch.bfloat16 else 30 * U * np.abs(x)
    x = np.where(see, x + bias, -np.inf)
    top = x.max(1, keepdims=True)
    e = np.exp(x - top)
    p = e / e.sum(1, keepdims=True)
    ref = p @ v
    w = np.zeros((D, D))
    at = 0
    for _, dims in o.groups(bits):
        w[np.ix_(range(at, at + len(dims)), dims)] = rot_k[len(dims)]
        at += len(dims)
    qa, kr, qr = np.abs(q) @ np.abs(w).T, np.abs(k @ w.T), np.abs(q @ w.T)
    dx = ((136 * U * qa + (144 * U + 2.0 ** -20) * qr) @ kr.T) / math.sqrt(D) + dcap + 4 * U * np.abs(bias)
    dx = np.where(see, dx + 4 * U * np.where(see, np.abs(x - top) + np.abs(x), 0.0), 0.0)
    move = np.expm1(2 * dx.max(1, keepdims=True))
    spread = p @ np.abs(v) + np.abs(ref)
    y = np.abs(v @ rot_v.T)
    weight = 2.0 ** -11 if out_dtype == torch.bfloat16 else 2.0 ** -21
    total = ((len(k) + 64) * U + weight + 8 * U) * (p @ y) + 132 * U * (p @ y)
    total = total + len(k) * 2.0 ** -25 * 5 / math.sqrt(D) / np.maximum(1.0, e.sum(1, keepdims=True))
    rounding = 2.0 ** -8 if out_dtype == torch.bfloat16 else U
    return ref, move * spread + total @ np.abs(rot_v) + rounding * np.abs(ref) + 1e-30


def expect(b, q, out_dtype, layer=0, cap=0.0, slopes=None, prefix=None, only=None):
    """Reference and bound of a call: q [tokens, Hq, 128]."""
    pool = b.pool
    G = pool.cfg.group
    ref, bound = np.zeros(q.shape), np.zeros(q.shape)
    for s, (n, total) in enumerate(zip(b.news, b.lens)):
        if n == 0 or (only is not None and s not in only):
            continue
        rows = slice(int(b.first[s]), int(b.first[s]) + n)
        pos = np.repeat(np.arange(total - n, total), G)
        see = np.arange(total)[None] <= pos[:, None]
        if prefix is not None:
            see |= (np.arange(total) < prefix[s])[None]
        for h in range(pool.cfg.n_kv_heads):
            hs = slice(h * G, (h + 1) * G)
            slope = None if slopes is None else np.tile(slopes[hs], n)
            r, t = attend(q[rows, hs].reshape(-1, D), b.rows(s, h, "k", layer), b.rows(s, h, "v", layer), see, pos,
                          pool.bits[layer, h], pool.rot_k, pool.rot_v, out_dtype, cap, slope)
            ref[rows, hs], bound[rows, hs] = r.reshape(n, G, D), t.reshape(n, G, D)
    return ref, bound


CASES = [
    # one token
    dict(news=[1], lens=[1], kv=1, group=1),
    dict(news=[1, 1, 1], lens=[64, 65, 300], kv=2, group=4, page=64, dtype="fp32"),
    dict(news=[1] * 6, lens=[1, 700, 63, 128, 129, 500], kv=2, group=8, k_budget=192, v_bits=3, kind="wide", page=128),
    dict(news=[1, 0, 1, 0, 0, 1], lens=[200, 50, 64, 0, 7, 191], kv=1, group=5, page=64, out="fp32"),
    dict(news=[1, 1], lens=[900, 100], kv=1, group=4, k_budget=512, v_bits=8, kind="uniform", splits=7),
    # a few tokens: part of one 32-row workgroup, and just more
    dict(news=[8, 3, 5], lens=[8, 100, 129], kv=2, group=4),
    dict(news=[9, 1, 4], lens=[200, 130, 64], kv=1, group=4, dtype="fp32", splits=3),
    dict(news=[33], lens=[33], kv=1, group=1, k_budget=64, v_bits=1, kind="uniform"),
    # chunks: 128 and 256 rows of a workgroup, splits, ragged
    dict(news=[150], lens=[150], kv=2, group=4, page=64),
    dict(news=[257, 31, 100], lens=[300, 31, 513], kv=1, group=8, k_budget=192, v_bits=3, kind="wide", page=128, dtype="fp32"),
    dict(news=[500], lens=[1500], kv=1, group=3, v_bits=5, k_budget=256, kind="wide", page=192, splits=4),
    dict(news=[300, 290], lens=[640, 290], kv=2, group=2, v_bits=6, k_budget=320, kind="wide", out="fp32", dtype="bf16"),
    # a chunk beside single tokens: two passes
    dict(news=[1, 200, 1, 1, 0, 2], lens=[400, 333, 64, 65, 10, 130], kv=2, group=4, pad=5),
    dict(news=[1] * 70 + [120] + [1] * 9, lens=[5 + (37 * i) % 200 for i in range(70)] + [300] + [20 + i for i in range(9)],
         kv=1, group=4, page=64, dtype="fp32"),
    # what else is seen, capped, biased
    dict(news=[100, 7], lens=[100, 70], kv=2, group=4, prefix=[64, 70]),
    dict(news=[1, 1], lens=[300, 200], kv=2, group=4, cap=20.0, bias=True),
    dict(news=[40, 100, 1], lens=[300, 100, 129], kv=1, group=8, cap=5.0, prefix=[0, 1000, 50], dtype="fp32"),
    dict(news=[200], lens=[400], kv=2, group=4, bias=True, dtype="fp32", page=128),
    dict(news=[300, 30], lens=[300, 500], kv=1, group=4, cap=50.0, bias=True, prefix=[17, -3], v_bits=3, k_budget=192, kind="wide"),
    dict(news=[3, 3], lens=[100, 40], kv=2, group=2, cap=30.0, dtype="fp32", qscale=0.05),
]


def run_case(rotations, news, lens, kv, group, page=64, k_budget=128, v_bits=2, kind="mixed", dtype="bf16", out=None, splits=0,
             prefix=None, cap=0.0, bias=False, pad=0, qscale=1.0, seed=1, layers=1, layer=0):
    pages = sum((t + page - 1) // page for t in lens) + 3
    pool = Packed(rotations, seed, layers=layers, batch=pages, kv=kv, group=group, cap=page, k_budget=k_budget, v_bits=v_bits,
                  kind=kind, dtype=dtype)
    b = Batch(pool, news, lens, seed=seed, pad=pad, spare=1)
    q, dq = pool.queries((b.n,), qscale)
    slopes = None
    if bias:
        slopes = (0.5 ** np.arange(1, kv * group + 1)).astype(np.float32)
    out_dtype = typed(out or dtype)
    got = torch.full((b.n, kv * group, D), 7.0, dtype=out_dtype, device="cuda")
    kw = dict(cap=cap, slopes=None if slopes is None else torch.from_numpy(slopes).cuda(),
              prefix=None if prefix is None else i32(prefix), n_splits=splits)
    bg.blockgtq_paged_attn(pool.cfg, pool.layout, layer, dq, b.chunk, pool.cache, out=got, **kw)
    return pool, b, q, dq, got, kw, slopes, out_dtype


@pytest.mark.parametrize("case", range(len(CASES)))
def test_paged_attn(rotations, case):
    c = CASES[case]
    pool, b, q, dq, got, kw, slopes, out_dtype = run_case(rotations, **c)
    ref, bound = expect(b, q, out_dtype, cap=c.get("cap", 0.0), slopes=slopes, prefix=c.get("prefix"))
    live = int(b.first[-1])
    check(f"case {case}", got[:live], ref[:live], bound[:live])
    assert (got[live:] == 7.0).all()  # rows behind the last sequence
    again = torch.full_like(got, 7.0)
    bg.blockgtq_paged_attn(pool.cfg, pool.layout, 0, dq, b.chunk, pool.cache, out=again, **kw)
    assert torch.equal(again, got)


@pytest.mark.parametrize("splits", [1, 2, 5, 64])
@pytest.mark.parametrize("news,lens", [([1, 1, 1], [300, 64, 511]), ([70, 1, 1], [400, 200, 65]), ([40, 300], [100, 600])])
def test_paged_attn_splits(rotations, news, lens, splits):
    """Any number of splits, those without a row among them."""
    pool, b, q, dq, got, kw, slopes, out_dtype = run_case(rotations, news, lens, 1, 4, splits=splits, out="fp32")
    ref, bound = expect(b, q, out_dtype)
    check(f"{splits} splits", got, ref, bound)


@pytest.mark.parametrize("v_bits", range(1, 9))
@pytest.mark.parametrize("k_budget", [64, 192, 256, 384, 512])
def test_paged_attn_widths(rotations, k_budget, v_bits):
    """Every value width with key rows of each register class, in both kinds of pass."""
    kind = "uniform" if k_budget in (64, 512) else "wide"
    for news, lens in (([1, 2], [100, 65]), ([150, 1], [200, 70])):
        pool, b, q, dq, got, kw, slopes, out_dtype = run_case(rotations, news, lens, 1, 4, k_budget=k_budget, v_bits=v_bits,
                                                              kind=kind, seed=k_budget + v_bits)
        ref, bound = expect(b, q, out_dtype)
        check(f"{k_budget} {v_bits} {news}", got, ref, bound)


def test_paged_attn_layers(rotations):
    for layer in (0, 2):
        pool, b, q, dq, got, kw, slopes, out_dtype = run_case(rotations, [1, 90], [70, 100], 2, 2, layers=3, layer=layer, out="fp32")
        ref, bound = expect(b, q, out_dtype, layer=layer)
        check(f"layer {layer}", got, ref, bound)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("news,lens,out,prefix", [
    ([20], [100], "fp32", None), ([20], [100], "bf16", None), ([200], [200], "fp32", None), ([200, 3], [300, 70], "bf16", None),
    ([40], [100], "bf16", [70]), ([1, 1], [70, 130], "bf16", None),
])
def test_unseen_rows_do_not_matter(rotations, news, lens, out, prefix, bad):
    """Radii that are not finite: rows that a token sees make its outputs NaN, others (later ones of the same tile, rows
    behind the sequence) do not touch them."""
    page, G = 64, 4
    for at in (lens[0] - max(1, news[0] // 2), lens[0] - 1, lens[0]):
        for which in ("k_norms", "v_norms"):
            pool = Packed(rotations, 2, batch=sum((t + page) // page for t in lens) + 1, kv=1, group=G, cap=page)
            b = Batch(pool, news, [t + 1 for t in lens], seed=2)  # pages for a row behind the sequences
            b.lens = lens
            b.per = [(t + page - 1) // page for t in lens]
            b.chunk = bg.Chunk(i32(b.first), i32(lens), i32(b.table), max(news), max(lens))
            q, dq = pool.queries((b.n,))
            out_dtype = typed(out)
            p, i = int(b.table[0, at // page]), at % page
            if which == "v_norms":
                pool.cache.v_norms[0, p, 0, i] = bad
            else:
                S = slots_of(pool, 0, 0)
                pool.cache.k_norms[0, p, 0, i * S:i * S + len(o.groups(pool.bits[0, 0]))] = bad
            kw = dict(prefix=None if prefix is None else i32(prefix + [0] * (len(news) - 1)))
            got = bg.blockgtq_paged_attn(pool.cfg, pool.layout, 0, dq, b.chunk, pool.cache, out_dtype=out_dtype, **kw)
            ref, bound = expect(b, q, out_dtype, prefix=None if prefix is None else prefix + [0] * (len(news) - 1))
            pos = np.arange(lens[0] - news[0], lens[0])
            sees = (pos >= at) | (at < (prefix[0] if prefix else 0)) if at < lens[0] else np.zeros(news[0], bool)
            clean = np.ones(b.n, bool)
            clean[:news[0]] = ~sees
            check(f"{which} at {at}", got[torch.from_numpy(clean).cuda()], ref[clean], bound[clean])
            assert torch.isnan(got[torch.from_numpy(~clean).cuda()].float()).all()


@pytest.mark.parametrize("new", [1, 5, 30, 300, 2500])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_infinite_radius_of_one_group(rotations, new, out):
    """Queries against the row's own direction: all of the group's products are -infinity, and the row is not dropped."""
    pool = Packed(rotations, 77, batch=1 + (new + 350) // 64, kv=1, cap=64, k_budget=192, v_bits=2, kind="wide")
    b = Batch(pool, [new], [new + 350 if new < 2500 else new], seed=new)
    groups = o.groups(pool.bits[0, 0])
    S, t = slots_of(pool, 0, 0), 13
    page = int(b.table[0, 0])
    keep = pool.cache.k_norms.clone()
    for g, (_, dims) in enumerate(groups):
        pool.cache.k_norms.copy_(keep)
        pool.cache.k_norms[0, page, 0, t * S + g] = math.inf
        for scale in (-1.0, 1.0):
            q = np.zeros((new, 4, D))
            q[:, :, dims] = scale * pool.k[0, page, 0, t, dims]
            got = bg.blockgtq_paged_attn(pool.cfg, pool.layout, 0, torch.from_numpy(q).cuda().to(torch.bfloat16), b.chunk,
                                         pool.cache, out_dtype=typed(out))
            seen = t if new == 2500 else 0  # (its first tokens come before the row)
            assert torch.isnan(got[seen:]).all() and torch.isfinite(got[:seen]).all(), (g, scale)


@pytest.mark.parametrize("new", [1, 5, 300])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_queries_that_are_not_finite(rotations, new, out, bad):
    """They make their own outputs not a number and no others."""
    pool = Packed(rotations, 5, batch=11, kv=1, cap=64, k_budget=192, v_bits=2, kind="wide")
    b = Batch(pool, [new], [650], seed=new)
    q, dq = pool.queries((new,))
    ref, bound = expect(b, q, typed(out))
    for i, dim in ((0, 0), (new // 2, 63), (new - 1, 100)):
        x = dq.clone()
        x[i, 2, dim] = bad
        got = bg.blockgtq_paged_attn(pool.cfg, pool.layout, 0, x, b.chunk, pool.cache, out_dtype=typed(out))
        assert torch.isnan(got[i, 2]).all(), (i, dim)
        fine = torch.ones((new, 4), dtype=torch.bool, device="cuda")
        fine[i, 2] = False
        check(f"{i} {dim}", got[fine], ref[fine.cpu().numpy()], bound[fine.cpu().numpy()])


def test_refused_sequences_and_pages(rotations):
    """Numbers that make no sense give NaN, in that sequence alone; nothing behind the sequences is written."""
    page = 64
    for news, lens in (([1, 1, 1, 1], [70, 66, 90, 64]), ([1, 60, 1, 2], [70, 130, 90, 64]), ([60, 70, 80, 60], [70, 130, 90, 64])):
        pool = Packed(rotations, 6, batch=14, kv=2, group=4, cap=page)
        b = Batch(pool, news, lens, seed=3, pad=4)
        q, dq = pool.queries((b.n,))
        ref, bound = expect(b, q, torch.float32)

        def run(what, gone, cu=None, ctx=None, table=None, max_new=max(news), max_ctx=max(lens), loose=()):
            for splits in (0, 1, 2):
                c = bg.Chunk(i32(b.first if cu is None else cu), i32(lens if ctx is None else ctx),
                             i32(b.table if table is None else table), max_new, max_ctx)
                got = torch.full((b.n, 8, D), 7.0, device="cuda")
                bg.blockgtq_paged_attn(pool.cfg, pool.layout, 0, dq, c, pool.cache, out=got, n_splits=splits)
                for s in range(4):
                    rows = slice(int(b.first[s]), int(b.first[s + 1]))
                    if s in gone:
                        assert torch.isnan(got[rows]).all(), (what, s, splits)
                    elif s not in loose:
                        check(f"{what} {s}", got[rows], ref[rows], bound[rows])
                assert (got[int(b.first[-1]):] == 7.0).all(), what
        run("fine", [])
        for x in (max(lens) + 1, news[1] - 1, -7, 2 ** 31 - 1, -2 ** 31):
            run(f"length {x}", [1], ctx=[lens[0], x, lens[2], lens[3]])
        if max(news) > 1:
            longest = [s for s in range(4) if news[s] == max(news)]
            run("max_new", longest, max_new=max(news) - 1)
        for x in (14, -1, 2 ** 31 - 1, -2 ** 31):
            table = b.table.copy()
            table[1, 0] = x  # its first page: every token of it attends it
            run(f"page {x}", [1], table=table)
            table = b.table.copy()
            table[2, 2:] = x  # one that no row needs
            run(f"unused page {x}", [], table=table)


def test_pages_shared_by_sequences(rotations):
    """Two sequences whose first rows lie in the same pages."""
    pool = Packed(rotations, 9, batch=8, kv=1, group=4, cap=64)
    b = Batch(pool, [1, 5], [200, 150], seed=1)
    b.table[1, :2] = b.table[0, :2]
    b.chunk = bg.Chunk(i32(b.first), i32(b.lens), i32(b.table), 5, 200)
    q, dq = pool.queries((b.n,))
    ref, bound = expect(b, q, torch.float32)
    check("shared pages", bg.blockgtq_paged_attn(pool.cfg, pool.layout, 0, dq, b.chunk, pool.cache), ref, bound)


def test_far_pages(rotations):
    """Pages whose codes lie beyond 2^32 bytes of a pool."""
    few = Packed(rotations, 3, batch=5, kv=1, group=4, cap=64, k_budget=512, v_bits=8, kind="uniform")
    pages = (1 << 32) // (64 * 32 * 4) + 600
    pool = bare_pool(rotations, 1, pages, 1, 64, 512, 8, "uniform", "bf16")
    at = torch.tensor([pages - 1, 3, pages - 300, 7, pages - 77], device="cuda")
    for n in ("k_codes", "k_norms", "v_codes", "v_norms"):
        getattr(pool.cache, n)[:, at] = getattr(few.cache, n)
    layout = few.layout
    for news, lens in (([1, 1], [150, 90]), ([100, 20], [150, 90])):
        b = Batch(few, news, lens, seed=2)
        b.chunk = bg.Chunk(i32(b.first), i32(lens), at[torch.from_numpy(b.table.clip(0, 4)).long().cuda()].int().contiguous(),
                           max(news), max(lens))
        q, dq = few.queries((b.n,))
        ref, bound = expect(b, q, torch.float32)
        check("far", bg.blockgtq_paged_attn(pool.cfg, layout, 0, dq, b.chunk, pool.cache), ref, bound)
        # appended there: the rows of a pool of those five pages alone
        near = bg.Cache(few.cfg)
        for n in ("k_codes", "k_norms", "v_codes", "v_norms"):
            getattr(near, n).copy_(getattr(few.cache, n))
        k, v = torch.randn((2, b.n, 1, D), device="cuda").to(torch.bfloat16)
        bg.blockgtq_paged_append(pool.cfg, layout, 0, k, v, b.chunk, pool.cache)
        bg.blockgtq_paged_append(few.cfg, layout, 0, k, v, bg.Chunk(i32(b.first), i32(lens), i32(b.table.clip(0, 4)), max(news), max(lens)), near)
        for n in ("k_codes", "k_norms", "v_codes", "v_norms"):
            assert torch.equal(getattr(pool.cache, n)[:, at], getattr(near, n)), n
            getattr(pool.cache, n)[:, at] = getattr(few.cache, n)


# ---------------------------------------------------------------- together

def serving(rotations, page=64, kv=2, group=4, seed=5):
    pool = Packed(rotations, seed, layers=2, batch=24, kv=kv, group=group, cap=page, k_budget=192, v_bits=3)
    for t in (pool.cache.k_codes, pool.cache.k_norms, pool.cache.v_codes, pool.cache.v_norms):
        t.zero_()
    rope = bg.Rope([10000.0 ** (-2 * i / 128) for i in range(64)])
    weights = [1 + 0.2 * torch.randn(D, generator=torch.Generator(device="cuda").manual_seed(s), device="cuda") for s in (1, 2)]

    def step(qkv, pos, chunk, layer, out, ws=None, stream=None):
        n, hq = qkv.shape[0], kv * group
        q, k = bg.blockgtq_norm_rope(pool.cfg, rope, qkv[:, :hq], qkv[:, hq:hq + kv], pos, q_weight=weights[0],
                                     k_weight=weights[1], stream=stream)
        bg.blockgtq_paged_append(pool.cfg, pool.layout, layer, k, qkv[:, hq + kv:], chunk, pool.cache, stream=stream)
        return q, bg.blockgtq_paged_attn(pool.cfg, pool.layout, layer, q, chunk, pool.cache, out=out, workspace=ws, stream=stream)
    return pool, step


def test_serving_steps(rotations):
    """Prompts in chunks, then tokens, of a ragged batch in two layers: the outputs are those of a cache per sequence."""
    pool, step = serving(rotations)
    kv, G, page = 2, 4, 64
    totals = [150, 70, 33]
    table = np.random.default_rng(1).permutation(24)[:15].reshape(3, 5).astype(np.int32)
    g = torch.Generator(device="cuda").manual_seed(9)
    x = [torch.randn((2, t + 3, (G + 2) * kv, D), generator=g, device="cuda").to(torch.bfloat16) for t in totals]
    cfg1 = bg.Config(n_layers=2, batch=1, n_kv_heads=kv, group=G, capacity=192, k_budget=192, v_bits=3)
    alone = [bg.Cache(cfg1) for _ in totals]
    have = [0, 0, 0]
    for news in ([100, 70, 0], [50, 0, 33], [1, 1, 1], [1, 0, 1], [1, 2, 1]):
        lens = [h + n for h, n in zip(have, news)]
        cu = np.concatenate([[0], np.cumsum(news)])
        chunk = bg.Chunk(i32(cu), i32(lens), i32(table), max(news), max(lens))
        for layer in range(2):
            qkv = torch.cat([x[s][layer, have[s]:lens[s]] for s in range(3)])
            pos = i32(np.concatenate([np.arange(have[s], lens[s]) for s in range(3)])[:, None])
            out = torch.empty((len(qkv), kv * G, D), device="cuda")
            q, _ = step(qkv, pos, chunk, layer, out)
            # by the cache of one sequence: its append and its causal prefill
            for s in range(3):
                if news[s] == 0:
                    continue
                rows = slice(int(cu[s]), int(cu[s + 1]))
                rope = bg.Rope([10000.0 ** (-2 * i / 128) for i in range(64)])
                w = 1 + 0.2 * torch.randn(D, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
                _, k = bg.blockgtq_norm_rope(pool.cfg, rope, None, qkv[rows, kv * G:kv * (G + 1)], pos[rows].contiguous(), k_weight=w)
                bg.blockgtq_quantize_append(cfg1, pool.layout, layer, k[None].contiguous(),
                                            qkv[rows, kv * (G + 1):][None].contiguous(), i32([have[s]]), alone[s])
                ref = bg.blockgtq_prefill_attn(cfg1, pool.layout, layer, q[rows][None].contiguous(), i32([have[s]]), lens[s] - 1, alone[s])[0]
                # (the prefill's weights are one fp16 part: 2^-11 of each weight, against values of norm below 30; a code
                # next to a threshold may be the neighbour's in the other kernel, in a row of hundreds)
                off = (out[rows] - ref).norm() / ref.norm()
                print(f"step {news} layer {layer} sequence {s}: {float(off):.2g}", flush=True)
                assert off < 2.0 ** -9
        have = lens


def test_captured_step(rotations):
    """A step captured once and replayed with other tokens, lengths and pages in the same buffers; eager work between."""
    for most, news_of in ((1, lambda i: [1, 1, 0] if i % 2 else [1, 1, 1]), (80, lambda i: [60 + i, 1, 3])):
        pool, step = serving(rotations, seed=6)
        n = most + 20
        static = {"qkv": torch.zeros((n, 12, D), dtype=torch.bfloat16, device="cuda"), "pos": torch.zeros((n, 1), dtype=torch.int32, device="cuda"),
                  "cu": torch.zeros(4, dtype=torch.int32, device="cuda"), "ctx": torch.zeros(3, dtype=torch.int32, device="cuda"),
                  "pages": torch.zeros((3, 7), dtype=torch.int32, device="cuda"), "out": torch.zeros((n, 8, D), device="cuda")}
        chunk = bg.Chunk(static["cu"], static["ctx"], static["pages"], most, 448)  # (7 pages)
        ws = torch.empty(bg.paged_workspace_bytes(pool.cfg, chunk, n), dtype=torch.uint8, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):  # (nothing to do yet: no sequence has a token)
            step(static["qkv"], static["pos"], chunk, 0, static["out"], ws)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(static["qkv"], static["pos"], chunk, 0, static["out"], ws)
        g = torch.Generator(device="cuda").manual_seed(3)
        rng = np.random.default_rng(2)
        have = [100, 64, 7]
        table = rng.permutation(24)[:21].reshape(3, 7).astype(np.int32)
        for i in range(5):
            news = news_of(i)
            lens = [h + c for h, c in zip(have, news)]
            static["qkv"].copy_(torch.randn((n, 12, D), generator=g, device="cuda"))
            static["pos"].copy_(torch.from_numpy(rng.integers(0, 999, (n, 1)).astype(np.int32)))
            static["cu"].copy_(i32(np.concatenate([[0], np.cumsum(news)])))
            static["ctx"].copy_(i32(lens))
            static["pages"].copy_(i32(table))
            static["out"].fill_(7.0)
            before = raw(pool.cache)
            graph.replay()
            torch.cuda.synchronize()
            replayed, cached = static["out"].clone(), raw(pool.cache)
            for a, c in zip((pool.cache.k_codes, pool.cache.k_norms, pool.cache.v_codes, pool.cache.v_norms), before):
                a.copy_(c)
            eager = torch.full_like(replayed, 7.0)
            step(static["qkv"], static["pos"], chunk, 0, eager)
            torch.cuda.synchronize()
            assert torch.equal(eager, replayed) and all(torch.equal(a, c) for a, c in zip(raw(pool.cache), cached))
            assert (replayed[sum(news):] == 7.0).all() and torch.isfinite(replayed[:sum(news)]).all()
            have = lens


def test_another_stream(rotations):
    pool, step = serving(rotations, seed=7)
    table = np.arange(12, dtype=np.int32).reshape(3, 4)
    chunk = bg.Chunk(i32([0, 90, 91, 94]), i32([90, 100, 3]), i32(table), 90, 100)
    qkv = torch.randn((94, 12, D), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(torch.bfloat16)
    pos = i32(np.arange(94)[:, None])
    _, here = step(qkv, pos, chunk, 0, torch.empty((94, 8, D), device="cuda"))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    _, there = step(qkv, pos, chunk, 0, torch.empty((94, 8, D), device="cuda"), stream=s)
    s.synchronize()
    assert torch.equal(here, there)
