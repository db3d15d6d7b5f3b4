"""GPU tests of the operators that read the packed cache, over the ranges that
a cache may hold: radii of every size, radii that are not finite, outputs in
both types, long reads, and each pass over several layers.

Tolerances as in test_gpu_cache_readers.py: element by element from the
roundings, or in the 2-norm where a single low part that is lost would be
invisible in a worst-case bound.  Radii are scaled by powers of two that keep
them normal fp16 numbers, so that a scaled cache holds exactly the scaled rows.
"""
import numpy as np
import pytest

from oracle import blockgtq_oracle as o
from paper_2606_24033_amd import blockgtq as bg
from paper_2606_24033_amd import synth
from tests.test_gpu_cache_readers import (D, Packed, attention_and_bound, check, expect_cross, expect_rows, expect_shared, i32,
                                          widths_of)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _require_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bg.lib()


@pytest.fixture(scope="module")
def rotations():
    return synth.rotations(7)


def key_radii(pk, layer, b, h):
    """The key radii of a head's rows as they lie in the cache, [capacity, groups] (a view)."""
    ng = len(o.groups(pk.bits[layer, h]))
    slots = ng + (ng & 1)
    return pk.cache.k_norms[layer, b, h, :pk.cfg.capacity * slots].view(pk.cfg.capacity, slots)[:, :ng]


def scale_rows(pk, key=1.0, value=1.0):
    """Radii of every row times powers of two (scalars, or one per cache row)."""
    cap = pk.cfg.capacity
    key, value = (np.broadcast_to(np.asarray(s, dtype=np.float64), (cap,)) for s in (key, value))
    for i in np.ndindex(pk.k.shape[:3]):
        r = key_radii(pk, *i)
        want = r.double() * torch.from_numpy(key.copy()).cuda()[:, None]
        r.copy_(want.half())
        assert torch.equal(r.double(), want)
        r = pk.cache.v_norms[i]
        want = r.double() * torch.from_numpy(value.copy()).cuda()
        r.copy_(want.half())
        assert torch.equal(r.double(), want)
    pk.k *= key[:, None]
    pk.v *= value[:, None]
    return pk


def norm_error(got, ref):
    return float(np.linalg.norm(got.double().cpu().numpy() - ref) / np.linalg.norm(ref))


# ---------------------------------------------------------------- rows read back

ROWS = [(1, 1, 128, 2, "mixed"), (2, 1, 192, 3, "wide"), (1, 2, 256, 5, "uniform"), (1, 1, 512, 8, "uniform"),
        (1, 1, 320, 1, "wide")]


@pytest.mark.parametrize("batch,kv,k_budget,v_bits,kind", ROWS)
def test_bf16_rows_are_rounded_once(rotations, batch, kv, k_budget, v_bits, kind):
    """A bf16 output is the fp32 one rounded: half a step of bf16 from a number that is itself off by the fp32 read's
    bound at most, also where the terms of an element cancel."""
    pk = Packed(rotations, 101, batch=batch, kv=kv, k_budget=k_budget, v_bits=v_bits, kind=kind)
    wide, half = (bg.blockgtq_dequantize_rows(pk.cfg, pk.layout, 0, pk.cache, i32([0] * batch), 192, out_dtype=t)
                  for t in (FP32, BF16))
    for n, a, b in zip("kv", wide, half):
        assert torch.equal(a.to(BF16), b)
        for s in range(batch):
            for h in range(kv):
                ref, bound = expect_rows(pk, 0, s, h, n, 0, 192, FP32)
                check(f"{n} fp32", a[s, :, h], ref, bound)
                check(f"{n} bf16", b[s, :, h], ref, bound + 2.0 ** -8 * (np.abs(ref) + bound))


@pytest.mark.parametrize("out_dtype", [FP32, BF16])
@pytest.mark.parametrize("k_budget,kind", [(192, "wide"), (128, "mixed")])
def test_key_groups_of_very_different_radii(rotations, k_budget, kind, out_dtype):
    """Each group's dims to the precision of its own radius, beside groups whose radii are 2^21 times as large."""
    pk = Packed(rotations, 102, k_budget=k_budget, kind=kind)
    groups = o.groups(pk.bits[0, 0])
    for g, (_, dims) in enumerate(groups):
        s = 2.0 ** (10 - round(21 * g / (len(groups) - 1)))
        key_radii(pk, 0, 0, 0)[:, g] *= s
        pk.k[0, 0, 0][:, dims] *= s
    k, _ = bg.blockgtq_dequantize_rows(pk.cfg, pk.layout, 0, pk.cache, i32([0]), 192, out_dtype=out_dtype)
    ref, bound = expect_rows(pk, 0, 0, 0, "k", 0, 192, FP32)
    if out_dtype == BF16:
        bound = bound + 2.0 ** -8 * (np.abs(ref) + bound)
    check("k", k[0, :, 0], ref, bound)


@pytest.mark.parametrize("out_dtype", [FP32, BF16])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_radius_that_is_not_finite_reads_back_in_its_place_only(rotations, bad, out_dtype):
    """A key group's radius: not finite in the group's dims of that row, every other number as without it.  A value
    radius: not finite in that row."""
    pk = Packed(rotations, 103, kv=2, k_budget=192, v_bits=3, kind="wide")
    args = (pk.cfg, pk.layout, 0, pk.cache, i32([0]), 192)
    k0, v0 = bg.blockgtq_dequantize_rows(*args, out_dtype=out_dtype)
    touched = torch.zeros(k0.shape, dtype=torch.bool, device="cuda")
    for h in range(2):
        for g, (_, dims) in enumerate(o.groups(pk.bits[0, h])):
            for row in (g, 40 + 3 * g, 191 - g):
                key_radii(pk, 0, 0, h)[row, g] = bad
                touched[0, row, h, torch.from_numpy(dims).cuda()] = True
    rows = torch.tensor([0, 31, 32, 100, 191], device="cuda")
    pk.cache.v_norms[0, 0, 1, rows] = bad
    k, v = bg.blockgtq_dequantize_rows(*args, out_dtype=out_dtype)
    assert torch.equal(k[~touched], k0[~touched]) and not torch.isfinite(k[touched]).any()
    assert not torch.isfinite(v[0, rows, 1]).any()
    v[0, rows, 1] = v0[0, rows, 1]
    assert torch.equal(v, v0)


@pytest.mark.parametrize("out_dtype,k_budget,v_bits,n_rows,pos,lens", [
    (BF16, 128, 2, 4160, [0, 0, 0, 0, 0, 0], None),
    (FP32, 192, 3, 4100, [60, 1, 33, 0, 64, 17], [4160, 4000, 65, 0, 3333, 2048]),
    (BF16, 512, 8, 3001, [1159, 0, 700, 31, -5, 4100], [4160] * 6),
])
def test_long_reads_are_the_short_reads(rotations, out_dtype, k_budget, v_bits, n_rows, pos, lens):
    """Reads of which a wave takes several tiles and a head several workgroups, against the same rows in short
    reads."""
    B, H, cap = 6, 6, 4160
    rng = np.random.default_rng(104)
    cfg = bg.Config(1, B, H, 1, cap, k_budget, v_bits, bg.BGTQ_BF16)
    bits = np.stack([[widths_of("uniform" if k_budget == 512 else "mixed", k_budget, rng) for _ in range(H)]])
    layout = bg.Layout(cfg, bits, synth.flat_rot_k(rotations[0]), rotations[1])
    cache = bg.Cache(cfg)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    for t in (cache.k_codes, cache.v_codes):
        t.random_(-2 ** 31, 2 ** 31 - 1, generator=g)
    for t in (cache.k_norms, cache.v_norms):
        t.uniform_(0.3, 3.0, generator=g)
    ctx = None if lens is None else i32(lens)
    shape = (B, n_rows, H, D)
    out = [torch.full(shape, 77.0, dtype=out_dtype, device="cuda") for _ in range(2)]
    bg.blockgtq_dequantize_rows(cfg, layout, 0, cache, i32(pos), n_rows, ctx_len=ctx, k_out=out[0], v_out=out[1])
    for at in range(0, n_rows, 192):
        m = min(192, n_rows - at)
        part = [torch.full((B, m, H, D), 77.0, dtype=out_dtype, device="cuda") for _ in range(2)]
        bg.blockgtq_dequantize_rows(cfg, layout, 0, cache, i32([p + at for p in pos]), m, ctx_len=ctx, k_out=part[0],
                                    v_out=part[1])
        for a, b in zip(out, part):
            assert torch.equal(a[:, at:at + m], b), f"rows {at} .. {at + m - 1}"


# ---------------------------------------------------------------- attention: radii of every size

NARROW, WIDE = (dict(kv=2, group=4), 6), (dict(kv=8, group=4), 1100)  # the second takes the passes with many query rows


@pytest.mark.parametrize("shape,n_q", [NARROW, WIDE])
@pytest.mark.parametrize("value", [2.0 ** -10, 2.0 ** -13, 2.0 ** -16, 2.0 ** 11, "rising", "falling"])
def test_value_radii_of_every_size(rotations, shape, n_q, value):
    """The bound of test_fp32_outputs_in_the_2_norm, 1e-5, holds for small, large and mixed value radii alike.  In bf16
    the output's rounding is 2^-8 of an element at most, and a weight is off by 2^-11, together below 2^-8 + 2^-10 in the
    2-norm (a weight's share of an output row cancels no further than the row itself: the values are independent)."""
    pk = Packed(rotations, 111, cap=640, dtype="fp32", k_budget=192, v_bits=3, **shape)
    t = np.arange(640)
    scale_rows(pk, value={"rising": 2.0 ** (-16 + t // 24), "falling": 2.0 ** (10 - t // 24)}[value]
               if isinstance(value, str) else value)
    assert (bg.cross_workspace_bytes(pk.cfg, 1, n_q, 0, 600) >= n_q * 32 * 512) == (n_q > 100)
    q, qd = pk.queries((1, 1, n_q))
    at = list(range(0, n_q, max(1, n_q // 6)))
    ref, _ = expect_cross(pk, q[:, :, at], [600], FP32)
    for dt, tol in ((FP32, 1e-5), (BF16, 2.0 ** -8 + 2.0 ** -10)):
        for splits in (0, 1, 3):
            out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32([600]), 600, pk.cache, n_splits=splits, out_dtype=dt)
            err = norm_error(out[:, at], ref[0])
            print(f"{n_q} query rows, {dt}, {splits} splits: {err:.3g}", flush=True)
            assert err <= tol, err


@pytest.mark.parametrize("shape,n_q", [NARROW, WIDE])
@pytest.mark.parametrize("key", [2.0 ** -7, 2.0 ** -11, 2.0 ** 9, "rising", "falling"])
def test_key_radii_of_every_size(rotations, shape, n_q, key):
    """Small key radii with large queries and the reverse give the logits of ordinary ones, to the same precision."""
    pk = Packed(rotations, 112, cap=640, dtype="fp32", k_budget=192, v_bits=3, **shape)
    t = np.arange(640)
    # mixed: from 2^-11 to 1, with queries for the largest
    radii = {"rising": 2.0 ** (-11 + np.minimum(t // 48, 11)), "falling": 2.0 ** -(np.minimum(t // 48, 11.0))}[key] \
        if isinstance(key, str) else key
    scale_rows(pk, key=radii)
    q, qd = pk.queries((1, 1, n_q), scale=1.0 if isinstance(key, str) else 1.0 / key)
    at = list(range(0, n_q, max(1, n_q // 6)))
    ref, _ = expect_cross(pk, q[:, :, at], [600], FP32)
    out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32([600]), 600, pk.cache)
    err = norm_error(out[:, at], ref[0])
    print(f"{n_q} query rows: {err:.3g}", flush=True)
    assert err <= 1e-5, err


def test_shared_prefix_with_radii_of_another_size(rotations):
    """Prefix and own rows whose value radii differ by 2^10 either way, in packed and plain workgroups."""
    for batch, kv, prefix_scale, own_scale in ((3, 2, 2.0 ** -12, 2.0 ** -2), (3, 2, 2.0 ** -2, 2.0 ** -12),
                                               (40, 8, 2.0 ** -12, 2.0 ** -2)):
        lens = [(37 * b) % 130 for b in range(batch)]
        kw = dict(kv=kv, group=4, k_budget=192, v_bits=3, dtype="fp32")
        pk = scale_rows(Packed(rotations, 113, batch=batch, cap=192, **kw), value=own_scale)
        pp = scale_rows(Packed(rotations, 114, cap=704, layout_of=pk, **kw), value=prefix_scale)
        q, qd = pk.queries((1, batch))
        ref, _ = expect_shared(pp, pk, q, 700, lens, FP32)
        out = bg.blockgtq_decode_attn_shared(pk.cfg, pk.layout, 0, qd[0], pp.cfg, pp.cache, i32([700]), 700, i32(lens), 130,
                                             pk.cache)
        err = norm_error(out, ref[0])
        print(f"{batch} sequences: {err:.3g}", flush=True)
        assert err <= 1e-5, err


@pytest.mark.parametrize("shape,n_q", [NARROW, WIDE])
@pytest.mark.parametrize("which", ["key", "value"])
def test_an_infinite_radius_reaches_every_query_that_sees_the_row(rotations, shape, n_q, which):
    """By the definition a row with an infinite radius has coordinates that are not finite, and so has every query's
    logit or output, whatever the query's sign: nothing is dropped silently.  Other heads and sequences are untouched."""
    pk = Packed(rotations, 115, batch=2, cap=640, k_budget=192, v_bits=3, **shape)
    q, qd = pk.queries((1, 2, n_q))
    args = (pk.cfg, pk.layout, 0, qd[0], i32([600, 500]), 600, pk.cache)
    for splits in (0, 1, 4):
        before = bg.blockgtq_cross_attn(*args, n_splits=splits)
        if which == "key":
            r = key_radii(pk, 0, 1, 1)
            keep = r[77, 0].clone()
            r[77, 0] = float("inf")
        else:
            r = pk.cache.v_norms[0, 1, 1][:, None]
            keep = r[77, 0].clone()
            r[77, 0] = float("inf")
        out = bg.blockgtq_cross_attn(*args, n_splits=splits)
        r[77, 0] = keep
        assert torch.isnan(out[1, :, 4:8]).all()
        out[1, :, 4:8] = before[1, :, 4:8]
        assert torch.equal(out, before)


# ---------------------------------------------------------------- passes over several layers, every row

@pytest.mark.parametrize("layers,batch,kv,group,tin,tout,n_q,longest", [
    (5, 67, 2, 4, "bf16", "bf16", 1, 200),   # 4 sequences to a workgroup
    (9, 33, 2, 4, "fp32", "fp32", 1, 200),
])
def test_many_short_sequences_of_several_layers(rotations, layers, batch, kv, group, tin, tout, n_q, longest):
    dt = BF16 if tout == "bf16" else FP32
    rng = np.random.default_rng(121)
    lens = [int(x) for x in rng.integers(0, longest + 1, batch)]
    lens[0], lens[1], lens[-1] = longest, 0, 1
    pk = Packed(rotations, 122, layers=layers, batch=batch, kv=kv, group=group, cap=256, dtype=tin, behind=float("nan"),
                lens=lens)
    q, qd = pk.queries((layers, batch, n_q))
    ref, bound = expect_cross(pk, q, lens, dt)
    out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, -1, qd, i32(lens), longest, pk.cache, out_dtype=dt)
    check("all layers", out, ref, bound)


@pytest.mark.parametrize("layers,batch,kv,group,n_q,lens,n_splits", [
    (2, 1, 8, 4, 1100, [577], 0),
    (3, 2, 4, 8, 500, [449, 130], 0),
    (2, 1, 4, 4, 301, [577], 6),
])
def test_many_bf16_query_rows_of_several_layers(rotations, layers, batch, kv, group, n_q, lens, n_splits):
    pk = Packed(rotations, 123, layers=layers, batch=batch, kv=kv, group=group, cap=640, k_budget=192, v_bits=3,
                behind=float("nan"), lens=lens)
    assert bg.cross_workspace_bytes(pk.cfg, layers, n_q, n_splits, max(lens)) >= layers * batch * n_q * kv * group * 512
    q, qd = pk.queries((layers, batch, n_q))
    at = [0, 1, 31, 32, n_q // 2, n_q - 1]
    ref, bound = expect_cross(pk, q[:, :, at], lens, FP32)
    out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, -1, qd, i32(lens), max(lens), pk.cache, n_splits=n_splits)
    check("all layers", out[:, :, at], ref, bound)
    one = bg.blockgtq_cross_attn(pk.cfg, pk.layout, layers - 1, qd[-1], i32(lens), max(lens), pk.cache, n_splits=n_splits)
    check("last layer", one[:, at], ref[-1], bound[-1])


@pytest.mark.parametrize("layers,batch,kv,group,prefix", [(2, 384, 4, 8, 1000), (3, 256, 4, 8, 700)])
def test_shared_prefix_wide_pass_of_several_layers(rotations, layers, batch, kv, group, prefix):
    lens = [(7 * b) % 41 for b in range(batch)]
    kw = dict(layers=layers, kv=kv, group=group, k_budget=192, v_bits=3)
    pk = Packed(rotations, 124, batch=batch, cap=64, **kw)
    pp = Packed(rotations, 125, cap=1024, layout_of=pk, behind=float("inf"), lens=[prefix], **kw)
    rows = layers * batch * kv * group
    assert bg.shared_workspace_bytes(pk.cfg, pp.cfg, layers, 0, prefix, 40) >= rows * (512 + 2 * 528)
    q, qd = pk.queries((layers, batch))
    out = bg.blockgtq_decode_attn_shared(pk.cfg, pk.layout, -1, qd, pp.cfg, pp.cache, i32([prefix]), prefix, i32(lens), 40,
                                         pk.cache, out_dtype=BF16)
    for li in range(layers):
        for b in (0, 1, 15, 16, 31, 32, batch - 1):
            for h in (0, kv - 1):
                hs = slice(group * h, group * h + group)
                k, v = (np.concatenate([getattr(pp, n)[li, 0, h, :prefix], getattr(pk, n)[li, b, h, :lens[b]]]) for n in "kv")
                check(f"layer {li} seq {b} head {h}", out[li, b, hs],
                      *attention_and_bound(q[li, b, hs], k, v, pk.bits[li, h], pk.rot_k, pk.rot_v, BF16))


@pytest.mark.parametrize("tout", ["bf16", "fp32"])
@pytest.mark.parametrize("batch,kv,group,n_q,lens,n_splits", [
    (1, 8, 4, 2048, [513], 0),          # 256 query rows to a workgroup
    (2, 4, 5, 40, [513, 70], 6),        # 128
])
def test_every_row_of_the_wide_passes_is_that_of_the_narrow_ones(rotations, tout, batch, kv, group, n_q, lens, n_splits):
    """Two fp32-grade results differ by 2e-5 of a row's 2-norm at most (1e-5 each); two bf16 roundings by 2^-8 each, and a
    weight's 2^-11 each."""
    dt = BF16 if tout == "bf16" else FP32
    pk = Packed(rotations, 126, batch=batch, kv=kv, group=group, cap=576, k_budget=192, v_bits=3)
    _, qd = pk.queries((batch, n_q))
    assert bg.cross_workspace_bytes(pk.cfg, 1, n_q, n_splits, max(lens)) >= batch * n_q * kv * group * 512
    out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd, i32(lens), max(lens), pk.cache, n_splits=n_splits, out_dtype=dt)
    per = 32 // group
    few = torch.cat([bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[:, i:i + per].contiguous(), i32(lens), max(lens), pk.cache,
                                            out_dtype=dt) for i in range(0, n_q, per)], 1)
    err = float(((out.double() - few.double()).norm(dim=-1) / few.double().norm(dim=-1)).max())
    print(f"{err:.3g}", flush=True)
    assert err <= (2e-5 if dt == FP32 else 2.0 ** -7 + 2.0 ** -10), err
