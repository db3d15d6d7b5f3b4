"""GPU tests of the operators that read the packed cache beside the decode:
rows read back, cross attention and the shared-prefix decode, against plain
formulas in 64 bits.

The caches hold random codes and radii written by the host in the documented
layout, so every code, width and position is under the test's control.

Tolerances, element by element, from the arithmetic alone (u = 2^-24):
 * a sum of n fp32 terms is off by at most n u times the sum of their
   magnitudes; an operand split into fp16 parts by 2^-21 of it, one rounded to
   fp16 by 2^-11; the output's own rounding is half a step (2^-8 of the value in
   bf16, 2^-24 in fp32);
 * logits: the query rotation (128 terms) and the product with the key (128
   terms) give |dx| <= D; weights then move by at most e^(2 D) - 1 relative;
 * a weight in fp16 (bf16 outputs) is off by 2^-11, one in two parts (fp32
   outputs) by 2^-21, or by half of fp16's smallest step.
"""
import math

import numpy as np
import pytest

from oracle import blockgtq_oracle as o
from paper_2606_24033_amd import blockgtq as bg
from paper_2606_24033_amd import synth
from tests import _parity as P

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U = 2.0 ** -24
D = 128


@pytest.fixture(scope="module", autouse=True)
def _require_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bg.lib()


@pytest.fixture(scope="module")
def rotations():
    return synth.rotations(7)


def widths_of(kind, budget, rng):
    """64 block widths that sum to the budget: all equal, or spread over 1 .. 8."""
    if kind == "uniform":
        return np.full(64, budget // 64, dtype=np.uint8)
    b = np.ones(64, dtype=np.int64)
    if kind == "wide":  # every width present, groups of odd block counts
        b[:8] = np.arange(1, 9)
    order = rng.permutation(64)
    i = 0
    while b.sum() < budget:
        j = order[int(64 * rng.random() ** 2)]
        if b[j] < 8:
            b[j] += 1
        i += 1
    return b.astype(np.uint8)


class Packed:
    """A configuration, its layout, a cache of random codes, and the rows it stands for in 64 bits."""

    def __init__(self, rotations, seed, layers=1, batch=1, kv=1, group=4, cap=192, k_budget=128, v_bits=2, kind="mixed",
                 dtype="bf16", behind=None, lens=None, layout_of=None, key_scale=1.0):
        rng = np.random.default_rng([seed, 11])
        self.cfg = bg.Config(n_layers=layers, batch=batch, n_kv_heads=kv, group=group, capacity=cap, k_budget=k_budget,
                             v_bits=v_bits, in_dtype=bg.BGTQ_BF16 if dtype == "bf16" else bg.BGTQ_FP32)
        self.rot_k, self.rot_v = rotations
        if layout_of is None:
            self.bits = np.stack([[widths_of(kind, k_budget, rng) for _ in range(kv)] for _ in range(layers)])
            self.layout = bg.Layout(self.cfg, self.bits, synth.flat_rot_k(self.rot_k), self.rot_v)
        else:
            self.bits, self.layout = layout_of.bits, layout_of.layout
        self.cache = bg.Cache(self.cfg)
        self.k = np.zeros((layers, batch, kv, cap, D))
        self.v = np.zeros_like(self.k)
        host = {n: getattr(self.cache, n).cpu().numpy() for n in ("k_codes", "k_norms", "v_codes", "v_norms")}
        for layer in range(layers):
            for h in range(kv):
                w = P.stream_widths(self.bits[layer, h])
                ng = len(o.groups(self.bits[layer, h]))
                slots = ng + (ng & 1)
                for b in range(batch):
                    codes = np.stack([rng.integers(0, 1 << int(x), cap) for x in w], 1)
                    kn = (key_scale * rng.uniform(0.3, 3.0, (cap, ng))).astype(np.float16).astype(np.float64)
                    vcodes = rng.integers(0, 1 << v_bits, (cap, D))
                    vn = rng.uniform(5.0, 17.0, cap).astype(np.float16).astype(np.float64)
                    self.k[layer, b, h] = o.dequantize_keys(codes, kn, self.bits[layer, h], self.rot_k)
                    self.v[layer, b, h] = o.dequantize_values(vcodes, vn, self.rot_v, v_bits)
                    if behind is not None:  # what lies behind a sequence's rows
                        kn[lens[b]:] = behind
                        vn[lens[b]:] = behind
                    host["k_codes"][layer, b, h] = o.pack_key_rows(codes, w).view(np.int32)
                    host["v_codes"][layer, b, h] = o.pack_value_tiles(vcodes, v_bits).reshape(cap // 32, D, v_bits).view(np.int32)
                    wide = np.zeros((cap, slots))
                    wide[:, :ng] = kn
                    host["k_norms"][layer, b, h, :cap * slots] = wide.reshape(-1)
                    host["v_norms"][layer, b, h] = vn
        for n, a in host.items():
            getattr(self.cache, n).copy_(torch.from_numpy(a))
        self.rng = rng

    def queries(self, shape, scale=1.0):
        q = synth.cast(scale * self.rng.standard_normal(shape + (self.cfg.n_q_heads, D)),
                       "bf16" if self.cfg.in_dtype == bg.BGTQ_BF16 else "fp32")
        t = torch.float32 if self.cfg.in_dtype == bg.BGTQ_FP32 else torch.bfloat16
        return q.astype(np.float64), torch.from_numpy(q).to(t).cuda()


def attention_and_bound(q, k, v, bits, rot_k, rot_v, out_dtype):
    """Attention of the rows q [n, 128] to k, v [T, 128] in 64 bits, and how far a kernel's output may be off."""
    if len(k) == 0:
        return np.zeros(q.shape), np.zeros(q.shape)
    x = q @ k.T / math.sqrt(D)
    e = np.exp(x - x.max(1, keepdims=True))
    p = e / e.sum(1, keepdims=True)
    ref = p @ v
    # logits: rotated operands, their magnitudes
    w = np.zeros((D, D))
    at = 0
    for _, dims in o.groups(bits):
        w[np.ix_(range(at, at + len(dims)), dims)] = rot_k[len(dims)]
        at += len(dims)
    qa, kr, qr = np.abs(q) @ np.abs(w).T, np.abs(k @ w.T), np.abs(q @ w.T)
    dx = ((136 * U * qa + (144 * U + 2.0 ** -20) * qr) @ kr.T) / math.sqrt(D) + 4 * U * np.abs(x - x.max(1, keepdims=True))
    move = np.expm1(2 * dx.max(1, keepdims=True))
    spread = p @ np.abs(v) + np.abs(ref)
    y = np.abs(v @ rot_v.T)
    weight = 2.0 ** -11 if out_dtype == torch.bfloat16 else 2.0 ** -21
    total = ((len(k) + 64) * U + weight + 8 * U) * (p @ y) + 132 * U * (p @ y)
    # weights below fp16's normal range: half its smallest step each, times a centroid below 5
    total = total + len(k) * 2.0 ** -25 * 5 / math.sqrt(D) / np.maximum(1.0, e.sum(1, keepdims=True))
    rounding = 2.0 ** -8 if out_dtype == torch.bfloat16 else U
    return ref, move * spread + total @ np.abs(rot_v) + rounding * np.abs(ref) + 1e-30


def check(what, got, ref, bound):
    off = np.abs(got.double().cpu().numpy() - ref)
    assert off.shape == bound.shape
    i = np.unravel_index(np.argmax(off - bound), off.shape)
    print(f"{what}: max err {off.max():.3g}, share of the bound {float(np.max(off / np.maximum(bound, 1e-30))):.3g}", flush=True)
    assert (off <= bound).all(), f"{what}: {int((off > bound).sum())} elements off, e.g. {off[i]:.3g} > {bound[i]:.3g} at {i}"


def expect_cross(pk, q, lens, out_dtype, layers=None):
    """Reference and bound of a call: q [L, B, n_q, Hq, 128]."""
    ref, bound = np.zeros(q.shape), np.zeros(q.shape)
    for li, layer in enumerate(layers if layers is not None else range(pk.cfg.n_layers)):
        for b in range(pk.cfg.batch):
            for h in range(pk.cfg.n_kv_heads):
                hs = slice(h * pk.cfg.group, (h + 1) * pk.cfg.group)
                rows = q[li, b, :, hs].reshape(-1, D)
                r, t = attention_and_bound(rows, pk.k[layer, b, h, :lens[b]], pk.v[layer, b, h, :lens[b]],
                                           pk.bits[layer, h], pk.rot_k, pk.rot_v, out_dtype)
                ref[li, b, :, hs], bound[li, b, :, hs] = (a.reshape(-1, pk.cfg.group, D) for a in (r, t))
    return ref, bound


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- rows read back

def expect_rows(pk, layer, b, h, which, pos, n, out_dtype):
    x = (pk.k if which == "k" else pk.v)[layer, b, h, pos:pos + n]
    if which == "k":
        total = np.zeros(x.shape)
        for _, dims in o.groups(pk.bits[layer, h]):
            rot = pk.rot_k[len(dims)]
            total[:, dims] = np.abs(x[:, dims] @ rot.T) @ np.abs(rot)
    else:
        total = np.abs(x @ pk.rot_v.T) @ np.abs(pk.rot_v)
    if out_dtype == torch.bfloat16:
        return x, 2.0 ** -8 * np.abs(x) + (2 * 2.0 ** -11 + 2.0 ** -20 + 136 * U) * total
    return x, U * np.abs(x) + (2.0 ** -21 + 140 * U) * total


@pytest.mark.parametrize("layers,batch,kv,k_budget,v_bits,kind,out_dtype,n_rows,pos,lens", [
    (1, 1, 1, 128, 2, "mixed", "fp32", 1, [0], None),
    (1, 1, 2, 192, 3, "wide", "bf16", 64, [64], None),
    (1, 2, 1, 192, 1, "wide", "fp32", 100, [3, 37], [90, 192]),
    (3, 2, 2, 128, 4, "uniform", "bf16", 17, [40, 0], [50, 5]),
    (1, 3, 1, 256, 5, "wide", "fp32", 70, [150, -9, 192], None),
    (2, 1, 1, 512, 8, "uniform", "fp32", 33, [31], [60]),
    (1, 1, 3, 64, 6, "uniform", "bf16", 192, [0], [192]),
    (1, 2, 1, 320, 7, "wide", "bf16", 40, [10, 20], [0, -5]),
    (2, 3, 2, 192, 2, "mixed", "fp32", 129, [1, 63, 100], [192, 64, 101]),
])
def test_dequantize_rows(rotations, layers, batch, kv, k_budget, v_bits, kind, out_dtype, n_rows, pos, lens):
    dt = torch.bfloat16 if out_dtype == "bf16" else torch.float32
    pk = Packed(rotations, 5, layers=layers, batch=batch, kv=kv, k_budget=k_budget, v_bits=v_bits, kind=kind)
    layer = -1 if layers > 1 else 0
    shape = ((layers,) if layers > 1 else ()) + (batch, n_rows, kv, D)
    for which in ("kv", "k", "v"):
        out = {n: torch.full(shape, 77.0, dtype=dt, device="cuda") for n in "kv"}
        bg.blockgtq_dequantize_rows(pk.cfg, pk.layout, layer, pk.cache, i32(pos), n_rows,
                                    ctx_len=None if lens is None else i32(lens),
                                    k_out=out["k"] if "k" in which else None, v_out=out["v"] if "v" in which else None)
        torch.cuda.synchronize()
        for n in "kv":
            got = out[n].view((layers, batch, n_rows, kv, D))
            for b in range(batch):
                end = min(pk.cfg.capacity, pk.cfg.capacity if lens is None else lens[b])
                keep = np.array([0 <= pos[b] + i < end for i in range(n_rows)])
                if n not in which:
                    keep[:] = False
                assert (got[:, b, torch.from_numpy(~keep).cuda()] == 77.0).all(), "a row that is not read was written"
                if keep.any():
                    i0, m = int(np.argmax(keep)), int(keep.sum())
                    for li in range(layers):
                        for h in range(kv):
                            ref, bound = expect_rows(pk, li, b, h, n, pos[b] + i0, m, dt)
                            check(f"{which}.{n} layer {li} seq {b} head {h}", got[li, b, i0:i0 + m, h], ref, bound)


def test_dequantize_one_layer_and_allocation(rotations):
    pk = Packed(rotations, 6, layers=3, batch=2, kv=2, k_budget=192, v_bits=3, kind="wide")
    k, v = bg.blockgtq_dequantize_rows(pk.cfg, pk.layout, 1, pk.cache, i32([5, 6]), 20, ctx_len=i32([9, 192]))
    assert k.shape == v.shape == (2, 20, 2, D) and k.dtype == torch.float32
    assert (k[0, 4:] == 0).all() and (v[0, 4:] == 0).all()
    for h in range(2):
        check("k", k[1, :, h], *expect_rows(pk, 1, 1, h, "k", 6, 20, torch.float32))
        check("v", v[1, :, h], *expect_rows(pk, 1, 1, h, "v", 6, 20, torch.float32))
    assert bg.blockgtq_dequantize_rows(pk.cfg, pk.layout, 1, pk.cache, i32([0, 0]), 0)[0].numel() == 0


@pytest.mark.parametrize("seed", range(6))
def test_dequantize_fp32_rounding_errors_are_independent(seed):
    """In the 2-norm.  An fp32 sum of 128 terms of one size: the k-th partial sum is about sqrt(k / 128) of the result,
    and its rounding at most u of that, uniformly: u sqrt(64 / 3) = 2.8e-7 of the result together.  Operands in two
    fp16 parts: 2^-22 / sqrt(3) each at most, two of them: 2e-7.  2^-20 = 9.5e-7 is about three times that; one matrix
    entry of 16384 with a wrong low part (2^-11 of it) is 2^-11 / 128 = 3.8e-6 or more in a dim's column."""
    rot = synth.rotations(seed)
    pk = Packed(rot, 60 + seed, batch=1, kv=2, cap=192, k_budget=192, v_bits=3, kind="uniform" if seed % 2 else "mixed")
    k, v = bg.blockgtq_dequantize_rows(pk.cfg, pk.layout, 0, pk.cache, i32([0]), 192)
    for name, got, ref in (("k", k, pk.k), ("v", v, pk.v)):
        off = np.moveaxis(got[0].double().cpu().numpy(), 1, 0) - ref[0, 0]
        err = np.linalg.norm(off, axis=1) / np.linalg.norm(ref[0, 0], axis=1)  # by head and dim
        print(f"{name}: {err.max():.3g}", flush=True)
        assert (err <= 2.0 ** -20).all(), f"{name}: {err.max():.3g} at {np.argwhere(err > 2.0 ** -20)[:5]}"


def test_dequantize_not_a_number_stays_in_its_row(rotations):
    pk = Packed(rotations, 8, cap=128, behind=float("nan"), lens=[70])
    k, v = bg.blockgtq_dequantize_rows(pk.cfg, pk.layout, 0, pk.cache, i32([0]), 128, out_dtype=torch.bfloat16)
    assert torch.isfinite(k[:, :70]).all() and torch.isfinite(v[:, :70]).all()
    assert torch.isnan(k[:, 70:]).all() and torch.isnan(v[:, 70:]).all()


# ---------------------------------------------------------------- cross attention

CROSS = [
    # layers, batch, kv, group, k_budget, v_bits, kind, in, out, n_q, lens, cap, n_splits
    (1, 1, 1, 1, 128, 2, "mixed", "bf16", "bf16", 1, [1], 64, 0),
    (1, 1, 1, 4, 128, 2, "mixed", "fp32", "fp32", 1, [64], 64, 0),
    (1, 2, 2, 4, 192, 3, "wide", "bf16", "bf16", 1, [65, 0], 128, 0),
    (1, 3, 1, 8, 192, 3, "mixed", "bf16", "fp32", 5, [63, 129, 191], 192, 0),
    (1, 1, 2, 3, 64, 1, "uniform", "bf16", "bf16", 11, [100], 128, 0),
    (1, 2, 1, 7, 256, 4, "wide", "fp32", "fp32", 9, [256, 31], 256, 3),
    (1, 1, 1, 5, 320, 5, "wide", "fp32", "bf16", 33, [200], 256, 0),
    (1, 1, 1, 6, 448, 6, "wide", "bf16", "fp32", 17, [700], 704, 2),
    (2, 2, 2, 4, 128, 7, "mixed", "bf16", "bf16", 8, [150, 77], 192, 0),
    (1, 1, 2, 8, 512, 8, "uniform", "bf16", "bf16", 70, [129], 192, 1),
    (3, 1, 2, 2, 192, 2, "wide", "fp32", "fp32", 2, [40], 64, 4),
    (1, 1, 1, 4, 128, 2, "uniform", "bf16", "fp32", 300, [1100], 1152, 0),
    (1, 4, 1, 1, 192, 3, "mixed", "bf16", "bf16", 260, [5, 64, 300, 448], 448, 0),
    (1, 1, 1, 8, 128, 2, "mixed", "bf16", "bf16", 3, [5000], 5056, 0),
]


@pytest.mark.parametrize("layers,batch,kv,group,k_budget,v_bits,kind,tin,tout,n_q,lens,cap,n_splits", CROSS)
def test_cross_attention(rotations, layers, batch, kv, group, k_budget, v_bits, kind, tin, tout, n_q, lens, cap, n_splits):
    dt = torch.bfloat16 if tout == "bf16" else torch.float32
    pk = Packed(rotations, 21, layers=layers, batch=batch, kv=kv, group=group, cap=cap, k_budget=k_budget, v_bits=v_bits,
                kind=kind, dtype=tin)
    q, qd = pk.queries((layers, batch, n_q))
    ref, bound = expect_cross(pk, q, lens, dt)
    if layers > 1:
        out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, -1, qd, i32(lens), max(lens), pk.cache, n_splits=n_splits, out_dtype=dt)
        check("all layers", out, ref, bound)
        one = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 1, qd[1], i32(lens), max(lens), pk.cache, n_splits=n_splits, out_dtype=dt)
        check("layer 1", one, ref[1], bound[1])
    else:
        out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32(lens), max(lens), pk.cache, n_splits=n_splits, out_dtype=dt)
        check("one layer", out, ref[0], bound[0])
        # a looser bound on the lengths changes the splits, not the result
        out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32(lens), cap, pk.cache, out_dtype=dt)
        check("max_ctx = capacity", out, ref[0], bound[0])


@pytest.mark.parametrize("behind", [float("nan"), float("inf"), 65504.0])
def test_cross_rows_behind_the_last_do_not_enter(rotations, behind):
    lens = [70, 1, 64]
    for dt in (torch.float32, torch.bfloat16):
        pk = Packed(rotations, 22, batch=3, cap=128, behind=behind, lens=lens)
        q, qd = pk.queries((1, 3, 20))
        ref, bound = expect_cross(pk, q, lens, dt)
        out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32(lens), 128, pk.cache, out_dtype=dt)
        check(f"behind {behind}", out, ref[0], bound[0])


def test_cross_lengths_outside_the_bound(rotations):
    """A length the host could not check makes its sequence NaN, and only that one."""
    pk = Packed(rotations, 23, batch=4, cap=128)
    q, qd = pk.queries((1, 4, 3))
    ref, bound = expect_cross(pk, q, [100, 0, 64, 7], torch.float32)
    out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32([100, -1, 101, 7]), 100, pk.cache)
    assert torch.isnan(out[1]).all() and torch.isnan(out[2]).all()
    for b in (0, 3):
        check(f"seq {b}", out[b], ref[0, b], bound[0, b])
    none = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32([0, 0, 0, 0]), 0, pk.cache, out_dtype=torch.bfloat16)
    assert (none == 0).all()
    assert bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0][:, :0].contiguous(), i32([0] * 4), 9, pk.cache).numel() == 0


def test_cross_large_and_small_logits(rotations):
    """Queries of very different sizes in one call: peaked and flat rows, tiny and huge rotated queries."""
    pk = Packed(rotations, 24, group=2, cap=192, dtype="fp32", key_scale=4.0)
    q, _ = pk.queries((1, 1, 40))
    q *= 10.0 ** np.linspace(-6, 1.5, 40)[None, None, :, None, None]
    q = q.astype(np.float32).astype(np.float64)
    ref, bound = expect_cross(pk, q, [150], torch.float32)
    qd = torch.from_numpy(q.astype(np.float32)).cuda()
    check("sizes", bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32([150]), 150, pk.cache), ref[0], bound[0])
    qd[0, 0, 3] = float("nan")
    out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32([150]), 150, pk.cache)
    assert torch.isnan(out[0, 3]).all()
    rest = [i for i in range(40) if i != 3]
    check("beside a NaN query", out[0, rest], ref[0, 0, rest], bound[0, 0, rest])


def test_cross_one_query_row_is_the_decode(rotations):
    pk = Packed(rotations, 25, batch=3, kv=2, group=8, k_budget=192, v_bits=3, cap=704)
    q, qd = pk.queries((3,))
    lens = [700, 1, 333]
    a = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[:, None], i32(lens), 700, pk.cache)[:, 0]
    b = bg.blockgtq_decode_attn(pk.cfg, pk.layout, 0, qd, i32(lens), 700, pk.cache)
    err = P.rel_err(a.double().cpu().numpy(), b.double().cpu().numpy())
    assert err <= P.tol_attention(), err


# ---------------------------------------------------------------- sequences that share a workgroup

PACKED = [
    # layers, batch, kv, group, k_budget, v_bits, kind, in, out, n_q, longest, n_splits: batches large enough that 2, 4 or 8
    # sequences share a workgroup, some of them not full
    (1, 65, 8, 4, 128, 2, "mixed", "bf16", "bf16", 1, 100, 0),     # 4 sequences
    (1, 67, 8, 4, 192, 3, "wide", "fp32", "fp32", 1, 300, 0),      # 2
    (1, 259, 4, 4, 128, 2, "uniform", "bf16", "fp32", 1, 300, 0),  # 8
    (9, 9, 2, 4, 128, 4, "mixed", "fp32", "bf16", 1, 200, 0),
    (1, 133, 4, 3, 320, 5, "wide", "bf16", "fp32", 3, 130, 0),     # 9 query rows a sequence: 2
    (1, 140, 4, 1, 512, 8, "uniform", "fp32", "fp32", 4, 200, 0),
    (1, 131, 4, 8, 256, 1, "mixed", "bf16", "bf16", 1, 500, 3),
    (1, 131, 4, 5, 192, 7, "mixed", "bf16", "fp32", 1, 500, 2),
]


@pytest.mark.parametrize("layers,batch,kv,group,k_budget,v_bits,kind,tin,tout,n_q,longest,n_splits", PACKED)
def test_cross_attention_of_many_short_sequences(rotations, layers, batch, kv, group, k_budget, v_bits, kind, tin, tout, n_q,
                                                 longest, n_splits):
    dt = torch.bfloat16 if tout == "bf16" else torch.float32
    rng = np.random.default_rng(91)
    lens = [int(x) for x in rng.integers(0, longest + 1, batch)]
    lens[0], lens[1], lens[-1], lens[5] = longest, 0, 64, 1
    cap = (longest + 63) // 64 * 64
    pk = Packed(rotations, 92, layers=layers, batch=batch, kv=kv, group=group, cap=cap, k_budget=k_budget, v_bits=v_bits,
                kind=kind, dtype=tin, behind=float("inf"), lens=lens)
    q, qd = pk.queries((layers, batch, n_q))
    bad = {2: -1, 6: longest + 1, batch - 2: 1 << 30}
    dev = i32([bad.get(b, n) for b, n in enumerate(lens)])
    qd[0, 7, 0, 0] = float("nan")
    ref, bound = expect_cross(pk, q, lens, dt)
    if layers > 1:
        out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, -1, qd, dev, longest, pk.cache, n_splits=n_splits, out_dtype=dt)
    else:
        out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], dev, longest, pk.cache, n_splits=n_splits, out_dtype=dt)[None]
    assert all(torch.isnan(out[:, b]).all() for b in bad) and (out[:, 1] == 0).all()
    if lens[7]:
        assert torch.isnan(out[0, 7, 0, 0]).all()
    out[0, 7, 0, 0] = 0
    ref[0, 7, 0, 0] = 0
    good = [b for b in range(batch) if b not in bad]
    check("good rows", out[:, good], ref[:, good], bound[:, good])


# ---------------------------------------------------------------- many query rows

WIDE = [
    # layers, batch, kv, group, k_budget, v_bits, kind, in, out, n_q, lens, cap, n_splits; sizes that take the passes with
    # 128 or 256 query rows to a workgroup (the workspace then holds the rotated queries)
    (1, 1, 8, 4, 128, 2, "mixed", "bf16", "bf16", 2048, [515], 576, 0),
    (1, 1, 8, 4, 192, 3, "wide", "bf16", "fp32", 2048, [512], 512, 0),
    (1, 1, 2, 8, 192, 3, "mixed", "bf16", "bf16", 2048, [513], 576, 0),
    (1, 1, 2, 8, 128, 4, "wide", "fp32", "fp32", 2047, [449], 512, 0),
    (2, 1, 2, 8, 128, 2, "mixed", "fp32", "fp32", 1500, [576], 576, 0),
    (1, 3, 4, 8, 256, 1, "uniform", "bf16", "fp32", 1001, [600, 0, 64], 640, 0),
    (1, 2, 8, 4, 320, 7, "wide", "bf16", "bf16", 1100, [577, 250], 640, 3),
    (1, 2, 8, 4, 512, 8, "uniform", "fp32", "fp32", 1100, [300, 577], 640, 2),
    (1, 1, 8, 5, 448, 6, "wide", "bf16", "bf16", 1700, [700], 704, 2),
    (1, 1, 8, 3, 128, 5, "mixed", "bf16", "fp32", 2731, [640], 640, 2),
    (1, 2, 2, 1, 128, 2, "wide", "fp32", "fp32", 400, [513, 70], 576, 6),
    (1, 2, 4, 5, 192, 3, "mixed", "bf16", "bf16", 40, [513, 0], 576, 6),
    (1, 2, 2, 4, 256, 1, "uniform", "bf16", "bf16", 100, [1, 513], 576, 6),
    (1, 1, 4, 3, 512, 8, "uniform", "fp32", "fp32", 150, [640], 640, 6),
]


@pytest.mark.parametrize("layers,batch,kv,group,k_budget,v_bits,kind,tin,tout,n_q,lens,cap,n_splits", WIDE)
def test_cross_attention_of_many_query_rows(rotations, layers, batch, kv, group, k_budget, v_bits, kind, tin, tout, n_q,
                                            lens, cap, n_splits):
    dt = torch.bfloat16 if tout == "bf16" else torch.float32
    pk = Packed(rotations, 71, layers=layers, batch=batch, kv=kv, group=group, cap=cap, k_budget=k_budget, v_bits=v_bits,
                kind=kind, dtype=tin, behind=float("nan"), lens=lens)
    assert bg.cross_workspace_bytes(pk.cfg, layers, n_q, n_splits, max(lens)) >= layers * batch * n_q * kv * group * 512
    q, qd = pk.queries((layers, batch, n_q))
    # positions whose rows are compared: the ends, the edges of workgroups, and some between
    at = sorted({0, 1, n_q - 1, *(min(n_q - 1, (r + d) // group) for r in (32, 128, 256, 512) for d in (-1, 0)),
                 *(int(i) for i in np.random.default_rng(3).integers(0, n_q, 9))})
    ref, bound = expect_cross(pk, q[:, :, at], lens, dt)
    if layers > 1:
        out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, -1, qd, i32(lens), max(lens), pk.cache, n_splits=n_splits, out_dtype=dt)
    else:
        out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32(lens), max(lens), pk.cache, n_splits=n_splits,
                                     out_dtype=dt)[None]
    check("compared rows", out[:, :, at], ref, bound)
    if dt == torch.float32:  # every other row against the 32-row passes (a few query rows to a call)
        few = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0, :, :7].contiguous(), i32(lens), max(lens), pk.cache)
        err = float((out[0, :, :7] - few).norm() / few.norm())
        assert err <= 1e-5, err


def test_many_query_rows_lengths_outside_the_bound_and_odd_queries(rotations):
    pk = Packed(rotations, 72, batch=4, kv=8, group=4, cap=640, dtype="fp32")
    lens, n_q = [600, 601, -3, 0], 600
    assert bg.cross_workspace_bytes(pk.cfg, 1, n_q, 0, 600) >= 4 * n_q * 32 * 512
    q, qd = pk.queries((1, 4, n_q))
    q[0, 0, 5] *= 1e-6
    q[0, 0, 6] *= 30.0
    q = q.astype(np.float32).astype(np.float64)
    qd = torch.from_numpy(q.astype(np.float32)).cuda()
    qd[0, 0, 9] = float("nan")
    out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32(lens), 600, pk.cache)
    assert torch.isnan(out[1]).all() and torch.isnan(out[2]).all() and (out[3] == 0).all() and torch.isnan(out[0, 9]).all()
    at = [0, 5, 6, 8, 10, 599]
    ref, bound = expect_cross(pk, q[:, :, at], [600, 0, 0, 0], torch.float32)
    check("seq 0", out[0, at], ref[0, 0], bound[0, 0])


def test_fp32_outputs_in_the_2_norm(rotations):
    """The worst-case bounds above are far from what independent roundings do.  A logit of size |x| is off by about
    2^-23 sqrt(sum of squared terms) from the operands' parts and the fp32 sums, below 2^-21 here (rotated terms of
    about 1, logits up to about 30: 30 2^-23 at the most from the scaling and the exponential's argument), a weight by
    as much again, so an output by less than 1e-5 of its size."""
    for shape, n_q in ((dict(kv=2, group=4), 6), (dict(kv=8, group=4), 1100)):
        pk = Packed(rotations, 73, cap=640, dtype="fp32", k_budget=192, v_bits=3, **shape)
        q, qd = pk.queries((1, 1, n_q))
        out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], i32([600]), 600, pk.cache)
        at = list(range(0, n_q, max(1, n_q // 6)))
        ref, _ = expect_cross(pk, q[:, :, at], [600], torch.float32)
        err = np.linalg.norm(out[:, at].double().cpu().numpy() - ref[0]) / np.linalg.norm(ref)
        print(f"{n_q} query rows: {err:.3g}", flush=True)
        assert err <= 1e-5, err


# ---------------------------------------------------------------- shared prefix

SHARED = [
    # layers, batch, kv, group, k_budget, v_bits, kind, in, out, prefix, lens, n_splits
    (1, 1, 1, 4, 128, 2, "mixed", "bf16", "bf16", 1, [0], 0),
    (1, 1, 1, 1, 128, 2, "mixed", "fp32", "fp32", 0, [1], 0),
    (1, 3, 2, 4, 192, 3, "wide", "bf16", "bf16", 130, [0, 64, 65], 0),
    (1, 5, 1, 8, 192, 2, "mixed", "bf16", "fp32", 600, [1, 2, 63, 129, 190], 3),
    (2, 9, 2, 4, 128, 2, "mixed", "bf16", "bf16", 64, [3] * 9, 0),
    (1, 33, 1, 4, 256, 4, "uniform", "fp32", "fp32", 257, list(range(33)), 0),
    (3, 2, 1, 6, 320, 5, "wide", "fp32", "fp32", 99, [40, 0], 2),
    (1, 64, 1, 2, 64, 1, "uniform", "bf16", "bf16", 1000, [7] * 64, 0),
    (1, 4, 1, 3, 512, 8, "uniform", "bf16", "bf16", 0, [0, 0, 5, 100], 0),
]


def expect_shared(pp, pk, q, prefix, lens, dt):
    ref, bound = np.zeros(q.shape), np.zeros(q.shape)
    for li in range(pk.cfg.n_layers):
        for b in range(pk.cfg.batch):
            for h in range(pk.cfg.n_kv_heads):
                hs = slice(h * pk.cfg.group, (h + 1) * pk.cfg.group)
                k, v = (np.concatenate([getattr(pp, n)[li, 0, h, :prefix], getattr(pk, n)[li, b, h, :lens[b]]]) for n in "kv")
                ref[li, b, hs], bound[li, b, hs] = attention_and_bound(q[li, b, hs], k, v, pk.bits[li, h], pk.rot_k,
                                                                       pk.rot_v, dt)
    return ref, bound


@pytest.mark.parametrize("layers,batch,kv,group,k_budget,v_bits,kind,tin,tout,prefix,lens,n_splits", SHARED)
def test_shared_prefix_decode(rotations, layers, batch, kv, group, k_budget, v_bits, kind, tin, tout, prefix, lens, n_splits):
    dt = torch.bfloat16 if tout == "bf16" else torch.float32
    kw = dict(layers=layers, kv=kv, group=group, k_budget=k_budget, v_bits=v_bits, kind=kind, dtype=tin)
    pk = Packed(rotations, 31, batch=batch, cap=192, behind=float("nan"), lens=lens, **kw)
    pp = Packed(rotations, 32, batch=1, cap=(prefix + 64) // 64 * 64, behind=float("inf"), lens=[prefix], layout_of=pk, **kw)
    q, qd = pk.queries((layers, batch))
    ref, bound = expect_shared(pp, pk, q, prefix, lens, dt)
    args = (pp.cfg, pp.cache, i32([prefix]), prefix, i32(lens), max(lens), pk.cache)
    if layers > 1:
        out = bg.blockgtq_decode_attn_shared(pk.cfg, pk.layout, -1, qd, *args, n_splits=n_splits, out_dtype=dt)
        check("all layers", out, ref, bound)
    one = bg.blockgtq_decode_attn_shared(pk.cfg, pk.layout, layers - 1, qd[-1], *args, n_splits=n_splits, out_dtype=dt)
    check("one layer", one, ref[-1], bound[-1])


@pytest.mark.parametrize("tout", ["bf16", "fp32"])
def test_shared_prefix_wide_pass(rotations, tout):
    """A batch and a prefix large enough for the passes with many query rows to a workgroup."""
    dt = torch.bfloat16 if tout == "bf16" else torch.float32
    batch, prefix = 384, 1000
    lens = [(7 * b) % 41 for b in range(batch)]
    kw = dict(kv=8, group=8, k_budget=192, v_bits=3)
    pk = Packed(rotations, 35, batch=batch, cap=64, **kw)
    pp = Packed(rotations, 36, cap=1024, layout_of=pk, behind=float("nan"), lens=[prefix], **kw)
    assert bg.shared_workspace_bytes(pk.cfg, pp.cfg, 1, 0, prefix, 40) >= batch * 64 * (512 + 3 * 528)
    q, qd = pk.queries((1, batch))
    out = bg.blockgtq_decode_attn_shared(pk.cfg, pk.layout, 0, qd[0], pp.cfg, pp.cache, i32([prefix]), prefix, i32(lens), 40,
                                         pk.cache, out_dtype=dt)
    for b in (0, 1, 15, 16, 31, 32, 300, 383):
        for h in (0, 7):
            hs = slice(8 * h, 8 * h + 8)
            k, v = (np.concatenate([getattr(pp, n)[0, 0, h, :prefix], getattr(pk, n)[0, b, h, :lens[b]]]) for n in "kv")
            check(f"seq {b} head {h}", out[b, hs], *attention_and_bound(q[0, b, hs], k, v, pk.bits[0, h], pk.rot_k, pk.rot_v, dt))


@pytest.mark.parametrize("layers,batch,kv,group,prefix,longest", [(1, 40, 8, 4, 500, 200), (4, 17, 8, 4, 300, 130),
                                                                  (1, 70, 4, 8, 700, 320)])
def test_shared_prefix_of_many_short_sequences(rotations, layers, batch, kv, group, prefix, longest):
    """The sequences' own rows in workgroups of several sequences, in one launch with the prefix's."""
    rng = np.random.default_rng(37)
    lens = [int(x) for x in rng.integers(0, longest + 1, batch)]
    lens[0], lens[1], lens[-1] = longest, 0, 1
    kw = dict(layers=layers, kv=kv, group=group)
    pk = Packed(rotations, 38, batch=batch, cap=320, behind=float("nan"), lens=lens, **kw)
    pp = Packed(rotations, 39, cap=704, layout_of=pk, behind=float("inf"), lens=[prefix], **kw)
    q, qd = pk.queries((layers, batch))
    dev = i32([longest + 1 if b == 4 else n for b, n in enumerate(lens)])
    out = bg.blockgtq_decode_attn_shared(pk.cfg, pk.layout, -1, qd, pp.cfg, pp.cache, i32([prefix]), prefix, dev, longest,
                                         pk.cache, out_dtype=torch.bfloat16)
    assert torch.isnan(out[:, 4]).all()
    for li in range(layers):
        for b in range(batch):
            for h in (0, kv - 1):
                if b == 4:
                    continue
                hs = slice(group * h, group * h + group)
                k, v = (np.concatenate([getattr(pp, n)[li, 0, h, :prefix], getattr(pk, n)[li, b, h, :lens[b]]]) for n in "kv")
                ref, bound = attention_and_bound(q[li, b, hs], k, v, pk.bits[li, h], pk.rot_k, pk.rot_v, torch.bfloat16)
                off = np.abs(out[li, b, hs].double().cpu().numpy() - ref)
                assert (off <= bound).all(), (li, b, h, float((off / bound).max()))


def test_shared_lengths_outside_the_bound(rotations):
    pk = Packed(rotations, 33, batch=3, cap=64)
    pp = Packed(rotations, 34, cap=128, layout_of=pk)
    q, qd = pk.queries((1, 3))
    out = bg.blockgtq_decode_attn_shared(pk.cfg, pk.layout, 0, qd[0], pp.cfg, pp.cache, i32([90]), 90, i32([4, 65, -2]), 64,
                                         pk.cache)
    ref, bound = expect_shared(pp, pk, q, 90, [4, 0, 0], torch.float32)
    check("seq 0", out[0], ref[0, 0], bound[0, 0])
    assert torch.isnan(out[1:]).all()
    for bad in (91, -1):
        out = bg.blockgtq_decode_attn_shared(pk.cfg, pk.layout, 0, qd[0], pp.cfg, pp.cache, i32([bad]), 90, i32([4, 5, 6]),
                                             64, pk.cache)
        assert torch.isnan(out).all()


# ---------------------------------------------------------------- long caches

def test_rows_beyond_32_bit_offsets(rotations):
    """Rows whose codes lie more than 2^32 bytes into the cache: read back, attended, and as a prefix.  The cache is
    zero (radius 0: logit 0, value 0) but for its last rows, whose keys are the query's own direction with logits far
    above ln(rows): they alone carry the output."""
    cap = (1 << 27) + (1 << 23)
    small = Packed(rotations, 81, cap=64, group=2, k_budget=128, v_bits=2, kind="uniform", dtype="fp32")
    cfg = bg.Config(1, 1, 1, 2, cap, 128, 2, bg.BGTQ_FP32)
    cache = bg.Cache(cfg)
    n0 = cap - 64
    assert n0 * 32 > 1 << 32
    rng = np.random.default_rng(82)
    d = rng.standard_normal(D)
    x = torch.from_numpy((40.0 * d + rng.standard_normal((1, 64, 1, D))).astype(np.float32)).cuda()
    v = torch.from_numpy(rng.standard_normal((1, 64, 1, D)).astype(np.float32)).cuda()
    bg.blockgtq_quantize_append(cfg, small.layout, 0, x, v, i32([n0]), cache)
    tail, head = bg.Cache(small.cfg), i32([0])
    bg.blockgtq_quantize_append(small.cfg, small.layout, 0, x, v, head, tail)
    near = bg.blockgtq_dequantize_rows(small.cfg, small.layout, 0, tail, head, 64)
    far = bg.blockgtq_dequantize_rows(cfg, small.layout, 0, cache, i32([n0]), 64)
    assert all(torch.equal(a, b) for a, b in zip(near, far))
    q = torch.from_numpy((d + 0.1 * rng.standard_normal((1, 1, 2, D))).astype(np.float32)).cuda()
    want = bg.blockgtq_cross_attn(small.cfg, small.layout, 0, q, i32([64]), 64, tail)
    got = bg.blockgtq_cross_attn(cfg, small.layout, 0, q, i32([cap]), cap, cache)
    assert float((got - want).abs().max()) <= 1e-5 * float(want.abs().max())
    empty = bg.Cache(small.cfg)
    got = bg.blockgtq_decode_attn_shared(small.cfg, small.layout, 0, q[:, 0].contiguous(), cfg, cache, i32([cap]), cap, i32([0]),
                                         0, empty)
    assert float((got - want[:, 0]).abs().max()) <= 1e-5 * float(want.abs().max())


# ---------------------------------------------------------------- together, streams, graphs

def test_prefix_packed_shared_read_back_and_copied(rotations):
    """A prefix is packed once and shared by a batch.  The same packed rows copied into every sequence's own cache,
    in front of its own rows, are the same rows when read back, and give the same step, as a decode and as cross
    attention."""
    rng = np.random.default_rng(41)
    B, H, G, n, own, cap = 3, 2, 4, 192, 64, 256
    pk = Packed(rotations, 42, batch=B, kv=H, group=G, cap=own, k_budget=192, v_bits=3, dtype="fp32")
    pcfg, wcfg = (bg.Config(1, b, H, G, c, 192, 3, bg.BGTQ_FP32) for b, c in ((1, n), (B, cap)))
    prefix, whole = bg.Cache(pcfg), bg.Cache(wcfg)
    x = [torch.from_numpy(rng.standard_normal((1, n, H, D)).astype(np.float32)).cuda() for _ in range(2)]
    bg.blockgtq_quantize_append(pcfg, pk.layout, 0, *x, i32([0]), prefix)
    for h in range(H):
        ng = len(o.groups(pk.bits[0, h]))
        s = ng + (ng & 1)
        for src, first, m in ((prefix, 0, n), (pk.cache, n, own)):
            whole.k_codes[0, :, h, first:first + m] = src.k_codes[0, :, h, :m]
            whole.k_norms[0, :, h, first * s:(first + m) * s] = src.k_norms[0, :, h, :m * s]
            whole.v_codes[0, :, h, first // 32:(first + m) // 32] = src.v_codes[0, :, h, :m // 32]
            whole.v_norms[0, :, h, first:first + m] = src.v_norms[0, :, h, :m]
    lens = [37, 5, 0]
    ctx = [n + m for m in lens]
    q, qd = pk.queries((B,))
    back = bg.blockgtq_dequantize_rows(pcfg, pk.layout, 0, prefix, i32([0]), n)
    mine = bg.blockgtq_dequantize_rows(pk.cfg, pk.layout, 0, pk.cache, i32([0] * B), own, ctx_len=i32(lens))
    copies = bg.blockgtq_dequantize_rows(wcfg, pk.layout, 0, whole, i32([0] * B), cap, ctx_len=i32(ctx))
    for one, rest, both in zip(back, mine, copies):
        assert torch.equal(both, torch.cat([one.expand(B, -1, -1, -1), rest], 1))
    shared = bg.blockgtq_decode_attn_shared(pk.cfg, pk.layout, 0, qd, pcfg, prefix, i32([n]), n, i32(lens), own, pk.cache)
    crossed = bg.blockgtq_cross_attn(wcfg, pk.layout, 0, qd[:, None], i32(ctx), max(ctx), whole)[:, 0]
    decoded = bg.blockgtq_decode_attn(wcfg, pk.layout, 0, qd, i32(ctx), max(ctx), whole)
    k, v = (t.double().cpu().numpy() for t in copies)
    for b in range(B):
        for h in range(H):
            hs = slice(h * G, (h + 1) * G)
            ref, bound = attention_and_bound(q[b, hs], k[b, :ctx[b], h], v[b, :ctx[b], h], pk.bits[0, h], pk.rot_k, pk.rot_v,
                                             torch.float32)
            bound = bound + 2.0 ** -20 * np.abs(v[b, :ctx[b], h]).max()  # (the rows read back are themselves rounded)
            check("shared", shared[b, hs], ref, bound)
            check("cross", crossed[b, hs], ref, bound)
            assert P.rel_err(decoded[b, hs].double().cpu().numpy(), ref) <= P.tol_attention()


def test_captured_and_replayed(rotations):
    """All three operators in one captured graph, replayed on new inputs with eager work in between."""
    pk = Packed(rotations, 51, batch=3, kv=2, cap=192)
    pp = Packed(rotations, 52, kv=2, cap=704, layout_of=pk)
    q, qd = pk.queries((3, 9))
    one = qd[:, 0].contiguous()
    lens, plen, pos = i32([192, 70, 1]), i32([700]), i32([1, 2, 3])
    n = bg.cross_workspace_bytes(pk.cfg, 1, 9, 0, 192)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(bg.shared_workspace_bytes(pk.cfg, pp.cfg, 1, 0, 700, 192), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(qd), torch.zeros(one.shape, device="cuda"), torch.zeros((3, 40, 2, D), device="cuda"),
            torch.zeros((3, 40, 2, D), device="cuda")]

    def step(outs, ws, ws2):
        bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd, lens, 192, pk.cache, out=outs[0], workspace=ws)
        bg.blockgtq_decode_attn_shared(pk.cfg, pk.layout, 0, one, pp.cfg, pp.cache, plen, 700, lens, 192, pk.cache,
                                       out=outs[1], workspace=ws2)
        bg.blockgtq_dequantize_rows(pk.cfg, pk.layout, 0, pk.cache, pos, 40, ctx_len=lens, k_out=outs[2], v_out=outs[3])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(outs, ws, ws2)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(outs, ws, ws2)
    for i in range(4):
        qd.copy_(pk.queries((3, 9))[1])
        one.copy_(qd[:, 0])
        lens.copy_(i32([[192, 70, 1], [0, 192, 64], [5, 6, 7], [65, 63, 0]][i]))
        plen.copy_(i32([[700], [1], [0], [333]][i]))
        pos.copy_(i32([i, 2 * i, 150]))
        for t in outs:
            t.zero_()
        ws.fill_(255)  # not a number, as fp32: no call relies on what a workspace held
        ws2.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        eager = [torch.zeros_like(t) for t in outs]
        step(eager, torch.full_like(ws, 255), torch.full_like(ws2, 255))
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b), f"replay {i}"


def test_on_another_stream(rotations):
    """Calls go to the stream that is given, or the current one: ordered behind slow work there."""
    pk = Packed(rotations, 53, batch=2, cap=128)
    q, qd = pk.queries((1, 2, 4))
    lens = [100, 128]
    ref, bound = expect_cross(pk, q, lens, torch.float32)
    late, ctx, pos = torch.zeros_like(qd[0]), i32(lens), i32([0, 0])
    big = torch.randn(4096, 4096, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(20):
            big = big @ big * 1e-4
        late.copy_(qd[0])
    out = torch.zeros(late.shape, device="cuda")
    ws = torch.empty(bg.cross_workspace_bytes(pk.cfg, 1, 4, 0, 128), dtype=torch.uint8, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, late, ctx, 128, pk.cache, out=out, workspace=ws, stream=s)
    with torch.cuda.stream(s):
        k, _ = bg.blockgtq_dequantize_rows(pk.cfg, pk.layout, 0, pk.cache, pos, 10)
    s.synchronize()
    check("stream", out, ref[0], bound[0])
    check("rows", k[1, :, 0], *expect_rows(pk, 0, 1, 0, "k", 0, 10, torch.float32))


def test_outputs_allocated_for_another_stream(rotations):
    """Outputs and workspaces that a call allocates belong to the stream it runs on: a late fill or a reuse on the
    current stream, behind slow work there, must not meet them."""
    pk = Packed(rotations, 54, batch=2, cap=640)
    q, qd = pk.queries((1, 2, 1))
    lens = [600, 640]
    ref, bound = expect_cross(pk, q, lens, torch.float32)
    ctx, pos = i32(lens), i32([0, 0])
    big = torch.randn(4096, 4096, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        big = big @ big * 1e-4
    k, v = bg.blockgtq_dequantize_rows(pk.cfg, pk.layout, 0, pk.cache, pos, 10, stream=s)
    out = bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd[0], ctx, 640, pk.cache, n_splits=10, stream=s)
    torch.cuda.synchronize()
    check("rows", k[1, :, 0], *expect_rows(pk, 0, 1, 0, "k", 0, 10, torch.float32))
    check("values", v[1, :, 0], *expect_rows(pk, 0, 1, 0, "v", 0, 10, torch.float32))
    check("stream", out, ref[0], bound[0])


def test_same_call_twice_gives_the_same_bits(rotations):
    pk = Packed(rotations, 54, batch=2, kv=2, cap=704)
    pp = Packed(rotations, 55, kv=2, cap=1088, layout_of=pk)
    q, qd = pk.queries((2, 7))
    for _ in range(2):
        runs = [(bg.blockgtq_cross_attn(pk.cfg, pk.layout, 0, qd, i32([700, 600]), 704, pk.cache),
                 bg.blockgtq_decode_attn_shared(pk.cfg, pk.layout, 0, qd[:, 0].contiguous(), pp.cfg, pp.cache, i32([1088]),
                                                1088, i32([700, 3]), 704, pk.cache)) for _ in range(3)]
        for r in runs[1:]:
            assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))
