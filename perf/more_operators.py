"""Serving steps over a paged packed cache, at the sizes that their speed is measured on.

Three operators, in the order in which a layer of a serving program calls them:
"rotate" is the norm of every query and key head with the rotation by the
token's position (one axis, or time, height and width), "append" quantizes and
packs the new rows of a ragged batch into the pages of their sequences, and
"attend" is the attention of those new tokens over the pages: causal, with a
prefix that all of a sequence's tokens see, logits capped by a tanh, a bias
that falls with the distance.  A case is one call of one layer.  Shapes are
those of this repository's workloads: a toy head, Qwen2.5-3B-shaped layers (2
KV heads, 8 query heads each), Llama-3.1-8B-shaped ones (8 KV heads, 4 query
heads each), K2V2 / K3V2 / K3V3 caches with greedy widths.  Inputs follow the
repository's synthetic recipe: log-normal block energies with three outlier
blocks, unit-normal values and queries, Haar rotations.  A pool of pages is a
packed cache whose "sequences" are the pages and whose capacity is a page's
rows; the page table gives each sequence its pages, in no order.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D, HALF = 128, 64


def _case(name, kind, **kw):
    c = {"kind": kind, "kv": 8, "group": 4, "k_budget": 128, "v_bits": 2, "dtype": "bf16", "seqs": 1, "page": 64,
         "new_lo": 1, "new_hi": 1, "ctx_lo": 0, "ctx_hi": 0, "chunks": 0, "axes": 1, "norm": True, "fused": True,
         "cap": 0.0, "bias": False, "prefix": 0}
    c.update(kw)
    return {"name": name, **c} if name else c


def listed():
    qwen = {"kv": 2, "group": 8, "k_budget": 192, "v_bits": 3}
    return [
        # the next token of one sequence: latency only
        _case("rotate_token", "rotate"),
        # a picture's patches (time, height, width) of a Qwen-shaped layer in fp32
        _case("rotate_picture_fp32", "rotate", dtype="fp32", new_hi=1037, axes=3, norm=False, fused=False, **qwen),
        # a long prompt of a Llama-shaped layer, read from the fused projection
        _case("rotate_prompt", "rotate", new_hi=32768, axes=3),
        # one token of each of a batch's sequences goes into its page
        _case("append_tokens_32", "append", seqs=32, ctx_lo=100, ctx_hi=1500),
        # ragged chunks that start inside value tiles, Qwen-shaped layer in fp32
        _case("append_chunks_fp32", "append", dtype="fp32", seqs=3, new_lo=1, new_hi=777, chunks=3, ctx_lo=800,
              ctx_hi=2501, page=128, **qwen),
        # a long prompt of a Llama-shaped layer
        _case("append_prompt", "append", new_hi=16384, ctx_hi=16384, ctx_lo=16384, page=256),
        # a toy head in fp32: the smallest attention, latency only
        _case("attend_toy_fp32", "attend", kv=1, k_budget=192, dtype="fp32", new_hi=5, ctx_lo=257, ctx_hi=257),
        # one generated token of each of 32 sequences, Llama-shaped layer
        _case("attend_tokens_32", "attend", seqs=32, ctx_lo=500, ctx_hi=8200),
        # a chunk of a prompt behind a long document, Qwen-shaped layer
        _case("attend_late_chunk", "attend", new_hi=512, ctx_lo=33111, ctx_hi=33111, page=256, **qwen),
        # one sequence's chunk beside the generated tokens of 15 others
        _case("attend_mixed_16", "attend", seqs=16, new_lo=1, new_hi=300, chunks=1, ctx_lo=301, ctx_hi=4097, k_budget=192),
        # capped logits with a bias by distance, two chunks in fp32
        _case("attend_capped_fp32", "attend", dtype="fp32", seqs=2, new_lo=333, new_hi=501, chunks=2, ctx_lo=2000,
              ctx_hi=4001, cap=30.0, bias=True, k_budget=192, page=128),
        # a whole prompt whose first 1000 tokens (a picture) see one another
        _case("attend_prompt_prefix", "attend", new_hi=8192, ctx_lo=8192, ctx_hi=8192, prefix=1000, page=128),
    ]


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    kv, group = rng.choice([(8, 4), (8, 4), (2, 8), (2, 8), (1, 4), (4, 6), (4, 1)])
    k_budget, v_bits = rng.choice([(128, 2), (128, 2), (192, 2), (192, 3), (192, 3), (256, 4)])
    kw = {"kv": kv, "group": group, "k_budget": k_budget, "v_bits": v_bits, "page": rng.choice([64, 64, 128, 256, 1024]),
          "dtype": rng.choice(["bf16", "bf16", "bf16", "fp32"])}
    kind = rng.choice(["rotate", "append", "attend", "attend", "attend"])
    if kind == "rotate":
        kw.update(new_hi=log(1, 12000), axes=rng.choice([1, 1, 2, 3, 4]), norm=rng.random() < 0.7, fused=rng.random() < 0.6)
        return _case("", kind, **kw)
    seqs = rng.choice([1, 2, 5, log(3, 64)])
    if kind == "append":
        chunks = rng.choice([0, 1, seqs])
        new = log(2, 6000 // chunks) if chunks else 1
        kw.update(seqs=seqs, chunks=chunks, new_lo=rng.randint(1, new), new_hi=new, ctx_lo=new)
        kw["ctx_hi"] = new + rng.choice([0, log(1, 2000)])
        return _case("", kind, **kw)
    chunks, ctx = rng.choice([0, 0, 1, min(seqs, 4)]), log(1, 12000)
    if chunks and seqs > 8:
        ctx = min(ctx, 4000)
    rows = 10 ** 9 // (seqs * ctx * kv * group)
    new = max(1, min(log(2, 4000), rows, ctx)) if chunks else 1
    kw.update(seqs=seqs, chunks=chunks, new_lo=rng.randint(1, new), new_hi=new, ctx_lo=rng.randint(new, ctx), ctx_hi=ctx,
              cap=rng.choice([0.0, 0.0, 20.0, 50.0]), bias=rng.random() < 0.3, prefix=rng.choice([0, 0, log(1, ctx)]))
    return _case("", kind, **kw)


# ---------------------------------------------------------------- sizes

def _news(c):
    """New tokens of each sequence: the first `chunks` ones have chunks spread over [new_lo, new_hi], the others one token."""
    if c["seqs"] == 1:
        return [c["new_hi"]]
    span = c["new_hi"] - c["new_lo"]
    return [c["new_hi"] - int(span * ((i * 0.6180339887498949) % 1.0)) if i < c["chunks"] else 1 for i in range(c["seqs"])]


def _lens(c):
    """Rows of each sequence, its new ones among them, spread over [ctx_lo, ctx_hi]."""
    span = c["ctx_hi"] - c["ctx_lo"]
    return [max(c["ctx_hi"] - int(span * ((i * 0.6180339887498949) % 1.0)), n) for i, n in enumerate(_news(c))]


def _prefixes(c):
    """Rows of each sequence that all of its tokens see: spread over [0, prefix]."""
    return [c["prefix"] - int(c["prefix"] * ((i * 0.6180339887498949) % 1.0)) for i in range(c["seqs"])]


def _row_bytes(c):
    """Packed bytes of one row: codes, about five group radii, the value radius."""
    return (2 * c["k_budget"] + D * c["v_bits"]) / 8 + 2 * 5 + 2


def work(c):
    esize, heads = 2 if c["dtype"] == "bf16" else 4, c["kv"] * c["group"]
    tokens = sum(_news(c))
    if c["kind"] == "rotate":
        n = tokens * (heads + c["kv"]) * D
        return {"bytes": 2 * n * esize + 4 * tokens * c["axes"], "flops": n * (3 + (4 if c["norm"] else 0))}
    if c["kind"] == "append":
        # rows in, packed and back as bf16 values; a key row by its groups' rotations (about 128^2 / 4 products), a
        # value row by the whole one, each there and back
        rows = tokens * c["kv"]
        return {"bytes": rows * (2 * D * esize + 2 * _row_bytes(c) + 2 * D * 2), "flops": rows * 4 * (D * D // 4 + D * D)}
    pairs = 0
    for n, t, p in zip(_news(c), _lens(c), _prefixes(c)):
        first = t - n + 1  # rows that the first new token sees, all below `see` seen by all
        see = min(p, t)
        whole = max(0, min(n, see - first + 1))
        pairs += whole * see + sum((first + whole, t)) * (n - whole) // 2
    rows = sum(_lens(c)) * c["kv"]
    return {"bytes": rows * _row_bytes(c) + 2 * tokens * heads * D * esize, "flops": 4 * D * heads * pairs}


# ---------------------------------------------------------------- inputs

def _lloyd_max(b):
    """The 2^b centroids of the Gaussian minimum-MSE quantizer, rounded to fp16 (Newton on c = E[x | cell])."""
    n = 1 << b
    pdf = lambda x: torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)  # noqa: E731
    tail = lambda x: 0.5 * torch.special.erfc(x / math.sqrt(2.0))  # noqa: E731
    p = (torch.arange(n, dtype=torch.float64) + 0.5) / n
    c = math.sqrt(3.0) * math.sqrt(2.0) * torch.special.erfinv(2 * p - 1)
    inf = torch.full((1,), math.inf, dtype=torch.float64)
    for _ in range(100):
        t = torch.cat([-inf, (c[1:] + c[:-1]) / 2, inf])
        lo, hi = t[:-1], t[1:]
        mass = torch.where(lo >= 0, tail(lo) - tail(hi), tail(-hi) - tail(-lo))
        mean = (pdf(lo) - pdf(hi)) / mass
        by_lo = torch.where(torch.isfinite(lo), pdf(lo) * (mean - lo) / mass, 0.0)
        by_hi = torch.where(torch.isfinite(hi), pdf(hi) * (hi - mean) / mass, 0.0)
        jac = torch.diag((by_lo + by_hi) / 2) + torch.diag(by_lo[1:] / 2, -1) + torch.diag(by_hi[:-1] / 2, 1)
        step = torch.linalg.solve(torch.eye(n, dtype=torch.float64) - jac, mean - c)
        while bool((torch.diff(c + step) <= 0).any()):
            step = step / 2
        c = c + step
        c = (c - c.flip(0)) / 2
        if float(step.abs().max()) < 1e-14:
            break
    return c.to(torch.float16)


_BOOKS = []


def _books():
    """Centroids (fp32 values of fp16 numbers) of the widths 1 .. 8."""
    if not _BOOKS:
        _BOOKS.extend(_lloyd_max(b).to(torch.float32) for b in range(1, 9))
    return _BOOKS


def _greedy(scores, budget):
    """Widths of the 64 blocks of each row of scores: one bit at a time to the largest score / 4^width."""
    bits = np.ones(scores.shape, dtype=np.int64)
    gain = scores / 4.0
    at = np.arange(len(scores))
    for _ in range(budget - HALF):
        i = np.argmax(np.where(bits < 8, gain, -1.0), axis=1)
        bits[at, i] += 1
        gain[at, i] /= 4.0
    return bits


def _haar(r, d):
    q, t = np.linalg.qr(r.standard_normal((d, d)))
    return (q * np.sign(np.diag(t))[None, :]).astype(np.float32)


def _rows_of_layout(bits, rot_k):
    """Stream-order tables of each (layer, KV head) row: source dim, width, first bit and group of every
    position, group sizes, and the key rotation as one matrix from natural dims to stream positions."""
    n = len(bits)
    t = {k: np.zeros((n, D), dtype=np.int64) for k in ("dim", "width", "bitoff", "grp", "gdim")}
    w, ng = np.zeros((n, D, D), dtype=np.float32), np.zeros(n, dtype=np.int64)
    for r in range(n):
        p = 0
        for b in range(1, 9):
            blocks = np.nonzero(bits[r] == b)[0]
            if not blocks.size:
                continue
            dims = np.stack([blocks, blocks + HALF], 1).reshape(-1)
            s = slice(p, p + dims.size)
            t["dim"][r, s], t["width"][r, s], t["grp"][r, s], t["gdim"][r, s] = dims, b, ng[r], dims.size
            w[r][np.ix_(np.arange(p, p + dims.size), dims)] = rot_k[dims.size]
            ng[r] += 1
            p += dims.size
        t["bitoff"][r] = np.cumsum(t["width"][r]) - t["width"][r]
    return t, w, ng


def _int32(words):
    """Values below 2^32 as the int32 of the same bits."""
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _normal(seed, what, shape):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + what * 7919 + 12345) % (1 << 62))
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _codes_of(z, width, edges, widths):
    """Codes of rotated coordinates: thresholds at or below each, of its position's width."""
    codes = torch.zeros(z.shape, dtype=torch.int64, device="cuda")
    for b in widths:
        codes = torch.where(width == b, torch.bucketize(z, edges[b - 1], right=True), codes)
    return codes


def _pack(s, c, seed, rows):
    """Pages of `rows` (a multiple of the page) quantized synthetic rows of each sequence, in the documented layout:
    [sequence, page of it, head, ...]."""
    H, bv, kw, B, P = c["kv"], c["v_bits"], s["kw"], c["seqs"], c["page"]
    n = rows // P
    dev = {"dtype": torch.int32, "device": "cuda"}
    out = {"k_codes": torch.zeros((B, n, H, P, kw), **dev),
           "k_norms": torch.zeros((B, n, H, P * 8), dtype=torch.float16, device="cuda"),
           "v_codes": torch.zeros((B, n, H, P // 32, D, bv), **dev),
           "v_norms": torch.zeros((B, n, H, P), dtype=torch.float16, device="cuda")}
    edges = [(t[1:] + t[:-1]) / 2 for t in (t.cuda() for t in _books())]
    step = max(1, (1 << 22) // (B * D * P))
    for h in range(H):
        width, w, grp, gdim = s["width"][h], s["w"][h], s["grp"][h], s["gdim"][h]
        ng, slots = int(s["ng_host"][h]), (int(s["ng_host"][h]) + 1) // 2 * 2
        widths = sorted(set(s["bits_host"][h].tolist()))
        for p0 in range(0, n, step):
            m = min(step, n - p0)
            k = _normal(seed + 31 * p0, 2 * (64 + h), (B, m * P, D)) * s["sigma"][h]
            v = _normal(seed + 31 * p0, 2 * (64 + h) + 1, (B, m * P, D))
            z = k @ w.T
            norm = ((z * z) @ (grp[:, None] == torch.arange(slots, device="cuda")).float()).sqrt()
            z = z * (gdim.float().sqrt() / norm[..., grp].clamp_min(1e-30))
            at, sh = s["bitoff"][h] // 32, s["bitoff"][h] % 32
            codes = _codes_of(z, width, edges, widths) << sh
            words = torch.zeros((B, m * P, kw + 1), dtype=torch.int64, device="cuda")
            words.index_add_(2, at, codes & 0xFFFFFFFF).index_add_(2, at + 1, codes >> 32)
            out["k_codes"][:, p0:p0 + m, h] = _int32(words[..., :kw]).view(B, m, P, kw)
            norm[..., ng:] = 0
            out["k_norms"][:, p0:p0 + m, h, :P * slots] = norm.reshape(B, m, -1).half()
            radius = v.norm(dim=-1)
            out["v_norms"][:, p0:p0 + m, h] = radius.half().view(B, m, P)
            code = torch.bucketize((v @ s["rot_v"].T) * (math.sqrt(D) / radius)[..., None], edges[bv - 1], right=True)
            code = code.view(B, m, P // 32, 32, D).transpose(3, 4) << s["v_sh"]
            words = torch.zeros((B, m, P // 32, D, bv + 1), dtype=torch.int64, device="cuda")
            words.index_add_(4, s["v_at"], code & 0xFFFFFFFF).index_add_(4, s["v_at"] + 1, code >> 32)
            out["v_codes"][:, p0:p0 + m, h] = _int32(words[..., :bv])
    return out


def _layout(s, c, r):
    """The layout of one layer's heads: widths from the energies that a calibration set shows, rotations, tables."""
    H = c["kv"]
    sigma = np.exp(r.standard_normal((H, HALF)))
    for row in sigma:
        row[r.choice(HALF, size=3, replace=False)] *= 8
    rot_k, rot_v = {d: _haar(r, d) for d in range(2, D + 1, 2)}, _haar(r, D)
    bits = _greedy(sigma ** 2 * r.uniform(0.95, 1.05, sigma.shape) + 1.0, c["k_budget"])
    t, w, ng = _rows_of_layout(bits, rot_k)
    s.update({k: torch.from_numpy(v).cuda() for k, v in t.items()})
    s.update(v_bits=c["v_bits"], kw=(2 * c["k_budget"] + 31) // 32, w=torch.from_numpy(w).cuda(), rot_k=rot_k,
             rot_v=torch.from_numpy(rot_v).cuda(), bits_host=bits, ng_host=ng,
             slots=torch.from_numpy((ng + 1) // 2 * 2).cuda(),
             sigma=torch.from_numpy(np.concatenate([sigma, sigma], 1).astype(np.float32)).cuda(),
             books=torch.cat(_books()).cuda(), edges=[((t[1:] + t[:-1]) / 2).double().cuda() for t in _books()])
    bit = torch.arange(32, device="cuda") * c["v_bits"]
    s["v_at"], s["v_sh"] = bit // 32, bit % 32


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(c, seed):
    H, G, B, kind = c["kv"], c["group"], c["seqs"], c["kind"]
    dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    r = np.random.default_rng([seed, 7])
    news, n = _news(c), sum(_news(c))
    s = {"kind": kind, "kv": H, "group": G, "type": dtype, "n": n}
    if kind == "rotate":
        s["qkv"] = _normal(seed, 1, (n, (G + 2) * H, D)).to(dtype) * 3
        if c["fused"]:  # the projection's output: queries, keys and values of a token beside one another
            s["q"], s["k"] = s["qkv"][:, :H * G], s["qkv"][:, H * G:H * (G + 1)]
        else:
            s["q"], s["k"] = s["qkv"][:, :H * G].contiguous(), s["qkv"][:, H * G:H * (G + 1)].contiguous()
        # time, height, width: a picture's rows and columns behind some text; late in a long context
        start = int(r.integers(0, 200000))
        s["pos"] = torch.stack([start + torch.arange(n) // 37 ** (a % 2) % (10 ** 6 if a == 0 else 37 + a)
                                for a in range(c["axes"])], 1).to(torch.int32).cuda().contiguous()
        s["axis"] = [min(i * c["axes"] // HALF, c["axes"] - 1) for i in range(HALF)]
        s["theta"] = [1e6 ** (-2.0 * i / D) for i in range(HALF)]
        s["eps"] = 1e-6
        s["weights"] = [1 + 0.2 * _normal(seed, 5 + i, (D,)) for i in range(2)] if c["norm"] else [None, None]
        s["axis_of"], s["theta_of"] = torch.tensor(s["axis"]).cuda(), torch.tensor(s["theta"], dtype=torch.float64).cuda()
        s["outs"] = [torch.empty((n, h, D), dtype=dtype, device="cuda") for h in (H * G, H)]
        if own:
            _handles(s, c, None)
        return s
    lens, P = _lens(c), c["page"]
    _layout(s, c, r)
    per = [(t + P - 1) // P for t in lens]
    most = max(max(per), 1)
    # every sequence's pages, anywhere in the pool, with a few free pages among them
    places = r.permutation(sum(per) + 3)
    table, at = np.full((B, most), -1, dtype=np.int64), 0
    for b, p in enumerate(per):
        table[b, :p] = places[at:at + p]
        at += p
    s.update(page=P, lens_host=lens, news_host=news, max_new=max(news), max_ctx=max(lens), table_host=table,
             pages=_int(table), lens=_int(lens), cu=_int(np.concatenate([[0], np.cumsum(news)])), pool_pages=sum(per) + 3)
    # each token's sequence and position; each sequence's tokens in a padded batch
    seq = np.repeat(np.arange(B), news)
    index = np.concatenate([np.arange(m) for m in news])
    s["seq"], s["index"] = torch.from_numpy(seq).cuda(), torch.from_numpy(index).cuda()
    s["pos"] = torch.from_numpy(index + np.repeat(np.array(lens) - np.array(news), news)).cuda()
    first = np.concatenate([[0], np.cumsum(news)[:-1]])
    s["token"] = torch.from_numpy(np.minimum(first[:, None] + np.arange(max(news)), n - 1)).cuda()
    shapes = {"k_codes": (H, P, s["kw"]), "k_norms": (H, P * 8), "v_codes": (H, P // 32, D, c["v_bits"]), "v_norms": (H, P)}
    half = ("k_norms", "v_norms")
    s["pool"] = {k: torch.zeros((1, s["pool_pages"]) + x, dtype=torch.float16 if k in half else torch.int32, device="cuda")
                 for k, x in shapes.items()}
    if kind == "append":
        s["k"] = (_normal(seed, 1, (n, H, D)) * s["sigma"]).to(dtype)
        s["v"] = _normal(seed, 2, (n, H, D)).to(dtype)
        # what is read back: of each page the new rows, from the first one on
        page, slot = table[seq, s["pos"].cpu().numpy() // P], s["pos"].cpu().numpy() % P
        lo, hi = np.full(s["pool_pages"], P), np.zeros(s["pool_pages"], dtype=np.int64)
        np.minimum.at(lo, page, slot)
        np.maximum.at(hi, page, slot + 1)
        s["rows"] = int((hi - lo).max())
        s["from"], s["to"] = _int(np.where(hi > 0, lo, -P)), _int(hi)
        s["out_at"] = torch.from_numpy(page).cuda(), torch.from_numpy(slot - lo[page]).cuda()
        s["outs"] = [torch.zeros((s["pool_pages"], s["rows"], H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    else:
        packed = _pack(s, c, seed, most * P)
        used = torch.from_numpy(table >= 0).cuda()
        for name, x in packed.items():
            s["pool"][name][0, torch.from_numpy(table[table >= 0]).cuda()] = x[used]
        s["q"] = _normal(seed, 3, (n, H * G, D)).to(dtype)
        s["cap"] = c["cap"]
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (i + 1) / (H * G)) for i in range(H * G)], device="cuda") if c["bias"] else None
        s["prefix"] = _int(_prefixes(c)) if c["prefix"] else None
        s["outs"] = torch.empty((n, H * G, D), dtype=dtype, device="cuda")
    if own:
        _handles(s, c, shapes)
    return s


def _handles(s, c, shapes):
    """What a program of the framework keeps: its configuration, layout, pool, batch and workspace."""
    from paper_2606_24033_amd import blockgtq as bg

    rotate = c["kind"] == "rotate"
    cfg = s["cfg"] = bg.Config(n_layers=1, batch=1 if rotate else s["pool_pages"], n_kv_heads=c["kv"], group=c["group"],
                               capacity=c["page"], k_budget=c["k_budget"], v_bits=c["v_bits"],
                               in_dtype=bg.BGTQ_BF16 if c["dtype"] == "bf16" else bg.BGTQ_FP32)
    if rotate:
        s["rope"] = bg.Rope(s["theta"], s["axis"])
        return
    flat = np.concatenate([s["rot_k"][d].reshape(-1) for d in range(2, D + 1, 2)])
    s["layout"] = bg.Layout(cfg, s["bits_host"], flat, s["rot_v"].cpu().numpy())
    s["packed"] = bg.Cache(cfg)
    for name in shapes:
        setattr(s["packed"], name, s["pool"][name])
    s["chunk"] = bg.Chunk(s["cu"], s["lens"], s["pages"], s["max_new"], s["max_ctx"])
    if c["kind"] == "attend":
        n = bg.paged_workspace_bytes(cfg, s["chunk"], s["n"], 0)
        s["ws"] = torch.zeros(n, dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------- the operators

def _plain_rotate(s):
    # the angle in 64 bits: far positions
    turn = s["pos"][:, s["axis_of"]].double() * s["theta_of"]
    cos, sin = torch.cos(turn).float()[:, None], torch.sin(turn).float()[:, None]

    def one(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * weight
        a, b = x[..., :HALF], x[..., HALF:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1).to(s["type"])

    return [one(s["q"], s["weights"][0]), one(s["k"], s["weights"][1])]


def _plain_append(s):
    """Codes from 64 bits (values next to a border), rows back from codes and radii held in 16 bits."""
    k, v = s["k"].double(), s["v"].double()
    # [heads, tokens, stream positions]
    z = k.transpose(0, 1) @ s["w"].double().transpose(1, 2)
    member = (s["grp"][:, :, None] == torch.arange(8, device="cuda")).double()
    norm = ((z * z) @ member).sqrt()
    of = s["grp"][:, None].expand(z.shape)
    z = z * (s["gdim"].double().sqrt()[:, None] / torch.take_along_dim(norm, of, 2).clamp_min(1e-300))
    width = s["width"][:, None]
    every = torch.stack([torch.bucketize(z, e, right=True) for e in s["edges"]])
    code = torch.take_along_dim(every, (width - 1).expand(z.shape)[None], 0)[0]
    y = s["books"][code + (1 << width) - 2] * torch.take_along_dim(norm.half().float(), of, 2)
    k = (y / s["gdim"].float().sqrt()[:, None]) @ s["w"]
    bv = s["v_bits"]
    radius = v.norm(dim=-1, keepdim=True)
    code = torch.bucketize((v @ s["rot_v"].double().T) * (math.sqrt(D) / radius.clamp_min(1e-300)), s["edges"][bv - 1], right=True)
    v = (s["books"][code + (1 << bv) - 2] * (radius.half().float() / math.sqrt(D))) @ s["rot_v"]
    outs = [torch.zeros_like(x) for x in s["outs"]]
    for x, rows in zip(outs, (k.transpose(0, 1), v)):
        x[s["out_at"]] = rows.to(x.dtype)
    return outs


def _unpack(words, at, sh, mask):
    """Bit fields (first word, shift, mask) of the last dimension's little-endian 32-bit words."""
    words = torch.nn.functional.pad(words, (0, 1)).to(torch.int64) & 0xFFFFFFFF
    low = torch.take_along_dim(words, at.expand(words.shape[:-1] + at.shape[-1:]), -1)
    high = torch.take_along_dim(words, (at + 1).expand(words.shape[:-1] + at.shape[-1:]), -1)
    return ((low | high << 32) >> sh) & mask


def _plain_rows(s):
    """The rows of every sequence by its page table: keys and values [sequences, KV heads, rows, 128] in fp32."""
    H, bv, P = s["kv"], s["v_bits"], s["page"]
    table = s["pages"].long().clamp_min(0)
    per = lambda x: x.view(1, 1, H, 1, -1)  # noqa: E731
    words = s["pool"]["k_codes"][0][table]
    B, n = words.shape[:2]
    code = _unpack(words, per(s["bitoff"] // 32), per(s["bitoff"] % 32), per((1 << s["width"]) - 1))
    y = s["books"][code + per((1 << s["width"]) - 2)]
    # row t's radii start at t times the head's slots
    at = torch.arange(P, device="cuda").view(1, 1, 1, P, 1) * per(s["slots"]) + per(s["grp"])
    norms = s["pool"]["k_norms"][0][table]
    radius = torch.take_along_dim(norms, at.expand(B, n, H, P, D).reshape(B, n, H, P * D), -1).view(y.shape).float()
    k = (y * radius / per(s["gdim"].float().sqrt())) @ s["w"]
    code = _unpack(s["pool"]["v_codes"][0][table], s["v_at"], s["v_sh"], (1 << bv) - 1)
    y = s["books"][code + ((1 << bv) - 2)].transpose(-1, -2).reshape(B, n, H, P, D)
    v = (y * (s["pool"]["v_norms"][0][table][..., None].float() / math.sqrt(D))) @ s["rot_v"]
    return [x.transpose(1, 2).reshape(B, H, n * P, D)[:, :, :s["max_ctx"]] for x in (k, v)]


def _plain_attend(s):
    """The sequences' tokens in a padded batch, one softmax over the rows that each of them sees."""
    H, G = s["kv"], s["group"]
    k, v = _plain_rows(s)
    B, n = k.shape[0], k.shape[2]
    q = s["q"].float()[s["token"]].view(B, -1, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    x = (q @ k.transpose(-1, -2)) / math.sqrt(D)
    if s["cap"]:
        x = s["cap"] * torch.tanh(x / s["cap"])
    x = x.view(B, H, -1, G, n)
    pos = s["pos"][s["token"]][:, None, :, None, None]
    row = torch.arange(n, device="cuda")
    if s["slopes"] is not None:
        x = x - s["slopes"].view(1, H, 1, G, 1) * (pos - row).abs()
    seen = row <= pos
    if s["prefix"] is not None:
        seen = seen | (row < torch.minimum(s["prefix"], s["lens"])[:, None, None, None, None])
    x = torch.where(seen, x, -math.inf)
    e = torch.exp(x - x.amax(-1, keepdim=True)).view(B, H, -1, n)
    out = (e @ v) / e.sum(-1, keepdim=True)
    out = out.view(B, H, -1, G, D).permute(0, 2, 1, 3, 4).reshape(B, -1, H * G, D)
    return out[s["seq"], s["index"]].to(s["type"])


def run(s):
    kind = s["kind"]
    if not own:
        return _plain_rotate(s) if kind == "rotate" else _plain_append(s) if kind == "append" else _plain_attend(s)
    from paper_2606_24033_amd import blockgtq as bg

    if kind == "rotate":
        return list(bg.blockgtq_norm_rope(s["cfg"], s["rope"], s["q"], s["k"], s["pos"], q_weight=s["weights"][0],
                                          k_weight=s["weights"][1], eps=s["eps"], q_out=s["outs"][0], k_out=s["outs"][1]))
    if kind == "append":
        bg.blockgtq_paged_append(s["cfg"], s["layout"], 0, s["k"], s["v"], s["chunk"], s["packed"])
        # what the pages now hold
        return list(bg.blockgtq_dequantize_rows(s["cfg"], s["layout"], 0, s["packed"], s["from"], s["rows"], ctx_len=s["to"],
                                                k_out=s["outs"][0], v_out=s["outs"][1]))
    return bg.blockgtq_paged_attn(s["cfg"], s["layout"], 0, s["q"], s["chunk"], s["packed"], cap=s["cap"], slopes=s["slopes"],
                                  prefix=s["prefix"], out=s["outs"], workspace=s["ws"])


# ---------------------------------------------------------------- 64 bits

def _bits_of(words):
    """Each row's words [rows, words] as its bits [rows, 32 words]."""
    return ((words[:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).flatten(1).double()


def _groups(s, h):
    """(first bit, width, dims) of each same-rate group of a head's key row, in ascending width."""
    at = 0
    for w in range(1, 9):
        blocks = np.nonzero(s["bits_host"][h] == w)[0]
        if len(blocks):
            dims = torch.from_numpy(np.stack([blocks, blocks + HALF], 1).reshape(-1)).cuda()
            yield at, w, dims
            at += w * len(dims)


def _rot(s, d):
    return torch.from_numpy(s["rot_k"][d].astype(np.float64)).cuda()


def _exact_rows(s, b, h):
    """Keys and values of one head of a sequence, bit by bit and group by group."""
    n, P, bv = s["lens_host"][b], s["page"], s["v_bits"]
    books = [x.double().cuda() for x in _books()]
    slots, keys, values = int(s["slots"][h]), [], []
    for p in s["table_host"][b, :(n + P - 1) // P]:
        bits = _bits_of(s["pool"]["k_codes"][0, p, h])
        radii = s["pool"]["k_norms"][0, p, h, :P * slots].view(P, slots).double()
        k = torch.zeros((P, D), dtype=torch.float64, device="cuda")
        for i, (at, w, dims) in enumerate(_groups(s, h)):
            d = len(dims)
            code = (bits[:, at:at + w * d].view(P, d, w) @ (2.0 ** torch.arange(w, device="cuda")).double()).long()
            k[:, dims] = (radii[:, i:i + 1] * books[w - 1][code] / math.sqrt(d)) @ _rot(s, d)
        bits = _bits_of(s["pool"]["v_codes"][0, p, h].reshape(-1, bv)).view(P // 32, D, 32, bv)
        code = (bits @ (2.0 ** torch.arange(bv, device="cuda")).double()).long().transpose(1, 2).reshape(P, D)
        radius = s["pool"]["v_norms"][0, p, h].double()[:, None]
        keys.append(k)
        values.append((radius * books[bv - 1][code] / math.sqrt(D)) @ s["rot_v"].double())
    return torch.cat(keys)[:n], torch.cat(values)[:n]


def _exact_append(s):
    outs = [torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in s["outs"]]
    books = [x.double().cuda() for x in _books()]

    def code(z, w):
        return books[w - 1][(z[..., None] >= (books[w - 1][1:] + books[w - 1][:-1]) / 2).sum(-1)]

    for h in range(s["kv"]):
        for i in range(0, s["n"], 4096):
            k, v = s["k"][i:i + 4096, h].double(), s["v"][i:i + 4096, h].double()
            page, slot = (x[i:i + 4096] for x in s["out_at"])
            back = torch.zeros_like(k)
            for _, w, dims in _groups(s, h):
                x, d = k[:, dims], len(dims)
                r = torch.linalg.vector_norm(x, dim=1, keepdim=True)
                back[:, dims] = (r.half().double() / math.sqrt(d)) * code(x @ _rot(s, d).T * (math.sqrt(d) / r), w) @ _rot(s, d)
            outs[0][page, slot, h] = back
            r, rot = torch.linalg.vector_norm(v, dim=1, keepdim=True), s["rot_v"].double()
            outs[1][page, slot, h] = (r.half().double() / math.sqrt(D)) * code(v @ rot.T * (math.sqrt(D) / r), s["v_bits"]) @ rot
    return outs


def exact(c, seed):
    s = prepare(c, seed)
    H, G = s["kv"], s["group"]
    if s["kind"] == "rotate":
        outs = []
        for x, weight in zip((s["q"], s["k"]), s["weights"]):
            x = x.double()
            if weight is not None:
                x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / D + s["eps"]) * weight.double()
            out = torch.zeros_like(x)
            for i in range(HALF):
                z = torch.polar(torch.ones(s["n"], dtype=torch.float64, device="cuda"),
                                s["pos"][:, s["axis"][i]].double() * s["theta"][i])
                z = z[:, None] * torch.complex(x[..., i], x[..., i + HALF])
                out[..., i], out[..., i + HALF] = z.real, z.imag
            outs.append(out)
        return outs
    if s["kind"] == "append":
        return _exact_append(s)
    out, first = torch.zeros((s["n"], H, G, D), dtype=torch.float64, device="cuda"), 0
    q = s["q"].double().view(-1, H, G, D)
    for b, (n, t) in enumerate(zip(s["news_host"], s["lens_host"])):
        see = 0 if s["prefix"] is None else min(_prefixes(c)[b], t)
        for h in range(H):
            k, v = _exact_rows(s, b, h)
            for i in range(0, n, 1024):
                at = slice(first + i, first + min(i + 1024, n))
                pos = torch.arange(t - n + i, t - n + min(i + 1024, n), device="cuda")[:, None, None]
                row = torch.arange(t, device="cuda")
                x = (q[at, h].reshape(-1, D) @ k.T / math.sqrt(D)).view(-1, G, t)
                if s["cap"]:
                    x = torch.tanh(x / s["cap"]) * s["cap"]
                if s["slopes"] is not None:
                    x = x - s["slopes"].double()[h * G:(h + 1) * G, None] * (pos - row).abs().double()
                x = x.masked_fill((row > pos) & (row >= see), -math.inf)
                out[at, h] = (torch.softmax(x, -1).view(-1, t) @ v).view(-1, G, D)
        first += n
    return out.view(s["n"], H * G, D)
