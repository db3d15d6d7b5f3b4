"""Operators that read the packed cache, at the sizes that their speed is measured on.

Three operators: "read" gives cache rows back as plain keys and values, "cross"
is the attention of query rows to another sequence's whole cache (an encoder's
states), "shared" one decode step of a batch whose sequences share a long
prefix.  A case is one call at one size.  Shapes are those of this repository's
workloads: a toy head, Qwen2.5-3B-shaped layers (2 KV heads, 8 query heads
each), Llama-3.1-8B-shaped ones (8 KV heads, 4 query heads each), K2V2 / K3V2 /
K3V3 caches with greedy widths.  Inputs follow the repository's synthetic
recipe: log-normal block energies with three outlier blocks, unit-normal values
and queries, Haar rotations.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D, HALF = 128, 64


def _case(name, kind, **kw):
    c = {"kind": kind, "layers": 1, "batch": 1, "kv": 8, "group": 4, "k_budget": 128, "v_bits": 2, "dtype": "bf16",
         "uniform": False, "lo": 0, "hi": 0, "rows": 0, "prefix": 0}
    c.update(kw)
    return {"name": name, **c} if name else c


def listed():
    qwen = {"kv": 2, "group": 8, "k_budget": 192, "v_bits": 3}
    return [
        # one page of every layer handed over to code that wants plain rows
        _case("read_page_all_layers", "read", layers=32, lo=1001, hi=1001, rows=16),
        # the ragged contexts of a few sequences read back in fp32, Qwen-shaped layer
        _case("read_ragged_fp32", "read", batch=3, rows=4999, lo=1200, hi=4999, dtype="fp32", **qwen),
        # a long prompt read back to be packed anew, Llama-shaped layer
        _case("read_llama_prompt", "read", rows=65536, lo=65536, hi=65536),
        # a toy head: the smallest cross attention, latency only
        _case("cross_toy_fp32", "cross", kv=1, k_budget=192, dtype="fp32", lo=257, hi=257, rows=5),
        # one generated token of a batch against its encoder states of ragged lengths
        _case("cross_token_batch8", "cross", batch=8, k_budget=192, lo=150, hi=1500, rows=1),
        # decoder prompts of a batch against ragged encoder states
        _case("cross_prompt_ragged", "cross", batch=4, lo=1000, hi=4097, rows=333),
        # a long decoder pass against a long document, Qwen-shaped layer
        _case("cross_long", "cross", lo=16385, hi=16385, rows=2048, **qwen),
        # two requests behind a short system prompt: latency
        _case("shared_pair", "shared", batch=2, prefix=500, lo=5, hi=40),
        # a toy head in fp32
        _case("shared_toy_fp32", "shared", kv=1, k_budget=192, dtype="fp32", batch=5, prefix=2049, lo=0, hi=129),
        # a chat service: many requests behind one instruction text
        _case("shared_chat_32", "shared", batch=32, prefix=8205, lo=1, hi=600),
        # many samples of one long document's continuation, Qwen-shaped layer
        _case("shared_document_64", "shared", batch=64, prefix=32768, lo=100, hi=2000, **qwen),
        # every layer of a Llama-shaped model in one call
        _case("shared_all_layers_16", "shared", layers=32, batch=16, prefix=4001, lo=20, hi=300),
    ]


def draw(rng):
    def log(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    kv, group = rng.choice([(8, 4), (8, 4), (2, 8), (2, 8), (1, 4), (4, 6), (4, 1)])
    k_budget, v_bits = rng.choice([(128, 2), (128, 2), (192, 2), (192, 3), (192, 3), (256, 4)])
    kw = {"kv": kv, "group": group, "k_budget": k_budget, "v_bits": v_bits,
          "dtype": rng.choice(["bf16", "bf16", "bf16", "fp32"]), "uniform": rng.random() < 0.15}
    kind = rng.choice(["read", "cross", "cross", "shared", "shared"])
    if kind == "read":
        if rng.random() < 0.4:  # a few rows of every layer
            kw.update(layers=rng.choice([8, 28, 32]), batch=rng.choice([1, 2]), rows=rng.randint(1, 100))
        else:
            kw.update(batch=rng.choice([1, 1, 2, 3]), rows=log(16, 10000))
        hi = kw["rows"] + rng.randint(0, 900)
        kw.update(lo=rng.randint(0, hi), hi=hi)
    elif kind == "cross":
        batch = rng.choice([1, 1, 2, 5, 8])
        hi = log(1, 12000)
        rows = rng.choice([1, rng.randint(2, 8), log(9, 1500)])
        kw.update(batch=batch, rows=max(1, min(rows, 5 * 10 ** 8 // (batch * hi * kv * group))), lo=rng.randint(0, hi), hi=hi)
    else:
        batch = log(1, 100)
        hi = rng.choice([log(1, 300), log(1, 1500)])
        kw.update(batch=batch, prefix=log(1, 40000), lo=rng.randint(0, hi), hi=hi)
    return _case("", kind, **kw)


# ---------------------------------------------------------------- sizes

def _lens(c):
    """Cache rows of each sequence (its own, behind a prefix), spread over [lo, hi]."""
    return [c["hi"] - int((c["hi"] - c["lo"]) * ((i * 0.6180339887498949) % 1.0)) for i in range(c["batch"])]


def _read_from(c):
    """First row that a read takes of every sequence: the last `rows` of the longest one."""
    return max(0, c["hi"] - c["rows"])


def _cap(n):
    return max(64, (n + 63) // 64 * 64)


def _row_bytes(c):
    """Packed bytes of one row: codes, about five group radii (one in a uniform layout), the value radius."""
    return (2 * c["k_budget"] + D * c["v_bits"]) / 8 + 2 * (1 if c["uniform"] else 5) + 2


def work(c):
    heads, esize = c["layers"] * c["kv"], 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "read":
        rows = heads * sum(max(0, min(c["rows"], n - _read_from(c))) for n in _lens(c))
        # a key row by its groups' rotations (about 128^2 / 4 products) and a value row by the whole one
        rotate = 2 * (D * D if c["uniform"] else D * D // 4) + 2 * D * D
        return {"bytes": rows * (_row_bytes(c) + 2 * D * esize), "flops": rows * rotate}
    n_q = c["rows"] if c["kind"] == "cross" else 1
    q = heads * c["group"] * D * c["batch"] * n_q
    rows = heads * (c["prefix"] + sum(_lens(c)))
    pairs = heads * c["group"] * (c["prefix"] * c["batch"] + n_q * sum(_lens(c)))
    return {"bytes": rows * _row_bytes(c) + 2 * q * esize, "flops": 4 * D * pairs}


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


def _pack(s, c, seed, what, batch, n, cap):
    """A packed cache of `cap` rows whose first n hold quantized synthetic keys and values (the inputs of every
    operator here): group radii and codes of the rotated rows, in the documented layout."""
    L, H, bv, kw = c["layers"], c["kv"], c["v_bits"], s["kw"]
    dev = {"dtype": torch.int32, "device": "cuda"}
    out = {"k_codes": torch.zeros((L, batch, H, cap, kw), **dev),
           "k_norms": torch.zeros((L, batch, H, cap * 8), dtype=torch.float16, device="cuda"),
           "v_codes": torch.zeros((L, batch, H, cap // 32, D, bv), **dev),
           "v_norms": torch.zeros((L, batch, H, cap), dtype=torch.float16, device="cuda")}
    books = [t.cuda() for t in _books()]
    edges = [(t[1:] + t[:-1]) / 2 for t in books]
    step = max(32, (1 << 22) // (batch * D) // 32 * 32)
    for layer in range(L):
        for h in range(H):
            r = layer * H + h
            width, w, grp, gdim = s["width"][r], s["w"][r], s["grp"][r], s["gdim"][r]
            ng, slots = int(s["ng_host"][r]), (int(s["ng_host"][r]) + 1) // 2 * 2
            widths = sorted(set(s["bits_host"][r].tolist()))
            for t0 in range(0, n, step):
                m = min(step, n - t0)
                key = (what * 64 + layer) * 64 + h
                k = _normal(seed + 31 * t0, 2 * key, (batch, m, D)) * s["sigma"][r]
                v = _normal(seed + 31 * t0, 2 * key + 1, (batch, m, D))
                z = k @ w.T
                norm = ((z * z) @ (grp[:, None] == torch.arange(slots, device="cuda")).float()).sqrt()
                z = z * (gdim.float().sqrt() / norm[..., grp].clamp_min(1e-30))
                codes = torch.zeros(z.shape, dtype=torch.int64, device="cuda")
                for b in widths:
                    codes = torch.where(width == b, torch.bucketize(z, edges[b - 1], right=True), codes)
                at, sh = s["bitoff"][r] // 32, s["bitoff"][r] % 32
                codes = codes << sh
                words = torch.zeros((batch, m, kw + 1), dtype=torch.int64, device="cuda")
                words.index_add_(2, at, codes & 0xFFFFFFFF).index_add_(2, at + 1, codes >> 32)
                out["k_codes"][layer, :, h, t0:t0 + m] = _int32(words[..., :kw])
                norm[..., ng:] = 0
                out["k_norms"][layer, :, h, t0 * slots:(t0 + m) * slots] = norm.reshape(batch, -1).half()
                radius = v.norm(dim=-1)
                out["v_norms"][layer, :, h, t0:t0 + m] = radius.half()
                code = torch.bucketize((v @ s["rot_v"].T) * (math.sqrt(D) / radius)[..., None], edges[bv - 1], right=True)
                tiles = (m + 31) // 32
                code = torch.nn.functional.pad(code, (0, 0, 0, tiles * 32 - m)).view(batch, tiles, 32, D).transpose(2, 3)
                at, sh = s["v_at"], s["v_sh"]
                code = code << sh
                words = torch.zeros((batch, tiles, D, bv + 1), dtype=torch.int64, device="cuda")
                words.index_add_(3, at, code & 0xFFFFFFFF).index_add_(3, at + 1, code >> 32)
                out["v_codes"][layer, :, h, t0 // 32:t0 // 32 + tiles] = _int32(words[..., :bv])
    return out


def prepare(c, seed):
    L, H, B, kind = c["layers"], c["kv"], c["batch"], c["kind"]
    r = np.random.default_rng([seed, 5])
    sigma = np.exp(r.standard_normal((L * H, HALF)))
    for row in sigma:
        row[r.choice(HALF, size=3, replace=False)] *= 8
    rot_k, rot_v = {d: _haar(r, d) for d in range(2, D + 1, 2)}, _haar(r, D)
    if c["uniform"]:
        bits = np.full((L * H, HALF), c["k_budget"] // HALF, dtype=np.int64)
    else:  # widths from the energies that a calibration set shows
        bits = _greedy(sigma ** 2 * r.uniform(0.95, 1.05, sigma.shape) + 1.0, c["k_budget"])
    t, w, ng = _rows_of_layout(bits, rot_k)
    s = {k: torch.from_numpy(v).cuda() for k, v in t.items()}
    bv = c["v_bits"]
    s.update(kind=kind, layers=L, kv=H, batch=B, group=c["group"], v_bits=bv, rows=c["rows"], kw=(2 * c["k_budget"] + 31) // 32,
             w=torch.from_numpy(w).cuda(), rot_v=torch.from_numpy(rot_v).cuda(), rot_k=rot_k, bits_host=bits, ng_host=ng,
             slots=torch.from_numpy((ng + 1) // 2 * 2).cuda(),
             sigma=torch.from_numpy(np.concatenate([sigma, sigma], 1).astype(np.float32)).cuda(),
             books=torch.cat([b for b in _books()]).cuda(), type=torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)
    bit = torch.arange(32, device="cuda") * bv
    s["v_at"], s["v_sh"] = bit // 32, bit % 32
    lens, cap = _lens(c), _cap(max(c["hi"], c["rows"] if kind == "read" else 0))
    s["lens_host"], s["max_ctx"] = lens, max(lens)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["cache"] = _pack(s, c, seed, 1, B, max(lens), cap)
    if kind == "read":
        s["from"] = _read_from(c)
        s["pos"] = torch.full((B,), s["from"], dtype=torch.int32, device="cuda")
        shape = (L, B, c["rows"], H, D) if L > 1 else (B, c["rows"], H, D)
        s["k_out"], s["v_out"] = (torch.zeros(shape, dtype=s["type"], device="cuda") for _ in range(2))
    else:
        shape = (L, B) if L > 1 else (B,)
        shape += (c["rows"],) if kind == "cross" else ()
        s["q"] = _normal(seed, 3, shape + (H * c["group"], D)).to(s["type"])
    if kind == "shared":
        s["prefix"] = c["prefix"]
        s["prefix_len"] = torch.tensor([c["prefix"]], dtype=torch.int32, device="cuda")
        s["prefix_cache"] = _pack(s, c, seed, 2, 1, c["prefix"], _cap(c["prefix"]))
    if own:
        _handles(s, c, cap)
    return s


def _handles(s, c, cap):
    """What a program of the framework keeps: its configurations, layout, caches, output and workspace."""
    from paper_2606_24033_amd import blockgtq as bg

    def cache_of(cfg, tensors):
        cache = bg.Cache(cfg)
        for name, x in tensors.items():
            setattr(cache, name, x)
        return cache

    def config(batch, capacity):
        return bg.Config(n_layers=c["layers"], batch=batch, n_kv_heads=c["kv"], group=c["group"], capacity=capacity,
                         k_budget=c["k_budget"], v_bits=c["v_bits"],
                         in_dtype=bg.BGTQ_BF16 if c["dtype"] == "bf16" else bg.BGTQ_FP32)

    cfg = s["cfg"] = config(c["batch"], cap)
    flat = np.concatenate([s["rot_k"][d].reshape(-1) for d in range(2, D + 1, 2)])
    s["layout"] = bg.Layout(cfg, s["bits_host"], flat, s["rot_v"].cpu().numpy())
    s["packed"], s["layer"] = cache_of(cfg, s["cache"]), -1 if c["layers"] > 1 else 0
    if s["kind"] != "read":
        s["out"] = torch.empty(s["q"].shape, dtype=s["type"], device="cuda")
        if s["kind"] == "cross":
            n = bg.cross_workspace_bytes(cfg, c["layers"], c["rows"], 0, s["max_ctx"])
        else:
            s["prefix_cfg"] = config(1, _cap(c["prefix"]))
            s["prefix_packed"] = cache_of(s["prefix_cfg"], s["prefix_cache"])
            n = bg.shared_workspace_bytes(cfg, s["prefix_cfg"], c["layers"], 0, c["prefix"], s["max_ctx"])
        s["ws"] = torch.zeros(n, dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------- the operators

def _unpack(words, at, sh, mask):
    """Bit fields (first word, shift, mask) of the last dimension's little-endian 32-bit words."""
    words = torch.nn.functional.pad(words, (0, 1)).to(torch.int64) & 0xFFFFFFFF
    low = torch.take_along_dim(words, at.expand(words.shape[:-1] + at.shape[-1:]), -1)
    high = torch.take_along_dim(words, (at + 1).expand(words.shape[:-1] + at.shape[-1:]), -1)
    return ((low | high << 32) >> sh) & mask


def _plain_rows(s, cache, t0, n):
    """Rows t0 .. t0 + n - 1 of a packed cache: keys and values [layers, batch, KV heads, n, 128] in fp32."""
    L, H, bv = s["layers"], s["kv"], s["v_bits"]
    per = lambda x: x.view(L, 1, H, 1, -1)  # noqa: E731
    words = cache["k_codes"][:, :, :, t0:t0 + n]
    code = _unpack(words, per(s["bitoff"] // 32), per(s["bitoff"] % 32), per((1 << s["width"]) - 1))
    y = s["books"][code + per((1 << s["width"]) - 2)]
    # token t's radii start at t times the row's slots
    t = torch.arange(t0, t0 + n, device="cuda").view(1, 1, 1, n, 1)
    at = (t * per(s["slots"]) + per(s["grp"])).expand(L, cache["k_norms"].shape[1], H, n, D)
    radius = torch.take_along_dim(cache["k_norms"], at.reshape(at.shape[:3] + (n * D,)), -1).view(at.shape).float()
    k = (y * radius / per(s["gdim"].float().sqrt())) @ s["w"].view(L, 1, H, D, D)
    first, last = t0 // 32, (t0 + n + 31) // 32
    code = _unpack(cache["v_codes"][:, :, :, first:last], s["v_at"], s["v_sh"], (1 << bv) - 1)
    y = s["books"][code + ((1 << bv) - 2)].transpose(-1, -2).flatten(3, 4)[:, :, :, t0 - 32 * first:][:, :, :, :n]
    v = (y * (cache["v_norms"][:, :, :, t0:t0 + n, None].float() / math.sqrt(D))) @ s["rot_v"]
    return k, v


def _softmax_terms(x, allowed):
    """exp(x - max) over the last dimension where `allowed` (0 elsewhere), and that max (-inf where nothing is)."""
    x = torch.where(allowed, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isinf(top), 0.0, top))
    return e, top


def _plain_read(s):
    k, v = _plain_rows(s, s["cache"], s["from"], s["rows"])
    keep = (torch.arange(s["rows"], device="cuda") + s["from"])[None, :] < s["lens"][:, None]
    keep = keep[None, :, None, :, None]
    out = [torch.where(keep, x, 0.0).transpose(2, 3).to(s["type"]) for x in (k, v)]
    return [x if s["layers"] > 1 else x[0] for x in out]


def _plain_attention(s, prefix):
    """One softmax over the prefix's rows (if any) and the sequence's own first lens[b] ones."""
    L, B, H, G, n = s["layers"], s["batch"], s["kv"], s["group"], s["max_ctx"]
    q = s["q"].float().view(L, B, -1, H, G, D).permute(0, 1, 3, 2, 4, 5).reshape(L, B, H, -1, D)
    k, v = _plain_rows(s, s["cache"], 0, n)
    allowed = (torch.arange(n, device="cuda")[None, :] < s["lens"][:, None])[None, :, None, None, :]
    e, top = _softmax_terms((q @ k.transpose(-1, -2)) / math.sqrt(D), allowed)
    if prefix:
        # every sequence's queries against the one prefix: its rows dequantized once
        kp, vp = _plain_rows(s, s["prefix_cache"], 0, s["prefix"])
        qp = q.transpose(1, 2).reshape(L, 1, H, -1, D)
        x = (qp @ kp.transpose(-1, -2)) / math.sqrt(D)
        top_p = x.amax(-1, keepdim=True)
        ep = torch.exp(x - top_p)
        back = lambda a: a.view(L, H, B, -1, a.shape[-1]).transpose(1, 2)  # noqa: E731
        sum_p, acc_p, top_p = back(ep.sum(-1, keepdim=True)), back(ep @ vp), back(top_p)
        both = torch.maximum(top, top_p)
        by, by_p = torch.exp(top - both), torch.exp(top_p - both)
        out = (by * (e @ v) + by_p * acc_p) / (by * e.sum(-1, keepdim=True) + by_p * sum_p)
    else:
        total = e.sum(-1, keepdim=True)
        out = (e @ v) / torch.where(total > 0, total, 1.0)
    out = out.view(L, B, H, -1, G, D).permute(0, 1, 3, 2, 4, 5).reshape(s["q"].shape)
    return out.to(s["type"])


def run(s):
    kind = s["kind"]
    if not own:
        return _plain_read(s) if kind == "read" else _plain_attention(s, kind == "shared")
    from paper_2606_24033_amd import blockgtq as bg

    if kind == "read":
        return list(bg.blockgtq_dequantize_rows(s["cfg"], s["layout"], s["layer"], s["packed"], s["pos"], s["rows"],
                                                ctx_len=s["lens"], k_out=s["k_out"], v_out=s["v_out"]))
    if kind == "cross":
        return bg.blockgtq_cross_attn(s["cfg"], s["layout"], s["layer"], s["q"], s["lens"], s["max_ctx"], s["packed"],
                                      out=s["out"], workspace=s["ws"])
    return bg.blockgtq_decode_attn_shared(s["cfg"], s["layout"], s["layer"], s["q"], s["prefix_cfg"], s["prefix_packed"],
                                          s["prefix_len"], s["prefix"], s["lens"], s["max_ctx"], s["packed"],
                                          out=s["out"], workspace=s["ws"])


# ---------------------------------------------------------------- 64 bits

class _Exact:
    """The rows of one (layer, KV head) in 64 bits, bit by bit and group by group."""

    def __init__(self, s, layer, h):
        self.s, self.layer, self.h, self.bits = s, layer, h, s["bits_host"][layer * s["kv"] + h]
        self.books = [b.double().cuda() for b in _books()]

    @staticmethod
    def _stream(words):
        """Each row's words [rows, words] as its bits [rows, 32 words]."""
        return ((words[:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).flatten(1).double()

    def keys(self, cache, b, n):
        bits = self._stream(cache["k_codes"][self.layer, b, self.h, :n])
        groups = [w for w in range(1, 9) if (self.bits == w).any()]
        slots = (len(groups) + 1) // 2 * 2
        radii = cache["k_norms"][self.layer, b, self.h, :n * slots].view(n, slots).double()
        out, at = torch.zeros((n, D), dtype=torch.float64, device="cuda"), 0
        for i, w in enumerate(groups):
            blocks = np.nonzero(self.bits == w)[0]
            dims = torch.from_numpy(np.stack([blocks, blocks + HALF], 1).reshape(-1)).cuda()
            d = len(dims)
            weight = (2.0 ** torch.arange(w, device="cuda")).double()
            code = (bits[:, at:at + w * d].view(n, d, w) @ weight).long()
            unit = self.books[w - 1][code] / math.sqrt(d)
            out[:, dims] = (radii[:, i:i + 1] * unit) @ torch.from_numpy(self.s["rot_k"][d].astype(np.float64)).cuda()
            at += w * d
        return out

    def values(self, cache, b, n):
        bv = self.s["v_bits"]
        tiles = cache["v_codes"][self.layer, b, self.h, :(n + 31) // 32]
        bits = self._stream(tiles.reshape(-1, bv)).view(len(tiles), D, 32, bv)
        code = (bits @ (2.0 ** torch.arange(bv, device="cuda")).double()).long().transpose(1, 2).reshape(-1, D)[:n]
        radius = cache["v_norms"][self.layer, b, self.h, :n].double()[:, None]
        return (radius * self.books[bv - 1][code] / math.sqrt(D)) @ self.s["rot_v"].double()


def exact(c, seed):
    s = prepare(c, seed)
    L, B, H, G, kind = s["layers"], s["batch"], s["kv"], s["group"], s["kind"]
    f64 = {"dtype": torch.float64, "device": "cuda"}
    if kind == "read":
        outs = [torch.zeros((L, B, s["rows"], H, D), **f64) for _ in range(2)]
    else:
        q = s["q"].double().view(L, B, -1, H, G, D)
        out = torch.zeros(q.shape, **f64)
    for layer in range(L):
        for h in range(H):
            e = _Exact(s, layer, h)
            if kind == "shared":
                kp, vp = e.keys(s["prefix_cache"], 0, s["prefix"]), e.values(s["prefix_cache"], 0, s["prefix"])
            for b, n in enumerate(s["lens_host"]):
                k, v = e.keys(s["cache"], b, n), e.values(s["cache"], b, n)
                if kind == "read":
                    for x, y in zip(outs, (k[s["from"]:], v[s["from"]:])):
                        x[layer, b, :min(len(y), s["rows"]), h] = y[:s["rows"]]
                    continue
                if kind == "shared":
                    k, v = torch.cat([kp, k]), torch.cat([vp, v])
                if len(k):
                    for i in range(0, q.shape[2], 1024):
                        x = q[layer, b, i:i + 1024, h].reshape(-1, D) @ k.T / math.sqrt(D)
                        out[layer, b, i:i + 1024, h] = (torch.softmax(x, -1) @ v).view(-1, G, D)
    if kind == "read":
        return [x if L > 1 else x[0] for x in outs]
    return out.view(s["q"].shape)
