"""Measured cases of the paged-cache and differential-attention operators.

Three operators: `append` (new keys and values into a paged cache, rotated on the way, with the queries of the same
tokens), `paged` (attention of one or a few new tokens over that cache) and `diff` (differential attention, over a prompt
or over the paged cache).  `run` computes them either in elementary torch operations (`own` false) or through the
library's entry points (`own` true).
"""
import math

import numpy as np
import torch

own = False

_E4M3_MAX = 448.0
_ROPE_BASE = 500000.0
_handle = None


# ------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # a chat with one user: one token enters the cache (Llama-3 8B heads), where the launch is what counts
        {"name": "append 1 token", "op": "append", "B": 1, "new": 1, "ragged": False, "ctx": 1000, "Hq": 32, "Hkv": 8, "dqk": 128,
         "dv": 128, "page": 16, "e4m3": False, "heads_first": False, "rot": 128, "rot_at": 0, "span": 128, "inter": False, "pad": 0},
        # a decode step of a serving batch into an 8-bit cache, two rows of the batch unused (a padded, captured step)
        {"name": "append 62 tokens e4m3", "op": "append", "B": 62, "new": 1, "ragged": False, "ctx": 700, "Hq": 64, "Hkv": 8, "dqk": 128,
         "dv": 128, "page": 32, "e4m3": True, "heads_first": True, "rot": 128, "rot_at": 0, "span": 128, "inter": False, "pad": 2},
        # prompts of different lengths enter the cache (Llama-3 8B heads)
        {"name": "append ragged prompts", "op": "append", "B": 7, "new": 4096, "ragged": True, "ctx": 5, "Hq": 32, "Hkv": 8, "dqk": 128,
         "dv": 128, "page": 64, "e4m3": False, "heads_first": False, "rot": 128, "rot_at": 0, "span": 128, "inter": False, "pad": 3},
        # prompts of 192/128 heads (a quarter of a key is rotated, in interleaved pairs) into an 8-bit cache
        {"name": "append prompts 192/128", "op": "append", "B": 3, "new": 1001, "ragged": True, "ctx": 0, "Hq": 32, "Hkv": 32, "dqk": 192,
         "dv": 128, "page": 48, "e4m3": True, "heads_first": True, "rot": 64, "rot_at": 128, "span": 192, "inter": True, "pad": 0},
        # one user's next token (Llama-3 8B heads), short context: latency
        {"name": "paged 1 short", "op": "paged", "B": 1, "Sq": 1, "min": 777, "max": 777, "Hq": 32, "Hkv": 8, "dqk": 128, "dv": 128,
         "page": 16, "e4m3": False, "heads_first": False},
        # an ordinary serving batch, lengths spread, small pages
        {"name": "paged 64 ragged", "op": "paged", "B": 64, "Sq": 1, "min": 65, "max": 4096, "Hq": 32, "Hkv": 8, "dqk": 128, "dv": 128,
         "page": 16, "e4m3": False, "heads_first": False},
        # two users with the longest context of the benchmark
        {"name": "paged 2 x 131072", "op": "paged", "B": 2, "Sq": 1, "min": 131001, "max": 131072, "Hq": 32, "Hkv": 8, "dqk": 128, "dv": 128,
         "page": 64, "e4m3": False, "heads_first": True},
        # an 8-bit cache with eight queries to a key head (DeepSeek 67B heads)
        {"name": "paged 48 e4m3", "op": "paged", "B": 48, "Sq": 1, "min": 300, "max": 8192, "Hq": 64, "Hkv": 8, "dqk": 128, "dv": 128,
         "page": 128, "e4m3": True, "heads_first": True},
        # 192/128 heads without grouping, two draft tokens a sequence, pages that are no power of two
        {"name": "paged 192/128 2 tokens", "op": "paged", "B": 5, "Sq": 2, "min": 100, "max": 4001, "Hq": 32, "Hkv": 32, "dqk": 192, "dv": 128,
         "page": 48, "e4m3": False, "heads_first": False},
        # differential attention over a short prompt of odd length
        {"name": "diff prompt 1001", "op": "diff", "B": 2, "Hq": 8, "Hkv": 8, "Sq": 1001, "Sk": 1001, "causal": True, "rows_first": False},
        # over a long prompt with grouped heads, tensors as a projection leaves them
        {"name": "diff prompt 4096", "op": "diff", "B": 1, "Hq": 32, "Hkv": 8, "Sq": 4096, "Sk": 4096, "causal": True, "rows_first": True},
        # one new token a sequence of differential attention over the paged cache
        {"name": "diff paged 32", "op": "diff_paged", "B": 32, "Sq": 1, "min": 33, "max": 8000, "Hq": 16, "Hkv": 4, "dqk": 128, "dv": 128,
         "page": 32, "e4m3": False, "heads_first": False},
    ]


_HEADS = ((32, 8), (14, 2), (12, 12), (16, 16), (64, 8), (8, 1), (6, 3), (40, 8))
_DIMS = ((64, 64), (128, 128), (128, 128), (192, 128))
_PAGES = (16, 32, 48, 64, 128, 256)


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "append", "paged", "paged", "paged", "diff", "diff_paged"))
    Hq, Hkv = rng.choice(_HEADS)
    if op == "diff":
        S, causal = _log_int(rng, 1, 4096), rng.random() < 0.7
        Sk = min(4096, S + rng.choice((0, 0, rng.randint(0, 500))))
        while Hq * S * Sk * (1 if causal else 2) > 32 * 4096 * 4096:
            S -= 1
        return {"op": op, "B": 1 if S > 1024 else rng.randint(1, 4), "Hq": Hq, "Hkv": Hkv, "Sq": S, "Sk": Sk, "causal": causal,
                "rows_first": rng.random() < 0.5}
    dqk, dv = (128, 128) if op == "diff_paged" else rng.choice(_DIMS)
    case = {"op": op, "B": _log_int(rng, 1, 96), "Hq": Hq, "Hkv": Hkv, "dqk": dqk, "dv": dv, "page": rng.choice(_PAGES),
            "e4m3": rng.random() < 0.4, "heads_first": rng.random() < 0.5}
    if op == "append":
        inter = rng.random() < 0.4
        rot, at, span = rng.choice(((dqk, 0, dqk), (dqk // 2, 0, dqk), (dqk // 2, dqk // 2, dqk), (64, 0, 64), (0, 0, dqk), (48, 16, dqk)))
        total = _log_int(rng, 1, 12000)
        per = max(1, total // case["B"])
        case.update({"new": per, "ragged": rng.random() < 0.6, "ctx": rng.randint(0, 900), "rot": rot, "rot_at": at, "span": span,
                     "inter": inter, "pad": rng.choice((0, 0, 1, 5))})
        return case
    most = (1 << 30) // (case["B"] * Hkv * (dqk + dv) * 2)
    hi = _log_int(rng, 16, max(16, min(131072, most)))
    case.update({"Sq": rng.choice((1, 1, 1, 2, 3, 5, 8)), "max": hi, "min": max(8, hi // rng.choice((1, 3, 40)))})
    case["max"] = max(case["max"], case["min"])
    return case


# ------------------------------------------------------------------------------------------------- inputs

def _spread(n, lo, hi):
    """n whole numbers from lo to hi, the last of them hi: the same for a case whatever the seed."""
    return [hi if i == n - 1 else lo + (i * 7919 + 4201) % (hi - lo + 1) for i in range(n)]


def _new_counts(c):
    return _spread(c["B"], max(1, c["new"] // 8), c["new"]) if c["ragged"] else [c["new"]] * c["B"]


def _lens(c):
    if c["op"] == "append":
        return [n + (c["ctx"] * (i + 1)) // c["B"] for i, n in enumerate(_new_counts(c))]
    return _spread(c["B"], c["min"], c["max"])


def _cache(c, lens, g):
    """A pool of pages in shuffled order, its block table, and the scales of an 8-bit cache."""
    dev, B, ps, Hkv = "cuda", c["B"], c["page"], c["Hkv"]
    need = [-(-n // ps) for n in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, device=dev, generator=g).to(torch.int32)
    table = torch.zeros((B, max(need)), dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    both = []
    for d in (c["dqk"], c["dv"]):
        shape = (pages, Hkv, ps, d) if c["heads_first"] else (pages, ps, Hkv, d)
        x = torch.randn(shape, dtype=torch.bfloat16, device=dev, generator=g)
        if c["e4m3"]:
            x = (x * 20).clamp_(-_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn)
        both.append(x if c["heads_first"] else x.permute(0, 2, 1, 3))
    s = {"k_cache": both[0], "v_cache": both[1], "table": table, "lens": torch.tensor(lens, dtype=torch.int32, device=dev),
         "k_scale": None, "v_scale": None}
    if c["e4m3"]:
        s["k_scale"] = (0.9 + 0.2 * torch.rand(Hkv, device=dev, generator=g)) / 20
        s["v_scale"] = (0.9 + 0.2 * torch.rand(Hkv, device=dev, generator=g)) / 20
    return s


def _diff_weights(c, g):
    return {"lam": 0.2 + 0.6 * torch.rand(c["Hq"], device="cuda", generator=g),
            "weight": 1 + 0.1 * torch.randn(128, device="cuda", generator=g), "eps": 1e-5, "out_scale": 0.2}


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, dtype=torch.bfloat16, device="cuda", generator=g)  # noqa: E731
    s = {"case": c}
    if c["op"] == "diff":
        def heads(H, S):
            return rand(c["B"], S, H, 128).permute(0, 2, 1, 3) if c["rows_first"] else rand(c["B"], H, S, 128)
        s.update(q=heads(c["Hq"], c["Sq"]), k=heads(c["Hkv"], c["Sk"]), v=heads(c["Hkv"], c["Sk"]), **_diff_weights(c, g))
        return s
    lens = _lens(c)
    s.update(_cache(c, lens, g))
    if c["op"] != "append":
        s["q"] = rand(c["B"] * c["Sq"], c["Hq"], c["dqk"])
        if c["op"] == "diff_paged":
            s.update(_diff_weights(c, g))
        return s
    counts, Hq, Hkv, dqk, dv = _new_counts(c), c["Hq"], c["Hkv"], c["dqk"], c["dv"]
    n, rows = sum(counts), sum(counts) + c["pad"]
    if dqk == dv:       # what one projection leaves: the queries, keys and values of a token behind one another
        x = rand(rows, Hq + 2 * Hkv, dqk)
        s["q"], s["k"], s["v"] = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    else:
        s["q"], s["k"], s["v"] = rand(rows, Hq, dqk), rand(rows, Hkv, dqk), rand(rows, Hkv, dv)
    s["q_out"] = torch.zeros(rows, Hq, dqk, dtype=torch.bfloat16, device="cuda")
    s["n"] = n
    s["cu"] = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    s["cos_sin"] = None
    if c["rot"]:
        half = c["rot"] // 2
        freq = _ROPE_BASE ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        angle = torch.arange(max(lens), dtype=torch.float64, device="cuda")[:, None] * freq
        s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    return s


# ------------------------------------------------------------------------------------------------- one pass

def _library(s):
    """The library, its handle (one a process, as a user's program has) and the state's view of its cache."""
    global _handle
    from paper_2609_21264_b200 import binding
    if _handle is None:
        _handle = binding.fa_create(device=0)
    if "k_cache" in s and "cache" not in s:
        s["cache"] = binding.PagedCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
        if s.get("cos_sin") is not None:
            c = s["case"]
            s["rope"] = binding.Rope(s["cos_sin"], offset=c["rot_at"], span=c["span"], interleaved=c["inter"])
    return binding


def run(state):
    s, c = state, state["case"]
    if own:
        lib = _library(s)
        if c["op"] == "append":
            lib.append_paged(_handle, s["k"], s["v"], s["cache"], s["table"], s["lens"], cu_seqlens=s["cu"], q=s["q"], q_out=s["q_out"],
                             rope=s.get("rope"))
            return s["k_cache"], s["v_cache"], s["q_out"]
        if c["op"] == "paged":
            return lib.forward_paged(_handle, s["q"], s["cache"], s["table"], s["lens"])
        if c["op"] == "diff_paged":
            return lib.forward_paged_diff(_handle, s["q"], s["cache"], s["table"], s["lens"], s["lam"], norm_weight=s["weight"],
                                          eps=s["eps"], out_scale=s["out_scale"])
        return lib.forward_diff(_handle, s["q"], s["k"], s["v"], s["lam"], causal=c["causal"], norm_weight=s["weight"], eps=s["eps"],
                                out_scale=s["out_scale"])
    if c["op"] == "append":
        return _plain_append(s, c)
    if c["op"] == "paged":
        return _plain_paged(s, c)
    if c["op"] == "diff_paged":
        return _plain_diff_paged(s, c)
    return _plain_diff(s, c)


def _turn(x, rows, c):
    """x [n, H, d] float, rotated by the rows [n, rot] of the table."""
    if rows is None:
        return x
    n, H, d = x.shape
    half = c["rot"] // 2
    cos, sin = rows[:, None, None, :half], rows[:, None, None, half:]
    x = x.reshape(n, H, d // c["span"], c["span"])
    part = x[..., c["rot_at"]:c["rot_at"] + c["rot"]]
    a, b = (part[..., 0::2], part[..., 1::2]) if c["inter"] else (part[..., :half], part[..., half:])
    y, z = a * cos - b * sin, b * cos + a * sin
    part = torch.stack([y, z], dim=-1).flatten(-2) if c["inter"] else torch.cat([y, z], dim=-1)
    return torch.cat([x[..., :c["rot_at"]], part, x[..., c["rot_at"] + c["rot"]:]], dim=-1).reshape(n, H, d)


def _plain_append(s, c):
    n, ps = s["n"], c["page"]
    t = torch.arange(n, device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["cu"][1:], t, right=True)
    pos = (s["lens"][b] - s["cu"][b + 1] + t).long()
    page, slot = s["table"][b, pos // ps].long(), pos % ps
    rows = None if s["cos_sin"] is None else s["cos_sin"][pos]
    k, v = _turn(s["k"][:n].float(), rows, c), s["v"][:n].float()
    s["q_out"][:n] = _turn(s["q"][:n].float(), rows, c).to(torch.bfloat16)
    if c["e4m3"]:
        k = (k / s["k_scale"][:, None]).clamp(-_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        v = (v / s["v_scale"][:, None]).clamp(-_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        s["k_cache"].view(torch.uint8).permute(0, 2, 1, 3)[page, slot] = k
        s["v_cache"].view(torch.uint8).permute(0, 2, 1, 3)[page, slot] = v
    else:
        s["k_cache"].permute(0, 2, 1, 3)[page, slot] = k.to(torch.bfloat16)
        s["v_cache"].permute(0, 2, 1, 3)[page, slot] = v.to(torch.bfloat16)
    return s["k_cache"], s["v_cache"], s["q_out"]


def _gathered(cache, scale, table):
    """The cache's rows [B, Hkv, pages * page, d] in 32 bits, in the order of the sequences."""
    B, P = table.shape
    _, Hkv, ps, d = cache.shape
    x = cache.view(torch.uint8) if cache.dtype != torch.bfloat16 else cache
    x = x.permute(0, 2, 1, 3)[table.long()]
    x = (x.view(cache.dtype).float()).reshape(B, P * ps, Hkv, d).transpose(1, 2)
    return x if scale is None else x * scale[:, None, None]


def _softmax(scores, seen):
    """Softmax over the last axis of what is seen, and the log of its sum."""
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = (scores - top).exp()
    total = p.sum(-1, keepdim=True)
    return p / total, (top + total.log()).squeeze(-1)


def _plain_paged(s, c):
    B, Sq, Hq, Hkv = c["B"], c["Sq"], c["Hq"], c["Hkv"]
    k, v = _gathered(s["k_cache"], s["k_scale"], s["table"]), _gathered(s["v_cache"], s["v_scale"], s["table"])
    n = k.shape[2]
    q = s["q"].float().reshape(B, Sq, Hkv, Hq // Hkv, c["dqk"]).transpose(1, 2).reshape(B, Hkv, Sq * (Hq // Hkv), c["dqk"])
    last = (s["lens"][:, None] - Sq + torch.arange(Sq, device="cuda")).repeat_interleave(Hq // Hkv, 1)
    seen = torch.arange(n, device="cuda") <= last[:, None, :, None]
    p, lse = _softmax(torch.matmul(q, k.transpose(2, 3)) * c["dqk"] ** -0.5, seen)
    o = torch.matmul(p, v).reshape(B, Hkv, Sq, Hq // Hkv, c["dv"]).transpose(1, 2).reshape(B * Sq, Hq, c["dv"])
    lse = lse.reshape(B, Hkv, Sq, Hq // Hkv).permute(1, 3, 0, 2).reshape(Hq, B * Sq)
    return o.to(torch.bfloat16), lse


def _normed(y, s):
    return s["out_scale"] * s["weight"] * y * torch.rsqrt(y.square().mean(-1, keepdim=True) + s["eps"])


def _plain_diff_paged(s, c):
    B, Sq, Hq, Hkv = c["B"], c["Sq"], c["Hq"], c["Hkv"]
    G = Hq // Hkv
    k, v = _gathered(s["k_cache"], s["k_scale"], s["table"]), _gathered(s["v_cache"], s["v_scale"], s["table"])
    q = s["q"].float().reshape(B, Sq, Hkv, G, 128).transpose(1, 2).reshape(B, Hkv, Sq * G, 128)
    last = (s["lens"][:, None] - Sq + torch.arange(Sq, device="cuda")).repeat_interleave(G, 1)
    seen = torch.arange(k.shape[2], device="cuda") <= last[:, None, :, None]
    one, _ = _softmax(torch.matmul(q[..., :64], k[..., :64].transpose(2, 3)) * 0.125, seen)
    two, _ = _softmax(torch.matmul(q[..., 64:], k[..., 64:].transpose(2, 3)) * 0.125, seen)
    lam = s["lam"].reshape(Hkv, 1, G).expand(Hkv, Sq, G).reshape(Hkv, Sq * G, 1)
    y = torch.matmul(one - lam * two, v)
    y = y.reshape(B, Hkv, Sq, G, 128).transpose(1, 2).reshape(B * Sq, Hq, 128)
    return _normed(y, s).to(torch.bfloat16)


def _plain_diff(s, c):
    G = c["Hq"] // c["Hkv"]
    q, k, v = s["q"].float(), s["k"].float().repeat_interleave(G, 1), s["v"].float().repeat_interleave(G, 1)
    i, j = torch.arange(c["Sq"], device="cuda")[:, None], torch.arange(c["Sk"], device="cuda")
    seen = (j <= i + (c["Sk"] - c["Sq"])) if c["causal"] else torch.ones_like(i * j, dtype=torch.bool)
    one, _ = _softmax(torch.matmul(q[..., :64], k[..., :64].transpose(2, 3)) * 0.125, seen)
    two, _ = _softmax(torch.matmul(q[..., 64:], k[..., 64:].transpose(2, 3)) * 0.125, seen)
    return _normed(torch.matmul(one - s["lam"][:, None, None] * two, v), s).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------- what cannot be done without

def work(case):
    c = case
    if c["op"] == "diff":
        rows = min(c["Sq"], c["Sk"]) if c["causal"] else 0
        back = c["Sk"] - c["Sq"]
        pairs = sum(max(0, min(c["Sk"], i + back + 1)) for i in range(c["Sq"])) if rows else c["Sq"] * c["Sk"]
        return {"bytes": c["B"] * 256 * (2 * c["Hq"] * c["Sq"] + 2 * c["Hkv"] * c["Sk"]), "flops": 2 * c["B"] * c["Hq"] * pairs * (128 + 256)}
    size, lens = (1 if c["e4m3"] else 2), _lens(c)
    if c["op"] == "append":
        n = sum(_new_counts(c))
        kv = c["Hkv"] * (c["dqk"] + c["dv"])
        return {"bytes": n * (kv * (2 + size) + c["Hq"] * c["dqk"] * 4 + c["rot"] * 4),
                "flops": n * 3 * (c["Hkv"] + c["Hq"]) * c["rot"] * (c["dqk"] // c["span"])}
    tokens = c["B"] * c["Sq"]
    flops = 2 * sum(lens) * c["Sq"] * c["Hq"] * ((128 + 256) if c["op"] == "diff_paged" else c["dqk"] + c["dv"])
    return {"bytes": sum(lens) * c["Hkv"] * (c["dqk"] + c["dv"]) * size + tokens * c["Hq"] * (c["dqk"] + c["dv"]) * 2, "flops": flops}


# ------------------------------------------------------------------------------------------------- the definition, in 64 bits

def _exact_turn(x, row, c):
    """One token's heads [H, d] in 64 bits, every pair turned by its angle's cosine and sine."""
    if row is None:
        return x
    y = x.clone()
    for first in range(c["rot_at"], c["dqk"], c["span"]):
        for i in range(c["rot"] // 2):
            a, b = (first + 2 * i, first + 2 * i + 1) if c["inter"] else (first + i, first + c["rot"] // 2 + i)
            y[..., a] = x[..., a] * row[..., i, None] - x[..., b] * row[..., c["rot"] // 2 + i, None]
            y[..., b] = x[..., b] * row[..., i, None] + x[..., a] * row[..., c["rot"] // 2 + i, None]
    return y


def _exact_rows(cache, scale, pages, n):
    """The first n rows [Hkv, n, d] of a sequence in 64 bits."""
    x = torch.cat([cache[p].double() for p in pages], dim=1)[:, :n]
    return x if scale is None else x * scale.double()[:, None, None]


def _exact_map(q, k, scale, last):
    """q [n, d], k [m, d]: the rows' probabilities over the keys up to `last` [n], and the log-sum-exp."""
    z = (q @ k.T) * scale
    z[torch.arange(k.shape[0], device=z.device)[None, :] > last[:, None]] = -math.inf
    lse = torch.logsumexp(z, dim=1)
    return torch.exp(z - lse[:, None]), lse


def _exact_norm(y, s):
    return s["out_scale"] * s["weight"].double() * y / torch.sqrt((y * y).mean(-1, keepdim=True) + s["eps"])


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "append":
        lens, counts, ps = _lens(c), _new_counts(c), c["page"]
        k_cache, v_cache, q_out = s["k_cache"].double(), s["v_cache"].double(), s["q_out"].double()
        table, at = s["table"].tolist(), 0
        for b, (n, m) in enumerate(zip(lens, counts)):
            row = None if s["cos_sin"] is None else s["cos_sin"][n - m:n].double()
            k, v = _exact_turn(s["k"][at:at + m].double(), row, c), s["v"][at:at + m].double()
            q_out[at:at + m] = _exact_turn(s["q"][at:at + m].double(), row, c)
            if c["e4m3"]:
                k, v = k / s["k_scale"].double()[:, None], v / s["v_scale"].double()[:, None]
            first = n - m
            for j in range(first // ps, (n - 1) // ps + 1):
                lo, hi = max(first, j * ps), min(n, (j + 1) * ps)
                k_cache[table[b][j], :, lo - j * ps:hi - j * ps] = k[lo - first:hi - first].transpose(0, 1)
                v_cache[table[b][j], :, lo - j * ps:hi - j * ps] = v[lo - first:hi - first].transpose(0, 1)
            at += m
        if c["e4m3"]:
            k_cache, v_cache = k_cache.clamp(-_E4M3_MAX, _E4M3_MAX), v_cache.clamp(-_E4M3_MAX, _E4M3_MAX)
        return k_cache, v_cache, q_out
    G = c["Hq"] // c["Hkv"]
    if c["op"] == "diff":
        o = torch.empty(c["B"], c["Hq"], c["Sq"], 128, dtype=torch.float64, device="cuda")
        last = torch.arange(c["Sq"], device="cuda") + (c["Sk"] - c["Sq"]) if c["causal"] else torch.full((c["Sq"],), c["Sk"], device="cuda")
        for b in range(c["B"]):
            for h in range(c["Hq"]):
                q, k, v = s["q"][b, h].double(), s["k"][b, h // G].double(), s["v"][b, h // G].double()
                one, two = (_exact_map(q[:, x], k[:, x], 0.125, last)[0] for x in (slice(0, 64), slice(64, 128)))
                o[b, h] = _exact_norm(one @ v - s["lam"][h].double() * (two @ v), s)
        return o
    Sq, lens, table = c["Sq"], _lens(c), s["table"].tolist()
    o = torch.empty(c["B"] * Sq, c["Hq"], c["dv"], dtype=torch.float64, device="cuda")
    lse = torch.empty(c["Hq"], c["B"] * Sq, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        pages = table[b][:-(-n // c["page"])]
        k, v = _exact_rows(s["k_cache"], s["k_scale"], pages, n), _exact_rows(s["v_cache"], s["v_scale"], pages, n)
        last = torch.arange(n - Sq, n, device="cuda")
        here = slice(b * Sq, (b + 1) * Sq)
        for h in range(c["Hq"]):
            q = s["q"][here, h].double()
            if c["op"] == "paged":
                p, lse[h, here] = _exact_map(q, k[h // G], c["dqk"] ** -0.5, last)
                o[here, h] = p @ v[h // G]
            else:
                one, two = (_exact_map(q[:, x], k[h // G][:, x], 0.125, last)[0] for x in (slice(0, 64), slice(64, 128)))
                o[here, h] = _exact_norm(one @ v[h // G] - s["lam"][h].double() * (two @ v[h // G]), s)
    return o if c["op"] == "diff_paged" else (o, lse)
