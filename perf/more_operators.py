"""Measured cases of the operators that decode drafted tokens over a paged cache.

Five operators, in the order in which a step of speculative decoding uses them: `layout` (what each token of a drafted tree
sees, and its position), `append` (the drafts' keys and values into the cache, rotated by given positions of one or several
axes), `tree` (attention of the drafts over the cache and over one another), `compact` (the accepted drafts moved up in the
caches of all layers) and `copy` (pages copied in the caches of all layers: a fork).  `run` computes them either in elementary
torch operations (`own` false) or through the library's entry points (`own` true).
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
        # one user, a small tree: the launch and a chain of look-ups are what counts
        {"name": "layout 1 x 26", "op": "layout", "B": 1, "T": 26, "ragged": False, "ctx": 1000},
        # a serving batch whose draft model grew trees of different sizes
        {"name": "layout 96 ragged", "op": "layout", "B": 96, "T": 64, "ragged": True, "ctx": 4000},
        # the same small tree into one user's cache (Llama-3 8B heads), at positions that follow the depth and not the slot
        {"name": "append 26 drafts", "op": "append", "B": 1, "T": 26, "ragged": False, "ctx": 1000, "Hq": 32, "Hkv": 8, "dqk": 128, "dv": 128,
         "page": 16, "e4m3": False, "heads_first": False, "rot": 128, "axes": 1, "by": "sections", "inter": False, "pad": 0},
        # prompts of text and pictures: every token has a time, a row and a column, each of which turns its own pairs
        {"name": "append pictures 3 axes", "op": "append", "B": 3, "T": 4001, "ragged": True, "ctx": 0, "Hq": 32, "Hkv": 8, "dqk": 128, "dv": 128,
         "page": 64, "e4m3": False, "heads_first": True, "rot": 128, "axes": 3, "by": "sections", "inter": False, "pad": 2},
        # one user's tree over a short context (Llama-3 8B heads): latency
        {"name": "tree 1 x 26", "op": "tree", "B": 1, "T": 26, "ragged": False, "min": 1003, "max": 1003, "Hq": 32, "Hkv": 8, "dqk": 128, "dv": 128,
         "page": 16, "e4m3": False, "heads_first": False},
        # an ordinary batch with large trees: 256 query rows to a key head
        {"name": "tree 16 x 64 ragged", "op": "tree", "B": 16, "T": 64, "ragged": True, "min": 129, "max": 8192, "Hq": 32, "Hkv": 8, "dqk": 128,
         "dv": 128, "page": 32, "e4m3": False, "heads_first": False},
        # an 8-bit cache with eight queries to a key head (DeepSeek 67B heads), small trees
        {"name": "tree 48 x 13 e4m3", "op": "tree", "B": 48, "T": 13, "ragged": True, "min": 300, "max": 8192, "Hq": 64, "Hkv": 8, "dqk": 128,
         "dv": 128, "page": 128, "e4m3": True, "heads_first": True},
        # two long contexts of 192/128 heads without grouping, pages that are no power of two
        {"name": "tree 192/128 2 x 20000", "op": "tree", "B": 2, "T": 31, "ragged": False, "min": 19001, "max": 20000, "Hq": 32, "Hkv": 32,
         "dqk": 192, "dv": 128, "page": 48, "e4m3": False, "heads_first": False},
        # one user's accepted path moved up in 32 layers
        {"name": "compact 1 x 26", "op": "compact", "B": 1, "T": 26, "ragged": False, "ctx": 1000, "accept": 5, "layers": 32, "Hkv": 8, "dqk": 128,
         "dv": 128, "page": 16, "e4m3": False, "heads_first": False},
        # a serving batch's accepted paths in 32 layers of an 8-bit cache
        {"name": "compact 64 e4m3", "op": "compact", "B": 64, "T": 40, "ragged": True, "ctx": 900, "accept": 7, "layers": 32, "Hkv": 8, "dqk": 128,
         "dv": 128, "page": 32, "e4m3": True, "heads_first": True},
        # a sequence is forked: its last page, of which a part is filled, in 32 layers
        {"name": "copy 1 page", "op": "copy", "n": 1, "pad": 0, "filled": True, "layers": 32, "Hkv": 8, "dqk": 128, "dv": 128, "page": 64,
         "e4m3": False, "heads_first": False},
        # a pool is put in order, or many sequences fork at once; some entries of the list unused (a captured step)
        {"name": "copy 192 pages", "op": "copy", "n": 192, "pad": 7, "filled": False, "layers": 16, "Hkv": 8, "dqk": 128, "dv": 128, "page": 64,
         "e4m3": False, "heads_first": True},
    ]


_HEADS = ((32, 8), (14, 2), (12, 12), (16, 16), (64, 8), (8, 1), (6, 3), (40, 8))
_DIMS = ((64, 64), (128, 128), (128, 128), (192, 128))
_PAGES = (16, 32, 48, 64, 128, 256)


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("layout", "append", "append", "tree", "tree", "tree", "compact", "copy"))
    if op == "layout":
        return {"op": op, "B": _log_int(rng, 1, 96), "T": _log_int(rng, 1, 64), "ragged": rng.random() < 0.6, "ctx": rng.randint(0, 4000)}
    Hq, Hkv = rng.choice(_HEADS)
    dqk, dv = rng.choice(_DIMS)
    case = {"op": op, "Hq": Hq, "Hkv": Hkv, "dqk": dqk, "dv": dv, "page": rng.choice(_PAGES), "e4m3": rng.random() < 0.4,
            "heads_first": rng.random() < 0.5}
    row = Hkv * (dqk + dv) * (1 if case["e4m3"] else 2)          # bytes of a key and its value
    if op == "copy":
        case.update({"layers": rng.choice((1, 4, 16, 32)), "pad": rng.choice((0, 3)), "filled": rng.random() < 0.5})
        case["n"] = _log_int(rng, 1, max(1, min(192, (700 << 20) // (row * case["page"] * case["layers"]))))
        return case
    case["B"], case["ragged"] = _log_int(rng, 1, 64), rng.random() < 0.6
    if op == "compact":
        case.update({"T": _log_int(rng, 2, 64), "ctx": rng.randint(0, 900), "layers": rng.choice((1, 4, 16, 32))})
        case["accept"] = rng.randint(1, min(12, case["T"]))
        while case["B"] * (case["ctx"] + case["T"] + case["page"]) * row * case["layers"] > (1 << 30):
            case["B"], case["layers"] = (case["B"] + 1) // 2, max(1, case["layers"] // 2)
        return case
    if op == "append":
        case["rot"] = rng.choice((dqk, dqk, 64, 48))
        total = _log_int(rng, 1, 9000)
        case.update({"T": max(1, total // case["B"]), "ctx": rng.randint(0, 900), "axes": rng.choice((1, 2, 3, 3)), "by": rng.choice(("sections", "turns")),
                     "inter": rng.random() < 0.4, "pad": rng.choice((0, 0, 1, 5))})
        return case
    case["T"] = _log_int(rng, 1, 64)
    most = min((700 << 20) // (case["B"] * row), 16 * 4160 * 64 * 32 // (case["B"] * case["T"] * Hq))
    hi = _log_int(rng, 70, max(70, min(40000, most)))
    case.update({"max": hi, "min": max(65, hi // rng.choice((1, 3, 40)))})
    return case


# ------------------------------------------------------------------------------------------------- inputs

def _spread(n, lo, hi):
    """n whole numbers from lo to hi, the last of them hi: the same for a case whatever the seed."""
    return [hi if i == n - 1 else lo + (i * 7919 + 4201) % (hi - lo + 1) for i in range(n)]


def _counts(c):
    return _spread(c["B"], max(1, c["T"] // 4), c["T"]) if c["ragged"] else [c["T"]] * c["B"]


def _lens(c):
    if c["op"] == "tree":
        return _spread(c["B"], c["min"], c["max"])
    return [n + (c["ctx"] * (i + 1)) // c["B"] for i, n in enumerate(_counts(c))]


def _accepted(c):
    return [min(n, 1 + (i * 5 + 2) % c["accept"]) if i < c["B"] - 1 else min(n, c["accept"]) for i, n in enumerate(_counts(c))]


def _axis_of_pair(c):
    """Which axis turns each pair: consecutive sections (the first half as long as the others), or in turns."""
    pairs, axes = c["rot"] // 2, c["axes"]
    if axes == 1:
        return [0] * pairs
    if c["by"] == "turns":
        return [i % axes for i in range(pairs)]
    unit = 2 * axes - 1
    return [min(axes - 1, (i * unit // pairs + 1) // 2) for i in range(pairs)]


def _pools(c, pages, g):
    """K and V pools of all layers, [layers, pages, Hkv, page, d] in either order of heads and slots."""
    both = []
    for d in (c["dqk"], c["dv"]):
        shape = (pages, c["Hkv"], c["page"], d) if c["heads_first"] else (pages, c["page"], c["Hkv"], d)
        x = torch.randn((c.get("layers", 1), *shape), dtype=torch.bfloat16, device="cuda", generator=g)
        if c["e4m3"]:
            x = (x * 20).clamp_(-_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn)
        both.append(x if c["heads_first"] else x.transpose(2, 3))
    return both


def _scales(c, g):
    return [(0.9 + 0.2 * torch.rand(c["Hkv"], device="cuda", generator=g)) / 20 if c["e4m3"] else None for _ in range(2)]


def _table(c, lens, g):
    """A block table over shuffled pages, and the number of pages."""
    need = [-(-n // c["page"]) for n in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    width = max(need)
    at = torch.arange(width, device="cuda")[None] + torch.tensor([0] + list(np.cumsum(need)[:-1]), device="cuda")[:, None]
    held = torch.arange(width, device="cuda")[None] < torch.tensor(need, device="cuda")[:, None]
    return torch.where(held, order[at.clamp(max=pages - 1)], 0).to(torch.int32), pages


def _trees(c, g):
    """A parent for every drafted token of every sequence [B, T]: an earlier token of the tree, or -1 (the last cached token)."""
    u = torch.rand(c["B"], c["T"], device="cuda", generator=g)
    at = torch.arange(c["T"], device="cuda")
    # (as a draft model grows them: half of the tokens continue a token not far before them)
    near = (at - 1 - (u * 2 * 4).long()).clamp(min=-1)
    return torch.where(u < 0.5, near, ((u - 0.5) * 2 * (at + 1)).long().clamp(max=at) - 1)


def _packed_rows(c):
    """Places [total] of the sequences' tokens in a [B * T] array."""
    return torch.cat([torch.arange(n) + b * c["T"] for b, n in enumerate(_counts(c))]).cuda()


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, dtype=torch.bfloat16, device="cuda", generator=g)  # noqa: E731
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"case": c}
    if c["op"] == "copy":
        n, pages = c["n"], 2 * c["n"] + 5
        s["k"], s["v"] = _pools(c, pages, g)
        order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
        none = torch.full((c["pad"],), -1, dtype=torch.int32, device="cuda")
        s["src"], s["dst"] = torch.cat([order[:n], none]), torch.cat([order[n:2 * n], none])
        s["slots"] = ints([1 + (i * 11 + 8) % c["page"] for i in range(n + c["pad"])]) if c["filled"] else None
        return s
    counts, lens = _counts(c), _lens(c)
    s["n"] = sum(counts)
    s["lens"], s["cu"] = ints(lens), ints([0] + list(np.cumsum(counts)))
    if c["op"] == "layout":
        s["parents"] = _trees(c, g).reshape(-1)[_packed_rows(c)].to(torch.int32)
        return s
    s["table"], pages = _table(c, lens, g)
    s["k"], s["v"] = _pools(c, pages, g)
    if c["op"] == "compact":
        # what was accepted: the first tokens of the tree as far as they were, then tokens from further down
        keep = torch.zeros(c["B"], c["accept"], dtype=torch.int64)
        pick = torch.Generator().manual_seed(seed)
        for b, (n, a) in enumerate(zip(counts, _accepted(c))):
            stay = int(torch.randint(0, a + 1, (1,), generator=pick))
            stay = max(stay, 2 * a - n)
            keep[b, :stay] = torch.arange(stay)
            keep[b, stay:a] = (a + torch.randperm(n - a, generator=pick)[:a - stay]).sort().values
        s["keep"], s["kept"] = keep.to(torch.int32).cuda(), ints(_accepted(c))
        return s
    s["k_scale"], s["v_scale"] = _scales(c, g)
    Hq, Hkv, dqk, dv = c["Hq"], c["Hkv"], c["dqk"], c["dv"]
    if c["op"] == "tree":
        s["q"] = rand(s["n"], Hq, dqk)
        s["mask"] = _packed_mask(_seen(_trees(c, g))).reshape(c["B"] * c["T"], -1)[_packed_rows(c)]
        return s
    rows = s["n"] + c["pad"]
    if dqk == dv:       # what one projection leaves: the queries, keys and values of a token behind one another
        x = rand(rows, Hq + 2 * Hkv, dqk)
        s["q"], s["k_new"], s["v_new"] = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    else:
        s["q"], s["k_new"], s["v_new"] = rand(rows, Hq, dqk), rand(rows, Hkv, dqk), rand(rows, Hkv, dv)
    s["q_out"] = torch.zeros(rows, Hq, dqk, dtype=torch.bfloat16, device="cuda")
    # the first axis goes on with the sequence, the others are places in a picture of 48 columns
    at = torch.cat([torch.arange(l - n, l) for n, l in zip(counts, lens)] + [torch.zeros(c["pad"], dtype=torch.int64)])
    away = int(torch.randint(0, 7, (1,), device="cuda", generator=g))
    s["pos"] = torch.stack([at + away, at // 48 + away, at % 48, at % 7][:c["axes"]]).to(torch.int32).cuda()
    half = c["rot"] // 2
    freq = _ROPE_BASE ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    angle = torch.arange(max(lens) + 8, dtype=torch.float64, device="cuda")[:, None] * freq
    s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    return s


# ------------------------------------------------------------------------------------------------- one pass

def _library(s):
    """The library, its handle (one a process, as a user's program has) and the state's view of its caches."""
    global _handle
    from paper_2609_21264_b200 import binding
    if _handle is None:
        _handle = binding.fa_create(device=0)
    if "k" in s and "cache" not in s:
        c = s["case"]
        each = [binding.PagedCache(k, v, s.get("k_scale"), s.get("v_scale")) for k, v in zip(s["k"], s["v"])]
        s["cache"] = each[0] if c["op"] in ("append", "tree") else binding.PagedCaches(each)
        if c["op"] == "append":
            s["rope"] = binding.Rope(s["cos_sin"], interleaved=c["inter"], axis_of_pair=_axis_of_pair(c))
    return binding


def run(state):
    s, c = state, state["case"]
    if own:
        lib = _library(s)
        if c["op"] == "layout":
            return lib.tree_layout(_handle, s["parents"], s["lens"], cu_seqlens=s["cu"], max_tokens=c["T"])
        if c["op"] == "append":
            lib.append_paged(_handle, s["k_new"], s["v_new"], s["cache"], s["table"], s["lens"], cu_seqlens=s["cu"], q=s["q"], q_out=s["q_out"],
                             rope=s["rope"], positions=s["pos"])
            return s["k"], s["v"], s["q_out"]
        if c["op"] == "tree":
            return lib.forward_paged_tree(_handle, s["q"], s["cache"], s["table"], s["lens"], s["mask"], cu_seqlens=s["cu"], max_tokens=c["T"])
        if c["op"] == "compact":
            return s["k"], s["v"], lib.compact_paged(_handle, s["cache"], s["table"], s["lens"], s["keep"], s["kept"], cu_seqlens=s["cu"])
        lib.copy_pages(_handle, s["cache"], s["src"], s["dst"], slots=s["slots"])
        return s["k"], s["v"]
    if c["op"] == "layout":
        return _plain_layout(s, c)
    if c["op"] == "append":
        return _plain_append(s, c)
    if c["op"] == "tree":
        return _plain_tree(s, c)
    if c["op"] == "compact":
        return _plain_compact(s, c)
    return _plain_copy(s, c)


def _seen(parents):
    """[B, T, T] truth values: token i sees token j, itself and its ancestors; by doubling of the paths."""
    B, T = parents.shape
    at = torch.arange(T, device=parents.device)
    a = ((at[None, None] == parents[:, :, None]) | (at[None, None] == at[None, :, None])).float()
    for _ in range(max(1, (T - 1).bit_length())):
        a = (torch.matmul(a, a) > 0).float()
    return a > 0


def _packed_mask(seen):
    """[B, T, words] int32: bit j % 32 of word j / 32 of a token says that it sees token j."""
    B, T, n = seen.shape
    words = -(-n // 32)
    wide = torch.zeros(B, T, words * 32, dtype=torch.int64, device=seen.device)
    wide[:, :, :n] = seen
    w = (wide.reshape(B, T, words, 32) << torch.arange(32, device=seen.device)).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _places(s, n):
    """Sequence and place among its drafted tokens of every token."""
    t = torch.arange(n, device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["cu"][1:], t, right=True)
    return b, (t - s["cu"][b]).long()


def _plain_layout(s, c):
    b, i = _places(s, s["n"])
    parents = torch.full((c["B"], c["T"]), -1, dtype=torch.int64, device="cuda")
    parents[b, i] = s["parents"].long()
    seen = _seen(parents)
    count = (s["cu"][1:] - s["cu"][:-1])[b]
    pos = s["lens"][b] - count + seen[b, i].sum(-1) - 1
    return _packed_mask(seen)[b, i], pos.to(torch.int32)


def _turn(x, cos, sin, c):
    """x [n, H, d] float, the first `rot` of its dimensions turned in pairs; cos and sin [n, 1, rot / 2]."""
    rot = c["rot"]
    part = x[..., :rot]
    a, b = (part[..., 0::2], part[..., 1::2]) if c["inter"] else (part[..., :rot // 2], part[..., rot // 2:])
    y, z = a * cos - b * sin, b * cos + a * sin
    part = torch.stack([y, z], dim=-1).flatten(-2) if c["inter"] else torch.cat([y, z], dim=-1)
    return torch.cat([part, x[..., rot:]], dim=-1)


def _plain_append(s, c):
    n, ps, half = s["n"], c["page"], c["rot"] // 2
    b, i = _places(s, n)
    at = (s["lens"][b] - (s["cu"][b + 1] - s["cu"][b])).long() + i
    page, slot = s["table"][b, at // ps].long(), at % ps
    axis = torch.tensor(_axis_of_pair(c), device="cuda")
    rows = s["pos"][:, :n][axis].long().T                                   # [n, half]
    pair = torch.arange(half, device="cuda")
    cos, sin = s["cos_sin"][rows, pair][:, None], s["cos_sin"][rows, half + pair][:, None]
    k, v = _turn(s["k_new"][:n].float(), cos, sin, c), s["v_new"][:n].float()
    s["q_out"][:n] = _turn(s["q"][:n].float(), cos, sin, c).to(torch.bfloat16)
    k_cache, v_cache = s["k"][0].permute(0, 2, 1, 3), s["v"][0].permute(0, 2, 1, 3)
    if c["e4m3"]:
        k = (k / s["k_scale"][:, None]).clamp(-_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        v = (v / s["v_scale"][:, None]).clamp(-_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        k_cache.view(torch.uint8)[page, slot] = k
        v_cache.view(torch.uint8)[page, slot] = v
    else:
        k_cache[page, slot] = k.to(torch.bfloat16)
        v_cache[page, slot] = v.to(torch.bfloat16)
    return s["k"], s["v"], s["q_out"]


def _gathered(cache, scale, table):
    """The cache's rows [B, Hkv, pages * page, d] in 32 bits, in the order of the sequences."""
    B, P = table.shape
    _, Hkv, ps, d = cache.shape
    x = cache.view(torch.uint8) if cache.dtype != torch.bfloat16 else cache
    x = x.permute(0, 2, 1, 3)[table.long()]
    x = (x.view(cache.dtype).float()).reshape(B, P * ps, Hkv, d).transpose(1, 2)
    return x if scale is None else x * scale[:, None, None]


def _plain_tree(s, c):
    B, T, Hq, Hkv = c["B"], c["T"], c["Hq"], c["Hkv"]
    G = Hq // Hkv
    k, v = _gathered(s["k"][0], s["k_scale"], s["table"]), _gathered(s["v"][0], s["v_scale"], s["table"])
    n = k.shape[2]
    b, i = _places(s, s["n"])
    q = torch.zeros(B, T, Hq, c["dqk"], device="cuda")
    q[b, i] = s["q"].float()
    mask = torch.zeros(B, T, s["mask"].shape[1], dtype=torch.int32, device="cuda")
    mask[b, i] = s["mask"]
    first = s["lens"] - (s["cu"][1:] - s["cu"][:-1])                        # the first drafted key
    j = torch.arange(n, device="cuda")[None] - first[:, None]               # [B, n]: its number among the drafts
    at = j.clamp(0, 32 * mask.shape[2] - 1)
    bit = (torch.gather(mask, 2, (at // 32)[:, None].expand(B, T, n).long()) >> (at % 32)[:, None]) & 1
    seen = (j[:, None] < 0) | ((bit == 1) & (torch.arange(n, device="cuda") < s["lens"][:, None])[:, None])
    q = q.reshape(B, T, Hkv, G, c["dqk"]).transpose(1, 2).reshape(B, Hkv, T * G, c["dqk"])
    x = torch.matmul(q, k.transpose(2, 3)) * c["dqk"] ** -0.5
    x.masked_fill_(~seen.repeat_interleave(G, 1)[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log()).squeeze(-1)
    o = o.reshape(B, Hkv, T, G, c["dv"]).transpose(1, 2).reshape(B, T, Hq, c["dv"])[b, i]
    lse = lse.reshape(B, Hkv, T, G).transpose(1, 2).reshape(B, T, Hq)[b, i].T
    return o.to(torch.bfloat16), lse.contiguous()


def _plain_compact(s, c):
    ps, a = c["page"], c["accept"]
    first = s["lens"] - (s["cu"][1:] - s["cu"][:-1])
    m = torch.arange(a, device="cuda", dtype=torch.int32)[None]
    live = m < s["kept"][:, None]
    # (unused places name the sequence's first kept token twice)
    src = (first[:, None] + torch.where(live, s["keep"], s["keep"][:, :1])).long()
    dst = (first[:, None] + torch.where(live, m, 0)).long()
    b = torch.arange(c["B"], device="cuda")[:, None]
    for x in (s["k"], s["v"]):
        y = (x.view(torch.uint8) if c["e4m3"] else x).permute(1, 3, 0, 2, 4)        # [pages, slots, layers, heads, d]
        y[s["table"][b, dst // ps].long(), dst % ps] = y[s["table"][b, src // ps].long(), src % ps]
    return s["k"], s["v"], first + s["kept"]


def _plain_copy(s, c):
    n, ps = c["n"], c["page"]
    src, dst = s["src"][:n].long(), s["dst"][:n].long()
    for x in (s["k"], s["v"]):
        y = x.view(torch.uint8) if c["e4m3"] else x                                  # [layers, pages, heads, slots, d]
        if s["slots"] is None:
            y[:, dst] = y[:, src]
        else:
            filled = (torch.arange(ps, device="cuda") < s["slots"][:n, None])[None, :, None, :, None]
            y[:, dst] = torch.where(filled, y[:, src], y[:, dst])
    return s["k"], s["v"]


# ------------------------------------------------------------------------------------------------- what cannot be done without

def work(case):
    c = case
    if c["op"] == "layout":
        n = sum(_counts(c))
        return {"bytes": n * (4 + 4 + 4 * -(-c["T"] // 32)) + c["B"] * 8, "flops": n}
    size = 1 if c["e4m3"] else 2
    row = c["Hkv"] * (c["dqk"] + c["dv"])
    if c["op"] == "copy":
        slots = sum(1 + (i * 11 + 8) % c["page"] for i in range(c["n"])) if c["filled"] else c["n"] * c["page"]
        return {"bytes": 2 * slots * row * size * c["layers"], "flops": 0}
    if c["op"] == "compact":
        # (what stays in its place is decided by the seed: half of the tokens on average)
        return {"bytes": 2 * max(1, sum(_accepted(c)) // 2) * row * size * c["layers"], "flops": 0}
    counts, lens = _counts(c), _lens(c)
    n = sum(counts)
    if c["op"] == "append":
        return {"bytes": n * (row * (2 + size) + c["Hq"] * c["dqk"] * 4 + c["rot"] * 4 + 4 * c["axes"]),
                "flops": n * 3 * (c["Hkv"] + c["Hq"]) * c["rot"]}
    flops = 2 * sum(m * l for m, l in zip(counts, lens)) * c["Hq"] * (c["dqk"] + c["dv"])
    return {"bytes": sum(lens) * row * size + n * c["Hq"] * (c["dqk"] + c["dv"]) * 2 + n * c["Hq"] * 4, "flops": flops}


# ------------------------------------------------------------------------------------------------- the definition, in 64 bits

def _exact_tree(s, c):
    lens, counts, table = _lens(c), _counts(c), s["table"].tolist()
    G, at = c["Hq"] // c["Hkv"], 0
    o = torch.empty(s["n"], c["Hq"], c["dv"], dtype=torch.float64, device="cuda")
    lse = torch.empty(c["Hq"], s["n"], dtype=torch.float64, device="cuda")
    for b, (n, m) in enumerate(zip(lens, counts)):
        pages, here = table[b][:-(-n // c["page"])], slice(at, at + m)
        k, v = (torch.cat([x[0, p].double() for p in pages], dim=1)[:, :n] for x in (s["k"], s["v"]))
        if c["e4m3"]:
            k, v = k * s["k_scale"].double()[:, None, None], v * s["v_scale"].double()[:, None, None]
        bits = [[(w >> e) & 1 for w in words for e in range(32)][:m] for words in s["mask"][here].tolist()]
        hidden = torch.zeros(m, n, dtype=torch.bool, device="cuda")
        hidden[:, n - m:] = torch.tensor(bits, device="cuda") == 0
        for h in range(c["Hq"]):
            z = (s["q"][here, h].double() @ k[h // G].T) / math.sqrt(c["dqk"])
            z[hidden] = -math.inf
            lse[h, here] = torch.logsumexp(z, dim=1)
            o[here, h] = torch.exp(z - lse[h, here][:, None]) @ v[h // G]
        at += m
    return o, lse


def _exact_append(s, c):
    lens, counts, ps, half, at = _lens(c), _counts(c), c["page"], c["rot"] // 2, 0
    k_cache, v_cache, q_out = s["k"].double(), s["v"].double(), s["q_out"].double()
    table, axis = s["table"].tolist(), _axis_of_pair(c)

    def turned(x, here):
        x = x.double()
        y = x.clone()
        for i in range(half):
            row = s["cos_sin"][s["pos"][axis[i], here].long()].double()
            p, r = (2 * i, 2 * i + 1) if c["inter"] else (i, half + i)
            cos, sin = row[:, i, None], row[:, half + i, None]
            y[..., p] = x[..., p] * cos - x[..., r] * sin
            y[..., r] = x[..., r] * cos + x[..., p] * sin
        return y

    for b, (n, m) in enumerate(zip(lens, counts)):
        here = slice(at, at + m)
        k, v = turned(s["k_new"][here], here), s["v_new"][here].double()
        q_out[here] = turned(s["q"][here], here)
        if c["e4m3"]:
            k, v = k / s["k_scale"].double()[:, None], v / s["v_scale"].double()[:, None]
        first = n - m
        for j in range(first // ps, (n - 1) // ps + 1):
            lo, hi = max(first, j * ps), min(n, (j + 1) * ps)
            k_cache[0, table[b][j], :, lo - j * ps:hi - j * ps] = k[lo - first:hi - first].transpose(0, 1)
            v_cache[0, table[b][j], :, lo - j * ps:hi - j * ps] = v[lo - first:hi - first].transpose(0, 1)
        at += m
    if c["e4m3"]:
        k_cache, v_cache = k_cache.clamp(-_E4M3_MAX, _E4M3_MAX), v_cache.clamp(-_E4M3_MAX, _E4M3_MAX)
    return k_cache, v_cache, q_out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "tree":
        return _exact_tree(s, c)
    if c["op"] == "append":
        return _exact_append(s, c)
    # (the other operators copy values and count: what they return is compared as it is)
    return None
