"""The operators of a serving step around an 8-bit block cache, and the sizes they are measured at.

A block cache holds keys and values in 8 bits in pages of 16 to 128 tokens, with one FP32 scale for each page and
key / value head.  A page table names the pages of each sequence, `lens` the tokens it holds, the call's own included.
Four operators work around it:

  rotate  RMS norm of every query and key head and the rotation of its first `rot` features by the row's position
  append  the new tokens' keys and values are quantised into their pages (a page's scale grows where it has to)
  read    the last tokens of each sequence come back as 16-bit values
  attn    softmax(scale q K^T) V over the cache, causal within a sequence's new rows, grouped query heads

`run` computes them in elementary torch operations in 32 bits, or, with `own`, through the library's entry points.
The rows of the sequences lie one after another; row_start[b] is the first row of sequence b.
"""
import math
import random

import torch

own = False

FP = {"bf16": torch.bfloat16, "f16": torch.float16}
Q8 = {"i8": torch.int8, "f8": torch.float8_e4m3fn}
TOP = {"i8": 127.0, "f8": 448.0}
EPS = 1e-6
POSITIONS = 32768          # rows of the rotation tables


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    c = lambda name, op, **kw: dict({"name": name, "op": op, "kind": "i8", "fp": "bf16", "page": 64, "new": 1, "ctx": 0,  # noqa: E731
                                     "ragged": False, "mix": 1, "pad": 0}, **kw)
    return [
        # one decode step of a small batch: a call of a few hundred kilobytes, where its latency is what counts
        c("rotate_step", "rotate", rows=16, nq=32, nkv=8, dh=128, rot=128, halves=True),
        # a prompt of one row less than a power of two, heads of 64 features of which half turn, neighbours paired
        c("rotate_prompt", "rotate", rows=16383, nq=32, nkv=32, dh=64, rot=32, halves=False, fp="f16"),
        # one token for each sequence of a batch at lengths of their own, read back with the tokens that share its page
        c("append_step", "append", B=64, nq=32, nkv=8, dh=128, ctx=4095, back=64, ragged=True),
        # prompts of different lengths written behind a cached prefix, e4m3 payload
        c("append_prompt", "append", B=5, nq=32, nkv=8, dh=128, ctx=1000, new=4096, back=4096, kind="f8", page=32, ragged=True),
        # a short prefix of one sequence, in the smallest pages
        c("read_prefix", "read", B=1, nq=16, nkv=16, dh=64, ctx=515, back=515, page=16, fp="f16"),
        # whole sequences of a batch
        c("read_batch", "read", B=8, nq=32, nkv=8, dh=128, ctx=8191, back=8191, page=128, ragged=True),
        # one sequence, one new token, a cache of a few pages
        c("attn_one", "attn", B=1, nq=16, nkv=16, dh=64, ctx=383, page=16, fp="f16"),
        # a batch of decode steps at lengths of their own
        c("attn_step", "attn", B=32, nq=32, nkv=8, dh=128, ctx=4095, ragged=True, pad=3),
        # two long documents, one new token each: few rows, a long axis
        c("attn_long", "attn", B=2, nq=32, nkv=4, dh=128, ctx=131071, page=128),
        # up to six drafted tokens for each sequence, checked in one call, e4m3 payload
        c("attn_drafts", "attn", B=16, nq=32, nkv=8, dh=128, ctx=6001, new=6, kind="f8", fp="f16", page=32, ragged=True),
        # a chunk of a prompt against what is cached already
        c("attn_chunk", "attn", B=1, nq=32, nkv=8, dh=128, ctx=6000, new=2048),
        # prompts of different lengths in one call, heads of 64 features, no grouping
        c("attn_prompts", "attn", B=6, nq=16, nkv=16, dh=64, ctx=100, new=1500, kind="f8", fp="f16", page=128, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "read", "attn", "attn", "attn"])
    dh = rng.choice([64, 128])
    nkv = rng.choice([1, 2, 4, 8, 16])
    group = rng.choice([1, 2, 3, 4, 5, 8])
    case = {"op": op, "kind": rng.choice(["i8", "f8"]), "fp": rng.choice(["bf16", "f16"]), "page": rng.choice([16, 32, 64, 128]),
            "nq": nkv * group, "nkv": nkv, "dh": dh, "new": 1, "ctx": 0, "ragged": rng.random() < 0.7, "mix": rng.randrange(1 << 20),
            "pad": rng.choice([0, 0, 1, 7])}
    if op == "rotate":
        case |= {"rows": _log(rng, 1, 8000), "rot": rng.choice([dh, dh // 2]), "halves": rng.random() < 0.5}
        return case
    if op == "append":
        case |= {"B": _log(rng, 1, 64), "ctx": _log(rng, 1, 4096) - 1, "new": 1 if rng.random() < 0.5 else _log(rng, 2, 4096)}
        top = 16e6
    elif op == "read":
        case |= {"B": _log(rng, 1, 16), "ctx": _log(rng, 1, 16384)}
        top = 48e6
    else:
        kind = rng.choice(["one", "one", "few", "many"])
        case |= {"B": _log(rng, 1, 64), "ctx": _log(rng, 1, 40000) - 1}
        case["new"] = {"one": 1, "few": rng.randint(2, 16), "many": _log(rng, 17, 1500)}[kind]
        if kind == "many":
            case["ctx"] = min(case["ctx"], 6000)
        top = 100e6
    # no drawn case costs more than the largest listed one of its operator: fewer sequences, then fewer heads
    cost = lambda: case["B"] * case["nkv"] * dh * (case["ctx"] + case["new"]) * 1.0  # noqa: E731
    pairs = lambda: case["B"] * case["nq"] * dh * case["new"] * (case["ctx"] + case["new"]) * 1.0  # noqa: E731
    while cost() > top or (op == "attn" and pairs() > 5e10):
        if case["B"] > 1:
            case["B"] //= 2
        elif case["nkv"] > 1:
            case["nkv"], case["nq"] = case["nkv"] // 2, case["nq"] // 2
        else:
            case["ctx"] //= 2
    if op == "append":
        case["back"] = case["new"] if case["new"] > 1 else case["page"]
    if op == "read":
        case["back"] = case["ctx"] if rng.random() < 0.5 else _log(rng, 1, case["ctx"])
    return case


def _lengths(case):
    """(tokens in the cache before the call's own, new tokens) of each sequence; a case's lengths are its own."""
    r, B, ctx, new = random.Random(case["mix"]), case["B"], case["ctx"], case["new"]
    if not case["ragged"]:
        return [ctx] * B, [new] * B
    held = [r.randint(ctx // 4, ctx) for _ in range(B)]
    fresh = [r.randint(max(1, new // 4), new) for _ in range(B)]
    held[0], fresh[0] = ctx, new
    if B > 3:
        held[1] = 0
        if new > 1:
            fresh[2] = 1
    return held, fresh


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def _plan(case):
    """What of a case is plain numbers: lengths with the new tokens, rows of the call's tensors, pages."""
    held, fresh = _lengths(case)
    if case["op"] == "read":
        fresh = [0] * case["B"]
    lens = [a + n for a, n in zip(held, fresh)]
    back = [min(case.get("back", 0), n) for n in lens]
    per = -(-max(1, case["ctx"] + (case["new"] if case["op"] != "read" else 0)) // case["page"])
    return {"lens": lens, "fresh": fresh, "back": back, "per": per, "max_len": per * case["page"]}


# ------------------------------------------------------------------------------------------------ what a program has in hand
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    fp, nq, nkv, dh = FP[case["fp"]], case["nq"], case["nkv"], case["dh"]
    S = {"case": case}
    if case["op"] == "rotate":
        rows = case["rows"]
        # queries, keys and values of a row lie side by side, as the projection writes them
        S["qkv"] = (normal(rows, (nq + 2 * nkv) * dh) * torch.exp(0.5 * normal((nq + 2 * nkv) * dh))).to(fp)
        S["q"], S["k"] = S["qkv"][:, :nq * dh], S["qkv"][:, nq * dh:(nq + nkv) * dh]
        S["q_out"], S["k_out"] = torch.zeros(rows, nq * dh, dtype=fp, device="cuda"), torch.zeros(rows, nkv * dh, dtype=fp, device="cuda")
        S["q_gamma"], S["k_gamma"] = 1 + 0.1 * normal(dh), 1 + 0.1 * normal(dh)
        first = random.Random(int(seed)).randrange(POSITIONS - rows)
        S["pos"] = torch.arange(first, first + rows, dtype=torch.int32, device="cuda")
        half = case["rot"] // 2
        turn = torch.arange(POSITIONS, dtype=torch.float64, device="cuda")[:, None] * \
            torch.pow(10000.0, -torch.arange(half, dtype=torch.float64, device="cuda") / half)[None]
        S["cos"], S["sin"] = turn.cos().float(), turn.sin().float()
    else:
        plan = _plan(case)
        B, page, per, kind = case["B"], case["page"], plan["per"], case["kind"]
        pages = B * per + 1                               # one page of the pool stays free
        for name in ("k", "v"):
            x = normal(pages, nkv, page, dh)
            if kind == "i8":
                S[name + "_cache"] = (x * 36).round().clamp(-127, 127).to(torch.int8)
            else:
                S[name + "_cache"] = (x * 120).clamp(-448, 448).to(torch.float8_e4m3fn)
            # what a page stands for: keys with products of about 1.5 sqrt(dh) against unit queries, values of about 1
            unit = {"i8": 1 / 36, "f8": 1 / 120}[kind] * (1.5 if name == "k" else 1.0)
            S[name + "_scale"] = unit * torch.exp(0.3 * normal(pages, nkv))
        S["table"] = torch.randperm(pages - 1, generator=g, device="cuda")[:B * per].to(torch.int32).reshape(B, per).contiguous()
        S["lens"] = torch.tensor(plan["lens"], dtype=torch.int32, device="cuda")
        S["max_len"] = plan["max_len"]
        if case["op"] in ("append", "attn"):
            S["start"] = torch.tensor(_starts(plan["fresh"]), dtype=torch.int32, device="cuda")
            S["most"] = max(plan["fresh"])
            rows = sum(plan["fresh"]) + case["pad"]
        if case["op"] in ("append", "read"):
            S["back_start"] = torch.tensor(_starts(plan["back"]), dtype=torch.int32, device="cuda")
            S["back_most"] = max(plan["back"])
            n_back = sum(plan["back"]) + case["pad"]
            S["k_back"], S["v_back"] = (torch.zeros(n_back, nkv * dh, dtype=fp, device="cuda") for _ in range(2))
        if case["op"] == "append":
            # a few features of the keys are larger throughout, as they are in trained models
            loud = torch.where(torch.rand(nkv * dh, generator=g, device="cuda") < 0.03, 6.0, 1.0)
            S["k"], S["v"] = (normal(rows, nkv * dh) * loud).to(fp), normal(rows, nkv * dh).to(fp)
        if case["op"] == "attn":
            S["q"] = normal(rows, nq * dh).to(fp)
            S["out"] = torch.zeros(rows, nq * dh, dtype=fp, device="cuda")
    if own:
        _describe(S)
    return S


_handle = None


def _describe(S):
    """The library's handle, and its views of the buffers above."""
    global _handle
    from paper_2310_17723_b200 import hero
    if _handle is None:
        _handle = hero.Handle()
    case = S["case"]
    S["h"] = _handle
    for name in ("q", "k", "v", "q_out", "k_out", "k_back", "v_back", "out"):
        if name in S:
            S["t_" + name] = hero.tensor(S[name])
    if case["op"] != "rotate":
        S["cache"] = hero.block_cache(S["k_cache"], S["v_cache"], S["k_scale"], S["v_scale"], S["table"], S["lens"], S["max_len"])
    if case["op"] == "attn":
        n = _handle.hero_block_attention_workspace_bytes(S["cache"], case["nq"], S["q"].shape[0], S["most"])
        S["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------ one pass
def run(S):
    case = S["case"]
    if own:
        return {"rotate": _own_rotate, "append": _own_append, "read": _own_read, "attn": _own_attn}[case["op"]](S, case)
    return {"rotate": _rotate, "append": _append, "read": _read, "attn": _attn}[case["op"]](S, case)


def _own_rotate(S, case):
    S["h"].hero_qk_norm_rope(S["t_q"], S["t_k"], S["t_q_out"], S["t_k_out"], case["nq"], case["nkv"], S["pos"], S["cos"], S["sin"],
                             q_gamma=S["q_gamma"], k_gamma=S["k_gamma"], eps=EPS, pairing="halves" if case["halves"] else "adjacent")
    return {"q": S["q_out"], "k": S["k_out"]}


def _own_append(S, case):
    S["h"].hero_block_cache_append(S["cache"], S["t_k"], S["t_v"], row_start=S["start"], max_rows=S["most"])
    S["h"].hero_block_cache_read(S["cache"], S["t_k_back"], S["t_v_back"], row_start=S["back_start"], max_rows=S["back_most"])
    return {"k": S["k_back"], "v": S["v_back"], "k_scale": S["k_scale"][:-1], "v_scale": S["v_scale"][:-1]}


def _own_read(S, case):
    S["h"].hero_block_cache_read(S["cache"], S["t_k_back"], S["t_v_back"], row_start=S["back_start"], max_rows=S["back_most"])
    return {"k": S["k_back"], "v": S["v_back"]}


def _own_attn(S, case):
    S["h"].hero_block_attention(S["cache"], S["t_q"], S["t_out"], case["nq"], row_start=S["start"], max_rows=S["most"],
                                workspace=S["workspace"])
    return S["out"]


def _turned(x, heads, gamma, S, case):
    rows, dh, rot = x.shape[0], case["dh"], case["rot"]
    y = x.float().reshape(rows, heads, dh)
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * gamma
    c, s = S["cos"][S["pos"].long()][:, None], S["sin"][S["pos"].long()][:, None]
    if case["halves"]:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        z = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        z = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([z, y[..., rot:]], -1).reshape(rows, heads * dh).to(x.dtype)


def _rotate(S, case):
    return {"q": _turned(S["q"], case["nq"], S["q_gamma"], S, case), "k": _turned(S["k"], case["nkv"], S["k_gamma"], S, case)}


def _row_index(start, rows):
    """Sequence of each row, its place in it, and whether it belongs to one at all."""
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(start[1:].long(), r, right=True).clamp(max=start.numel() - 2)
    return b, r - start[b].long(), r < start[-1]


def _values(S, name, pages):
    """FP32 values of the pages named, [..., heads, tokens, features]."""
    code = S[name + "_cache"].view(torch.uint8)[pages].view(S[name + "_cache"].dtype)
    return code.float() * S[name + "_scale"][pages][..., None, None]


def _append_one(S, case, name):
    page, nkv, dh, kind, most = case["page"], case["nkv"], case["dh"], case["kind"], S["most"]
    x, cache, scale = S[name], S[name + "_cache"], S[name + "_scale"]
    lens, start = S["lens"].long(), S["start"].long()
    n = start[1:] - start[:-1]
    begin = lens - n
    j = begin[:, None] // page + torch.arange((most + page - 2) // page + 1, device="cuda")             # [B, touched pages]
    pos = j[..., None] * page + torch.arange(page, device="cuda")                                       # [B, touched, page]
    new = (pos >= begin[:, None, None]) & (pos < lens[:, None, None])
    old = pos < begin[:, None, None]
    touched = new.any(-1)
    at = torch.where(touched, S["table"].long().gather(1, j.clamp(max=S["table"].shape[1] - 1)), cache.shape[0] - 1)
    row = (start[:-1, None, None] + pos - begin[:, None, None]).clamp(0, x.shape[0] - 1)
    fresh = x[row].float().reshape(*row.shape, nkv, dh).transpose(2, 3)                                 # [B, touched, heads, page, dh]
    mask = new[:, :, None, :, None]
    most_now = torch.where(mask, fresh.abs(), 0.0).amax((-1, -2)) / TOP[kind]
    s_old = torch.where(old.any(-1)[..., None], scale[at], 0.0)
    s = torch.maximum(s_old, most_now)
    y = torch.where(mask, fresh, torch.where(old[:, :, None, :, None], _values(S, name, at), 0.0))
    y = torch.where(s[..., None, None] > 0, y / s[..., None, None], 0.0).clamp(-TOP[kind], TOP[kind])
    code = y.round().to(torch.int8) if kind == "i8" else y.to(torch.float8_e4m3fn)
    # tokens of the page that are neither old nor new keep what they hold
    keep = (new | old)[:, :, None, :, None]
    code = torch.where(keep, code.view(torch.uint8), cache.view(torch.uint8)[at])
    cache.view(torch.uint8)[at] = code
    scale[at] = s


def _read_one(S, case, name, out):
    page, nkv, dh = case["page"], case["nkv"], case["dh"]
    start = S["back_start"].long()
    b, i, real = _row_index(S["back_start"], out.shape[0])
    pos = (S["lens"].long()[b] - (start[b + 1] - start[b]) + i).clamp(0, S["max_len"] - 1)
    at = S["table"].long()[b, pos // page]
    code = S[name + "_cache"].view(torch.uint8)[at, :, pos % page].view(S[name + "_cache"].dtype)       # [rows, heads, dh]
    y = (code.float() * S[name + "_scale"][at][..., None]).reshape(out.shape).to(out.dtype)
    return torch.where(real[:, None], y, out)


def _append(S, case):
    _append_one(S, case, "k")
    _append_one(S, case, "v")
    return dict(_read(S, case), k_scale=S["k_scale"][:-1], v_scale=S["v_scale"][:-1])


def _read(S, case):
    return {"k": _read_one(S, case, "k", S["k_back"]), "v": _read_one(S, case, "v", S["v_back"])}


def _attn(S, case):
    B, nq, nkv, dh, most = case["B"], case["nq"], case["nkv"], case["dh"], S["most"]
    group, rows = nq // nkv, S["q"].shape[0]
    lens, start = S["lens"].long(), S["start"].long()
    n = start[1:] - start[:-1]
    i = torch.arange(most, device="cuda")
    q = S["q"][(start[:-1, None] + i).clamp(max=rows - 1)].float().reshape(B, most, nkv, group, dh)
    q = q.permute(0, 2, 1, 3, 4).reshape(B, nkv, most * group, dh)
    at = S["table"].long()
    k = _values(S, "k", at).transpose(1, 2).reshape(B, nkv, -1, dh)                                     # [B, heads, tokens, dh]
    s = (q @ k.transpose(-1, -2)).mul_(dh ** -0.5).reshape(B, nkv, most, group, -1)
    del k
    key = torch.arange(s.shape[-1], device="cuda")
    seen = key <= (lens - n)[:, None, None] + i[None, :, None]                                          # [B, rows, tokens]
    s.masked_fill_(~seen[:, None, :, None], float("-inf"))
    e = s.sub_(s.amax(-1, keepdim=True)).exp_()
    total = e.sum(-1, keepdim=True)
    v = torch.where((key < lens[:, None])[:, None, :, None], _values(S, "v", at).transpose(1, 2).reshape(B, nkv, -1, dh), 0.0)
    o = (e.reshape(B, nkv, most * group, -1) @ v).reshape(B, nkv, most, group, dh) / total
    o = o.permute(0, 2, 1, 3, 4).reshape(B, most, nq * dh).to(S["out"].dtype)
    b, r, real = _row_index(S["start"], rows)
    return torch.where(real[:, None], o[b, r.clamp(max=most - 1)], S["out"])


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    nq, nkv, dh = case["nq"], case["nkv"], case["dh"]
    if case["op"] == "rotate":
        n = case["rows"] * (nq + nkv) * dh
        return {"bytes": 2 * 2 * n + case["rows"] * (case["rot"] * 4 + 4), "flops": 8 * n}
    p = _plan(case)
    page = case["page"]
    pages = sum(-(-n // page) for n in p["lens"])
    if case["op"] == "read":
        n = sum(p["back"]) * nkv * dh
        return {"bytes": 2 * n * (1 + 2) + 2 * 4 * nkv * (sum(p["back"]) // page + 1), "flops": 2 * n}
    if case["op"] == "append":
        new, back = sum(p["fresh"]) * nkv * dh, sum(p["back"]) * nkv * dh
        return {"bytes": 2 * new * (2 + 1) + 2 * back * (1 + 2), "flops": 6 * new + 2 * back}
    rows = sum(p["fresh"])
    pairs = sum(n * (a - n) + n * (n + 1) // 2 for a, n in zip(p["lens"], p["fresh"]))
    return {"bytes": 2 * sum(p["lens"]) * nkv * dh + 2 * 4 * pages * nkv + 2 * 2 * rows * nq * dh, "flops": 4 * pairs * nq * dh}


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    S = prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "read": _exact_read, "attn": _exact_attn}[case["op"]](S, case)


def _exact_rotate(S, case):
    dh, rot = case["dh"], case["rot"]
    turn = torch.complex(S["cos"].double(), S["sin"].double())[S["pos"].long()]                          # e^(i angle)

    def one(x, heads, gamma):
        y = x.double().reshape(x.shape[0], heads, dh)
        y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / dh + EPS) * gamma.double()
        first = torch.arange(rot // 2, device="cuda") if case["halves"] else torch.arange(0, rot, 2, device="cuda")
        second = first + (rot // 2 if case["halves"] else 1)
        z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        return y.reshape(x.shape[0], heads * dh)

    return {"q": one(S["q"], case["nq"], S["q_gamma"]), "k": one(S["k"], case["nkv"], S["k_gamma"])}


def _tokens(S, case, name, b, n):
    """The first n tokens that sequence b's pages stand for, [n, heads, features], in 64 bits."""
    at = S["table"][b, :max(1, -(-n // case["page"]))].long()
    y = S[name + "_cache"][at].to(torch.float32).double() * S[name + "_scale"][at].double()[:, :, None, None]
    return y.transpose(1, 2).reshape(-1, case["nkv"], case["dh"])[:n]


def _exact_read(S, case):
    p, got = _plan(case), {}
    for name in ("k", "v"):
        out = torch.zeros(S[name + "_back"].shape, dtype=torch.float64, device="cuda")
        at = 0
        for b, n in enumerate(p["back"]):
            out[at:at + n] = _tokens(S, case, name, b, p["lens"][b])[p["lens"][b] - n:].flatten(1)
            at += n
        got[name] = out
    return got


def _exact_append(S, case):
    p, page, top, got = _plan(case), case["page"], TOP[case["kind"]], {}
    for name in ("k", "v"):
        out = torch.zeros(S[name + "_back"].shape, dtype=torch.float64, device="cuda")
        scale = S[name + "_scale"].double()
        row = at = 0
        for b, (n, m) in enumerate(zip(p["lens"], p["fresh"])):
            held = n - m
            full = -(-n // page) * page
            y = torch.zeros(full, case["nkv"], case["dh"], dtype=torch.float64, device="cuda")
            y[:held] = _tokens(S, case, name, b, held)
            y[held:n] = S[name][row:row + m].double().reshape(m, case["nkv"], case["dh"])
            row += m
            first = held // page                                       # pages before this one are not touched
            z = y[first * page:].reshape(-1, page, case["nkv"], case["dh"])
            pos = torch.arange(first * page, full, device="cuda").reshape(-1, page)
            s = (z.abs() * (pos >= held)[..., None, None]).amax((1, 3)) / top
            pages = S["table"][b, first:full // page].long()
            if held % page:
                s[0] = torch.maximum(s[0], scale[pages[0]])
            scale[pages] = s
            w = torch.where(s[:, None, :, None] > 0, z / s[:, None, :, None], 0.0).clamp(-top, top)
            w = w.round() if case["kind"] == "i8" else w.float().to(torch.float8_e4m3fn).double()
            y[first * page:] = (w * s[:, None, :, None]).reshape(-1, case["nkv"], case["dh"])
            k = p["back"][b]
            out[at:at + k] = y[n - k:n].flatten(1)
            at += k
        got[name], got[name + "_scale"] = out, scale[:-1]
    return got


def _exact_attn(S, case):
    p, nq, nkv, dh = _plan(case), case["nq"], case["nkv"], case["dh"]
    out = torch.zeros(S["out"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, (n, m) in enumerate(zip(p["lens"], p["fresh"])):
        k, v = _tokens(S, case, "k", b, n), _tokens(S, case, "v", b, n)
        hidden = torch.arange(n, device="cuda")[None] > torch.arange(n - m, n, device="cuda")[:, None]
        for h in range(nq):
            s = S["q"][row:row + m, h * dh:(h + 1) * dh].double() @ k[:, h // (nq // nkv)].T / math.sqrt(dh)
            out[row:row + m, h * dh:(h + 1) * dh] = torch.softmax(s.masked_fill(hidden, -math.inf), -1) @ v[:, h // (nq // nkv)]
        row += m
    return out
