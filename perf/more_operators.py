"""The operators of a mixture of experts around W8A8 layers, and the sizes they are measured at.

A router gives every token a logit for each of E experts; the token is worked on by the k experts with the largest ones and
gets the weighted sum of what they give.  Three operators do that:

  route    top k of every row of logits, their weights, and the order of the (token, expert) pairs by expert
  linear   the products of the rows of each expert with that expert's weights, with scales, bias, activation and rounding
  combine  residual + weighted sum of each token's rows, with LayerNorm and quantisation of the result
  experts  all of them behind one another, as a layer calls them: route, two products, combine

`run` computes them in elementary torch operations in 32 bits (scores of the router in 64), or, with `own`, through the
library's entry points.  Sorted rows: the pairs ordered by expert, then by token; offset[e] is the first row of expert e.
"""
import math
import random

import torch

own = False

FP = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    c = lambda name, op, **kw: dict({"name": name, "op": op, "kind": "i8", "fp": "bf16", "pad": 0, "score": "softmax", "renorm": True,  # noqa: E731
                                     "bias": False, "logits": "f32"}, **kw)
    return [
        # the router of one decode step of a small batch: a call of a few kilobytes, where its latency is what counts
        c("route_step", "route", T=16, E=64, k=6),
        # a long prompt of one token less than a power of two, many experts, 16-bit logits (which tie)
        c("route_prompt", "route", T=16383, E=128, k=8, logits="bf16"),
        # sigmoid scores, a bias that balances the experts' load in the choice alone, a batch padded to 5000 rows
        c("route_balanced", "route", T=5000, E=256, k=8, score="sigmoid", bias=True, pad=77),
        # one new token in a small model: the first product, biases and GELU, INT8 out
        c("linear_one", "linear", T=1, E=8, k=2, K=1024, N=4096, act="gelu_erf", gated=False, gather=True, out="i8", fp="f16"),
        # a decode step of a batch over many small experts: bound by the weights of every expert that has a token
        c("linear_step", "linear", T=64, E=64, k=6, K=2048, N=2816, act="silu", gated=True, gather=True, out="i8", fp="f16"),
        # a prompt: about a thousand rows for each expert, more for the popular ones
        c("linear_prompt", "linear", T=8192, E=64, k=8, K=2048, N=2048, act="silu", gated=True, gather=True, out="i8"),
        # e4m3 operands, the second product: rows in sorted order, 16-bit out, ragged and padded
        c("linear_f8", "linear", T=3001, E=16, k=4, K=4096, N=1024, act="none", gated=False, gather=False, out="fp", kind="f8", pad=9),
        # modules left in 16 bits
        c("linear_bf16", "linear", T=2000, E=8, k=2, K=1024, N=4096, act="gelu_tanh", gated=False, gather=True, out="fp", kind="bf16"),
        # the sum behind a decode step, onto the residual stream
        c("combine_step", "combine", T=64, E=64, k=6, H=2048, y="i8", norm=False, fp="f16"),
        # the sum behind a prompt with the next LayerNorm, token-wise INT8 out
        c("combine_prompt", "combine", T=8192, E=64, k=8, H=2048, y="fp", norm=True),
        # the whole expert part of a layer for one decode step
        c("experts_step", "experts", T=32, E=32, k=4, H=2048, F=1024, y="fp", norm=True),
        # ... and for a prompt, the second product's output in INT8 with a scale for each expert and feature
        c("experts_prompt", "experts", T=4096, E=64, k=8, H=2048, F=1024, y="i8", norm=True, fp="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "linear", "linear", "linear", "combine", "experts"])
    E = rng.choice([4, 8, 16, 33, 60, 64, 128])
    T = _log(rng, 1, 8192)
    case = {"op": op, "kind": "i8", "fp": rng.choice(["bf16", "f16"]), "T": T, "E": E, "k": rng.randint(1, min(8, E)),
            "pad": rng.choice([0, 0, 1, 5]), "score": rng.choice(["softmax", "sigmoid"]), "renorm": rng.random() < 0.7,
            "bias": rng.random() < 0.5, "logits": rng.choice(["f32", "bf16", "f16"])}
    if op == "route":
        return case | {"T": _log(rng, 1, 16383), "E": rng.choice([E, 200, 256])}
    size = lambda lo, hi, step: max(step, _log(rng, lo, hi) // step * step)  # noqa: E731
    if op == "combine":
        case |= {"H": size(256, 4096, 16), "y": rng.choice(["i8", "fp"]), "norm": rng.random() < 0.5}
        while case["T"] * case["k"] * case["H"] > 1.3e8:
            case["T"] //= 2
        return case
    if op == "experts":
        case |= {"H": size(256, 4096, 16), "F": size(128, 2048, 16), "y": rng.choice(["i8", "fp"]), "norm": rng.random() < 0.7}
        while case["E"] * case["H"] * case["F"] > 1.4e8:
            case["F"] = max(16, case["F"] // 32 * 16)
        while case["T"] * case["k"] * case["H"] * case["F"] > 6e10:
            case["T"] //= 2
        return case
    kind = rng.choice(["i8", "i8", "f8", "bf16", "f16"])
    case |= {"kind": kind, "K": size(256, 4096, 16), "N": size(256, 4096, 32), "act": rng.choice(["none", "gelu_erf", "gelu_tanh", "silu"]),
             "gated": rng.random() < 0.5, "gather": rng.random() < 0.5, "out": rng.choice(["fp", "i8"]) if kind == "i8" else "fp"}
    if kind in FP:
        case["fp"] = kind
    while case["E"] * case["N"] * case["K"] > 2.7e8:
        case["N"] = max(32, case["N"] // 64 * 32)
    while case["T"] * case["k"] * case["N"] * case["K"] > 2.7e11 / (1 if kind in ("i8", "f8") else 2):
        case["T"] //= 2
    return case


# ------------------------------------------------------------------------------------------------ what a program has in hand
def _order(ids, E):
    """offset [E + 1], token of each sorted row, sorted row of each pair, from the experts chosen (-1: none)."""
    T, k = ids.shape
    flat = torch.where(ids < 0, E, ids).reshape(-1).long()
    by, at = torch.sort(flat, stable=True)
    offset = torch.searchsorted(by, torch.arange(E + 1, device=ids.device))
    place = torch.empty_like(at)
    place[at] = torch.arange(T * k, device=ids.device)
    token = torch.where(by < E, at // k, -1)
    row = torch.where(flat < E, place, -1).reshape(T, k)
    return offset.int(), token.int(), row.int()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 6151 + 29)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    codes = lambda *s: (normal(*s) * 36).round_().clamp_(-127, 127).to(torch.int8)  # noqa: E731
    zeros = lambda *s, dtype: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    op, T, E, k, fp = case["op"], case["T"], case["E"], case["k"], FP[case["fp"]]
    rows = T + case["pad"]                                  # rows of the padded batch; the first T are tokens
    S = {"case": case, "n_tokens": torch.tensor([T], dtype=torch.int32, device="cuda")}
    # experts of different popularity, as trained routers have them
    S["logits"] = (normal(rows, E) + 0.4 * normal(E)).to(FP[case["logits"]])
    S["select_bias"] = 0.1 * normal(E) if case["bias"] else None
    S["expert"], S["row"] = zeros(rows, k, dtype=torch.int32), zeros(rows, k, dtype=torch.int32)
    S["weight"] = zeros(rows, k, dtype=torch.float32)
    S["offset"], S["token"] = zeros(E + 1, dtype=torch.int32), torch.full((rows * k,), -1, dtype=torch.int32, device="cuda")
    if op != "route":                                       # what the router has left behind
        got = _route(S, case)
        for name in ("expert", "weight", "offset", "token", "row"):
            S[name].copy_(got[name])
        S["cap"] = int((S["offset"][1:] - S["offset"][:-1]).max())
        R = rows * k
    if op == "linear":
        K, N, kind = case["K"], case["N"], case["kind"]
        n_a, n_out = rows if case["gather"] else R, N // 2 if case["gated"] else N
        if kind == "i8":
            S["a"], S["w"] = codes(n_a, K), codes(E, N, K)
            S["rs"] = torch.exp(0.2 * normal(n_a)) / 36
            S["cs"] = torch.exp(0.2 * normal(E, N)) / (36 * math.sqrt(K))
        elif kind == "f8":
            S["a"], S["w"] = ((normal(*s) * 100).clamp_(-448, 448).to(torch.float8_e4m3fn) for s in ((n_a, K), (E, N, K)))
            S["rs"] = torch.exp(0.2 * normal(n_a)) / 100
            S["cs"] = torch.exp(0.2 * normal(E, N)) / (100 * math.sqrt(K))
        else:
            S["a"], S["w"] = normal(n_a, K).to(fp), (normal(E, N, K) / math.sqrt(K)).to(fp)
            S["rs"] = S["cs"] = None
        S["b"] = 0.1 * normal(E, N)
        S["s_out"] = 4 / 127                                # static scale of an INT8 output
        S["post"] = torch.full((E, n_out), 127 / 4, device="cuda") if case["out"] == "i8" else None
        S["out"] = zeros(R, n_out, dtype=torch.int8 if case["out"] == "i8" else fp)
        S["values"] = zeros(R, n_out, dtype=fp)
    if op in ("combine", "experts"):
        H = case["H"]
        S["y_scale"] = torch.exp(0.3 * normal(E, H)) / 36 if case["y"] == "i8" else None
        S["y"] = codes(R, H) if case["y"] == "i8" else normal(R, H).to(fp)
        S["h"] = (2 * normal(rows, H)).to(fp)               # the residual stream
        S["h_out"] = zeros(rows, H, dtype=fp)
        S["gamma"], S["beta"] = 1 + 0.1 * normal(H), 0.1 * normal(H)
        S["x_out"], S["x_scale"], S["values"] = zeros(rows, H, dtype=torch.int8), zeros(rows, dtype=torch.float32), zeros(rows, H, dtype=fp)
    if op == "experts":
        F = case["F"]
        S["a"], S["rs"] = codes(rows, H), torch.exp(0.2 * normal(rows)) / 36
        S["w1"], S["cs1"] = codes(E, 2 * F, H), torch.exp(0.2 * normal(E, 2 * F)) / (36 * math.sqrt(H))
        S["b1"] = 0.1 * normal(E, 2 * F)
        S["post1"] = torch.exp(0.2 * normal(E, F)) * (127 / 4)        # one over the static scales of the hidden features
        S["hidden"] = zeros(R, F, dtype=torch.int8)
        S["w2"], S["cs2"] = codes(E, H, F), torch.exp(0.2 * normal(E, H)) / (36 * 12 * math.sqrt(F))
        S["b2"] = 0.1 * normal(E, H)
        S["post2"] = 1 / S["y_scale"] if case["y"] == "i8" else None
    if own:
        _describe(S)
    return S


_handle = None


def _describe(S):
    """The library's handle, its views of the buffers above, and the router's workspace."""
    global _handle
    from paper_2310_17723_b200 import hero
    if _handle is None:
        _handle = hero.Handle()
    case, h = S["case"], _handle
    S["hero"] = h
    S["t_logits"] = hero.tensor(S["logits"])
    n = h.hero_moe_route_workspace_bytes(S["logits"].shape[0], case["E"], case["k"])
    S["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    if "a" in S:
        S["t_a"] = hero.tensor(S["a"]) if S["rs"] is None else hero.tensor(S["a"], "twq", S["rs"])
    for name in ("h", "h_out", "out", "hidden"):
        if name in S:
            S["t_" + name] = hero.tensor(S[name])
    if "y" in S:
        S["t_y"] = hero.tensor(S["y"]) if S["y_scale"] is None else hero.tensor(S["y"], "fwq", S["y_scale"])
        S["t_x_out"] = hero.tensor(S["x_out"], "twq", S["x_scale"])


# ------------------------------------------------------------------------------------------------ one pass
def run(S):
    case = S["case"]
    if own:
        return {"route": _own_route, "linear": _own_linear, "combine": _own_combine, "experts": _own_experts}[case["op"]](S, case)
    return {"route": _route, "linear": _linear, "combine": _combine, "experts": _experts}[case["op"]](S, case)


def _own_route(S, case):
    S["hero"].hero_moe_route(S["t_logits"], S["expert"], S["weight"], S["offset"], S["token"], S["row"], score=case["score"],
                             renorm=case["renorm"], select_bias=S["select_bias"], n_tokens=S["n_tokens"], workspace=S["workspace"])
    return {n: S[n] for n in ("expert", "weight", "offset", "token", "row")}


def _own_linear(S, case):
    S["hero"].hero_moe_linear(S["t_a"], S["w"], S["t_out"], S["offset"], token=S["token"] if case["gather"] else None, w_scale=S["cs"],
                              bias=S["b"], act=case["act"], gated=case["gated"], post_scale=S["post"])
    return torch.mul(S["out"], S["s_out"], out=S["values"]) if case["out"] == "i8" else S["out"]


def _own_combine(S, case):
    S["hero"].hero_moe_combine(S["t_y"], S["row"], S["weight"], expert=S["expert"], residual=S["t_h"], fp_out=S["t_h_out"],
                               out=S["t_x_out"] if case["norm"] else None, gamma=S["gamma"] if case["norm"] else None,
                               beta=S["beta"] if case["norm"] else None, eps=EPS)
    if not case["norm"]:
        return {"h": S["h_out"]}
    return {"h": S["h_out"], "x": torch.mul(S["x_out"], S["x_scale"][:, None], out=S["values"])}


def _own_experts(S, case):
    _own_route(S, case)
    S["hero"].hero_moe_linear(S["t_a"], S["w1"], S["t_hidden"], S["offset"], token=S["token"], w_scale=S["cs1"], bias=S["b1"], act="silu",
                              gated=True, post_scale=S["post1"])
    S["hero"].hero_moe_linear(S["t_hidden"], S["w2"], S["t_y"], S["offset"], w_scale=S["cs2"], bias=S["b2"], post_scale=S["post2"])
    return _own_combine(S, case)


def _route(S, case):
    k, rows = case["k"], S["logits"].shape[0]
    x = S["logits"].double()
    score = torch.sigmoid(x) if case["score"] == "sigmoid" else torch.softmax(x, -1)
    key = x if S["select_bias"] is None else score + S["select_bias"].double()
    ids = torch.sort(key, dim=-1, descending=True, stable=True)[1][:, :k]
    w = score.gather(1, ids)
    if case["renorm"]:
        w = w / w.sum(-1, keepdim=True)
    real = torch.arange(rows, device="cuda")[:, None] < S["n_tokens"]
    ids, w = torch.where(real, ids, -1), torch.where(real, w, 0.0)
    offset, token, row = _order(ids, case["E"])
    return {"expert": ids.int(), "weight": w.float(), "offset": offset, "token": token, "row": row}


def _act(v, act):
    if act == "gelu_erf":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    return v / (1 + torch.exp(-v)) if act == "silu" else v


def _products(a, rs, w, cs, bias, post, act, gated, offset, token, cap, out):
    """The sorted rows' products, in `out`'s type; rows behind the last expert's keep what `out` holds."""
    R = out.shape[0]
    offset = offset.long()
    place = (offset[:-1, None] + torch.arange(cap, device="cuda")).clamp(max=R - 1)       # [experts, rows of the fullest one]
    at = place if token is None else token[place].long().clamp(min=0)
    v = torch.bmm(a.view(torch.int8)[at].view(a.dtype).float() if a.element_size() == 1 else a[at].float(), w.float().transpose(1, 2))
    if rs is not None:
        v = v * rs[at][..., None] * cs[:, None]
    v = v + bias[:, None]
    y = _act(v[..., :v.shape[-1] // 2], act) * v[..., v.shape[-1] // 2:] if gated else _act(v, act)
    if post is not None:
        y = y * post[:, None]
    if out.dtype == torch.int8:
        y = y.round().clamp(-127, 127)
    r = torch.arange(R, device="cuda")
    e = torch.searchsorted(offset[1:], r, right=True).clamp(max=w.shape[0] - 1)
    return torch.where((r < offset[-1])[:, None], y[e, (r - offset[e]).clamp(0, cap - 1)].to(out.dtype), out)


def _linear(S, case):
    y = _products(S["a"], S["rs"], S["w"], S["cs"], S["b"], S["post"], case["act"], case["gated"], S["offset"],
                  S["token"] if case["gather"] else None, S["cap"], S["out"])
    return (y * S["s_out"]).to(S["values"].dtype) if case["out"] == "i8" else y


def _sum(S, case, y, row, weight, expert):
    some = row >= 0
    at = row.clamp(min=0).long()
    v = y[at].float()                                                                      # [tokens, k, features]
    if S["y_scale"] is not None:
        v = v * S["y_scale"][expert.clamp(min=0).long()]
    h = (S["h"].float() + (v * torch.where(some, weight, 0.0)[..., None]).sum(1)).to(S["h"].dtype)
    if not case["norm"]:
        return {"h": h}
    r = h.float()
    d = r - r.mean(-1, keepdim=True)
    n = d / torch.sqrt((d * d).mean(-1, keepdim=True) + EPS) * S["gamma"] + S["beta"]
    s = n.abs().amax(-1, keepdim=True) / 127
    s = torch.where(s > 0, s, 1.0)
    return {"h": h, "x": ((n / s).round().clamp(-127, 127) * s).to(h.dtype)}


def _combine(S, case):
    return _sum(S, case, S["y"], S["row"], S["weight"], S["expert"])


def _experts(S, case):
    p = _route(S, case)
    hidden = _products(S["a"], S["rs"], S["w1"], S["cs1"], S["b1"], S["post1"], "silu", True, p["offset"], p["token"], S["cap"], S["hidden"])
    one = torch.ones(hidden.shape[0], device="cuda")
    y = _products(hidden, one, S["w2"], S["cs2"], S["b2"], S["post2"], "none", False, p["offset"], None, S["cap"], S["y"])
    return _sum(S, case, y, p["row"], p["weight"], p["expert"])


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def _busy(case):
    """Experts that have a row, about: those that some of T k independent choices fall on."""
    return case["E"] * (1 - (1 - 1 / case["E"]) ** (case["T"] * case["k"]))


def work(case):
    T, E, k = case["T"], case["E"], case["k"]
    R, out = T * k, {"bf16": 2, "f16": 2, "f32": 4}
    route = {"bytes": T * E * out[case["logits"]] + R * 16 + 4 * E, "flops": T * E * (k + 4)}
    product = lambda rows, K, N, ein, gather, n_out, eout: {  # noqa: E731
        "bytes": _busy(case) * N * K * ein + (min(T, rows) if gather else rows) * K * ein + rows * n_out * eout + _busy(case) * N * 8,
        "flops": 2 * rows * N * K}
    total = {"bytes": 0, "flops": 0}

    def add(w):
        for n in total:
            total[n] += w[n]

    if case["op"] in ("route", "experts"):
        add(route)
    if case["op"] == "linear":
        add(product(R, case["K"], case["N"], 1 if case["kind"] in ("i8", "f8") else 2, case["gather"],
                    case["N"] // 2 if case["gated"] else case["N"], 1 if case["out"] == "i8" else 2))
    if case["op"] == "experts":
        add(product(R, case["H"], 2 * case["F"], 1, True, case["F"], 1))
        add(product(R, case["F"], case["H"], 1, False, case["H"], 1 if case["y"] == "i8" else 2))
    if case["op"] in ("combine", "experts"):
        H = case["H"]
        add({"bytes": R * H * (1 if case["y"] == "i8" else 2) + T * H * (4 + (1 if case["norm"] else 0)) + R * 12, "flops": (2 * R + 8 * T) * H})
    return total


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    S = prepare(case, seed)
    if case["op"] == "route":
        return dict(_exact_route(S, case))
    if case["op"] == "linear":
        y = _exact_linear(S["a"], S["rs"], S["w"], S["cs"], S["b"], S["post"], case["act"], case["gated"], S["offset"],
                          S["token"] if case["gather"] else None, case["out"] == "i8", S["out"].shape)
        return y * S["s_out"] if case["out"] == "i8" else y
    p, y = {n: S[n] for n in ("expert", "weight", "offset", "token", "row")}, S["y"].double()
    if case["op"] == "experts":
        p = _exact_route(S, case)
        hidden = _exact_linear(S["a"], S["rs"], S["w1"], S["cs1"], S["b1"], S["post1"], "silu", True, p["offset"], p["token"], True, S["hidden"].shape)
        y = _exact_linear(hidden, None, S["w2"], S["cs2"], S["b2"], S["post2"], "none", False, p["offset"], None, case["y"] == "i8", S["y"].shape)
        y = y if case["y"] == "i8" else y.to(FP[case["fp"]]).double()                      # as it is stored between the two
    H, T = case["H"], case["T"]
    h = S["h"].double()
    for j in range(case["k"]):
        v = y[p["row"][:T, j].long()]
        if S["y_scale"] is not None:
            v = v * S["y_scale"].double()[p["expert"][:T, j].long()]
        h[:T] += v * p["weight"][:T, j, None].double()
    if not case["norm"]:
        return {"h": h}
    r = h.to(FP[case["fp"]]).double()                     # the normalisation reads the residual stream as it is stored
    n = torch.nn.functional.layer_norm(r, (H,), S["gamma"].double(), S["beta"].double(), EPS)
    s = n.abs().amax(-1, keepdim=True) / 127
    return {"h": h, "x": (n / s).round() * s}


def _exact_route(S, case):
    T, E, k, rows = case["T"], case["E"], case["k"], S["logits"].shape[0]
    x = S["logits"][:T].double().cpu()
    score = 1 / (1 + torch.exp(-x)) if case["score"] == "sigmoid" else torch.exp(x - torch.logsumexp(x, -1, keepdim=True))
    key = x.clone() if S["select_bias"] is None else score + S["select_bias"].double().cpu()
    expert, weight = torch.full((rows, k), -1, dtype=torch.int32), torch.zeros(rows, k, dtype=torch.float64)
    for j in range(k):
        best = key == key.amax(-1, keepdim=True)
        e = torch.where(best, torch.arange(E), E).amin(-1)                                 # the lowest index among the largest
        expert[:T, j], weight[:T, j] = e.int(), score[torch.arange(T), e]
        key[torch.arange(T), e] = -math.inf
    if case["renorm"]:
        weight[:T] /= weight[:T].sum(-1, keepdim=True)
    row, token, offset = torch.full((rows, k), -1, dtype=torch.int32), torch.full((rows * k,), -1, dtype=torch.int32), [0]
    for e in range(E):
        t, j = torch.nonzero(expert == e, as_tuple=True)
        row[t, j] = torch.arange(offset[-1], offset[-1] + len(t), dtype=torch.int32)
        token[offset[-1]:offset[-1] + len(t)] = t.int()
        offset.append(offset[-1] + len(t))
    got = {"expert": expert, "weight": weight, "offset": torch.tensor(offset, dtype=torch.int32), "token": token, "row": row}
    return {n: v.cuda() for n, v in got.items()}


def _exact_linear(a, rs, w, cs, bias, post, act, gated, offset, token, rounded, shape):
    out = torch.zeros(shape, dtype=torch.float64, device="cuda")
    at = offset.tolist()
    for e, (lo, hi) in enumerate(zip(at[:-1], at[1:])):
        if lo == hi:
            continue
        rows = torch.arange(lo, hi, device="cuda") if token is None else token[lo:hi].long()
        x = a.double()[rows] if token is None else a[:, :].to(torch.float32)[rows].double()
        if rs is not None:
            x = x * rs[rows].double()[:, None]
        v = x @ (w[e].to(torch.float32).double() * (1.0 if cs is None else cs[e].double()[:, None])).T + bias[e].double()
        u, f = (v[:, :v.shape[1] // 2], v[:, v.shape[1] // 2:]) if gated else (v, 1.0)
        if act in ("gelu_erf", "gelu_tanh"):
            u = torch.nn.functional.gelu(u, approximate="none" if act == "gelu_erf" else "tanh")
        elif act == "silu":
            u = u * torch.sigmoid(u)
        y = u * f if post is None else u * f * post[e].double()
        out[lo:hi] = y.round().clamp(-127, 127) if rounded else y
    return out
