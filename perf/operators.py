"""Operators beside the MoE layer, as cases that can be timed and compared.

``route``   routing from logits: softmax or sigmoid scores, a balance bias that chooses and never weighs, groups of experts, top-k,
            renormalised weights, and the stable grouping of the assignments by expert.
``linear``  one matrix of 8-bit codes with a scale for each output channel: the tokens are quantised to 8 bits with a scale each,
            multiplied in whole numbers and scaled.
``up``      the first half of 8-bit experts: the same product over the tokens of every expert, gathered by the routing, with
            silu(gate) * up behind it.
``down``    their second half: activations quantised, multiplied by their expert's matrix, and summed back into their tokens with the
            routing's weights.

With ``own`` the calls are those of ``paper_2510_26730_amd.binding``; without it the same operators are written in elementary torch
operations.  Sums of 8-bit products pass 24 bits and scores meet at the border of a top-k, so both are formed in 64 bits there.
"""
import math

import numpy as np
import torch

own = False

SMALLEST = 2.0 ** -126      # a row's scale is at least this
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def _route(name, T, E, k, score, groups, kept, best, bias, renorm, scale, dtype):
    return {"name": name, "op": "route", "T": T, "E": E, "k": k, "score": score, "groups": groups, "kept": kept, "best": best,
            "bias": bias, "renorm": renorm, "scale": scale, "dtype": dtype}


def _linear(name, M, K, N, dtype, out):
    return {"name": name, "op": "linear", "M": M, "K": K, "N": N, "dtype": dtype, "out": out}


def _experts(name, op, T, E, k, d, F, dtype):
    return {"name": name, "op": op, "T": T, "E": E, "k": k, "d": d, "F": F, "dtype": dtype}


def listed():
    return [
        # one sequence being decoded, 64 experts, plain softmax: nothing but latency
        _route("route_1", 1, 64, 6, "softmax", 1, 1, 1, False, False, 1.0, "f32"),
        # a decode batch over 256 experts in 8 groups, sigmoid scores with a balance bias, four groups kept by their two best
        _route("route_sigmoid_64", 64, 256, 8, "sigmoid", 8, 4, 2, True, True, 2.5, "f32"),
        # a prompt chunk with decode tokens, 60 experts, logits as a 16-bit gate leaves them
        _route("route_1056", 1056, 60, 4, "softmax", 1, 1, 1, False, True, 1.0, "bf16"),
        # many prompts at once: bound by reading the logits
        _route("route_sigmoid_32768", 32768, 256, 8, "sigmoid", 8, 4, 2, True, True, 2.5, "f32"),
        # a projection of one decoded token: every weight read once
        _linear("linear_1", 1, 4096, 4096, "bf16", "bf16"),
        # a decode batch through the first matrix of a shared FFN
        _linear("linear_64", 64, 2048, 5632, "bf16", "bf16"),
        # a ragged prompt chunk, sizes that no tile divides, fp16 in and 32 bits out
        _linear("linear_517", 517, 5640, 2049, "f16", "f32"),
        # whole prompts through the widest matrix there is here: bound by the matrix cores
        _linear("linear_8192", 8192, 4096, 14336, "bf16", "bf16"),
        # a decode batch of 64 small experts: a few tokens each, bound by reading the weights
        _experts("up_32", "up", 32, 64, 6, 2048, 1408, "bf16"),
        # prompts through eight wide experts
        _experts("up_4096", "up", 4096, 8, 2, 4096, 14336, "bf16"),
        # the second half of the decode batch, summed back into its tokens
        _experts("down_32", "down", 32, 64, 6, 2048, 1408, "bf16"),
        # a prompt of 1024 tokens with 32 decode tokens over 64 experts, some of them with few tokens and some with hundreds
        _experts("down_1056", "down", 1056, 64, 6, 2048, 1408, "bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["route", "linear", "up", "down"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        E = groups * _log(rng, max(2, 8 // groups), 256 // groups)
        kept = rng.randint(1, groups)
        k = rng.randint(1, min(8, kept * (E // groups)))
        score = rng.choice(["softmax", "sigmoid"])
        return {"op": op, "T": _log(rng, 1, 32768), "E": E, "k": k, "score": score, "groups": groups, "kept": kept,
                "best": rng.choice([1, 2]), "bias": rng.random() < 0.5, "renorm": rng.random() < 0.5,
                "scale": rng.choice([1.0, 2.5]), "dtype": dtype}
    if op == "linear":
        M, K, N = _log(rng, 1, 8192), _log(rng, 256, 14336), _log(rng, 256, 14336)
        while M * K * N > 8192 * 4096 * 14336:
            M = max(1, M // 2)
        return {"op": op, "M": M, "K": K, "N": N, "dtype": dtype, "out": rng.choice(["bf16", "f16", "f32"])}
    E = _log(rng, 4, 256)
    k = rng.randint(1, min(8, E))
    d, F = _log(rng, 256, 4096), _log(rng, 128, 14336)
    while E * d * F > 8 * 4096 * 14336:
        F = max(128, F // 2) if F > 128 else F
        E = max(k, E // 2)
    T = _log(rng, 1, 4096)
    while T * k * d * F > 4096 * 2 * 4096 * 14336:
        T = max(1, T // 2)
    return {"op": op, "T": T, "E": E, "k": k, "d": d, "F": F, "dtype": dtype}


# ---- inputs ------------------------------------------------------------------------------------

def _codes(gen, *shape):
    """Codes of weights, whose rows are 16-byte aligned: normal, the largest of a row near 127."""
    *lead, K = shape
    pitch = (K + 15) // 16 * 16
    c = torch.empty(*lead, pitch, dtype=torch.int8, device="cuda")
    flat = c.view(-1, pitch)
    for r in range(0, flat.shape[0], 16384):
        part = flat[r:r + 16384]
        part.copy_(torch.empty(part.shape, device="cuda").normal_(generator=gen).mul_(36).round_().clamp_(-127, 127))
    return c[..., :K]


def _choices(gen, T, E, k):
    """Experts of each token in ascending order, some more popular than others."""
    popular = -0.6 * torch.log(torch.randperm(E, generator=gen, device="cuda").float() + 1)
    noise = -torch.log(-torch.log(torch.rand(T, E, generator=gen, device="cuda").clamp_(1e-6, 1 - 1e-6)))
    return (popular + noise).topk(k, dim=1).indices.sort(dim=1).values


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    c = dict(case)
    dev = dict(device="cuda")
    ty = TYPES[c["dtype"]]
    i32 = dict(dtype=torch.int32, device="cuda")
    if c["op"] == "route":
        T, E, k = c["T"], c["E"], c["k"]
        lean = torch.randn(E, generator=gen, **dev)
        logits = (1.5 * torch.randn(T, E, generator=gen, **dev) + 0.5 * lean).to(ty)
        bias = (0.1 * torch.randn(E, generator=gen, **dev) - 0.05 * lean) if c["bias"] else None
        # room for what the call leaves in between: counts of every expert in every tile of 16 tokens, and their prefixes
        work = torch.empty(4096 + 16 * E * (T // 16 + 2), dtype=torch.uint8, **dev)
        return {"case": c, "logits": logits, "bias": bias, "work": work, "ids": torch.empty(T, k, **i32),
                "w": torch.empty(T, k, **dev), "counts": torch.empty(E, **i32), "offsets": torch.empty(E + 1, **i32),
                "perm": torch.empty(T * k, **i32), "inv_perm": torch.empty(T * k, **i32)}
    if c["op"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        x = torch.randn(M, K, generator=gen, **dev).to(ty)
        s = (0.02 / 36) * (0.5 + torch.rand(N, generator=gen, **dev))
        return {"case": c, "x": x, "wq": _codes(gen, N, K), "ws": s, "out": torch.empty(M, N, dtype=TYPES[c["out"]], **dev),
                "work": torch.empty(_work_bytes(M, K), dtype=torch.uint8, **dev)}
    T, E, k, d, F = c["T"], c["E"], c["k"], c["d"], c["F"]
    ids = _choices(gen, T, E, k).reshape(-1)
    perm = torch.sort(ids, stable=True).indices
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(T * k, **dev)
    counts = torch.bincount(ids, minlength=E)
    offsets = torch.cat([torch.zeros(1, dtype=counts.dtype, **dev), counts.cumsum(0)])
    st = {"case": c, "most": int(counts.max()), "perm": perm.int(), "inv_perm": inv.int(), "offsets": offsets.int()}
    if c["op"] == "up":
        st.update(x=torch.randn(T, d, generator=gen, **dev).to(ty), wq=_codes(gen, E, 2 * F, d),
                  ws=(0.02 / 36) * (0.5 + torch.rand(E, 2 * F, generator=gen, **dev)),
                  out=torch.empty(T * k, F, dtype=ty, **dev), work=torch.empty(_work_bytes(T, d), dtype=torch.uint8, **dev))
    else:
        act = torch.nn.functional.silu(torch.randn(T * k, F, generator=gen, **dev)) * torch.randn(T * k, F, generator=gen, **dev)
        w = torch.rand(T, k, generator=gen, **dev) + 0.1
        st.update(x=act.to(ty), wq=_codes(gen, E, d, F), ws=(0.02 / 36) * (0.5 + torch.rand(E, d, generator=gen, **dev)),
                  w=w / w.sum(1, keepdim=True), y=torch.empty(T * k, d, **dev), out=torch.empty(T, d, dtype=ty, **dev),
                  work=torch.empty(_work_bytes(T * k, F), dtype=torch.uint8, **dev))
    return st


def _work_bytes(rows, K):
    """Room for the rows' codes and scales, and for what a split product leaves in between."""
    return (64 << 20) + rows * ((K + 127) // 128 * 128 + 4) + 4096


# ---- plain forms -------------------------------------------------------------------------------

def _plain_route(st):
    c = st["case"]
    T, E, k = c["T"], c["E"], c["k"]
    z = st["logits"].double()
    if c["score"] == "softmax":
        e = torch.exp(z - z.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    else:
        score = 1 / (1 + torch.exp(-z))
    choose = score if st["bias"] is None else score + st["bias"].double()
    if c["groups"] > 1:
        by = choose.view(T, c["groups"], -1)
        best = by.sort(dim=2, descending=True).values[:, :, :c["best"]].sum(2)
        keep = best.sort(dim=1, descending=True, stable=True).indices[:, :c["kept"]]
        live = torch.zeros(T, c["groups"], dtype=torch.bool, device="cuda").scatter_(1, keep, True)
        choose = torch.where(live[:, :, None], by, -math.inf).view(T, E)
    ids = choose.sort(dim=1, descending=True, stable=True).indices[:, :k].sort(dim=1).values
    w = score.gather(1, ids)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    flat = ids.reshape(-1)
    perm = flat.sort(stable=True).indices
    inv = torch.empty_like(perm).scatter_(0, perm, torch.arange(T * k, device="cuda"))
    counts = torch.zeros(E, dtype=torch.int64, device="cuda").scatter_add_(0, flat, torch.ones_like(flat))
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return ids.int(), (w * c["scale"]).float(), counts.int(), offsets.int(), perm.int(), inv.int()


def _plain_quant(x):
    """Codes (as 64-bit numbers) and scales of each row."""
    v = x.double()
    s = (v.abs().amax(1) / 127).float().clamp(min=SMALLEST).double()
    return torch.round(v / s[:, None]), s


def _plain_grouped(q, s, st):
    """The rows' products with their expert's matrix, scaled: padded to as many rows as the fullest expert has."""
    o, rows = st["offsets"].long(), q.shape[0]
    at = o[:-1, None] + torch.arange(st["most"], device="cuda")
    live = at < o[1:, None]
    x = q[at.clamp(max=rows - 1)].transpose(1, 2).contiguous()
    y = torch.bmm(st["wq"].double(), x) * st["ws"].double()[:, :, None]
    return y.transpose(1, 2)[live] * s[:, None]


def _plain(st):
    c = st["case"]
    if c["op"] == "route":
        return _plain_route(st)
    q, s = _plain_quant(st["x"])
    if c["op"] == "linear":
        return (torch.mm(q, st["wq"].double().t()) * s[:, None] * st["ws"].double()).to(TYPES[c["out"]])
    ty = TYPES[c["dtype"]]
    if c["op"] == "up":
        tok = st["perm"].long() // c["k"]
        gu = _plain_grouped(q[tok], s[tok], st).float()
        g, u = gu[:, :c["F"]], gu[:, c["F"]:]
        return (g / (1 + torch.exp(-g)) * u).to(ty)
    y = _plain_grouped(q, s, st).float()[st["inv_perm"].long()].view(c["T"], c["k"], c["d"])
    return (y * st["w"][:, :, None]).sum(1).to(ty)


# ---- the framework's calls ---------------------------------------------------------------------

def _own(st):
    from paper_2510_26730_amd import binding as ef
    c, s = st["case"], torch.cuda.current_stream()
    if c["op"] == "route":
        ef.ef_route_scores(st["logits"], st["bias"], st["ids"], st["w"], st["counts"], st["offsets"], st["perm"], st["inv_perm"],
                           st["work"], sigmoid=c["score"] == "sigmoid", n_groups=c["groups"], groups_kept=c["kept"],
                           group_best=c["best"], renorm=c["renorm"], scale=c["scale"], stream=s)
        return st["ids"], st["w"], st["counts"], st["offsets"], st["perm"], st["inv_perm"]
    if c["op"] == "linear":
        ef.ef_matmul_q8(st["x"], st["wq"], st["ws"], st["out"], st["work"], stream=s)
    elif c["op"] == "up":
        ef.ef_matmul_q8(st["x"], st["wq"], st["ws"], st["out"], st["work"], offsets=st["offsets"], rows=st["perm"], row_div=c["k"],
                        swiglu=True, stream=s)
    else:
        ef.ef_matmul_q8(st["x"], st["wq"], st["ws"], st["y"], st["work"], offsets=st["offsets"], stream=s)
        ef.ef_combine(st["y"], st["w"], st["inv_perm"], st["out"], stream=s)
    return st["out"]


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ---------------------------------------------------------------

def _experts_in_use(T, E, k):
    """Expected number of experts that any token takes, for the popularities of prepare()."""
    p = np.arange(1, E + 1) ** -0.6
    p = np.minimum(1.0, k * p / p.sum())
    return float(np.sum(1 - (1 - p) ** T))


def work(case):
    c = case
    if c["op"] == "route":
        T, E, k = c["T"], c["E"], c["k"]
        return {"bytes": T * E * SIZE[c["dtype"]] + 16 * T * k + 8 * E + (4 * E if c["bias"] else 0), "flops": 0}
    if c["op"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        return {"bytes": M * K * SIZE[c["dtype"]] + N * (K + 4) + M * N * SIZE[c["out"]], "flops": 2 * M * K * N}
    T, E, k, d, F = c["T"], c["E"], c["k"], c["d"], c["F"]
    n, size, rows = _experts_in_use(T, E, k), SIZE[c["dtype"]], T * k
    if c["op"] == "up":
        return {"bytes": T * d * size + n * 2 * F * (d + 4) + rows * (F * size + 4), "flops": 4 * rows * d * F}
    return {"bytes": rows * F * size + n * d * (F + 4) + T * d * size + 8 * rows, "flops": 2 * rows * d * F}


# ---- the definition in 64 bits -------------------------------------------------------------------

def _exact_route(st):
    c = st["case"]
    z = st["logits"].double().cpu().numpy()
    T, E, k = c["T"], c["E"], c["k"]
    if c["score"] == "softmax":
        p = np.exp(z - z.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
    else:
        p = 1 / (1 + np.exp(-z))
    sel = p + (0 if st["bias"] is None else st["bias"].double().cpu().numpy())
    if c["groups"] > 1:
        per = E // c["groups"]
        top = -np.sort(-sel.reshape(T, c["groups"], per), axis=2)[:, :, :c["best"]].sum(2)
        rank = np.argsort(np.argsort(-top, axis=1, kind="stable"), axis=1, kind="stable")
        sel = np.where(np.repeat(rank < c["kept"], per, axis=1), sel, -np.inf)
    ids = np.sort(np.argsort(-sel, axis=1, kind="stable")[:, :k], axis=1)
    w = np.take_along_axis(p, ids, 1)
    if c["renorm"]:
        w = w / w.sum(1, keepdims=True)
    perm = np.argsort(ids.reshape(-1), kind="stable")
    inv = np.empty(T * k, np.int64)
    inv[perm] = np.arange(T * k)
    counts = np.bincount(ids.reshape(-1), minlength=E)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).int()  # noqa: E731
    return i32(ids), torch.from_numpy(w * c["scale"]), i32(counts), i32(offsets), i32(perm), i32(inv)


def _exact_codes(x):
    v = x.to(torch.float64)
    scale = torch.clamp((v.abs().max(dim=1).values / 127.0).to(torch.float32), min=SMALLEST).to(torch.float64)
    return torch.div(v, scale[:, None]).round(), scale


def _exact_product(q, w):
    """Whole-number products: pieces of 512 columns, whose sums 32-bit floats hold exactly, added up in 64 bits."""
    total = torch.zeros(q.shape[0], w.shape[0], dtype=torch.float64, device=q.device)
    for a in range(0, q.shape[1], 512):
        total += torch.mm(q[:, a:a + 512].float(), w[:, a:a + 512].float().t())
    return total


def exact(case, seed):
    st = prepare(case, seed)
    c = st["case"]
    if c["op"] == "route":
        return _exact_route(st)
    q, s = _exact_codes(st["x"])
    if c["op"] == "linear":
        out = _exact_product(q, st["wq"])
        out *= st["ws"].double()
        out *= s[:, None]
        return out
    off = st["offsets"].tolist()
    row = st["perm"].long() // c["k"] if c["op"] == "up" else torch.arange(c["T"] * c["k"], device="cuda")
    parts = []
    for e in range(c["E"]):
        r = row[off[e]:off[e + 1]]
        if len(r):
            y = _exact_product(q[r], st["wq"][e]) * st["ws"][e].double() * s[r][:, None]
            parts.append(y[:, :c["F"]] * torch.sigmoid(y[:, :c["F"]]) * y[:, c["F"]:] if c["op"] == "up" else y)
    y = torch.cat(parts)
    if c["op"] == "up":
        return y
    out = torch.zeros(c["T"], c["d"], dtype=torch.float64, device="cuda")
    for j in range(c["k"]):
        out += st["w"][:, j, None].double() * y[st["inv_perm"].view(c["T"], c["k"])[:, j].long()]
    return out
