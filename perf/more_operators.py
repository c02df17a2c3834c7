"""What a decoder's training step has around the compressed linear layers, as measurable cases.

kind     what one pass is
  attn   attention over packed documents, scores capped by a tanh or with a bias that falls with the distance; a forward pass or
         forward and backward
  embed  the vocabulary table's rows of a batch, scaled, and the table's gradient (a dense matrix, summed over equal tokens)
  clip   the norm over all gradients of a model and the gradients times min(1, max_norm / (norm + 1e-6)); with `rank` the linears'
         gradients are pairs of factors, whose products are never formed, and the small factor is what is scaled

Attention: query i sees the keys j of its own document that are at most i (causal) and less than `window` behind it, or that belong to
the document's first `prefix` tokens; rows of no document are zeros.  score = f(q.k / sqrt(d)) - slope |i - j| with f(x) =
cap tanh(x / cap) or x.  `direction`: "step" is a forward and a backward pass, "fwd" the first alone.  `run()` is the plain form, in
32 bits and rounded once, or where `own` is set the calls of the library.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a decoder layer's attention on four sequences of 4096, four query heads to a key head, a training step
        {"name": "attn_step", "kind": "attn", "direction": "step", "n": 16384, "docs": 4, "ragged": 0, "behind": 0, "heads": 32, "kv": 8, "d": 128,
         "causal": True, "cap": 0.0, "bias": False, "prefix": False, "window": 0, "dtype": "bf16"},
        # instruction tuning: conversations of odd lengths in one row, each with a prompt that sees all of itself, capped scores
        {"name": "attn_step_docs", "kind": "attn", "direction": "step", "n": 8191, "docs": 23, "ragged": 5, "behind": 13, "heads": 16, "kv": 16, "d": 64,
         "causal": True, "cap": 30.0, "bias": False, "prefix": True, "window": 0, "dtype": "bf16"},
        # evaluation of a long document with a bias by distance
        {"name": "attn_fwd_long", "kind": "attn", "direction": "fwd", "n": 16384, "docs": 1, "ragged": 0, "behind": 0, "heads": 16, "kv": 4, "d": 128,
         "causal": True, "cap": 0.0, "bias": True, "prefix": False, "window": 0, "dtype": "bf16"},
        # a layer with a sliding window and heads of 80 channels
        {"name": "attn_step_window", "kind": "attn", "direction": "step", "n": 6001, "docs": 2, "ragged": 1, "behind": 0, "heads": 20, "kv": 4, "d": 80,
         "causal": True, "cap": 50.0, "bias": False, "prefix": False, "window": 1000, "dtype": "bf16"},
        # a small float32 model's layer, each token sees the whole of its document
        {"name": "attn_step_f32", "kind": "attn", "direction": "step", "n": 1031, "docs": 3, "ragged": 2, "behind": 0, "heads": 8, "kv": 8, "d": 64,
         "causal": False, "cap": 0.0, "bias": True, "prefix": False, "window": 0, "dtype": "f32"},
        # one short sentence: little work, launches count
        {"name": "attn_tiny", "kind": "attn", "direction": "step", "n": 77, "docs": 1, "ragged": 0, "behind": 0, "heads": 8, "kv": 2, "d": 64,
         "causal": True, "cap": 0.0, "bias": False, "prefix": False, "window": 0, "dtype": "bf16"},
        # the table of 128000 words on 16384 tokens of text, whose words are as unequal as in text, a training step
        {"name": "embed_step_large", "kind": "embed", "n": 16384, "d": 4096, "v": 128000, "padded": 0.0, "scale": 64.0, "dtype": "bf16", "dw_dtype": "bf16"},
        # padded batches of short texts, gradient in float32
        {"name": "embed_step_padded", "kind": "embed", "n": 32768, "d": 1024, "v": 32000, "padded": 0.3, "scale": 1.0, "dtype": "bf16", "dw_dtype": "f32"},
        # a handful of tokens and a small odd vocabulary in float32
        {"name": "embed_step_f32", "kind": "embed", "n": 33, "d": 520, "v": 1001, "padded": 0.1, "scale": 22.8, "dtype": "f32", "dw_dtype": "f32"},
        # all gradients of six layers with 4096 features
        {"name": "clip_layers", "kind": "clip", "layers": 6, "d": 4096, "kv": 1024, "f": 14336, "rank": 0, "dtype": "bf16", "max_norm": 1.0},
        # the same for gradients kept as factors of rank 256
        {"name": "clip_factors", "kind": "clip", "layers": 4, "d": 4096, "kv": 1024, "f": 14336, "rank": 256, "dtype": "bf16", "max_norm": 1.0},
        # many small tensors of odd sizes in float32
        {"name": "clip_small_f32", "kind": "clip", "layers": 6, "d": 131, "kv": 67, "f": 353, "rank": 0, "dtype": "f32", "max_norm": 0.1},
    ]


SCORES = 4 * 32 * 4096 * 4096   # scores of the largest listed case


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "attn", "embed", "embed", "clip", "clip"])
    f32 = rng.random() < 0.25
    case = {"kind": kind, "dtype": "f32" if f32 else "bf16"}
    if kind == "attn":
        while True:
            n = int(_log(rng, 1, 2048 if f32 else 16384))
            kv = rng.choice([1, 2, 3, 4, 8, 16])
            case |= {"direction": rng.choice(["fwd", "step", "step"]), "n": n, "docs": max(1, min(n, int(_log(rng, 1, 40)))),
                     "ragged": rng.randrange(1, 1000), "behind": rng.choice([0, 0, 0, min(n // 3, 29)]), "heads": kv * rng.choice([1, 1, 2, 4, 5, 8]),
                     "kv": kv, "d": rng.choice([128, 128, 64, 64, 96, 8 * rng.randrange(2, 16)]), "causal": rng.random() < 0.8,
                     "cap": rng.choice([0.0, 0.0, 30.0, 50.0]), "bias": rng.random() < 0.3}
            case["prefix"] = case["causal"] and rng.random() < 0.25
            case["window"] = int(_log(rng, 1, n + 1)) if case["causal"] and not case["prefix"] and rng.random() < 0.25 else 0
            longest = max(b - a for a, b in _documents(case))
            if case["docs"] * case["heads"] * longest ** 2 <= SCORES // (16 if f32 else 1) // (1 if case["d"] <= 64 else 2):
                return case
    if kind == "embed":
        while True:
            n, d, v = int(_log(rng, 1, 4096 if f32 else 65536)), 8 * int(_log(rng, 2, 1024)), int(_log(rng, 2, 160000))
            if v * d <= 128000 * 4096 and n * d <= 16384 * 8192:
                return {**case, "n": n, "d": d, "v": v, "padded": rng.choice([0.0, 0.0, 0.3, 0.8]), "scale": rng.choice([1.0, math.sqrt(d)]),
                        "dw_dtype": "f32" if f32 or rng.random() < 0.4 else "bf16"}
    rank = rng.choice([0, 0, 8 * int(_log(rng, 1, 65))])
    q = 8 if rank else 1
    d, layers = q * int(_log(rng, 64 / q, (1024 if f32 else 4096) / q)), rng.randrange(1, 7)
    return {**case, "layers": layers, "d": d, "kv": q * (d // q // rng.choice([1, 2, 4]) or 1), "f": q * int(d * rng.uniform(1.5, 3.5) / q),
            "rank": min(rank, d // 8 * 8), "max_norm": rng.choice([0.01, 1.0, 1e6])}


# ---- inputs --------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _documents(case):
    """(first token, one past the last) of every document; `ragged` picks their lengths, 0: equal ones."""
    n, docs = case["n"] - case["behind"], case["docs"]
    if not case["ragged"]:
        cuts = [n * i // docs for i in range(docs + 1)]
    else:
        rng = random.Random(case["ragged"])
        cuts = [0, *sorted(rng.randrange(n + 1) for _ in range(docs - 1)), n]
    return list(zip(cuts, cuts[1:]))


def _shapes(case):
    """The weights of a layer, [out, in], and its two vectors."""
    d, kv, f = case["d"], case["kv"], case["f"]
    return [(d, d), (kv, d), (kv, d), (d, d), (f, d), (f, d), (d, f)], [d, d]


def prepare(case, seed):
    g, dt, s = _gen(seed), TYPES[case["dtype"]], dict(case)
    if case["kind"] == "attn":
        n, hq, hk, d = case["n"], case["heads"], case["kv"], case["d"]
        # q, k and v are column blocks of one projection's rows
        s["qkv"] = torch.randn(n, (hq + 2 * hk) * d, generator=g, device=DEV).to(dt)
        s["qkv"][:, : hq * d] *= 2.0
        docs = _documents(case)
        s["starts"] = torch.tensor([a for a, _ in docs] + [docs[-1][1]], dtype=torch.int64, device=DEV)
        s["prefixes"] = torch.tensor([(b - a) // 3 for a, b in docs], dtype=torch.int64, device=DEV) if case["prefix"] else None
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device=DEV, dtype=torch.float32) / hq) if case["bias"] else None
        if case["direction"] == "step":
            s["do"] = (torch.randn(n, hq * d, generator=g, device=DEV) * 0.01).to(dt)
    elif case["kind"] == "embed":
        n, d, v = case["n"], case["d"], case["v"]
        s["w"] = (torch.randn(v, d, generator=g, device=DEV) * 0.02).to(dt)
        # the r-th most frequent word has a share of about 1 / r, as in text
        ids = (v ** torch.rand(n, generator=g, device=DEV, dtype=torch.float64)).long().clamp_(1, v) - 1
        s["ids"] = torch.where(torch.rand(n, generator=g, device=DEV) < case["padded"], -1, ids)
        s["dy"] = (torch.randn(n, d, generator=g, device=DEV) * 0.01).to(dt)
    else:
        linears, vectors = _shapes(case)
        normal = lambda *size: torch.randn(*size, generator=g, device=DEV) * 1e-3  # noqa: E731
        s["dense"], s["left"], s["gr"] = [], [], []
        for _ in range(case["layers"]):
            for d_out, d_in in linears:
                if case["rank"]:
                    s["left"].append((normal(d_in, case["rank"]) * 3e3).to(dt))
                    s["gr"].append((normal(d_out, case["rank"])).to(dt))
                else:
                    s["dense"].append(normal(d_out, d_in).to(dt))
            s["dense"] += [normal(c) for c in vectors]
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------
def _plain_attn(s):
    dt, n, hq, hk, d = TYPES[s["dtype"]], s["n"], s["heads"], s["kv"], s["d"]
    longest = max(1, max(b - a for a, b in _documents(s)))
    # [documents, heads, longest, channels]; rows behind a document are masked
    at = torch.arange(longest, device=DEV)
    first, length = s["starts"][:-1], s["starts"].diff()
    there = at < length.unsqueeze(1)
    rows = torch.where(there, first.unsqueeze(1) + at, 0)
    q, k, v = (t.reshape(n, -1, d)[rows].float().transpose(1, 2) for t in s["qkv"].split((hq * d, hk * d, hk * d), 1))
    k, v = k.repeat_interleave(hq // hk, 1), v.repeat_interleave(hq // hk, 1)
    scale = 1.0 / math.sqrt(d)
    z = (q @ k.transpose(2, 3).contiguous()).mul_(scale)
    if s["cap"]:
        z = z.div_(s["cap"]).tanh_()
        slope_of_cap = 1.0 - z * z if s["direction"] == "step" else None
        z = z.mul_(s["cap"])
    gap = at.unsqueeze(1) - at
    if s["bias"]:
        z -= s["slopes"].view(-1, 1, 1) * gap.abs()
    seen = there.unsqueeze(1) & there.unsqueeze(2)
    if s["causal"]:
        near = gap >= 0
        if s["window"]:
            near = near & (gap < s["window"])
        if s["prefixes"] is not None:
            near = near | (at < s["prefixes"].view(-1, 1, 1))
        seen = seen & near
    z.masked_fill_(~seen.unsqueeze(1), -math.inf)
    top = z.amax(3, keepdim=True).clamp_min(-3e38)
    p = z.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    lse = (top + total.log()).squeeze(3)
    p = p.div_(total.clamp_min(1e-30))

    def back(t, like):   # [documents, heads, longest, channels] -> [n, heads * channels]
        full = torch.zeros(n, *like, device=DEV)
        full[rows[there]] = t.transpose(1, 2)[there]
        return full.flatten(1).to(dt)

    full = torch.full((n, hq), -math.inf, device=DEV)
    full[rows[there]] = lse.transpose(1, 2)[there]
    out = {"o": back(p @ v, (hq, d)), "lse": full.t().contiguous()}
    if s["direction"] == "step":
        do = (s["do"].reshape(n, hq, d)[rows].float() * there.view(*there.shape, 1, 1)).transpose(1, 2)
        dv = p.transpose(2, 3).contiguous() @ do
        dz = do @ v.transpose(2, 3).contiguous()
        dz = dz.sub_((p * dz).sum(3, keepdim=True)).mul_(p)
        if s["cap"]:
            dz *= slope_of_cap
        dq, dk = (dz @ k).mul_(scale), (dz.transpose(2, 3).contiguous() @ q).mul_(scale)
        groups = lambda t: t.unflatten(1, (hk, hq // hk)).sum(2)  # noqa: E731
        out |= {"dq": back(dq, (hq, d)), "dk": back(groups(dk), (hk, d)), "dv": back(groups(dv), (hk, d))}
    return out


def _plain_embed(s):
    counts = s["ids"] >= 0
    ids = s["ids"].clamp_min(0)
    y = torch.where(counts.unsqueeze(1), s["w"][ids].float() * s["scale"], 0.0)
    dy = torch.where(counts.unsqueeze(1), s["dy"].float() * s["scale"], 0.0)
    dw = torch.zeros(s["v"], s["d"], device=DEV).index_add_(0, ids, dy)
    return {"y": y.to(TYPES[s["dtype"]]), "dw": dw.to(TYPES[s["dw_dtype"]])}


def _plain_clip(s):
    squares = [t.float().square().sum(dtype=torch.float64) for t in s["dense"]]
    squares += [(g.float() @ x.float().t()).square().sum(dtype=torch.float64) for x, g in zip(s["left"], s["gr"])]
    norm = torch.stack(squares).sum().sqrt().float()
    factor = (s["max_norm"] / (norm + 1e-6)).clamp_max(1.0)
    return {"norm": norm, "grads": [(t.float() * factor).to(t.dtype) for t in s["dense"] + s["gr"]]}


# ---- the library's calls -------------------------------------------------------------------------------------
def _own_attn(acc, s):
    dt, n, hq, hk, d = TYPES[s["dtype"]], s["n"], s["heads"], s["kv"], s["d"]
    ld = (hq + 2 * hk) * d
    desc = acc.make_attn_desc(n, hq, hk, d, ldq=ld, ldk=ld, ldv=ld, docs=s["docs"], window=s["window"], cap=s["cap"], io_dtype=_code(acc, s["dtype"]),
                              flags=acc.ACC_ATTN_CAUSAL if s["causal"] else 0)
    q, k, v = s["qkv"].split((hq * d, hk * d, hk * d), 1)
    masks = s["starts"], s["prefixes"], s["slopes"]
    o, lse = torch.empty(n, hq * d, dtype=dt, device=DEV), torch.empty(hq, n, device=DEV)
    step = s["direction"] == "step"
    ws = torch.empty(acc.acc_attn_workspace_bytes(desc, step), dtype=torch.uint8, device=DEV)
    acc.acc_attn_fwd(desc, q, k, v, *masks, o, lse, ws)
    out = {"o": o, "lse": lse}
    if step:
        out["dq"], out["dk"], out["dv"] = torch.empty(n, ld, dtype=dt, device=DEV).split((hq * d, hk * d, hk * d), 1)
        acc.acc_attn_bwd(desc, q, k, v, *masks, o, lse, s["do"], out["dq"], out["dk"], out["dv"], ws)
    return out


def _own_embed(acc, s):
    n, d, v = s["n"], s["d"], s["v"]
    desc = acc.make_embed_desc(n, d, v, scale=s["scale"], io_dtype=_code(acc, s["dtype"]), dw_dtype=_code(acc, s["dw_dtype"]))
    y = torch.empty(n, d, dtype=TYPES[s["dtype"]], device=DEV)
    acc.acc_embed_fwd(desc, s["w"], s["ids"], y)
    dw = torch.empty(v, d, dtype=TYPES[s["dw_dtype"]], device=DEV)
    ws = torch.empty(acc.acc_embed_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    acc.acc_embed_bwd(desc, s["ids"], s["dy"], dw, ws)
    return {"y": y, "dw": dw}


def _own_clip(acc, s):
    result = torch.empty(2, device=DEV)
    outs = [torch.empty_like(t) for t in s["dense"] + s["gr"]]
    dense = acc.make_grad_list(s["dense"])
    factors = acc.make_factor_list(s["left"], s["gr"], acc.ACC_FLAG_W_OUT_IN)
    ws = torch.empty(acc.acc_grad_norm_workspace_bytes(dense, factors), dtype=torch.uint8, device=DEV)
    acc.acc_grad_norm(dense, factors, s["max_norm"], result, ws)
    acc.acc_grad_scale(acc.make_grad_list(s["dense"] + s["gr"], outs), result[1:])
    return {"norm": result[0], "grads": outs}


def _code(acc, name):
    return acc.ACC_BF16 if name == "bf16" else acc.ACC_F32


def run(s):
    if own:
        from paper_2605_01255_amd import binding
        return {"attn": _own_attn, "embed": _own_embed, "clip": _own_clip}[s["kind"]](binding, s)
    return {"attn": _plain_attn, "embed": _plain_embed, "clip": _plain_clip}[s["kind"]](s)


# ---- what a pass cannot do without ---------------------------------------------------------------------------
def _seen(case):
    """Pairs of a query and a key that it sees, over all documents of one head."""
    total = 0
    for a, b in _documents(case):
        n = b - a
        if not case["causal"]:
            total += n * n
        elif case["window"]:
            w = min(case["window"], n)
            total += w * (w + 1) // 2 + (n - w) * w
        else:
            p = n // 3 if case["prefix"] else 0
            total += p * p + (n * (n + 1) - p * (p + 1)) // 2
    return total


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "attn":
        n, hq, hk, d = case["n"], case["heads"], case["kv"], case["d"]
        rows, step = n * d * es, case["direction"] == "step"
        b = rows * (2 * hq + 2 * hk) + 4 * n * hq
        products = 2
        if step:   # q, k, v, o, do, lse; dq, dk, dv.  Two products give the probabilities and their gradients, three the gradients
            b += rows * (4 * hq + 4 * hk) + 4 * n * hq
            products += 5
        return {"bytes": b, "flops": products * 2 * d * hq * _seen(case)}
    if case["kind"] == "embed":
        n, d, v = case["n"], case["d"], case["v"]
        live = int(n * (1 - case["padded"]))
        words = min(v, live)   # rows of the table that are read, at most
        return {"bytes": words * d * es + 8 * n + n * d * es + 8 * n + live * d * es + v * d * (4 if case["dw_dtype"] == "f32" else 2),
                "flops": 3 * live * d}
    linears, vectors = _shapes(case)
    rank, flops, b = case["rank"], 0, 0
    for rows, cols in linears:
        if rank:   # read both factors, write one; the two r x r products of their rows
            b += (2 * rows + cols) * rank * es
            flops += 2 * (rows + cols) * rank * rank
        else:
            b += 2 * rows * cols * es
            flops += 3 * rows * cols
    b += sum(8 * c for c in vectors)
    return {"bytes": b * case["layers"], "flops": flops * case["layers"]}


# ---- 64 bits, from the definitions ---------------------------------------------------------------------------
def _exact_attn(case, s):
    n, hq, hk, d = case["n"], case["heads"], case["kv"], case["d"]
    step = case["direction"] == "step"
    zeros = lambda h: torch.zeros(n, h, d, dtype=torch.float64, device=DEV)  # noqa: E731
    out = {"o": zeros(hq), "lse": torch.full((hq, n), -math.inf, dtype=torch.float64, device=DEV)}
    if step:
        out |= {"dq": zeros(hq), "dk": zeros(hk), "dv": zeros(hk)}
    rows = s["qkv"].double().view(n, hq + 2 * hk, d)
    for doc, (a, b) in enumerate(_documents(case)):
        if a == b:
            continue
        i = torch.arange(a, b, device=DEV).view(-1, 1)
        j = i.view(1, -1)
        hidden = torch.zeros(b - a, b - a, dtype=torch.bool, device=DEV)
        if case["causal"]:
            hidden |= j > i
            if case["window"]:
                hidden |= i - j >= case["window"]
            if case["prefix"]:
                hidden &= j >= a + (b - a) // 3
        for h in range(hq):
            q, k, v = (rows[a:b, x].detach().requires_grad_(step) for x in (h, hq + h * hk // hq, hq + hk + h * hk // hq))
            z = q.mm(k.t()) / d ** 0.5
            if case["cap"]:
                z = torch.tanh(z / case["cap"]) * case["cap"]
            if case["bias"]:
                z = z - s["slopes"][h].double() * (i - j).abs()
            z = torch.where(hidden, torch.full_like(z, -math.inf), z)
            lse = torch.logsumexp(z, 1)
            o = torch.exp(z - lse.view(-1, 1)).mm(v)
            out["o"][a:b, h], out["lse"][h, a:b] = o.detach(), lse.detach()
            if step:
                dq, dk, dv = torch.autograd.grad(o, (q, k, v), s["do"][a:b, h * d:(h + 1) * d].double())
                out["dq"][a:b, h] = dq
                out["dk"][a:b, h * hk // hq] += dk
                out["dv"][a:b, h * hk // hq] += dv
    return {name: t if name == "lse" else t.flatten(1) for name, t in out.items()}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attn":
        return _exact_attn(case, s)
    if case["kind"] == "embed":
        counts = (s["ids"] >= 0).nonzero().squeeze(1)
        ids = s["ids"][counts]
        y = torch.zeros(case["n"], case["d"], dtype=torch.float64, device=DEV)
        y[counts] = s["w"].double().index_select(0, ids) * case["scale"]
        order = torch.argsort(ids, stable=True)   # equal words next to each other, their sum the difference of two running ones
        words, times = torch.unique_consecutive(ids[order], return_counts=True)
        ends = times.cumsum(0)
        sums = torch.zeros(len(ids) + 1, case["d"], dtype=torch.float64, device=DEV)
        torch.cumsum(s["dy"].index_select(0, counts[order]).double(), 0, out=sums[1:])
        dw = torch.zeros(case["v"], case["d"], dtype=torch.float64, device=DEV)
        dw[words] = (sums[ends] - sums[ends - times]) * case["scale"]
        return {"y": y, "dw": dw}
    total = sum(float(torch.linalg.vector_norm(t.double())) ** 2 for t in s["dense"])
    total += sum(float(torch.linalg.vector_norm(x.double() @ g.double().t())) ** 2 for x, g in zip(s["left"], s["gr"]))
    norm = math.sqrt(total)
    factor = min(1.0, case["max_norm"] / (norm + 1e-6))
    return {"norm": torch.tensor(norm, dtype=torch.float64), "grads": [t.double() * factor for t in s["dense"] + s["gr"]]}
