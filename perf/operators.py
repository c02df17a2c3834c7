"""The operators beside the compressed linear layer that a training step is made of, as measurable cases.

kind      what one pass is
  pack    an activation into its 8-bit checkpoint and back
  linear  a linear layer that keeps its input as an 8-bit checkpoint: y and, from the checkpoint, the weight's gradient
  gated   SiLU(gate) * up with gate and up kept as 8-bit checkpoints, and its gradients from them
  ce      the vocabulary's product and its softmax cross entropy without the logits: per-token losses, and the gradients

An 8-bit checkpoint holds one power-of-two scale 2^e for every 32 consecutive tokens of a channel, e the least whole number
>= -100 for which the block's largest magnitude is at most 448 (e4m3) or 127 (int8) times 2^e, and every element over 2^e rounded
to nearest even.  What is not finite comes back as NaN and does not count for the scale.

`direction`: "step" is a forward and a backward pass, "fwd" and "bwd" are one of them.  `run()` is the plain form, in 32 bits and
rounded once, or where `own` is set the calls of the library.
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 32
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
TOP = 1.875 * 2.0 ** 127   # finite magnitudes above are kept as this


def listed():
    return [
        # the input of an attention projection, kept between forward and backward
        {"name": "pack_e4m3", "kind": "pack", "n": 16384, "c": 4096, "ld": 4096, "dtype": "bf16", "format": "e4m3"},
        # an odd number of tokens out of a wider float32 buffer: little data, launches count
        {"name": "pack_short_f32", "kind": "pack", "n": 77, "c": 520, "ld": 1040, "dtype": "f32", "format": "int8"},
        # a square projection of a decoder layer on 16384 tokens, a training step
        {"name": "linear_step", "kind": "linear", "direction": "step", "n": 16384, "d_in": 4096, "d_out": 4096, "w_out_in": True,
         "dtype": "bf16", "format": "int8"},
        # the backward pass alone at sizes that are no multiples of a tile, weights as [d_in, d_out], gradient in float32
        {"name": "linear_bwd_ragged", "kind": "linear", "direction": "bwd", "n": 2049, "d_in": 1032, "d_out": 1544, "w_out_in": False,
         "dtype": "bf16", "dw_dtype": "f32", "format": "e4m3"},
        # the small float32 layer of the repository's first configuration
        {"name": "linear_tiny_f32", "kind": "linear", "direction": "step", "n": 256, "d_in": 256, "d_out": 512, "w_out_in": True,
         "dtype": "f32", "format": "int8"},
        # the gated activation of an MLP with 8192 channels on 16384 tokens, a training step
        {"name": "gated_step", "kind": "gated", "direction": "step", "n": 16384, "f": 8192, "dtype": "bf16", "format": "int8"},
        # its backward pass on an odd batch, which also forms the activation again for the product behind it
        {"name": "gated_bwd_again", "kind": "gated", "direction": "bwd", "n": 3001, "f": 2728, "dtype": "bf16", "format": "e4m3", "again": True},
        # one token in float32
        {"name": "gated_one_f32", "kind": "gated", "direction": "step", "n": 1, "f": 1408, "dtype": "f32", "format": "int8"},
        # loss and gradients of a fine-tuning batch over a vocabulary of 128000: two tokens in five belong to prompts and have no loss
        {"name": "ce_step_large", "kind": "ce", "direction": "step", "n": 8192, "d": 4096, "v": 128000, "dtype": "bf16", "ignored": 0.4},
        # evaluation of a short document: the losses alone
        {"name": "ce_fwd", "kind": "ce", "direction": "fwd", "n": 1024, "d": 2048, "v": 32000, "dtype": "bf16", "ignored": 0.0},
        # a small float32 model with an odd vocabulary
        {"name": "ce_step_f32", "kind": "ce", "direction": "step", "n": 515, "d": 520, "v": 10007, "dtype": "f32", "ignored": 0.1},
        # the score of one token: the vocabulary's matrix is read once and that is all
        {"name": "ce_one", "kind": "ce", "direction": "fwd", "n": 1, "d": 2048, "v": 50257, "dtype": "bf16", "ignored": 0.0},
    ]


LARGEST = 8192 * 4096 * 128000   # multiply-adds of one product of the largest listed case


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _width(rng, lo, hi):
    """A width of a layer: most are multiples of 64, one in four only of 8."""
    q = 8 if rng.random() < 0.25 else 64
    return max(q, int(_log(rng, lo, hi)) // q * q)


def draw(rng):
    kind = rng.choice(["pack", "linear", "linear", "gated", "gated", "ce", "ce", "ce"])
    f32 = rng.random() < 0.25
    case = {"kind": kind, "dtype": "f32" if f32 else "bf16"}
    if kind == "ce":
        while True:
            n, d = int(_log(rng, 1, 2048 if f32 else 16384)), _width(rng, 64, 2048 if f32 else 8192)
            v = int(_log(rng, 512, 32768 if f32 else 160000))
            if n * d * v <= LARGEST // (16 if f32 else 1) and v * d <= 1 << 29:
                break
        return {**case, "direction": rng.choice(["fwd", "step", "step"]), "n": n, "d": d, "v": v,
                "ignored": rng.choice([0.0, 0.0, 0.2, 0.5, 0.9])}
    case["format"] = rng.choice(["e4m3", "int8"])
    n = int(_log(rng, 1, 4096 if f32 else 32768))
    if kind == "linear":
        top = 2048 if f32 else 8192
        d_in, d_out = _width(rng, 64, top), _width(rng, 64, top)
        case |= {"direction": rng.choice(["step", "bwd"]), "n": n, "d_in": d_in, "d_out": d_out, "w_out_in": rng.random() < 0.6}
        if not f32 and rng.random() < 0.3:
            case["dw_dtype"] = "f32"
        return case
    width = _width(rng, 64, 8192)
    if kind == "gated":
        return {**case, "direction": rng.choice(["step", "bwd"]), "n": n, "f": width, "again": rng.random() < 0.4}
    return {**case, "n": n, "c": width, "ld": width * rng.choice([1, 1, 2])}


# ---- inputs --------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _activation(g, n, c, dt, scale=1.0, ld=None):
    """N(0, scale^2) with eight channels twenty times as large, as activations of trained models have them; rows `ld` apart."""
    x = torch.randn(n, c, generator=g, device=DEV) * scale
    x[:, torch.arange(8, device=DEV) * max(1, c // 8) % c] *= 20.0
    buf = torch.zeros(n, ld or c, dtype=dt, device=DEV)
    buf[:, :c] = x.to(dt)
    return buf[:, :c]


def _dense(g, rows, cols, dt, scale):
    return (torch.randn(rows, cols, generator=g, device=DEV) * scale).to(dt)


def _scale_of(largest, fmt):
    m, e = torch.frexp(largest)
    top, bits = (0.875, 9) if fmt == "e4m3" else (127 / 128, 7)
    return torch.where(largest > 0, e - bits + (m > top), -100).clamp_min(-100)


def _blocks(x):
    """[n, c] -> [blocks, 32, c], filled up with zeros."""
    n, c = x.shape
    return torch.nn.functional.pad(x, (0, 0, 0, -n % BLOCK)).reshape(-1, BLOCK, c)


def _pack(x, fmt):
    """The checkpoint of x [n, c]: its bytes [n, c] and a byte of exponent (e + 127) for every block and channel."""
    b = _blocks(x.float())
    fine = torch.isfinite(b)
    b = b.clamp(-TOP, TOP)
    e = _scale_of(torch.where(fine, b.abs(), 0.0).amax(1), fmt)
    y = torch.ldexp(b, -e.unsqueeze(1))
    if fmt == "e4m3":
        q = torch.where(fine, y, math.nan).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        q = torch.where(fine, y.round(), -128.0).to(torch.int8).view(torch.uint8)
    return q.reshape(-1, x.shape[1])[: x.shape[0]].contiguous(), (e + 127).to(torch.uint8)


def _unpack(q, e, fmt):
    """The values that a checkpoint stands for, in float32."""
    if fmt == "e4m3":
        y = q.view(torch.float8_e4m3fn).float()
    else:
        y = q.view(torch.int8).float()
        y = torch.where(y == -128.0, math.nan, y)
    y = torch.ldexp(_blocks(y), e.int().unsqueeze(1) - 127)
    return y.reshape(-1, q.shape[1])[: q.shape[0]]


def prepare(case, seed):
    g = _gen(seed)
    dt, s = TYPES[case["dtype"]], dict(case)
    if case["kind"] == "pack":
        s["x"] = _activation(g, case["n"], case["c"], dt, ld=case["ld"])
    elif case["kind"] == "linear":
        n, d_in, d_out = case["n"], case["d_in"], case["d_out"]
        s["x"] = _activation(g, n, d_in, dt)
        s["w"] = _dense(g, *((d_out, d_in) if case["w_out_in"] else (d_in, d_out)), dt, 0.02)
        s["dy"] = _dense(g, n, d_out, dt, 0.01)
        if case["direction"] == "bwd":
            s["q"], s["e"] = _pack(s.pop("x"), case["format"])
    elif case["kind"] == "gated":
        # gate and up are the two halves of one projection's rows
        both = _activation(g, case["n"], 2 * case["f"], dt, 1.6)
        s["gate"], s["up"] = both[:, : case["f"]], both[:, case["f"]:]
        s["dh"] = _dense(g, case["n"], case["f"], dt, 0.01)
        if case["direction"] == "bwd":
            s["q_gate"], s["e_gate"] = _pack(s.pop("gate"), case["format"])
            s["q_up"], s["e_up"] = _pack(s.pop("up"), case["format"])
    else:
        n, d, v = case["n"], case["d"], case["v"]
        s["x"] = _dense(g, n, d, dt, 1.0)
        s["w"] = _dense(g, v, d, dt, 1.3 / math.sqrt(d))   # logits of a spread of 1.3
        t = torch.randint(0, v, (n,), generator=g, device=DEV)
        s["targets"] = torch.where(torch.rand(n, generator=g, device=DEV) < case["ignored"], -100, t)
        # the gradient of the mean over the tokens that count
        s["dloss"] = torch.ones(n, device=DEV) / (s["targets"] >= 0).sum().clamp_min(1)
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------
def _plain_linear(s):
    dt, fmt = TYPES[s["dtype"]], s["format"]
    w = s["w"].float().t() if s["w_out_in"] else s["w"].float()   # [d_in, d_out]
    out = {}
    if s["direction"] == "step":
        out["y"] = (s["x"].float() @ w).to(dt)
        x = _unpack(*_pack(s["x"], fmt), fmt)
    else:
        x = _unpack(s["q"], s["e"], fmt)
    dy = s["dy"].float()
    out["dx"] = (dy @ w.t()).to(dt)
    out["dw"] = (dy.t() @ x if s["w_out_in"] else x.t() @ dy).to(TYPES[s.get("dw_dtype", s["dtype"])])
    return out


def _plain_gated(s):
    dt, fmt, out = TYPES[s["dtype"]], s["format"], {}
    if s["direction"] == "step":
        gate, up = s["gate"].float(), s["up"].float()
        out["h"] = (gate * torch.sigmoid(gate) * up).to(dt)
        gate, up = (_unpack(*_pack(t, fmt), fmt) for t in (s["gate"], s["up"]))
    else:
        gate, up = _unpack(s["q_gate"], s["e_gate"], fmt), _unpack(s["q_up"], s["e_up"], fmt)
    sg, dh = torch.sigmoid(gate), s["dh"].float()
    out["dgate"] = (dh * up * sg * (1 + gate * (1 - sg))).to(dt)
    out["dup"] = (dh * gate * sg).to(dt)
    if s.get("again"):
        out["h_again"] = (gate * sg * up).to(dt)
    return out


def _plain_ce(s):
    dt, x, w, t = TYPES[s["dtype"]], s["x"].float(), s["w"].float(), s["targets"]
    z = x @ w.t()
    lse, rows, counts = torch.logsumexp(z, 1), torch.arange(t.numel(), device=DEV), t >= 0
    out = {"loss": torch.where(counts, lse - z[rows, t.clamp_min(0)], 0.0)}
    if s["direction"] == "step":
        dz = z.sub_(lse.unsqueeze(1)).exp_()
        dz[rows, t.clamp_min(0)] -= 1.0
        dz *= torch.where(counts, s["dloss"], 0.0).unsqueeze(1)
        out["dx"], out["dw"] = (dz @ w).to(dt), (dz.t() @ x).to(dt)
    return out


# ---- the library's calls -------------------------------------------------------------------------------------
def _own_pack(acc, s):
    x = s["x"]
    desc = acc.make_act8_desc(s["n"], s["c"], ldx=s["ld"], io_dtype=_code(acc, s["dtype"]), format=_format(acc, s))
    q, e = acc.alloc_act8(desc, DEV)
    acc.acc_act8_pack(desc, x, q, e)
    back = torch.empty(s["n"], s["ld"], dtype=x.dtype, device=DEV)[:, : s["c"]]
    acc.acc_act8_unpack(desc, q, e, back)
    return {"x": back}


def _own_linear(acc, s):
    n, d_in, d_out, dt, code, fmt = s["n"], s["d_in"], s["d_out"], TYPES[s["dtype"]], _code(acc, s["dtype"]), _format(acc, s)
    dw_dtype = s.get("dw_dtype", s["dtype"])
    desc = acc.make_desc(n, d_in, d_out, 8, io_dtype=code, dw_dtype=_code(acc, dw_dtype), flags=acc.ACC_FLAG_W_OUT_IN if s["w_out_in"] else 0)
    out = {}
    if s["direction"] == "step":
        q, e = acc.alloc_act8(acc.make_act8_desc(n, d_in, io_dtype=code, format=fmt), DEV)
        out["y"] = torch.empty(n, d_out, dtype=dt, device=DEV)
        acc.acc_linear_fwd_act8(desc, fmt, s["x"], s["w"], out["y"], q, e)
    else:
        q, e = s["q"], s["e"]
    out["dx"] = torch.empty(n, d_in, dtype=dt, device=DEV)
    out["dw"] = torch.empty(s["w"].shape, dtype=TYPES[dw_dtype], device=DEV)
    ws = torch.empty(acc.acc_linear_act8_workspace_bytes(desc), dtype=torch.uint8, device=DEV)
    acc.acc_linear_bwd_act8(desc, fmt, s["dy"], s["w"], q, e, out["dx"], out["dw"], ws)
    return out


def _own_gated(acc, s):
    n, f, dt = s["n"], s["f"], TYPES[s["dtype"]]
    desc = acc.make_gated_desc(n, f, ldg=2 * f, io_dtype=_code(acc, s["dtype"]), format=_format(acc, s))
    out = {}
    if s["direction"] == "step":
        kept = acc.alloc_gated_act8(desc, DEV)
        out["h"] = torch.empty(n, f, dtype=dt, device=DEV)
        acc.acc_gated_fwd_act8(desc, s["gate"], s["up"], out["h"], *kept)
    else:
        kept = s["q_gate"], s["e_gate"], s["q_up"], s["e_up"]
    both = torch.empty(n, 2 * f, dtype=dt, device=DEV)
    out["dgate"], out["dup"] = both[:, :f], both[:, f:]
    if s.get("again"):
        out["h_again"] = torch.empty(n, f, dtype=dt, device=DEV)
    acc.acc_gated_bwd_act8(desc, s["dh"], *kept, out["dgate"], out["dup"], out.get("h_again"))
    return out


def _own_ce(acc, s):
    n, d, v, code = s["n"], s["d"], s["v"], _code(acc, s["dtype"])
    desc = acc.make_ce_desc(n, d, v, io_dtype=code, dw_dtype=code)
    loss, stats = torch.empty(n, device=DEV), torch.empty(2, n, device=DEV)
    ws = torch.empty(acc.acc_linear_ce_workspace_bytes(desc, s["direction"] == "step"), dtype=torch.uint8, device=DEV)
    acc.acc_linear_ce_fwd(desc, s["x"], s["w"], s["targets"], loss, stats, ws)
    out = {"loss": loss}
    if s["direction"] == "step":
        out["dx"], out["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
        acc.acc_linear_ce_bwd(desc, s["x"], s["w"], s["targets"], stats, s["dloss"], out["dx"], out["dw"], ws)
    return out


def _code(acc, name):
    return acc.ACC_BF16 if name == "bf16" else acc.ACC_F32


def _format(acc, s):
    return acc.ACC_ACT8_E4M3 if s["format"] == "e4m3" else acc.ACC_ACT8_INT8


def run(s):
    if own:
        from paper_2605_01255_amd import binding
        return {"pack": _own_pack, "linear": _own_linear, "gated": _own_gated, "ce": _own_ce}[s["kind"]](binding, s)
    if s["kind"] == "pack":
        return {"x": _unpack(*_pack(s["x"], s["format"]), s["format"]).to(s["x"].dtype)}
    return {"linear": _plain_linear, "gated": _plain_gated, "ce": _plain_ce}[s["kind"]](s)


# ---- what a pass cannot do without ---------------------------------------------------------------------------
def work(case):
    es, n = 2 if case["dtype"] == "bf16" else 4, case["n"]
    blocks = -(-n // BLOCK)
    if case["kind"] == "pack":
        c = case["c"]
        return {"bytes": 2 * n * c * es + 2 * (n + blocks) * c, "flops": 4 * n * c}
    if case["kind"] == "linear":
        d_in, d_out = case["d_in"], case["d_out"]
        dw = d_in * d_out * (4 if case.get("dw_dtype", case["dtype"]) == "f32" else 2)
        kept = (n + blocks) * d_in
        b = kept + n * d_out * es + d_in * d_out * es + n * d_in * es + dw
        if case["direction"] == "step":
            b += n * d_in * es + n * d_out * es + kept + d_in * d_out * es
        return {"bytes": b, "flops": 2 * n * d_in * d_out * (3 if case["direction"] == "step" else 2)}
    if case["kind"] == "gated":
        f = case["f"]
        kept = 2 * (n + blocks) * f
        b = kept + 3 * n * f * es + (n * f * es if case.get("again") else 0)
        if case["direction"] == "step":
            b += 3 * n * f * es + kept
        return {"bytes": b, "flops": (30 if case["direction"] == "step" else 20) * n * f}
    d, v = case["d"], case["v"]
    b = n * d * es + v * d * es + 8 * n + 4 * n
    flops = 2 * n * d * v
    if case["direction"] == "step":
        # backward: the inputs again, the gradients; the product that gives the logits back, and the gradients' two.  Tokens
        # without a loss have no part in them (their losses are 0 too, and need no logits).
        b += n * d * es + v * d * es + 8 * n + 4 * n + n * d * es + v * d * es
        flops = 8 * n * d * v
    return {"bytes": b, "flops": int(flops * (1 - case["ignored"]))}


# ---- 64 bits, from the definitions ---------------------------------------------------------------------------
def _exact_kept(x, fmt):
    """What a checkpoint of x gives back, in float64."""
    n, c = x.shape
    x = x.double()
    fine = torch.isfinite(x)
    x = torch.where(fine, x, torch.zeros_like(x)).clamp(-TOP, TOP)
    block = torch.arange(n, device=x.device) // BLOCK
    largest = torch.zeros(-(-n // BLOCK), c, dtype=x.dtype, device=x.device)
    largest = largest.scatter_reduce(0, block.unsqueeze(1).expand(n, c), x.abs(), "amax")
    top = 448.0 if fmt == "e4m3" else 127.0
    e = torch.ceil(torch.log2(largest.clamp_min(2.0 ** -200) / top))
    e = torch.where(largest > top * torch.exp2(e), e + 1, e)
    e = torch.where(largest <= top * torch.exp2(e - 1), e - 1, e).clamp_min(-100.0)
    scale = torch.exp2(e)[block]
    y = x / scale
    if fmt == "e4m3":
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))).clamp_min(-6.0) - 3.0)
        y = torch.round(y / step) * step
    else:
        y = torch.round(y)
    return torch.where(fine, y * scale, torch.full_like(y, math.nan))


def _exact_read(q, e, fmt):
    """The values of given checkpoint bytes, in float64, by a table of the 256 of them."""
    code = torch.arange(256, dtype=torch.float64, device=q.device)
    if fmt == "e4m3":
        low, exp = code % 128 % 8, torch.floor(code % 128 / 8)
        table = torch.where(exp == 0, low * 2.0 ** -9, (8 + low) * torch.exp2(exp - 10))
        table = torch.where(code % 128 == 127, torch.full_like(table, math.nan), table) * torch.where(code >= 128, -1.0, 1.0)
    else:
        table = torch.where(code >= 128, code - 256, code)
        table[128] = math.nan
    rows = torch.arange(q.shape[0], device=q.device) // BLOCK
    return table[q.long()] * torch.exp2(e.double() - 127)[rows]


def exact(case, seed):
    s = prepare(case, seed)
    fmt = case.get("format")
    if case["kind"] == "pack":
        return {"x": _exact_kept(s["x"], fmt)}
    if case["kind"] == "linear":
        w = s["w"].double().t() if case["w_out_in"] else s["w"].double()
        out = {"y": s["x"].double() @ w} if case["direction"] == "step" else {}
        x = _exact_kept(s["x"], fmt) if case["direction"] == "step" else _exact_read(s["q"], s["e"], fmt)
        dy = s["dy"].double()
        dw = x.t() @ dy
        return {**out, "dx": dy @ w.t(), "dw": dw.t() if case["w_out_in"] else dw}
    if case["kind"] == "gated":
        out = {}
        if case["direction"] == "step":
            gate, up = s["gate"].double(), s["up"].double()
            out["h"] = gate / (1 + torch.exp(-gate)) * up
            gate, up = _exact_kept(s["gate"], fmt), _exact_kept(s["up"], fmt)
        else:
            gate, up = _exact_read(s["q_gate"], s["e_gate"], fmt), _exact_read(s["q_up"], s["e_up"], fmt)
        dh, ex = s["dh"].double(), torch.exp(-gate)
        out["dgate"] = dh * up * ((1 + ex + gate * ex) / (1 + ex) ** 2)
        out["dup"] = dh * gate / (1 + ex)
        if case.get("again"):
            out["h_again"] = gate / (1 + ex) * up
        return out
    n, v = case["n"], case["v"]
    w, keep = s["w"].double(), s["targets"] >= 0
    loss, dx, dw = torch.zeros(n, dtype=torch.float64, device=DEV), torch.zeros(n, case["d"], dtype=torch.float64, device=DEV), torch.zeros_like(w)
    rows = torch.nonzero(keep).squeeze(1)
    for part in rows.split(2048):
        x, t = s["x"][part].double(), s["targets"][part]
        z = x @ w.t()
        z -= z.amax(1, keepdim=True)
        p = torch.exp(z)
        total = p.sum(1, keepdim=True)
        loss[part] = torch.log(total.squeeze(1)) - z.gather(1, t.unsqueeze(1)).squeeze(1)
        if case["direction"] == "step":
            dz = p.div_(total)
            dz.scatter_add_(1, t.unsqueeze(1), torch.full_like(dz[:, :1], -1.0))
            dz *= s["dloss"][part].double().unsqueeze(1)
            dx[part] = dz @ w
            dw += dz.t() @ x
    return {"loss": loss, "dx": dx, "dw": dw} if case["direction"] == "step" else {"loss": loss}
