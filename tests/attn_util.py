"""Attention over documents in float64 on the CPU, from its definition, with a bound for every element of what a kernel may give.

The bounds count roundings (half a step: 2^-8 of the value in bfloat16, 2^-24 in float):
  a score      d products summed in float, 2^-24 d sum |q||k|, three more factors, the cap's tanh to 2^-21 of the cap (its exponential
               and reciprocal to one step each, weighted by at most 1 / 2 and 2), the bias' product and difference
  P            twice the largest error of a row's scores (its own and the log-sum-exp's), the sum over the keys, the exponential
  O            P rounded as an operand (bfloat16), the result rounded: |O| + sum P |V|; the sum in float
  delta        dO . O with O as rounded: sum |dO| |error of O|; where no row sees more than 64 keys (bfloat16) sum P dP: P's and dP's errors
  dS           P (dP - delta): P's error, dP's sum over d, delta's error; rounded as an operand (bfloat16)
  dQ, dK, dV   the operands' errors through the product, its sum in float, the result rounded
"""
import math

import torch


class Case:
    """Inputs of one call: q, k and v as column blocks of one matrix, documents `cuts` (row numbers) or sequences of `seq` rows."""

    def __init__(self, n, heads, kv, d, dtype="bf16", cuts=None, seq=0, causal=True, window=0, cap=0.0, prefix=None, bias=False, scale=0.0, seed=0,
                 size=1.0):
        g = torch.Generator().manual_seed(seed * 1000 + n)
        self.n, self.heads, self.kv, self.d, self.dtype = n, heads, kv, d, dtype
        self.tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.cuts, self.seq, self.causal, self.window, self.cap = cuts, seq, causal, window, cap
        self.scale = scale
        self.qkv = (torch.randn(n, (heads + 2 * kv) * d, generator=g) * size).to(self.tdt)
        self.dO = torch.randn(n, heads * d, generator=g).to(self.tdt)
        self.starts = None if cuts is None else torch.tensor(cuts, dtype=torch.int64)
        self.prefix = None if prefix is None else torch.tensor(prefix, dtype=torch.int64)
        self.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]) if bias else None

    def documents(self):
        if self.cuts is not None:
            return list(zip(self.cuts, self.cuts[1:]))
        s = self.seq or self.n
        return [(a, min(a + s, self.n)) for a in range(0, self.n, s)]

    def seen(self):
        """[n, n]: whether query i sees key j."""
        out = torch.zeros(self.n, self.n, dtype=torch.bool)
        i = torch.arange(self.n)
        for e, (a, b) in enumerate(self.documents()):
            inside = (i >= a) & (i < b)
            m = torch.ones(self.n, self.n, dtype=torch.bool)
            if self.causal:
                m = i[:, None] >= i
                if self.window:
                    m = m & (i[:, None] - i < self.window)
                if self.prefix is not None:
                    m = m | (i < a + min(int(self.prefix[e]), b - a))
            out |= m & inside[:, None] & inside
        return out

    def split(self, t):
        return t.split((self.heads * self.d, self.kv * self.d, self.kv * self.d), 1)

    def exact(self):
        """{name: (value, bound)} for o, lse, dq, dk, dv."""
        n, d, group = self.n, self.d, self.heads // self.kv
        u, e = 2.0 ** -24, (2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24)
        operand = e if self.dtype == "bf16" else 0.0
        heads_of = lambda t, h: t.double().reshape(n, h, d).transpose(0, 1)  # noqa: E731
        q, k, v = (heads_of(t, h) for t, h in zip(self.split(self.qkv), (self.heads, self.kv, self.kv)))
        k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
        do = heads_of(self.dO, self.heads)
        scale = self.scale or 1.0 / math.sqrt(d)
        seen = self.seen()
        raw = scale * q @ k.transpose(1, 2)
        z_err = (d + 4) * u * scale * q.abs() @ k.abs().transpose(1, 2)
        z, slope = raw, torch.ones_like(raw)
        if self.cap:
            t = torch.tanh(raw / self.cap)
            z, slope = self.cap * t, 1 - t * t
            z_err = z_err + self.cap * 2.0 ** -21
        if self.slopes is not None:
            gap = (torch.arange(n)[:, None] - torch.arange(n)).abs().double()
            bias = self.slopes.double().view(-1, 1, 1) * gap
            z_err = z_err + 4 * u * bias
            z = z - bias
        z_err = z_err + 4 * u * z.abs()
        z = z.masked_fill(~seen, -math.inf)
        lse = torch.logsumexp(z, 2)
        empty = ~seen.any(1)
        p = torch.where(seen, torch.exp(z - lse.masked_fill(empty, 0.0).unsqueeze(2)), 0.0)
        most = torch.where(seen, z_err, 0.0).amax(2)
        sums = (n + 24) * u
        lse_err = most + sums + 4 * u * lse.masked_fill(empty, 0.0).abs()
        p_rel = (most + lse_err + sums).unsqueeze(2) * 1.1
        o = p @ v
        o_err = (p_rel + operand + sums) * (p @ v.abs()) + e * o.abs()
        dp = do @ v.transpose(1, 2)
        dp_err = (d + 4) * u * do.abs() @ v.abs().transpose(1, 2)
        delta = (do * o).sum(2, keepdim=True)
        delta_err = (do.abs() * o_err).sum(2, keepdim=True) + (d + 4) * u * (do * o).abs().sum(2, keepdim=True)
        longest = max([b - a for a, b in self.documents()], default=0)
        if self.dtype == "bf16" and min(longest, self.window or longest) <= 64:   # from P and dP, and not from O as rounded
            delta_err = (p * dp.abs() * (p_rel + 4 * u) + p * dp_err).sum(2, keepdim=True) + sums * (p * dp.abs()).sum(2, keepdim=True)
        ds = p * (dp - delta) * slope
        slope_err = 2.0 ** -20 if self.cap else 0.0
        ds_err = ds.abs() * (p_rel + operand + 8 * u) + p * slope * (dp_err + delta_err) + p * (dp - delta).abs() * slope_err
        back = lambda t: t.transpose(0, 1).reshape(n, -1)  # noqa: E731
        shared = lambda t: back(t.unflatten(0, (self.kv, group)).sum(1))  # noqa: E731
        dq, dk, dv = scale * ds @ k, scale * ds.transpose(1, 2) @ q, p.transpose(1, 2) @ do
        dq_err = scale * (ds_err + sums * ds.abs()) @ k.abs()
        dk_err = scale * (ds_err + sums * group * ds.abs()).transpose(1, 2) @ q.abs()
        dv_err = (p * (p_rel + operand + sums * group)).transpose(1, 2) @ do.abs()
        slack = 1e-30
        return {"o": (back(o), back(o_err) * 1.05 + slack), "lse": (lse, lse_err * 1.05 + slack),
                "dq": (back(dq), back(dq_err + (e + 4 * u) * dq.abs()) * 1.05 + slack),
                "dk": (shared(dk), (shared(dk_err) + (e + 4 * u) * shared(dk).abs()) * 1.05 + slack),
                "dv": (shared(dv), (shared(dv_err) + (e + 4 * u) * shared(dv).abs()) * 1.05 + slack)}

    # ---- the library's calls, on the GPU -----------------------------------------------------------------------
    def desc(self, acc):
        ld = (self.heads + 2 * self.kv) * self.d
        return acc.make_attn_desc(self.n, self.heads, self.kv, self.d, ldq=ld, ldk=ld, ldv=ld, docs=0 if self.cuts is None else len(self.cuts) - 1,
                                  seq=self.seq, window=self.window, scale=self.scale, cap=self.cap,
                                  io_dtype=acc.ACC_BF16 if self.dtype == "bf16" else acc.ACC_F32, flags=acc.ACC_ATTN_CAUSAL if self.causal else 0)

    def to_gpu(self):
        gpu = lambda t: None if t is None else t.cuda()  # noqa: E731
        return {name: gpu(getattr(self, name)) for name in ("qkv", "dO", "starts", "prefix", "slopes")}

    def outputs(self):
        """What the calls write, filled with NaN so that what stays unwritten is seen."""
        nan = lambda *s, dt=self.tdt: torch.full(s, math.nan, dtype=dt, device="cuda")  # noqa: E731
        return {"o": nan(self.n, self.heads * self.d), "lse": nan(self.heads, self.n, dt=torch.float32),
                "dqkv": nan(self.n, (self.heads + 2 * self.kv) * self.d)}

    def call(self, acc, t, out, ws=None, backward=True, stream=None):
        desc = self.desc(acc)
        if ws is None:
            ws = torch.empty(max(16, acc.acc_attn_workspace_bytes(desc, True)), dtype=torch.uint8, device="cuda").fill_(0xFF)
        masks = t["starts"], t["prefix"], t["slopes"]
        acc.acc_attn_fwd(desc, *self.split(t["qkv"]), *masks, out["o"], out["lse"], ws, stream=stream)
        if backward:
            acc.acc_attn_bwd(desc, *self.split(t["qkv"]), *masks, out["o"], out["lse"], t["dO"], *self.split(out["dqkv"]), ws, stream=stream)

    def run(self, acc, backward=True):
        t, out = self.to_gpu(), self.outputs()
        self.call(acc, t, out, backward=backward)
        torch.cuda.synchronize()
        return out

    def check(self, out, backward=True):
        want = self.exact()
        got = {"o": out["o"], "lse": out["lse"]}
        if backward:
            got["dq"], got["dk"], got["dv"] = self.split(out["dqkv"])
        for name, t in got.items():
            value, bound = want[name]
            t = t.cpu().double()
            infinite = torch.isinf(value)
            assert torch.equal(t[infinite], value[infinite]), name
            off = (t - value).abs()[~infinite]
            worst = (off / bound[~infinite]).max() if off.numel() else torch.tensor(0.0)
            assert bool(worst <= 1.0), (name, float(worst), float(off.max()))
