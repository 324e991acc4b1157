"""More operators of a query encoder as cases that can be timed and compared: a gated encoder, trained by a larger one's
most probable labels and served in 8 bits.

A case is a dict of plain values.  ``op`` names the operator and ``way`` the direction:

  rms        root-mean-square norm of x + residual, its output in the inputs' type or in 8 bits   (forward | backward)
  q8         matrix product of operands in 8 bits with a scale for each 128 columns, its epilogue with bias, activation,
             gate and residual, its output in a wide type or in 8 bits again                       (forward)
  gated      act(x Wg^T + bg) (x Wu^T + bu), W the rows of Wg and then those of Wu                 (forward | backward)
  distill    divergence from a teacher's top labels over the whole vocabulary                      (forward | backward)

8 bits: codes are OCP e4m3, a scale is a power of two (a byte b stands for 2^(b - 127)), the least one under which the largest
finite value of its 128 columns is at most 448.  What a call leaves in 8 bits is returned as the values that it stands for.

Batch sizes, vocabularies and the encoder's width are those of the repository's workloads and of the query encoder beside it
(1 to 100,000 queries, 100 to 200,000 labels, width 1024, hidden 4096).
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
_BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}
_BLOCK = 128          # columns that share a scale


def listed():
    return [
        # one user's query between two layers: latency
        dict(op="rms", way="forward", name="norm, one query", dtype="bfloat16", m=1, d=1024, residual=True, quantize=True, pad=0),
        # the throughput batch between two layers, on its way into a product in 8 bits
        dict(op="rms", way="forward", name="norm, 10,000 queries", dtype="bfloat16", m=10_000, d=1024, residual=True, quantize=True, pad=0),
        # training on the largest batch: the weight's gradient over all of its rows, the residual path's gradient added
        dict(op="rms", way="backward", name="norm backward", dtype="bfloat16", m=100_000, d=1024, residual=True, quantize=False, pad=0),
        # one query through the widest layer: one read of the weights, half as many bytes as in bfloat16
        dict(op="q8", way="forward", name="8 bits, one query", dtype="bfloat16", m=1, k=1024, n=4096, act="gelu", gated=False, bias=True,
             residual=False, quantize=False, pad=0),
        # the throughput batch back to the encoder's width, added to what it branched off from
        dict(op="q8", way="forward", name="8 bits, 10,000 queries", dtype="bfloat16", m=10_000, k=4096, n=1024, act="none", gated=False,
             bias=True, residual=True, quantize=False, pad=0),
        # full precision outside of the product, nothing a multiple of anything, rows cut out of a wider table
        dict(op="q8", way="forward", name="8 bits, odd sizes", dtype="float32", m=1777, k=777, n=333, act="silu", gated=False, bias=True,
             residual=True, quantize=False, pad=5),
        # the throughput batch through the gated layer that the product above follows, 8 bits in and out
        dict(op="q8", way="forward", name="gated in 8 bits", dtype="bfloat16", m=10_000, k=1024, n=4096, act="silu", gated=True, bias=False,
             residual=False, quantize=True, pad=0),
        # one query through the gated layer: one read of both projections
        dict(op="gated", way="forward", name="gated, one query", dtype="bfloat16", m=1, k=1024, n=4096, act="silu", bias=True, save=False, pad=0),
        # the throughput batch, pre-activations kept for training
        dict(op="gated", way="forward", name="gated, 10,000 queries", dtype="bfloat16", m=10_000, k=1024, n=4096, act="silu", bias=True, save=True, pad=0),
        # the same layer's gradients in training
        dict(op="gated", way="backward", name="gated backward", dtype="bfloat16", m=10_000, k=1024, n=4096, act="silu", bias=True, save=True, pad=0),
        # a small batch against the largest vocabulary's teacher
        dict(op="distill", way="forward", name="distillation, 200,000 labels", dtype="bfloat16", m=64, v=200_000, top=64, masked=0.1, t=2.0, pad=0),
        # the throughput batch's gradient over 10,000 labels
        dict(op="distill", way="backward", name="distillation gradient", dtype="bfloat16", m=10_000, v=10_000, top=32, masked=0.1, t=2.0, pad=0),
    ]


def _size(rng, lo, hi, step=16):
    """A length between lo and hi, spread over its logarithm: odd ones and multiples alike."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v - v % step if rng.random() < 0.5 and v > step else v


def draw(rng):
    op = rng.choice(["rms", "rms", "q8", "q8", "q8", "gated", "gated", "distill", "distill"])
    dtype = rng.choice(["float32", "bfloat16", "bfloat16", "float16"])
    pad = rng.choice([0, 0, 0, 8, 5])
    if op == "rms":
        d, way = _size(rng, 16, 8192), rng.choice(["forward", "forward", "backward"])
        return dict(op=op, way=way, dtype=dtype, m=_size(rng, 1, min(100_000, 50_000_000 // d)), d=d, residual=rng.random() < 0.7,
                    quantize=way == "forward" and rng.random() < 0.5, pad=pad)
    if op == "distill":
        v = _size(rng, 100, 200_000)
        m = _size(rng, 1, max(2, min(20_000, 50_000_000 // v)))
        return dict(op=op, way=rng.choice(["forward", "backward"]), dtype=dtype, m=m, v=v, top=rng.choice([1, 8, 32, 64, 200]),
                    masked=rng.choice([0.0, 0.1, 0.9]), t=rng.choice([1.0, 2.0, 4.0]), pad=pad)
    k, n, act = _size(rng, 16, 4096), _size(rng, 16, 4096), rng.choice(["none", "relu", "gelu", "silu"])
    most = 10_000 * 1024 * 4096 // (k * n) // (8 if dtype == "float32" else 1)
    m = _size(rng, 1, max(2, min(20_000, most)))
    if op == "q8":
        return dict(op=op, way="forward", dtype=dtype, m=m, k=k, n=n, act=act, gated=rng.random() < 0.5, bias=rng.random() < 0.7,
                    residual=rng.random() < 0.4, quantize=rng.random() < 0.4, pad=pad)
    return dict(op=op, way=rng.choice(["forward", "forward", "backward"]), dtype=dtype, m=m, k=k, n=n, act=act, bias=rng.random() < 0.7,
                save=rng.random() < 0.5, pad=pad)


# ------------------------------------------------------------------ work


def _held_bytes(m, d):
    """Of m rows of d values in 8 bits."""
    return m * d + m * -(-d // _BLOCK)


def work(case):
    s, m = _BYTES[case["dtype"]], case["m"]
    if case["op"] == "rms":
        d = case["d"]
        if case["way"] == "backward":     # dy, the sum, the residual path's gradient; dx; the weight and its gradient
            return dict(bytes=m * d * s * (3 + case["residual"]) + 2 * d * s + 4 * m, flops=12 * m * d)
        out = 2 * m * d if case["quantize"] else m * d * s
        return dict(bytes=m * d * s * (1 + 2 * case["residual"]) + out + d * s + 4 * m, flops=6 * m * d)
    if case["op"] == "distill":
        v, top = case["v"], case["top"]
        return dict(bytes=m * v * s * (1 if case["way"] == "forward" else 2) + 8 * m * top + 12 * m, flops=(4 if case["way"] == "forward" else 6) * m * v)
    k, n = case["k"], case["n"]
    if case["op"] == "q8":
        rows = n * (1 + case["gated"])
        out = 2 * m * n if case["quantize"] else m * n * s
        return dict(bytes=_held_bytes(m, k) + _held_bytes(rows, k) + rows * s * case["bias"] + m * n * s * case["residual"] + out, flops=2 * m * rows * k)
    if case["way"] == "forward":
        return dict(bytes=(m * k + 2 * n * k + m * n * (1 + 2 * case["save"]) + 2 * n * case["bias"]) * s, flops=4 * m * n * k)
    return dict(bytes=(2 * m * k + 4 * n * k + 3 * m * n + 2 * n * case["bias"]) * s, flops=8 * m * n * k)


# ------------------------------------------------------------------ inputs


def _cut(x, pad):
    """The same values as rows of a wider table, where pad > 0."""
    if not pad:
        return x
    wide = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _codes(v):
    """(codes, scales) of float32 rows: e4m3 with the columns filled up to whole blocks with zeros, and a byte per block in rows of
    whole 32-bit words."""
    v = torch.nn.functional.pad(v, (0, -v.shape[1] % _BLOCK)).unflatten(1, (-1, _BLOCK))
    most = torch.where(torch.isfinite(v), v.abs(), torch.zeros_like(v)).amax(2)
    part, power = torch.frexp(most)
    power = torch.where(most > 0, (power - 9 + (part > 0.875).int()).clamp_min(-127), torch.zeros_like(power))
    codes = (v * torch.exp2(-power.float())[:, :, None]).to(torch.float8_e4m3fn).flatten(1)
    scales = (power + 127).to(torch.uint8)
    return codes, torch.nn.functional.pad(scales, (0, -scales.shape[1] % 4))


def _values(codes, scales):
    """What they stand for, in float32."""
    c = codes.float().unflatten(1, (-1, _BLOCK))
    return (c * torch.exp2(scales[:, :c.shape[1]].float() - 127)[:, :, None]).flatten(1)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    T, m, pad = _TYPES[case["dtype"]], case["m"], case["pad"]

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(std).add_(mean)

    def activations(m, d):
        """Some columns are far larger than the others."""
        x = normal(m, d)
        x[:, torch.randint(0, d, (1 + d // 200,), generator=g, device="cuda")] *= 12.0
        return x

    s = dict(case=case)
    if case["op"] == "rms":
        d = case["d"]
        s["x"] = _cut(activations(m, d).to(T), pad)
        s["r"] = _cut(normal(m, d, std=2.0).to(T), pad) if case["residual"] else None
        s["g"] = normal(d, std=0.2, mean=1.0).to(T)
        if case["way"] == "backward":
            s["rstd"] = (s["x"].float().square().mean(1) + 1e-6).rsqrt()
            s["dy"] = _cut(normal(m, d, std=0.1).to(T), pad)
    elif case["op"] == "distill":
        v, top = case["v"], case["top"]
        x = normal(m, v, std=2.0)
        teacher = normal(m, v).add_(x)
        if case["masked"]:
            gone = torch.rand((m, v), generator=g, device="cuda") < case["masked"]
            if m > 8:
                gone[m // 3] = True              # nothing is left of this row
            x[gone] = -math.inf
            teacher[gone] = -math.inf
        s["x"] = _cut(x.to(T), pad)
        val, ids = teacher.topk(min(top, v), dim=1)
        fill = (0, top - val.shape[1])
        s["val"] = torch.nn.functional.pad(val, fill, value=-math.inf).contiguous()
        s["ids"] = torch.nn.functional.pad(ids.int().masked_fill(val == -math.inf, -1), fill, value=-1).contiguous()
        if case["way"] == "backward":
            s["lse"] = torch.logsumexp(s["x"].float() / case["t"], 1)
            s["dl"] = normal(m)
    else:
        k, n = case["k"], case["n"]
        rows = n * (2 if case["op"] == "gated" or case["gated"] else 1)
        x, w = activations(m, k), normal(rows, k, std=k ** -0.5)
        s["b"] = normal(rows, std=0.1).to(T) if case["bias"] else None
        if case["op"] == "q8":
            s["x"], s["w"] = _codes(x), _codes(w)
            if pad:
                s["x"] = (_cut(s["x"][0], 16), s["x"][1])
            s["r"] = _cut(normal(m, n).to(T), pad) if case["residual"] else None
        else:
            s["x"], s["w"] = _cut(x.to(T), pad), w.to(T)
            if case["way"] == "backward":
                s["z"] = normal(m, 2 * n).to(T)
                s["dy"] = _cut(normal(m, n, std=0.1).to(T), pad)
    return s


# ------------------------------------------------------------------ one pass


def run(s):
    if own:
        return _own(s)
    case = s["case"]
    return {"rms": _plain_rms, "q8": _plain_q8, "gated": _plain_gated, "distill": _plain_distill}[case["op"]](s, case)


def _own(s):
    from paper_2506_00812_amd import binding as vf
    case = s["case"]
    op, forward = case["op"], case["way"] == "forward"
    if op == "rms":
        if not forward:
            return vf.rms_norm_backward(s["dy"], s["x"], s["rstd"], s["g"], d_total=s["r"])
        y, *more = vf.rms_norm(s["x"], s["g"], residual=s["r"], eps=1e-6, save=True, quantize=case["quantize"])
        return (vf.dequantize(y, torch.bfloat16) if case["quantize"] else y, *more)
    if op == "q8":
        y = vf.linear_q8(vf.Q8(*s["x"], case["k"]), vf.Q8(*s["w"], case["k"]), s["b"], residual=s["r"], activation=case["act"],
                         gated=case["gated"], dtype=_TYPES[case["dtype"]], quantize=case["quantize"])
        return vf.dequantize(y, torch.bfloat16) if case["quantize"] else y
    if op == "gated":
        if forward:
            return vf.gated_linear(s["x"], s["w"], s["b"], activation=case["act"], save=case["save"])
        return vf.gated_linear_backward(s["dy"], s["x"], s["w"], s["z"], activation=case["act"], bias=case["bias"])
    if forward:
        return vf.distill(s["x"], s["ids"], s["val"], temperature=case["t"])
    return vf.distill_backward(s["x"], s["lse"], s["ids"], s["val"], s["dl"], temperature=case["t"])


def _rounded(y, case):
    """The output as it is kept: in the case's type, or as the values of its 8 bits (which bfloat16 holds exactly)."""
    if case["quantize"]:
        return _values(*_codes(y))[:, :y.shape[1]].to(torch.bfloat16)
    return y.to(_TYPES[case["dtype"]])


def _plain_rms(s, case):
    T = _TYPES[case["dtype"]]
    x, g = s["x"].float(), s["g"].float()
    if case["way"] == "forward":
        if s["r"] is not None:
            total = (x + s["r"].float()).to(T)
            x = total.float()
        rstd = (x.square().mean(1) + 1e-6).rsqrt()
        y = _rounded(x * rstd[:, None] * g, case)
        return (y, rstd) if s["r"] is None else (y, total, rstd)
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    h, dg = x * rstd, dy * g
    dx = rstd * (dg - h * (dg * h).mean(1, keepdim=True))
    if s["r"] is not None:
        dx = dx + s["r"].float()
    return dx.to(T), (dy * h).sum(0).to(T)


def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        a = 1 / (1 + torch.exp(-z))
        return a * (1 + z * (1 - a))
    return torch.ones_like(z)


def _plain_q8(s, case):
    z = _values(*s["x"]) @ _values(*s["w"]).t()
    if s["b"] is not None:
        z = z + s["b"].float()
    if case["gated"]:
        gate, up = z.chunk(2, 1)
        y = _act(gate, case["act"]) * up
    else:
        y = _act(z, case["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return _rounded(y, case)


def _plain_gated(s, case):
    T = _TYPES[case["dtype"]]
    x, w = s["x"].float(), s["w"].float()
    if case["way"] == "forward":
        z = x @ w.t()
        if s["b"] is not None:
            z = z + s["b"].float()
        gate, up = z.chunk(2, 1)
        y = (_act(gate, case["act"]) * up).to(T)
        return (y, z.to(T)) if case["save"] else y
    dy = s["dy"].float()
    gate, up = s["z"].float().chunk(2, 1)
    dz = torch.cat([dy * up * _slope(gate, case["act"]), dy * _act(gate, case["act"])], 1)
    return (dz @ w).to(T), (dz.t() @ x).to(T), dz.sum(0).to(T) if case["bias"] else None


def _teacher(s, case):
    """(entries, q, log q): which of the teacher's entries count, their probabilities among themselves and the logarithms of these."""
    there = (s["ids"] >= 0) & (s["val"] > -math.inf)
    u = torch.where(there, s["val"] / case["t"], torch.full_like(s["val"], -math.inf))
    most = u.amax(1, keepdim=True)
    u = u - torch.where(most > -math.inf, most, torch.zeros_like(most))
    e = u.exp()
    total = e.sum(1, keepdim=True)
    total = torch.where(total > 0, total, torch.ones_like(total))
    return there, e / total, u - total.log()


def _plain_distill(s, case):
    x = s["x"].float() / case["t"]
    there, q, log_q = _teacher(s, case)
    at = s["ids"].clamp_min(0).long()
    if case["way"] == "forward":
        most = x.amax(1)
        most = torch.where(most > -math.inf, most, torch.zeros_like(most))
        lse = most + (x - most[:, None]).exp().sum(1).log()
        terms = q * (log_q - (x.gather(1, at) - lse[:, None]))
        return torch.where(q > 0, terms, torch.zeros_like(terms)).sum(1), lse
    lse = s["lse"][:, None]
    p = torch.where(lse > -math.inf, (x - lse).exp(), torch.zeros_like(x))
    p = torch.where(there.any(1, keepdim=True), p, torch.zeros_like(p))
    p.scatter_add_(1, at, torch.where(there & (lse > -math.inf), -q, torch.zeros_like(q)))
    return (p * (s["dl"] / case["t"])[:, None]).to(s["x"].dtype)


# ------------------------------------------------------------------ the definitions in 64 bits


def _wide(held):
    codes, scales = held
    at = torch.arange(codes.shape[1], device=codes.device) // _BLOCK
    return codes.to(torch.float64) * 2.0 ** (scales.to(torch.float64)[:, at] - 127)


def _in_8_bits(y):
    """The values that 8 bits keep of y."""
    m, d = y.shape
    at = torch.arange(d, device=y.device) // _BLOCK
    most = torch.zeros((m, int(at[-1]) + 1), dtype=y.dtype, device=y.device)
    most.scatter_reduce_(1, at.expand(m, d), y.abs(), "amax")
    unit = torch.where(most > 0, 2.0 ** torch.ceil(torch.log2(most.clamp_min(1e-300) / 448)), torch.ones_like(most)).clamp_min(2.0 ** -127)[:, at]
    u = y / unit
    step = 2.0 ** (torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(u / step) * step * unit


def _bend(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "silu":
        return z * torch.special.expit(z)
    return z


def exact(case, seed):
    s = prepare(case, seed)
    D = torch.float64
    T = _TYPES[case["dtype"]]
    if case["op"] == "rms":
        x, g, d = s["x"].to(D), s["g"].to(D), case["d"]
        if case["way"] == "forward":
            total = x if s["r"] is None else (x + s["r"].to(D)).to(T).to(D)
            rstd = 1 / torch.sqrt(torch.linalg.vecdot(total, total) / d + 1e-6)
            y = total * (rstd[:, None] * g)
            y = _in_8_bits(y) if case["quantize"] else y
            return (y, rstd) if s["r"] is None else (y, total, rstd)
        dy, rstd = s["dy"].to(D), s["rstd"].to(D)
        along = torch.linalg.vecdot(dy * g, x) / d
        dx = rstd[:, None] * dy * g - x * (rstd ** 3 * along)[:, None]
        return dx if s["r"] is None else dx + s["r"].to(D), torch.mv((dy * x).t(), rstd)
    if case["op"] == "distill":
        t, ids, v = case["t"], s["ids"].long(), case["v"]
        x = s["x"].to(D) / t
        rows = torch.arange(len(x), device=x.device)[:, None]
        u = (s["val"].to(D) / t).masked_fill(ids < 0, -math.inf)
        none = torch.isneginf(u).all(1)
        q = torch.softmax(u.masked_fill(none[:, None], 0.0), 1).masked_fill(none[:, None], 0.0)
        if case["way"] == "forward":
            lse = torch.logsumexp(x, 1)
            cross = (q * (x[rows, ids.clamp_min(0)] - lse[:, None])).masked_fill(q == 0, 0.0)
            return torch.special.xlogy(q, q).sum(1) - cross.sum(1), lse
        dx = torch.exp(x - s["lse"].to(D)[:, None])
        dx.index_put_((rows.expand_as(ids), ids.clamp_min(0)), -q, accumulate=True)
        dx.masked_fill_((none | torch.isneginf(s["lse"]))[:, None], 0.0)
        return dx * (s["dl"].to(D) / t)[:, None]
    n = case["n"]
    if case["op"] == "q8":
        z = torch.mm(_wide(s["x"]), _wide(s["w"]).t())
    elif case["way"] == "forward":
        z = torch.mm(s["x"].to(D), s["w"].to(D).t())
    if case["way"] == "forward":
        if s["b"] is not None:
            z += s["b"].to(D)
        y = _bend(z[:, :n], case["act"]) * z[:, n:] if z.shape[1] > n else _bend(z, case["act"])
        if case["op"] == "q8":
            y = y if s["r"] is None else y + s["r"].to(D)
            return _in_8_bits(y) if case["quantize"] else y
        return (y, z) if case["save"] else y
    dy, gate, up = s["dy"].to(D), s["z"][:, :n].to(D), s["z"][:, n:].to(D)
    if case["act"] == "none":
        slope = torch.ones_like(gate)
    elif case["act"] == "relu":
        slope = torch.heaviside(gate, torch.zeros_like(gate))
    elif case["act"] == "gelu":
        slope = torch.special.ndtr(gate) + gate * torch.exp(-gate * gate / 2) / math.sqrt(2 * math.pi)
    else:
        a = torch.special.expit(gate)
        slope = a + gate * a * torch.special.expit(-gate)
    a, b = dy * up * slope, dy * _bend(gate, case["act"])
    w, x = s["w"].to(D), s["x"].to(D)
    dx = torch.mm(a, w[:n]) + torch.mm(b, w[n:])
    dw = torch.cat([torch.mm(a.t().contiguous(), x), torch.mm(b.t().contiguous(), x)])
    return dx, dw, torch.cat([a.sum(0), b.sum(0)]) if case["bias"] else None
