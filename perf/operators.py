"""Timed cases of the microscaled operators: what workers send at a synchronization, in 4 or 8 bits.

A row is one worker's difference from the model all workers share.  Blocks of 32 elements share a
power of two (one byte, 2^(byte - 127)); an element is an E2M1 (4 bits, two to a byte, the even one
in the low half) or an E4M3 (8 bits) number.  Kinds of passes:

    send     mx_quantize, then mx_dequantize of what was sent: the message's values and the new residual
    read     mx_dequantize of received rows on top of the shared model: every worker's parameters
    sync     mx_average: the new model, broadcast to every row, and the variance of every tensor
    product  mx_product: the K x K inner products of the workers' rows for every tensor

Sizes follow the framework's workloads (65K to 138M parameters, 4 to 32 workers, 1 to 400 tensors) and
the odd shapes of its tests.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 32
# format: (bits of an element, exponent of the largest power of two, largest value's fraction bits in
# an fp32 mantissa, least exponent, fraction bits)
_FORMATS = {"e2m1": (4, 2, 0x400000, 0, 1), "e4m3": (8, 8, 0x600000, -6, 3)}
_DEFAULT = dict(kind="send", format="e2m1", K=8, P=65536, T=1, lo=64, seed_sizes=1002, fixed="", pad=True,
                base=True, residual=True, two=False)


def _case(name=None, **kw):
    c = dict(_DEFAULT, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    vgg = dict(K=8, P=138_000_000, T=32, seed_sizes=1004, fixed="102000000,16800000,4100000")
    return [
        # the smallest workload's message, without error feedback: launches count
        _case("send_k4_p65k", K=4, P=65_536, residual=False),
        # five workers, ragged tensors in packed rows that are not 16-byte aligned
        _case("send_k5_p1m_packed", K=5, P=1_000_003, T=19, lo=3, pad=False),
        # a ResNet50-sized vector in 8 bits, 16 workers, error feedback
        _case("send_k16_p26m_e4m3", K=16, P=25_600_000, T=161, seed_sizes=1003, format="e4m3"),
        # the 138M-parameter vector (VGG16-sized), error feedback: the bandwidth-bound message
        _case("send_k8_p138m", **vgg),
        # one worker's 8-bit message of 1001 parameters, read back: the smallest call
        _case("read_k1_p1001_e4m3", kind="read", K=1, P=1001, format="e4m3", base=False),
        # a ResNet18-sized vector: every worker's parameters from what it sent
        _case("read_k8_p11m", kind="read", K=8, P=11_200_000, T=62),
        # the smallest workload's sync
        _case("sync_k4_p65k", kind="sync", K=4, P=65_536),
        # 400 small tensors, 32 workers, 8 bits
        _case("sync_k32_p1m2_t400_e4m3", kind="sync", K=32, P=1_200_000, T=400, lo=16, seed_sizes=1005, format="e4m3"),
        # the bandwidth-bound sync
        _case("sync_k8_p138m_t32", kind="sync", **vgg),
        # how alike the workers' messages are, per tensor: 400 small tensors, against the messages of the sync before
        _case("product_k32_p1m2_t400", kind="product", K=32, P=1_200_000, T=400, lo=16, seed_sizes=1005, two=True),
        # the same of one sync's messages among themselves, 8 bits, 16 workers
        _case("product_k16_p26m_t161_e4m3", kind="product", K=16, P=25_600_000, T=161, seed_sizes=1003, format="e4m3"),
        # the 138M-parameter vector
        _case("product_k8_p138m_t32", kind="product", **vgg),
    ]


_MOST_ELEMENTS = 8 * 138_000_000     # K P of the largest listed case


def draw(rng):
    kind = rng.choice(["send", "send", "read", "sync", "sync", "product", "product"])
    K = rng.choice([2, 4, 8, 16, 32]) if rng.random() < 0.6 else rng.randint(1, 100)
    most_p = min(138e6, _MOST_ELEMENTS / (2 * K))
    P = int(math.exp(rng.uniform(math.log(33), math.log(most_p))))
    T = int(math.exp(rng.uniform(0, math.log(min(400, max(2, P // 8))))))
    return _case(kind=kind, format=rng.choice(["e2m1", "e2m1", "e4m3"]), K=K, P=P, T=T, lo=rng.randint(1, 64),
                 seed_sizes=rng.randint(1, 100_000), pad=rng.random() < 0.7, base=rng.random() < 0.8,
                 residual=rng.random() < 0.8, two=rng.random() < 0.4)


def _sizes(c):
    """Tensor sizes: the fixed ones, then log-uniform shares of the rest."""
    fixed = [int(v) for v in c["fixed"].split(",")] if c["fixed"] else []
    n, rest = c["T"] - len(fixed), c["P"] - sum(fixed)
    s = np.exp(np.random.default_rng(c["seed_sizes"]).uniform(math.log(c["lo"]), math.log(2.4e6), n))
    ends = np.floor(np.cumsum(s) * (rest / s.sum())).astype(np.int64)
    ends[-1] = rest
    return fixed + [int(v) for v in np.diff(ends, prepend=0)]


def _stride(n):
    """The least odd number of 256s that holds n."""
    q = -(-n // 256)
    return 256 * (q + 1 - q % 2)


def _rows(K, P, pad):
    ld = _stride(P) if pad else P
    return torch.zeros((K, ld), device="cuda")[:, :P]


def _pad_blocks(v):
    K, P = v.shape
    return torch.nn.functional.pad(v, (0, -P % BLOCK)).view(K, -1, BLOCK)


def _encode(d, fmt):
    """(values before the scale, scale bytes) of blocks d [..., 32]: round to nearest, ties to even."""
    _, emax, most, emin, frac = _FORMATS[fmt]
    bits = d.abs().amax(-1).view(torch.int32)
    e, man = bits >> 23, bits & 0x7FFFFF
    byte = torch.where(e == 255, 255, (e - emax + (man > most)).clamp(min=0))
    v = d * ((254 - byte.clamp(max=253)) << 23).view(torch.float32)[..., None]
    ve = ((v.view(torch.int32) >> 23) & 255) - 127
    step = ((ve.clamp(min=emin) - frac + 127) << 23).view(torch.float32)
    return torch.round(v / step) * step, byte.to(torch.uint8)


def _scale(byte):
    """2^(byte - 127) in fp32 (byte 0 is a subnormal number, 255 is NaN)."""
    b = byte.to(torch.int32)
    s = torch.where(b == 0, torch.full_like(b, 0x400000), b << 23).view(torch.float32)
    return torch.where(b == 255, torch.full_like(s, math.nan), s)


def _tables():
    v4 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    v4 = torch.tensor(v4 + [-v for v in v4], device="cuda")
    i = torch.arange(256, device="cuda")
    lut4 = torch.stack([v4[i & 15], v4[i >> 4]], -1)
    lut8 = torch.arange(256, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).float()[:, None]
    return {"e2m1": lut4, "e4m3": lut8}


def _pack(v, fmt):
    """Codes of values before the scale, as bytes of a row."""
    if fmt == "e4m3":
        return v.to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2)
    a = v.abs()
    i = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a * 0.5 + 4)).to(torch.uint8)
    i = (i | (v < 0).to(torch.uint8) * 8).flatten(-2)
    return i[..., 0::2] | (i[..., 1::2] << 4)


def _received(c, deltas):
    """Rows as they arrive: codes and scale bytes, each row's at a stride of an odd number of 256 bytes."""
    fmt, K, P = c["format"], c["K"], c["P"]
    n = -(-P // BLOCK)
    codes = torch.zeros((K, _stride(n * BLOCK * _FORMATS[fmt][0] // 8)), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((K, _stride(n)), dtype=torch.uint8, device="cuda")
    for k in range(K if deltas is not None else 0):
        v, byte = _encode(_pad_blocks(deltas[k:k + 1]), fmt)
        b = _pack(v, fmt)
        codes[k, :b.shape[1]] = b[0]
        scales[k, :n] = byte[0]
    return codes, scales


def _deltas(c, sizes, gen):
    """What the workers' local steps leave: a common drift and each worker's noise, of another size in
    every tensor; every fifteenth tensor of several is frozen and does not move at all."""
    K, P = c["K"], c["P"]
    d = _rows(K, P, c["pad"])
    d.copy_(torch.randn((K, P), generator=gen, device="cuda"))
    d.add_(torch.randn((P,), generator=gen, device="cuda"), alpha=0.5)
    rng = np.random.default_rng(c["seed_sizes"])
    amp = 10.0 ** rng.uniform(-4, -1, len(sizes))
    amp[14::15] = 0.0
    d.mul_(torch.repeat_interleave(torch.tensor(amp, device="cuda", dtype=torch.float32),
                                   torch.tensor(sizes, device="cuda"), output_size=P))
    return d


def prepare(case, seed):
    c, sizes = case, _sizes(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    K, P, fmt = c["K"], c["P"], c["format"]
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    st = {"c": c, "sizes": sizes, "offsets": torch.from_numpy(off).cuda(), "base": None, "lut": _tables()[fmt]}
    if c["base"]:
        st["base"] = torch.randn((P,), generator=gen, device="cuda")
    d = _deltas(c, sizes, gen)
    if c["kind"] == "send":
        # x: the replicas; residual: what the last message left out, up to half of a step
        st["residual"] = None
        st["residual_out"] = _rows(K, P, c["pad"])
        if c["residual"]:
            st["residual"] = _rows(K, P, c["pad"])
            st["residual"].copy_(d).mul_(torch.rand((K, P), generator=gen, device="cuda").sub_(0.5).mul_(0.2))
        if c["base"]:
            d.add_(st["base"])
        st["x"] = d
        st["codes"], st["scales"] = _received(c, None)
        st["values"] = _rows(K, P, c["pad"])
        return st
    st["codes"], st["scales"] = _received(c, d)
    if c["kind"] == "product" and c["two"]:
        st["codes2"], st["scales2"] = _received(c, _deltas(c, sizes, gen))
    if c["kind"] == "read":
        st["values"] = _rows(K, P, c["pad"])
    if c["kind"] == "sync":
        st["x"], st["base_out"] = _rows(K, P, c["pad"]), torch.zeros((P,), device="cuda")
    return st


def _decode(st, codes, scales):
    c = st["c"]
    n = -(-c["P"] // BLOCK)
    v = st["lut"][codes[:, :n * BLOCK * _FORMATS[c["format"]][0] // 8].long()]
    v = v.view(c["K"], n, BLOCK) * _scale(scales[:, :n])[..., None]
    return v.view(c["K"], -1)[:, :c["P"]]


def _inner(a, b):
    """a b^T of [K, n] rows: the long side in runs, whose products are summed."""
    K, n = a.shape
    whole = n - n % 4096
    out = a[:, whole:] @ b[:, whole:].t().contiguous()
    if whole:
        a, b = a[:, :whole].reshape(K, -1, 4096), b[:, :whole].reshape(K, -1, 4096)
        out += torch.bmm(a.transpose(0, 1).contiguous(), b.permute(1, 2, 0).contiguous()).sum(0)
    return out


def _run_plain(st):
    c = st["c"]
    if c["kind"] == "send":
        d = st["x"] if st["base"] is None else st["x"] - st["base"]
        d = d if st["residual"] is None else d + st["residual"]
        v, byte = _encode(_pad_blocks(d), c["format"])
        v = (v * _scale(byte)[..., None]).view(c["K"], -1)[:, :c["P"]]
        return {"values": v, "residual": torch.where(v.isnan(), 0.0, d - v)}
    v = _decode(st, st["codes"], st["scales"])
    if c["kind"] == "read":
        return {"values": v if st["base"] is None else st["base"] + v}
    if c["kind"] == "sync":
        mean = v.sum(0, dtype=torch.float64) / c["K"]
        dev = (v - mean).square_().sum(0) / c["K"]
        var = torch.stack([t.sum() for t in torch.split(dev, st["sizes"])])
        base = (mean if st["base"] is None else st["base"] + mean).float()
        return {"x": base.expand(c["K"], -1).contiguous(), "base": base, "var": var}
    w = _decode(st, st["codes2"], st["scales2"]) if c["two"] else v
    pairs = zip(torch.split(v, st["sizes"], 1), torch.split(w, st["sizes"], 1))
    return {"product": torch.stack([_inner(a.double(), b.double()) for a, b in pairs]).float()}


def _run_own(st):
    import paper_2007_06134_amd as A
    c = st["c"]
    fmt = A.MX_E2M1 if c["format"] == "e2m1" else A.MX_E4M3
    rows = A.MxRows(st["codes"], st["scales"], c["P"], fmt)
    if c["kind"] == "send":
        A.mx_quantize(st["x"], st["base"], st["residual"], residual_out=st["residual_out"], out=rows)
        return {"values": A.mx_dequantize(rows, out=st["values"]), "residual": st["residual_out"]}
    if c["kind"] == "read":
        return {"values": A.mx_dequantize(rows, st["base"], out=st["values"])}
    if c["kind"] == "sync":
        base, var = A.mx_average(rows, st["offsets"], st["base"], x=st["x"], base_out=st["base_out"])
        return {"x": st["x"], "base": base, "var": var}
    other = A.MxRows(st["codes2"], st["scales2"], c["P"], fmt) if c["two"] else None
    return {"product": A.mx_product(rows, st["offsets"], other)}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    c = case
    K, P, n = c["K"], c["P"], c["K"] * c["P"]
    base = 4 * P if c["base"] else 0
    row = n * (_FORMATS[c["format"]][0] / 8 + 1 / BLOCK)
    if c["kind"] == "send":      # x, base and the residual in; the message, its values and the residual out
        return {"bytes": int(4 * n + base + (4 * n if c["residual"] else 0) + row + 8 * n), "flops": 8 * n}
    if c["kind"] == "read":
        return {"bytes": int(row + base + 4 * n), "flops": 2 * n}
    if c["kind"] == "sync":
        return {"bytes": int(row + base + 4 * n + 4 * P + 8 * c["T"]), "flops": 5 * n}
    rows = 2 * row if c["two"] else row
    return {"bytes": int(rows + 4 * c["T"] * K * K), "flops": 2 * n * K}


# ---- the definition in 64 bits, apart from the plain form above -----------------------------------

def _grid(fmt):
    """The non-negative numbers of a format, ascending: sum of fraction bits times powers of two."""
    _, _, _, emin, frac = _FORMATS[fmt]
    top = 2 if fmt == "e2m1" else 8
    g = [m * 2.0 ** (emin - frac) for m in range(2 ** frac)]
    g += [(1 + m / 2 ** frac) * 2.0 ** e for e in range(emin, top + 1) for m in range(2 ** frac)]
    return g if fmt == "e2m1" else g[:-1]     # (E4M3's last code is NaN)


def _two(e):
    """2^e in 64 bits, from its exponent field (pow is not exact)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_rows(codes, scales, P, fmt):
    g = torch.tensor(_grid(fmt), device="cuda", dtype=torch.float64)
    n, b = -(-P // BLOCK), codes.long()
    if fmt == "e2m1":
        b = torch.stack([b % 16, b // 16], -1).flatten(-2)
    half = 8 if fmt == "e2m1" else 128
    v = g[(b % half).clamp(max=len(g) - 1)]
    v[(b % half) >= len(g)] = math.nan
    v = torch.where(b >= half, -v, v)[..., :n * BLOCK]
    s = _two(scales[..., :n].long() - 127)
    s[scales[..., :n] == 255] = math.nan
    return (v.view(*v.shape[:-1], n, BLOCK) * s[..., None]).flatten(-2)[..., :P]


def _exact_round(d, fmt):
    """The message's values of one row d (64 bits): the nearest of the scaled grid, ties to the even code."""
    g = torch.tensor(_grid(fmt), device="cuda", dtype=torch.float64)
    blocks = torch.nn.functional.pad(d, (0, -len(d) % BLOCK)).view(-1, BLOCK)
    most = blocks.abs().amax(1)
    e = torch.ceil(torch.log2((most / g[-1]).clamp(min=2.0 ** -140)))
    e += (most > g[-1] * _two(e)).double()          # log2 beside a power of two
    e -= (most <= g[-1] * _two(e - 1)).double()
    s = _two(e.clamp(min=-127))[:, None]
    a = blocks.abs() / s
    i = torch.searchsorted(g, a.clamp(max=float(g[-1]))).clamp(min=1)
    lo, hi = g[i - 1], g[i]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (i % 2 == 0))
    return (torch.where(up, hi, lo) * torch.sign(blocks) * s).flatten()[:len(d)]


def exact(case, seed):
    c = case
    if c["K"] * c["P"] > 5e8:
        return None
    st = prepare(case, seed)
    fmt, P = c["format"], c["P"]
    if c["kind"] == "send":
        # the difference that is sent is an fp32 number by definition: each sum rounded to fp32
        values, left = [], []
        for k in range(c["K"]):
            d = st["x"][k].double()
            if st["base"] is not None:
                d = (d - st["base"].double()).float().double()
            if st["residual"] is not None:
                d = (d + st["residual"][k].double()).float().double()
            values.append(_exact_round(d, fmt))
            left.append(d - values[-1])
        return {"values": torch.stack(values), "residual": torch.stack(left)}
    v = torch.stack([_exact_rows(st["codes"][k], st["scales"][k], P, fmt) for k in range(c["K"])])
    base = st["base"].double() if st["base"] is not None else torch.zeros((P,), device="cuda", dtype=torch.float64)
    if c["kind"] == "read":
        return {"values": base + v}
    ends = np.cumsum(st["sizes"])
    spans = [slice(int(e - n), int(e)) for e, n in zip(ends, st["sizes"])]
    if c["kind"] == "sync":
        mean = v.mean(0)
        new = base + mean
        var = [float((v[:, s] - mean[s]).square().sum()) / c["K"] for s in spans]
        return {"x": new.expand(c["K"], -1).contiguous(), "base": new,
                "var": torch.tensor(var, dtype=torch.float64)}
    w = torch.stack([_exact_rows(st["codes2"][k], st["scales2"][k], P, fmt) for k in range(c["K"])]) if c["two"] else v
    out = torch.zeros((len(spans), c["K"], c["K"]), dtype=torch.float64, device="cuda")
    for t, s in enumerate(spans):
        for j in range(c["K"]):
            out[t, j] = (w[:, s] * v[j, s]).sum(1)
    return {"product": out}
