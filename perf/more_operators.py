"""The layer in 4-bit floating point, and what follows its ReduceScatter in training: dropout, residual, layer norm.

`listed()` and `draw()` give cases, `prepare()` a case's device data, `run()` one pass through an operator (in plain form,
or by the library's entry points where `own` is set), `work()` the bytes and operations that pass cannot do without,
`exact()` its outputs from the definition in 64 bits.

A case's "op" is one of
  quant_mxf4     rows to 4-bit floats with a power-of-two scale per 32 elements, and back to values
  gemm_mxf4      product of two such matrices
  gemm_mxf4_grouped  the same with a weight matrix per expert, rows sorted by expert
  layer_norm     of residual + dropout(x), the sum written too     (bwd: its gradients, the weight's reduced over the rows)
  dropout        from a counter-based generator, its mask not stored, a residual added    (bwd: its gradient)
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-5


def listed():
    return [
        # activations of eight sequences in a decoding step, to 4 bits and back (what a simulated 4-bit layer computes with)
        {"name": "quant_decode", "op": "quant_mxf4", "M": 8, "K": 4096, "pad": 0, "dtype": "bf16"},
        # gated activations of a long prompt before the MLP down-projection of one of eight ranks
        {"name": "quant_prompt", "op": "quant_mxf4", "M": 8192, "K": 3584, "pad": 0, "dtype": "bf16"},
        # one decoding step of sixteen sequences through that down-projection: bound by reading the weight
        {"name": "gemm_decode", "op": "gemm_mxf4", "M": 16, "N": 8192, "K": 3584, "dtype": "bf16", "bias": False},
        # the whole prompt through it: bound by the tensor cores
        {"name": "gemm_prompt", "op": "gemm_mxf4", "M": 8192, "N": 8192, "K": 3584, "dtype": "bf16", "bias": False},
        # 32 decoding tokens, eight of 64 experts each: a few rows per expert, bound by reading the experts' weights
        {"name": "grouped_decode", "op": "gemm_mxf4_grouped", "T": 32, "top": 8, "G": 64, "N": 4096, "K": 1024, "dtype": "bf16", "drop": 0.0},
        # a prompt of 4096 tokens, four of 32 experts each, some assignments over capacity and dropped
        {"name": "grouped_prompt", "op": "gemm_mxf4_grouped", "T": 4096, "top": 4, "G": 32, "N": 4096, "K": 1024, "dtype": "bf16", "drop": 0.05},
        # the norm behind an attention out-projection in a decoding step of eight sequences: residual, no dropout; latency
        {"name": "norm_decode", "op": "layer_norm", "M": 8, "K": 4096, "pad": 0, "dtype": "bf16", "wdtype": "bf16", "p": 0.0, "residual": True, "bwd": False},
        # the same in training: a rank's shard of the tokens, dropout of the reduced output, statistics kept
        {"name": "norm_train", "op": "layer_norm", "M": 8192, "K": 5120, "pad": 0, "dtype": "bf16", "wdtype": "fp32", "p": 0.1, "residual": True, "bwd": False},
        # its backward pass, with the gradient that comes down the residual stream
        {"name": "norm_train_bwd", "op": "layer_norm", "M": 8192, "K": 5120, "pad": 0, "dtype": "bf16", "wdtype": "fp32", "p": 0.1, "residual": True, "bwd": True},
        # a ragged shard of rows of an odd length in 32 bits, a plain layer norm's backward pass
        {"name": "norm_ragged_bwd", "op": "layer_norm", "M": 777, "K": 1021, "pad": 3, "dtype": "fp32", "wdtype": "fp32", "p": 0.0, "residual": False, "bwd": True},
        # dropout of a long batch's embeddings
        {"name": "dropout_train", "op": "dropout", "M": 16384, "K": 4096, "pad": 0, "dtype": "bf16", "p": 0.1, "residual": False, "bwd": False},
        # the gradient of a dropout in half precision, rows of an odd length
        {"name": "dropout_ragged_bwd", "op": "dropout", "M": 1001, "K": 2051, "pad": 5, "dtype": "fp16", "p": 0.3, "residual": False, "bwd": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quant_mxf4", "gemm_mxf4", "gemm_mxf4_grouped", "layer_norm", "layer_norm", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "quant_mxf4":
        while True:
            M, K = _log(rng, 1, 16384), _log(rng, 128, 32768)
            if M * K <= 8192 * 3584:
                break
        return {"op": op, "M": M, "K": K, "pad": rng.choice([0, 0, 8, 3]), "dtype": dtype}
    if op == "gemm_mxf4":
        while True:
            M, N, K = _log(rng, 1, 16384), _log(rng, 512, 16384), _log(rng, 256, 8192)
            if M * N * K <= 8192 * 8192 * 3584 and M * N <= 1 << 26:
                break
        return {"op": op, "M": M, "N": N, "K": K, "dtype": dtype, "bias": rng.random() < 0.3}
    if op == "gemm_mxf4_grouped":
        G = rng.choice([4, 8, 16, 32, 60, 64, 128])
        top = rng.randint(1, min(8, G))
        while True:
            T, N, K = _log(rng, 1, 16384), _log(rng, 512, 8192), _log(rng, 256, 4096)
            if T * top * N * K <= 4096 * 4 * 4096 * 1024 and G * N * K <= 1 << 28 and T * top * N <= 1 << 26:
                break
        return {"op": op, "T": T, "top": top, "G": G, "N": N, "K": K, "dtype": dtype, "drop": rng.choice([0.0, 0.05])}
    while True:
        M, K = _log(rng, 1, 32768), _log(rng, 64, 16384)
        if M * K * SIZE[dtype] <= 8192 * 5120 * 2:
            break
    c = {"op": op, "M": M, "K": K, "pad": rng.choice([0, 0, 0, 8, 3]), "dtype": dtype, "p": rng.choice([0.0, 0.1, 0.1, 0.5]), "bwd": rng.random() < 0.5}
    if op == "layer_norm":
        # dropout comes with the residual that it is added to
        c["residual"] = c["p"] > 0 or rng.random() < 0.5
        c["wdtype"] = rng.choice([dtype, "fp32"])
    else:
        c["p"] = rng.choice([0.05, 0.1, 0.3, 0.5])
        c["residual"] = not c["bwd"] and rng.random() < 0.5
    return c


def _padded(rows, cols, pitch, dtype):
    return torch.zeros(rows, pitch, dtype=dtype, device="cuda")[:, :cols]


def _up(n, m):
    return -(-n // m) * m


def _activations(gen, rows, cols):
    """Gated activations: silu(g) u, with a few channels that are much larger than the rest."""
    g = torch.randn(rows, cols, generator=gen, device="cuda")
    u = torch.randn(rows, cols, generator=gen, device="cuda")
    loud = 1 + 20 * (torch.rand(cols, generator=gen, device="cuda") < 0.004)
    return torch.nn.functional.silu(g) * u * loud


def _codes(rows, cols):
    """Places for codes (two per byte, rows on 16-byte boundaries) and scales (rows on 4-byte boundaries)."""
    return (_padded(rows, -(-cols // 2), _up(-(-cols // 2), 16), torch.uint8),
            _padded(rows, -(-cols // 32), _up(-(-cols // 32), 4), torch.uint8))


def _pow2(e):
    """2^e, put together from its bits: exact."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _mxf4_plain(x):
    """Codes and scale bytes of the rows of x.  64 bits: which side of the middle of two levels a value lies on."""
    M, K = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -K % 32)).view(M, -1, 32)
    amax = v.abs().amax(2, keepdim=True)
    fine = torch.isfinite(amax)
    e = torch.clamp(torch.frexp(torch.where(fine & (amax > 0), amax, 2.0**-130)).exponent - 3, -127, 127)
    a = torch.where(fine, v.abs(), 0.0) * _pow2(-e)
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte()
            + (a >= 3.5).byte() + (a > 5).byte())
    code = (code + 8 * (torch.signbit(v) & fine).byte()).view(M, -1)
    byte = torch.where(fine, e + 127, 255).to(torch.uint8)[:, :, 0]
    return (code[:, 0::2] + 16 * code[:, 1::2])[:, :-(-K // 2)], byte


def _values_plain(q, scale, K):
    """The fp32 values that codes and scales stand for (a product of 1.5 and 2^e at most: exact)."""
    level = torch.tensor([0.0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=q.device)
    code = torch.stack([q & 15, q >> 4], -1).flatten(-2)[..., :K]
    s = torch.where(scale == 255, math.nan, _pow2(scale.long() - 127).float())
    return level[code.int()] * s.repeat_interleave(32, -1)[..., :K]


def _quantised(gen, rows, cols, weight):
    """An operand of the product: activations, or a weight of normal values, quantised."""
    q, s = _codes(rows, cols)
    step = max(1, (1 << 25) // cols)
    for r in range(0, rows, step):
        n = min(step, rows - r)
        x = torch.randn(n, cols, generator=gen, device="cuda") / math.sqrt(cols) if weight else _activations(gen, n, cols)
        q[r:r + n], s[r:r + n] = _mxf4_plain(x)
    return q, s


def _matrix(gen, M, K, pad, dtype, spread=1.0, shift=0.0):
    x = _padded(M, K, K + pad, dtype)
    x.copy_(torch.randn(M, K, generator=gen, device="cuda") * spread + shift)
    return x


def prepare(case, seed):
    c, gen = case, torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": dict(case)}
    dtype = TYPES[c["dtype"]]
    if c["op"] == "quant_mxf4":
        M, K = c["M"], c["K"]
        s["x"], s["values"] = _padded(M, K, K + c["pad"], dtype), _padded(M, K, K + c["pad"], dtype)
        s["x"].copy_(_activations(gen, M, K))
        s["q"], s["scale"] = _codes(M, K)
    elif c["op"] == "gemm_mxf4":
        M, N, K = c["M"], c["N"], c["K"]
        s["a"], s["sa"] = _quantised(gen, M, K, False)
        s["b"], s["sb"] = _quantised(gen, N, K, True)
        s["bias"] = torch.randn(N, generator=gen, device="cuda") if c["bias"] else None
        s["out"] = torch.zeros(M, N, dtype=dtype, device="cuda")
    elif c["op"] == "gemm_mxf4_grouped":
        n, G, N, K = c["T"] * c["top"], c["G"], c["N"], c["K"]
        wish = torch.randn(c["T"], G, generator=gen, device="cuda") + torch.randn(G, generator=gen, device="cuda") * 0.5
        ids = wish.topk(c["top"], dim=1).indices.flatten()
        kept = torch.rand(n, generator=gen, device="cuda") >= c["drop"]
        count = torch.bincount(ids[kept], minlength=G)
        s["offsets"] = torch.cat([count.new_zeros(1), count.cumsum(0)]).int()
        s["most"] = max(1, int(count.max()))
        s["a"], s["sa"] = _quantised(gen, n, K, False)
        b, sb = _quantised(gen, G * N, K, True)
        s["b"], s["sb"] = b.unflatten(0, (G, N)), sb.unflatten(0, (G, N))
        s["out"] = torch.zeros(n, N, dtype=dtype, device="cuda")
    else:
        M, K, pad = c["M"], c["K"], c["pad"]
        s["rng"] = torch.tensor([seed * 0x9E3779B97F4A7C15 % (1 << 63), seed % 1000], dtype=torch.int64, device="cuda")
        s["row0"] = 4096  # a shard in the middle of the tokens
        if c["op"] == "dropout":
            s["x"] = _matrix(gen, M, K, pad, dtype)
            s["out"] = _padded(M, K, K + pad, dtype)
            s["residual"] = _matrix(gen, M, K, pad, dtype, 2.0) if c["residual"] else None
            return s
        wdtype = TYPES[c["wdtype"]]
        s["weight"] = (1 + 0.1 * torch.randn(K, generator=gen, device="cuda")).to(wdtype)
        s["bias"] = (0.1 * torch.randn(K, generator=gen, device="cuda")).to(wdtype)
        if c["bwd"]:
            s["h"] = _matrix(gen, M, K, pad, dtype, 2.0, 0.3)
            h = s["h"].double()
            s["mean"] = h.mean(1).float()
            s["rstd"] = torch.rsqrt(h.var(1, correction=0) + EPS).float()
            s["dout"] = _matrix(gen, M, K, pad, dtype)
            s["dx"] = _padded(M, K, K + pad, dtype)
            s["dhidden"] = _matrix(gen, M, K, pad, dtype) if c["residual"] else None
            s["dresidual"] = _padded(M, K, K + pad, dtype) if c["p"] > 0 else None
            s["dweight"], s["dbias"] = torch.zeros(K, device="cuda"), torch.zeros(K, device="cuda")
        else:
            s["x"] = _matrix(gen, M, K, pad, dtype)
            s["residual"] = _matrix(gen, M, K, pad, dtype, 2.0, 0.3) if c["residual"] else None
            s["hidden"] = _padded(M, K, K + pad, dtype) if c["residual"] else None
            s["out"] = _padded(M, K, K + pad, dtype)
            s["mean"], s["rstd"] = torch.zeros(M, device="cuda"), torch.zeros(M, device="cuda")
    return s


def _run_own(s):
    from paper_2609_11562_b200 import entwine as E

    c = s["case"]
    if c["op"] == "quant_mxf4":
        E.quant_mxf4(s["x"], s["q"], s["scale"])
        E.dequant_mxf4(s["q"], s["scale"], s["values"])
        return s["values"]
    if c["op"] == "gemm_mxf4":
        E.gemm_mxf4(s["a"], s["sa"], s["b"], s["sb"], s["out"], bias=s["bias"])
        return s["out"]
    if c["op"] == "gemm_mxf4_grouped":
        E.gemm_mxf4_grouped(s["a"], s["sa"], s["b"], s["sb"], s["offsets"], s["out"])
        return s["out"]
    if c["op"] == "dropout":
        if c["bwd"]:
            E.dropout_bwd(s["x"], s["out"], c["p"], s["rng"], row0=s["row0"])
        else:
            E.dropout(s["x"], s["out"], c["p"], s["rng"], row0=s["row0"], residual=s["residual"])
        return s["out"]
    if c["bwd"]:
        if "work" not in s:
            s["work"] = torch.empty(E.layer_norm_bwd_work(c["M"], c["K"]), device="cuda")
        E.layer_norm_bwd(s["dout"], s["h"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"], s["dbias"], s["work"],
                         dhidden=s["dhidden"], dresidual=s["dresidual"], p=c["p"], rng=s["rng"], row0=s["row0"])
        return {k: s[k] for k in ("dx", "dresidual", "dweight", "dbias") if s[k] is not None}
    E.layer_norm(s["x"], s["weight"], s["bias"], s["out"], eps=EPS, mean=s["mean"], rstd=s["rstd"], residual=s["residual"],
                 hidden=s["hidden"], p=c["p"], rng=s["rng"], row0=s["row0"])
    return {k: s[k] for k in ("out", "hidden", "mean", "rstd") if s[k] is not None}


def _kept(s, M, K, p):
    """What dropout multiplies each element with: 0, or 1 over the share that is kept.  Ten rounds of Philox4x32 (Salmon,
    Moraes, Dror, Shaw 2011) on 64-bit integers; the high half of a product is read from its bits, whatever its sign."""
    seed, offset = s["rng"][0], s["rng"][1]
    low = 0xFFFFFFFF
    k0, k1 = seed & low, (seed >> 32) & low
    dev = s["rng"].device
    x = torch.arange(-(-K // 8), device=dev).expand(M, -1)
    y = (s["row0"] + torch.arange(M, device=dev))[:, None].expand_as(x)
    z, w = (offset & low).expand_as(x), ((offset >> 32) & low).expand_as(x)
    for _ in range(10):
        a, b = x * 0xD2511F53, z * 0xCD9E8D57
        x, y, z, w = ((b >> 32) & low) ^ y ^ k0, b & low, ((a >> 32) & low) ^ w ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([x, y, z, w], -1)
    number = torch.stack([words & 0xFFFF, words >> 16], -1).reshape(M, -1)[:, :K]
    t = int(round(p * 65536))
    return torch.where(number >= t, 65536 / (65536 - t), 0.0)


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    dtype = TYPES[c["dtype"]]
    if c["op"] == "quant_mxf4":
        return _values_plain(*_mxf4_plain(s["x"]), c["K"]).to(dtype)
    if c["op"] == "gemm_mxf4":
        y = _values_plain(s["a"], s["sa"], c["K"]) @ _values_plain(s["b"], s["sb"], c["K"]).T
        return (y if s["bias"] is None else y + s["bias"]).to(dtype)
    if c["op"] == "gemm_mxf4_grouped":
        # each expert's rows in a block of the longest expert's length, one batched product, and back
        off, n = s["offsets"].long(), s["a"].shape[0]
        at = (off[:-1, None] + torch.arange(s["most"], device=off.device)).clamp(max=n - 1)
        y = torch.bmm(_values_plain(s["a"], s["sa"], c["K"])[at], _values_plain(s["b"], s["sb"], c["K"]).transpose(1, 2))
        r = torch.arange(n, device=off.device)
        g = (torch.searchsorted(off, r, right=True) - 1).clamp(max=c["G"] - 1)
        y = y[g, (r - off[g]).clamp(max=s["most"] - 1)]
        return torch.where((r < off[-1])[:, None], y, 0.0).to(dtype)
    M, K = c["M"], c["K"]
    if c["op"] == "dropout":
        y = s["x"].float() * _kept(s, M, K, c["p"])
        return (y if s["residual"] is None else y + s["residual"].float()).to(dtype)
    w = s["weight"].float()
    if c["bwd"]:
        dy, xh = s["dout"].float(), (s["h"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * w
        dh = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        if s["dhidden"] is not None:
            dh = dh + s["dhidden"].float()
        out = {"dx": (dh * _kept(s, M, K, c["p"]) if c["p"] > 0 else dh).to(dtype)}
        if s["dresidual"] is not None:
            out["dresidual"] = dh.to(dtype)
        # 64 bits: long sums
        return {**out, "dweight": (dy * xh).double().sum(0).float(), "dbias": dy.double().sum(0).float()}
    h = s["x"].float()
    if c["p"] > 0:
        h = h * _kept(s, M, K, c["p"])
    if s["residual"] is not None:
        h = h + s["residual"].float()
    hidden = h.to(dtype)
    h = hidden.float()  # what is normalised is what was written
    mean = h.mean(1)
    d = h - mean[:, None]
    rstd = torch.rsqrt((d * d).mean(1) + EPS)
    out = {"out": (d * rstd[:, None] * w + s["bias"].float()).to(dtype), "mean": mean, "rstd": rstd}
    return {**out, "hidden": hidden} if s["hidden"] is not None else out


def work(case):
    c = case
    size = SIZE[c["dtype"]]
    if c["op"] == "quant_mxf4":
        return {"bytes": c["M"] * c["K"] * (2 * size + 1) + c["M"] * c["K"] // 16, "flops": 4 * c["M"] * c["K"]}
    if c["op"] == "gemm_mxf4":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": (M + N) * K * 17 // 32 + M * N * size + 4 * N * c["bias"], "flops": 2 * M * N * K}
    if c["op"] == "gemm_mxf4_grouped":
        n, N, K = c["T"] * c["top"] * (1 - c["drop"]), c["N"], c["K"]
        # experts that get no row need not be read
        used = c["G"] * (1 - (1 - 1 / c["G"]) ** n)
        return {"bytes": int((n + used * N) * K * 17 / 32 + n * N * size), "flops": int(2 * n * N * K)}
    n = c["M"] * c["K"]
    if c["op"] == "dropout":
        return {"bytes": n * size * (3 if c["residual"] else 2), "flops": n * (3 if c["residual"] else 2)}
    if c["bwd"]:
        moved = 3 + (1 if c["residual"] else 0) + (1 if c["p"] > 0 else 0)
        return {"bytes": n * size * moved + 8 * c["M"] + c["K"] * (8 + SIZE[c["wdtype"]]), "flops": 14 * n}
    return {"bytes": n * size * (4 if c["residual"] else 2) + 8 * c["M"] + 2 * c["K"] * SIZE[c["wdtype"]], "flops": 9 * n}


def _decode64(q, scale, K):
    """Values from the fields of a code: (-1)^s m 2^(max(e, 1) - 2) with e its exponent, m = f/2 (+1 where e > 0)."""
    n = np.empty(q.shape[:-1] + (2 * q.shape[-1],), np.uint8)
    n[..., 0::2], n[..., 1::2] = q & 15, q >> 4
    n = n[..., :K]
    e, f = (n >> 1) & 3, n & 1
    v = np.ldexp(np.where(e > 0, 1.0, 0.0) + 0.5 * f, np.maximum(e, 1).astype(np.int32) - 1)
    v = np.where(n & 8, -v, v)
    return v * np.ldexp(1.0, np.repeat(scale, 32, axis=-1)[..., :K].astype(np.int32) - 127)


def _wide(q, scale, K):
    rows = [torch.from_numpy(_decode64(a.cpu().numpy(), b.cpu().numpy(), K)).cuda() for a, b in zip(q.split(4096), scale.split(4096))]
    return torch.cat(rows)


def _kept64(s, M, K, p):
    """The generator again, on unsigned 64-bit integers of the host."""
    seed, offset = (int(v) for v in s["rng"].tolist())
    u, low, half = np.uint64, np.uint64(0xFFFFFFFF), np.uint64(32)
    key = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    groups = -(-K // 8)
    ctr = [np.tile(np.arange(groups, dtype=u), M), np.repeat(np.arange(s["row0"], s["row0"] + M, dtype=u), groups),
           np.full(M * groups, offset & 0xFFFFFFFF, u), np.full(M * groups, (offset >> 32) & 0xFFFFFFFF, u)]
    for _ in range(10):
        p0, p1 = ctr[0] * u(0xD2511F53), ctr[2] * u(0xCD9E8D57)
        ctr = [(p1 >> half) ^ ctr[1] ^ u(key[0]), p1 & low, (p0 >> half) ^ ctr[3] ^ u(key[1]), p0 & low]
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    number = np.stack(ctr, 1).astype("<u4").view("<u2").reshape(M, -1)[:, :K]
    t = int(np.rint(p * 65536))
    return torch.from_numpy(np.where(number < t, 0.0, 65536.0 / (65536 - t))).cuda()


def exact(case, seed):
    s, c = prepare(case, seed), case
    f = torch.float64
    if c["op"] == "quant_mxf4":
        M, K = c["M"], c["K"]
        out = torch.empty(M, K, dtype=f, device="cuda")
        power = torch.from_numpy(np.ldexp(1.0, np.arange(-256, 257))).cuda()
        for k in range(0, K, 32):
            x = s["x"][:, k:k + 32].to(f)
            amax = x.abs().max(dim=1, keepdim=True).values
            # amax = m 2^n with m in [1/2, 1): the power of two below it is 2^(n-1)
            unit = power[256 + torch.clamp(torch.frexp(amax).exponent.long() - 3, -127, 127)]
            v = x / unit
            step = power[256 - 2 + torch.frexp(v.abs().clamp(min=1.0)).exponent.long()]
            out[:, k:k + 32] = (torch.round(v / step) * step).clamp(-6, 6) * unit
        return out
    if c["op"] == "gemm_mxf4":
        y = torch.mm(_wide(s["a"], s["sa"], c["K"]), _wide(s["b"], s["sb"], c["K"]).t())
        return y if s["bias"] is None else y + s["bias"].to(f)
    if c["op"] == "gemm_mxf4_grouped":
        out = torch.zeros(s["out"].shape, dtype=f, device="cuda")
        off = s["offsets"].tolist()
        for g in range(c["G"]):
            r = slice(off[g], off[g + 1])
            if off[g] < off[g + 1]:
                out[r] = torch.mm(_wide(s["a"][r], s["sa"][r], c["K"]), _wide(s["b"][g], s["sb"][g], c["K"]).t())
        return out
    M, K = c["M"], c["K"]
    kept = _kept64(s, M, K, c["p"]) if c["p"] > 0 else torch.ones(M, K, dtype=f, device="cuda")
    if c["op"] == "dropout":
        y = torch.mul(s["x"].to(f), kept)
        return y if s["residual"] is None else s["residual"].to(f) + y
    w = s["weight"].to(f)
    if c["bwd"]:
        dy, rstd = s["dout"].to(f), s["rstd"].to(f).unsqueeze(1)
        xh = (s["h"].to(f) - s["mean"].to(f).unsqueeze(1)) * rstd
        g = torch.mul(dy, w)
        dot = torch.linalg.vecdot(g, xh).unsqueeze(1) / K
        dh = (g - g.sum(1, keepdim=True) / K - dot * xh) * rstd
        if s["dhidden"] is not None:
            dh = dh + s["dhidden"].to(f)
        out = {"dx": kept * dh, "dweight": torch.einsum("mk,mk->k", dy, xh), "dbias": torch.einsum("mk->k", dy)}
        return {**out, "dresidual": dh} if s["dresidual"] is not None else out
    h = s["x"].to(f) * kept
    if s["residual"] is not None:
        h = s["residual"].to(f) + h
    h = h.to(TYPES[c["dtype"]]).to(f)
    mean = h.sum(1) / K
    rstd = 1 / torch.sqrt(h.var(1, correction=0) + EPS)
    out = {"out": (h - mean.unsqueeze(1)) * rstd.unsqueeze(1) * w + s["bias"].to(f), "mean": mean, "rstd": rstd}
    return {**out, "hidden": h} if s["hidden"] is not None else out
