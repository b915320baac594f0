"""The quantised and the expert form of the row-parallel layer, in plain form and by the library's entry points.

`listed()` and `draw()` give cases, `prepare()` a case's device data, `run()` one pass through an operator,
`work()` the bytes and operations that pass cannot do without, `exact()` its outputs from the definition in 64 bits.

A case's "op" is one of
  quant_i8       rows to int8 with a scale each
  gemm_i8        int8 product with token and channel scales
  gemm_i8_grouped  the same with a weight matrix per expert, rows sorted by expert
  moe_dispatch   tokens sorted by expert          (bwd: its gradient)
  moe_combine    back with weights applied        (bwd: its gradients)
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "int8": torch.int8}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4, "int8": 1}


def listed():
    return [
        # activations of eight sequences in a decoding step, before the int8 product of an attention out-projection
        {"name": "quant_decode", "op": "quant_i8", "M": 8, "K": 4096, "pitch": 4096, "dtype": "bf16"},
        # gated activations of a long prompt before the MLP down-projection of one of eight ranks
        {"name": "quant_prompt", "op": "quant_i8", "M": 8192, "K": 3584, "pitch": 3584, "dtype": "bf16"},
        # one decoding step of sixteen sequences through that down-projection: bound by reading the weight
        {"name": "gemm_decode", "op": "gemm_i8", "M": 16, "N": 8192, "K": 3584, "pitch": 3584, "dtype": "bf16", "bias": False},
        # the whole prompt through it: bound by the tensor cores
        {"name": "gemm_prompt", "op": "gemm_i8", "M": 8192, "N": 8192, "K": 3584, "pitch": 3584, "dtype": "bf16", "bias": False},
        # a ragged batch of tokens, an odd reduction length in padded rows, a bias and half-precision outputs
        {"name": "gemm_ragged", "op": "gemm_i8", "M": 777, "N": 5120, "K": 1021, "pitch": 1024, "dtype": "fp16", "bias": True},
        # 32 decoding tokens, eight of 64 experts each: a few rows per expert, bound by reading the experts' weights
        {"name": "grouped_decode", "op": "gemm_i8_grouped", "T": 32, "top": 8, "G": 64, "N": 4096, "K": 1024, "pitch": 1024, "dtype": "bf16", "drop": 0.0},
        # a prompt of 4096 tokens, four of 32 experts each, some assignments over capacity and dropped
        {"name": "grouped_prompt", "op": "gemm_i8_grouped", "T": 4096, "top": 4, "G": 32, "N": 4096, "K": 1024, "pitch": 1024, "dtype": "bf16", "drop": 0.05},
        # 16 decoding tokens to eight of 64 experts each: latency
        {"name": "dispatch_decode", "op": "moe_dispatch", "T": 16, "H": 4096, "top": 8, "G": 64, "dtype": "bf16", "ids": "int64", "drop": 0.0, "bwd": False},
        # a long batch of quantised rows to eight of 128 experts each, scales travelling along
        {"name": "dispatch_prompt", "op": "moe_dispatch", "T": 16384, "H": 4096, "top": 8, "G": 128, "dtype": "int8", "ids": "int32", "drop": 0.02, "bwd": False},
        # the gradient of the dispatch in a training step
        {"name": "dispatch_train", "op": "moe_dispatch", "T": 8192, "H": 5120, "top": 4, "G": 32, "dtype": "bf16", "ids": "int64", "drop": 0.02, "bwd": True},
        # the weighted return of a few decoding tokens, one expert having dropped some
        {"name": "combine_decode", "op": "moe_combine", "T": 16, "H": 4096, "top": 8, "G": 64, "dtype": "bf16", "ids": "int32", "drop": 0.1, "bwd": False},
        # both gradients of the weighted return in a training step
        {"name": "combine_train", "op": "moe_combine", "T": 8192, "H": 5120, "top": 4, "G": 32, "dtype": "bf16", "ids": "int32", "drop": 0.02, "bwd": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quant_i8", "gemm_i8", "gemm_i8_grouped", "moe_dispatch", "moe_combine"])
    if op == "quant_i8":
        while True:
            M, K = _log(rng, 1, 16384), _log(rng, 256, 32768)
            if M * K <= 1 << 26:
                break
        return {"op": op, "M": M, "K": K, "pitch": -(-K // 16) * 16 + 16 * rng.randrange(2), "dtype": rng.choice(["bf16", "fp16", "fp32"])}
    if op == "gemm_i8":
        while True:
            M, N, K = _log(rng, 1, 16384), _log(rng, 512, 16384), _log(rng, 256, 8192)
            if M * N * K <= 8192 * 8192 * 3584:
                break
        return {"op": op, "M": M, "N": N, "K": K, "pitch": -(-K // 16) * 16 + 16 * rng.randrange(2), "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                "bias": rng.random() < 0.3}
    G = rng.choice([4, 8, 16, 32, 60, 64, 128])
    top = rng.randint(1, min(8, G))
    if op == "gemm_i8_grouped":
        while True:
            T, N, K = _log(rng, 1, 16384), _log(rng, 512, 8192), _log(rng, 256, 4096)
            if T * top * N * K <= 4096 * 4 * 4096 * 4096 and G * N * K <= 1 << 29 and T * top * N <= 1 << 28:
                break
        return {"op": op, "T": T, "top": top, "G": G, "N": N, "K": K, "pitch": -(-K // 16) * 16,
                "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "drop": rng.choice([0.0, 0.05])}
    bwd = rng.random() < 0.5
    while True:
        T, H = _log(rng, 1, 32768), _log(rng, 256, 8192)
        if T * top * H <= 8192 * 4 * 5120:
            break
    types = ["bf16", "bf16", "fp16", "fp32"] + (["int8"] if op == "moe_dispatch" and not bwd else [])
    return {"op": op, "T": T, "H": H, "top": top, "G": G, "dtype": rng.choice(types), "ids": rng.choice(["int32", "int64"]), "drop": rng.choice([0.0, 0.02, 0.3]), "bwd": bwd}


def _padded(rows, cols, pitch, dtype):
    return torch.zeros(rows, pitch, dtype=dtype, device="cuda")[:, :cols]


def _activations(gen, rows, cols):
    """Gated activations: silu(g) u, with a few channels that are much larger than the rest."""
    g = torch.randn(rows, cols, generator=gen, device="cuda")
    u = torch.randn(rows, cols, generator=gen, device="cuda")
    loud = 1 + 20 * (torch.rand(cols, generator=gen, device="cuda") < 0.004)
    return torch.nn.functional.silu(g) * u * loud


def _levels(gen, rows, cols, pitch):
    """An int8 operand with the spread of a quantised normal row, in rows of `pitch` elements."""
    out = _padded(rows, cols, pitch, torch.int8)
    step = max(1, (1 << 27) // cols)
    for r in range(0, rows, step):
        n = min(step, rows - r)
        out[r:r + n] = (torch.randn(n, cols, generator=gen, device="cuda") * 32).round_().clamp_(-127, 127).to(torch.int8)
    return out


def _routing(gen, T, top, G, drop, dtype):
    """The `top` best of G experts for each token, some experts more wanted than others; a share dropped."""
    wish = torch.randn(T, G, generator=gen, device="cuda") + torch.randn(G, generator=gen, device="cuda") * 0.5
    best = wish.topk(top, dim=1)
    ids = best.indices
    if drop:
        ids = torch.where(torch.rand(T, top, generator=gen, device="cuda") < drop, -1, ids)
    return ids.to(dtype), torch.softmax(best.values, dim=1)


def _places(ids, G):
    """Stable order by expert: (offsets [G+1], row of each assignment or -1, flat assignments in row order)."""
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < G), flat, G)
    sorted_key, order = torch.sort(key, stable=True)
    offsets = torch.searchsorted(sorted_key, torch.arange(G + 1, device=ids.device))
    row = torch.empty_like(order)
    row[order] = torch.arange(order.numel(), device=ids.device)
    return offsets.int(), torch.where(key < G, row, -1).int().view(ids.shape), order


def prepare(case, seed):
    c, gen = case, torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": dict(case)}
    dtype = TYPES[c["dtype"]]
    if c["op"] == "quant_i8":
        s["x"] = _padded(c["M"], c["K"], c["pitch"], dtype)
        s["x"].copy_(_activations(gen, c["M"], c["K"]))
        s["q"] = _padded(c["M"], c["K"], c["pitch"], torch.int8)
        s["scale"] = torch.zeros(c["M"], device="cuda")
    elif c["op"] == "gemm_i8":
        M, N, K = c["M"], c["N"], c["K"]
        s["a"], s["b"] = _levels(gen, M, K, c["pitch"]), _levels(gen, N, K, c["pitch"])
        s["sa"] = torch.rand(M, generator=gen, device="cuda") * 0.05 + 0.005
        s["sb"] = (torch.rand(N, generator=gen, device="cuda") + 0.5) / (32 * math.sqrt(K))
        s["bias"] = torch.randn(N, generator=gen, device="cuda") if c["bias"] else None
        s["out"] = torch.zeros(M, N, dtype=dtype, device="cuda")
    elif c["op"] == "gemm_i8_grouped":
        n, G, N, K = c["T"] * c["top"], c["G"], c["N"], c["K"]
        ids, _ = _routing(gen, c["T"], c["top"], G, c["drop"], torch.int64)
        s["offsets"], _, _ = _places(ids, G)
        s["most"] = int(s["offsets"].diff().max())
        s["a"], s["b"] = _levels(gen, n, K, c["pitch"]), _levels(gen, G * N, K, c["pitch"]).unflatten(0, (G, N))
        s["sa"] = torch.rand(n, generator=gen, device="cuda") * 0.05 + 0.005
        s["sb"] = (torch.rand(G, N, generator=gen, device="cuda") + 0.5) / (32 * math.sqrt(K))
        s["out"] = torch.zeros(n, N, dtype=dtype, device="cuda")
    else:
        T, H, top, G = c["T"], c["H"], c["top"], c["G"]
        s["ids"], s["w"] = _routing(gen, T, top, G, c["drop"], torch.int32 if c["ids"] == "int32" else torch.int64)
        offsets, row_of, _ = _places(s["ids"], G)
        if c["op"] == "moe_dispatch" and not c["bwd"]:
            if c["dtype"] == "int8":
                s["x"] = _levels(gen, T, H, H)
                s["x_scale"] = torch.rand(T, generator=gen, device="cuda") * 0.05 + 0.005
                s["row_scale"] = torch.zeros(T * top, device="cuda")
            else:
                s["x"] = torch.randn(T, H, generator=gen, device="cuda").to(dtype)
            s["rows"] = torch.zeros(T * top, H, dtype=dtype, device="cuda")
            s["offsets"] = torch.zeros(G + 1, dtype=torch.int32, device="cuda")
            s["row_of"] = torch.zeros(T, top, dtype=torch.int32, device="cuda")
        else:
            s["row_of"] = row_of
            s["y"] = torch.randn(T * top, H, generator=gen, device="cuda").to(dtype)
            s["out"] = torch.zeros(T, H, dtype=dtype, device="cuda")
            if c["op"] == "moe_combine" and c["bwd"]:
                s["dout"] = torch.randn(T, H, generator=gen, device="cuda").to(dtype)
                s["dy"] = torch.zeros(T * top, H, dtype=dtype, device="cuda")
                s["dw"] = torch.zeros(T, top, device="cuda")
    return s


def _run_own(s):
    from paper_2609_11562_b200 import entwine as E

    c = s["case"]
    if c["op"] == "quant_i8":
        E.quant_i8(s["x"], s["q"], s["scale"])
        return {"q": s["q"], "scale": s["scale"]}
    if c["op"] == "gemm_i8":
        E.gemm_i8(s["a"], s["sa"], s["b"], s["sb"], s["out"], bias=s["bias"])
        return s["out"]
    if c["op"] == "gemm_i8_grouped":
        E.gemm_i8_grouped(s["a"], s["sa"], s["b"], s["sb"], s["offsets"], s["out"])
        return s["out"]
    if c["op"] == "moe_dispatch" and c["bwd"]:
        E.moe_dispatch_bwd(s["y"], s["row_of"], s["out"])
        return s["out"]
    if c["op"] == "moe_dispatch":
        E.moe_dispatch(s["x"], s["ids"], c["G"], s["rows"], s["offsets"], s["row_of"],
                       x_scale=s.get("x_scale"), row_scale=s.get("row_scale"))
        return {k: s[k] for k in ("rows", "row_scale", "offsets", "row_of") if k in s}
    if c["bwd"]:
        E.moe_combine_bwd(s["dout"], s["y"], s["w"], s["row_of"], s["dy"], s["dw"])
        return {"dy": s["dy"], "dw": s["dw"]}
    E.moe_combine(s["y"], s["w"], s["row_of"], s["out"])
    return s["out"]


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    dtype = TYPES[c["dtype"]]
    if c["op"] == "quant_i8":
        # 64 bits: which side of a half a quotient lies on
        x = s["x"].double()
        amax = x.abs().amax(1, keepdim=True)
        q = torch.round(x * 127 / torch.where(amax > 0, amax, 1.0))
        return {"q": q.to(torch.int8), "scale": (amax[:, 0] / 127).float()}
    if c["op"] == "gemm_i8":
        y = (s["a"].float() @ s["b"].float().T) * s["sa"][:, None] * s["sb"]
        return (y if s["bias"] is None else y + s["bias"]).to(dtype)
    if c["op"] == "gemm_i8_grouped":
        # each expert's rows in a block of the longest expert's length, one batched product, and back
        off, n = s["offsets"].long(), s["a"].shape[0]
        at = (off[:-1, None] + torch.arange(s["most"], device=off.device)).clamp(max=n - 1)
        y = torch.bmm(s["a"][at].float(), s["b"].float().transpose(1, 2)) * s["sa"][at][:, :, None] * s["sb"][:, None, :]
        r = torch.arange(n, device=off.device)
        g = (torch.searchsorted(off, r, right=True) - 1).clamp(max=c["G"] - 1)
        y = y[g, (r - off[g]).clamp(max=s["most"] - 1)]
        return torch.where((r < off[-1])[:, None], y, 0.0).to(dtype)
    if c["op"] == "moe_dispatch" and not c["bwd"]:
        offsets, row_of, order = _places(s["ids"], c["G"])
        used = torch.arange(order.numel(), device=order.device) < offsets[-1]
        rows = torch.where(used[:, None], s["x"][order // c["top"]], torch.zeros((), dtype=dtype, device=order.device))
        out = {"rows": rows}
        if "x_scale" in s:
            out["row_scale"] = torch.where(used, s["x_scale"][order // c["top"]], 0.0)
        return {**out, "offsets": offsets, "row_of": row_of}
    there = s["row_of"] >= 0
    at = s["row_of"].clamp(min=0).long()
    if c["op"] == "moe_dispatch":
        return (s["y"].float()[at] * there[:, :, None]).sum(1).to(dtype)
    w = torch.where(there, s["w"], 0.0)
    if not c["bwd"]:
        return (s["y"].float()[at] * w[:, :, None]).sum(1).to(dtype)
    g = s["dout"].float()
    n = s["y"].shape[0]
    # one row more than there are: the place of what was dropped
    dy = torch.zeros(n + 1, c["H"], dtype=dtype, device=g.device)
    dy[torch.where(there, at, n)] = (w[:, :, None] * g[:, None, :]).to(dtype)
    dw = (s["y"].float()[at] * g[:, None, :]).sum(2)
    return {"dy": dy[:-1], "dw": torch.where(there, dw, 0.0)}


def work(case):
    c = case
    size = SIZE[c["dtype"]]
    if c["op"] == "quant_i8":
        return {"bytes": c["M"] * c["K"] * (size + 1) + 4 * c["M"], "flops": 3 * c["M"] * c["K"]}
    if c["op"] == "gemm_i8":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": M * K + N * K + M * N * size + 4 * (M + N), "flops": 2 * M * N * K}
    n = c["T"] * c["top"] * (1 - c["drop"])
    if c["op"] == "gemm_i8_grouped":
        N, K = c["N"], c["K"]
        # experts that get no row need not be read
        used = c["G"] * (1 - (1 - 1 / c["G"]) ** n)
        return {"bytes": int(n * K + used * N * (K + 4) + n * N * size + 4 * n), "flops": int(2 * n * N * K)}
    T, H, ids = c["T"], c["H"], c["T"] * c["top"] * 4
    if c["op"] == "moe_dispatch":
        return {"bytes": int((T + n) * H * size + 2 * ids), "flops": int(n * H) if c["bwd"] else 0}
    if c["bwd"]:
        return {"bytes": int((T + 2 * n) * H * size + 3 * ids), "flops": int(3 * n * H)}
    return {"bytes": int((T + n) * H * size + 2 * ids), "flops": int(2 * n * H)}


def exact(case, seed):
    s, c = prepare(case, seed), case
    f = torch.float64
    if c["op"] == "quant_i8":
        return {"q": None, "scale": s["x"].to(f).abs().max(dim=1).values / 127}
    if c["op"] == "gemm_i8":
        y = torch.mm(s["a"].to(f), s["b"].to(f).t())
        y = torch.einsum("mn,m,n->mn", y, s["sa"].to(f), s["sb"].to(f))
        return y if s["bias"] is None else y + s["bias"].to(f)
    if c["op"] == "gemm_i8_grouped":
        out = torch.zeros(s["out"].shape, dtype=f, device="cuda")
        off = s["offsets"].tolist()
        for g in range(c["G"]):
            r = slice(off[g], off[g + 1])
            out[r] = torch.mm(s["a"][r].to(f), s["b"][g].to(f).t()) * torch.outer(s["sa"][r].to(f), s["sb"][g].to(f))
        return out
    if c["op"] == "moe_dispatch" and not c["bwd"]:
        kept = [(s["ids"] == g).nonzero()[:, 0] for g in range(c["G"])]
        t = torch.cat(kept)
        out = {}
        if c["dtype"] != "int8":
            out["rows"] = torch.zeros(s["rows"].shape, dtype=f, device="cuda")
            out["rows"][:t.numel()] = s["x"][t].to(f)
        if "x_scale" in s:
            out["row_scale"] = torch.zeros(s["row_scale"].shape, dtype=f, device="cuda")
            out["row_scale"][:t.numel()] = s["x_scale"][t].to(f)
        return {"rows": out.get("rows"), "row_scale": out.get("row_scale"), "offsets": None, "row_of": None}
    out = torch.zeros(s["out"].shape, dtype=f, device="cuda")
    if c["op"] == "moe_combine" and c["bwd"]:
        dy, dw = torch.zeros(s["y"].shape, dtype=f, device="cuda"), torch.zeros(s["w"].shape, dtype=f, device="cuda")
    for j in range(c["top"]):
        t = (s["row_of"][:, j] >= 0).nonzero()[:, 0]
        r = s["row_of"][t, j].long()
        w = s["w"][t, j].to(f) if c["op"] == "moe_combine" else torch.ones(t.numel(), dtype=f, device="cuda")
        if c["bwd"] and c["op"] == "moe_combine":
            dy[r] = s["dout"][t].to(f) * w[:, None]
            dw[t, j] = torch.linalg.vecdot(s["dout"][t].to(f), s["y"][r].to(f))
        else:
            out.index_add_(0, t, s["y"][r].to(f) * w[:, None])
    return {"dy": dy, "dw": dw} if c["op"] == "moe_combine" and c["bwd"] else out
