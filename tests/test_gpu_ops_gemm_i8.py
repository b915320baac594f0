"""Int8 product with token and channel scales through the C ABI, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E

FLOATING = (torch.bfloat16, torch.float16, torch.float32)
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}


def _levels(rows, cols, seed, pitch=None):
    """int8 values over the whole range, -128 among them, in rows of `pitch`; what lies behind a row is not zero."""
    pitch = -(-cols // 16) * 16 if pitch is None else pitch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-128, 128, (rows, pitch), generator=g, device="cuda", dtype=torch.int8)[:, :cols]


def _scales(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.rand(n, generator=g, device="cuda") * 0.02 + 0.001


def _check(out, a, sa, b, sb, bias):
    """The sum is exact; its conversion to fp32, the two products and the addition are off by at most 2^-24 each, the
    rounding to the type by half a step."""
    acc = a.double() @ b.double().T
    p = acc * sa.double()[:, None] * sb.double()
    ref = p if bias is None else p + bias.double()
    u, half = 2.0 ** -24, torch.finfo(out.dtype).eps / 2
    add = 0.0 if bias is None else bias.double().abs()
    tol = u * (3 * p.abs() + add) * (1 + 2.0 ** -7) + half * ref.abs() * (1 + 2.0 ** -20) + TINY[out.dtype]
    if out.dtype == torch.float16:
        over = ref.abs() >= 65520 - tol
        assert bool((out.double().abs()[over] >= 65504 - tol[over]).all())
        ref, tol, got = ref[~over], tol[~over], out.double()[~over]
    else:
        got = out.double()
    assert bool(torch.isfinite(got).all())
    worst = ((got - ref).abs() / tol).max().item() if got.numel() else 0.0
    assert worst <= 1.0, worst


def _dtype_id(v):
    return str(v).replace("torch.", "") if isinstance(v, torch.dtype) else None


SHAPES = [(1, 1, 1), (1, 128, 128), (1, 1000, 4096), (2, 7, 15), (15, 129, 16), (16, 8, 127), (17, 300, 129), (31, 128, 1021),
          (33, 513, 640), (64, 256, 256), (65, 100, 64), (100, 1000, 1000), (128, 384, 512), (129, 257, 2049), (200, 96, 96), (255, 640, 160),
          (256, 512, 1024), (257, 1025, 520), (300, 64, 4096), (511, 130, 33), (1000, 777, 1021), (2049, 1024, 256), (64, 8192, 512),
          (300, 5000, 200), (129, 8197, 136), (1000, 3000, 1021), (4500, 700, 128), (260, 40000, 48)]


@pytest.mark.parametrize("dtype", FLOATING, ids=_dtype_id)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_i8_matches_the_definition(M, N, K, dtype):
    a, b = _levels(M, K, 1), _levels(N, K, 2)
    sa, sb = _scales(M, 3), _scales(N, 4)
    for bias, extra in ((None, 0), (torch.randn(N, device="cuda"), 5)):
        store = torch.full((M, N + extra), -9.0, dtype=dtype, device="cuda")
        out = store[:, :N]
        E.gemm_i8(a, sa, b, sb, out, bias=bias)
        _check(out, a, sa, b, sb, bias)
        assert bool((store[:, N:] == -9).all())
    E.ops_status()


def test_gemm_i8_pitches_and_exact_sums():
    """Padded rows of different lengths; unit scales give the integer sum itself while fp32 holds it."""
    M, N, K = 130, 200, 1000
    a, b = _levels(M, K, 1, 1008), _levels(N, K, 2, 1200)
    out = torch.empty(M, N, device="cuda")
    E.gemm_i8(a, torch.ones(M, device="cuda"), b, torch.ones(N, device="cuda"), out)
    assert torch.equal(out.double(), a.double() @ b.double().T)
    # one row: its distance to the next does not matter
    E.gemm_i8(a[:1], torch.ones(1, device="cuda"), b, torch.ones(N, device="cuda"), out[:1])
    assert torch.equal(out[:1].double(), a[:1].double() @ b.double().T)


@pytest.mark.parametrize("M,N", [(3, 5), (300, 5), (300, 5000)])
def test_gemm_i8_largest_sum(M, N):
    """K at its limit and every product at its largest: 2147467264, one step below int32's end in fp32's eyes."""
    K = 131071
    for sign in (1, -1):
        a = torch.full((M, K + 1), -128, dtype=torch.int8, device="cuda")[:, :K]
        b = torch.full((N, K + 1), -128 if sign > 0 else 127, dtype=torch.int8, device="cuda")[:, :K]
        out = torch.empty(M, N, device="cuda")
        E.gemm_i8(a, torch.ones(M, device="cuda"), b, torch.ones(N, device="cuda"), out)
        want = np.float32(128 * 128 * K if sign > 0 else -128 * 127 * K)
        assert bool((out == float(want)).all())


def test_gemm_i8_scales_that_are_not_finite():
    """A token whose scale is NaN gives a row of NaN and leaves the others alone; a zero scale gives the bias."""
    M, N, K = 20, 140, 256
    a, b, sa, sb = _levels(M, K, 1), _levels(N, K, 2), _scales(M, 3), _scales(N, 4)
    sa[7], sa[9] = float("nan"), 0.0
    bias = torch.randn(N, device="cuda")
    out = torch.empty(M, N, dtype=torch.float32, device="cuda")
    E.gemm_i8(a, sa, b, sb, out, bias=bias)
    assert bool(out[7].isnan().all()) and torch.equal(out[9], bias)
    keep = [i for i in range(M) if i != 7]
    _check(out[keep], a[keep], sa[keep], b, sb, bias)


# rows per expert: empty experts first, in the middle and last, one row, tile ends, everything in one
GROUPS = [([0, 3, 0, 1, 16, 17, 0], 128, 128), ([5], 100, 64), ([0, 0, 40, 0], 257, 300), ([1] * 33, 130, 1021), ([64, 65, 63, 0, 128], 384, 512),
          ([300, 1, 0, 255, 257], 200, 640), ([1000, 0, 0, 24], 129, 96), ([7] * 100 + [0] * 28, 256, 256), ([0, 0, 0], 64, 64), ([513, 700], 512, 160),
          ([0, 3, 0, 1, 16, 17, 0, 64, 65, 33, 31, 129, 0], 3333, 192), ([300, 1, 0, 255, 257, 513], 1800, 640), ([1] * 33, 1300, 1021),
          ([0] * 500 + [40] + [0] * 400 + [1, 2], 1024, 80), ([5000, 0, 70], 2000, 112)]


def _grouped(counts, N, K, dtype, bias, spare, seed=0, first=0, expert_pad=0):
    G, M = len(counts), first + sum(counts) + spare
    off = torch.tensor(np.cumsum([first] + counts), dtype=torch.int32, device="cuda")
    pitch = -(-K // 16) * 16
    a = _levels(max(M, 1), K, seed + 1)[:M]
    b = torch.randint(-128, 128, (G, N * pitch + expert_pad), device="cuda", dtype=torch.int8)
    b = b[:, :N * pitch].unflatten(1, (N, pitch))[:, :, :K]
    sa, sb = _scales(M, seed + 3), _scales(G * N, seed + 4).view(G, N)
    bs = torch.randn(G, N, device="cuda") if bias else None
    out = torch.full((M, N), -9.0, dtype=dtype, device="cuda")
    E.gemm_i8_grouped(a, sa, b, sb, off, out, bias=bs)
    o = off.tolist()
    for g in range(G):
        r = slice(o[g], o[g + 1])
        _check(out[r], a[r], sa[r], b[g], sb[g], None if bs is None else bs[g])
    assert bool((out[:first] == -9).all()) and bool((out[o[-1]:] == -9).all())


@pytest.mark.parametrize("dtype", FLOATING, ids=_dtype_id)
@pytest.mark.parametrize("counts,N,K", GROUPS, ids=[f"G{len(c)}_rows{sum(c)}_N{n}_K{k}" for c, n, k in GROUPS])
def test_grouped_matches_the_definition(counts, N, K, dtype):
    _grouped(counts, N, K, dtype, False, 0)
    _grouped(counts, N, K, dtype, True, 40, seed=7, expert_pad=48)
    _grouped(counts, N, K, dtype, False, 3, first=9)


def test_grouped_offsets_out_of_order_or_range_stay_inside():
    """What no dispatch writes: bounds outside the rows and decreasing ones; rows without an expert stay as they were."""
    M, N, K = 50, 130, 64
    a, b, sa, sb = _levels(M, K, 1), _levels(4 * N, K, 2).view(4, N, K), _scales(M, 3), _scales(4 * N, 4).view(4, N)
    off = torch.tensor([-5, 10, 4, 30, 900], dtype=torch.int32, device="cuda")   # [0,10), none, [4,30), [30,50)
    out = torch.full((M, N), -9.0, device="cuda")
    E.gemm_i8_grouped(a, sa, b, sb, off, out)
    _check(out[:4], a[:4], sa[:4], b[0], sb[0], None)
    _check(out[10:30], a[10:30], sa[10:30], b[2], sb[2], None)
    _check(out[30:], a[30:], sa[30:], b[3], sb[3], None)


@pytest.mark.parametrize("M,N", [(4, 1536), (600, 1536), (600, 2560)])
def test_gemm_i8_repeats_bitwise_and_replays(M, N):
    """Same bits on every call, in a captured first call, and with two graphs on streams of their own at once."""
    K = 1408
    a, b, sa, sb = _levels(M, K, 1), _levels(N, K, 2), _scales(M, 3), _scales(N, 4)
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    E.gemm_i8(a, sa, b, sb, out)
    again = torch.empty_like(out)
    for _ in range(3):
        again.fill_(float("nan"))
        E.gemm_i8(a, sa, b, sb, again)
        assert torch.equal(out, again)
    side, graphs, outs, ins = [torch.cuda.Stream() for _ in range(2)], [], [], []
    torch.cuda.synchronize()
    for i, s in enumerate(side):
        outs.append(torch.empty_like(out))
        ins.append(a.clone())
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            E.gemm_i8(ins[i], sa, b, sb, outs[i])
        graphs.append(g)
    for round_ in range(3):
        for i in range(2):
            ins[i].copy_(_levels(M, K, 50 + 2 * round_ + i))
            outs[i].fill_(float("nan"))
        torch.cuda.synchronize()
        for g, s in zip(graphs, side):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            E.gemm_i8(ins[i], sa, b, sb, again)
            assert torch.equal(outs[i], again)
    E.ops_status()


def test_weight_offsets_beyond_32_bits():
    """Experts whose matrices start more than 2^32 bytes behind the first."""
    G, N, K = 70, 8192, 8192
    b = torch.empty(G, N, K, dtype=torch.int8, device="cuda")
    b[0], b[-1] = _levels(N, K, 1), _levels(N, K, 2)
    counts = [3] + [0] * (G - 2) + [5]
    off = torch.tensor(np.cumsum([0] + counts), dtype=torch.int32, device="cuda")
    a, sa, sb = _levels(8, K, 3), _scales(8, 4), _scales(G * N, 5).view(G, N)
    out = torch.empty(8, N, device="cuda")
    E.gemm_i8_grouped(a, sa, b, sb, off, out)
    _check(out[:3], a[:3], sa[:3], b[0], sb[0], None)
    _check(out[3:], a[3:], sa[3:], b[-1], sb[-1], None)


def test_quantised_expert_layer():
    """The operators as they are used together: quantise, sort, product per expert, weighted return; against the layer
    in 64 bits on the quantised values, and against the unquantised layer within the quantisation's own error."""
    T, H, N, n_experts, k = 150, 256, 384, 16, 4
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
    weight = torch.randn(n_experts, N, H, generator=g, device="cuda") / 16
    wish, ids = torch.randn(T, n_experts, generator=g, device="cuda").topk(k, dim=1)
    ids[::7, 1] = -1
    w = torch.softmax(wish, dim=1)
    wq, ws = torch.empty(n_experts * N, H, dtype=torch.int8, device="cuda"), torch.empty(n_experts * N, device="cuda")
    E.quant_i8(weight.view(-1, H), wq, ws)
    xq, xs = torch.empty(T, H, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    rows, rs = torch.zeros(T * k, H, dtype=torch.int8, device="cuda"), torch.zeros(T * k, device="cuda")
    off, row_of = torch.empty(n_experts + 1, dtype=torch.int32, device="cuda"), torch.empty(T, k, dtype=torch.int32, device="cuda")
    y, out = torch.empty(T * k, N, dtype=torch.float32, device="cuda"), torch.empty(T, N, dtype=torch.float32, device="cuda")
    E.quant_i8(x, xq, xs)
    E.moe_dispatch(xq, ids, n_experts, rows, off, row_of, x_scale=xs, row_scale=rs)
    E.gemm_i8_grouped(rows, rs, wq.view(n_experts, N, H), ws.view(n_experts, N), off, y)
    E.moe_combine(y, w, row_of, out)
    E.ops_status()
    there = (ids >= 0)
    deq = (xq.double() * xs.double()[:, None])
    wdeq = (wq.double() * ws.double()[:, None]).view(n_experts, N, H)[ids.clamp(min=0)]      # [T, k, N, H]
    each = torch.einsum("th,tknh->tkn", deq, wdeq) * there[:, :, None]
    ref, mag = (each * w.double()[:, :, None]).sum(1), (each.abs() * w.double()[:, :, None]).sum(1)
    # three roundings of 2^-24 in each product, k + 1 in the sum
    assert bool(((out.double() - ref).abs() <= (k + 5) * 2.0 ** -24 * mag * (1 + 2.0 ** -7) + 1e-30).all())
    # each value is off by at most half a level: |error| <= (scale_x |w|_1 + scale_w |x|_1 + H scale_x scale_w / 2) / 2 per product
    full = weight.double()[ids.clamp(min=0)]
    plain = (torch.einsum("th,tknh->tkn", x.double(), full) * (w.double() * there)[:, :, None]).sum(1)
    wsc = ws.double().view(n_experts, N)[ids.clamp(min=0)]
    bound = (xs.double()[:, None, None] * full.abs().sum(-1) + wsc * x.double().abs().sum(1)[:, None, None] + H * xs.double()[:, None, None] * wsc / 2) / 2
    bound = (bound * (w.double() * there)[:, :, None]).sum(1)
    assert bool(((ref - plain).abs() <= bound * (1 + 1e-5)).all())
