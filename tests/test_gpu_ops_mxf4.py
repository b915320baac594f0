"""4-bit floats with a scale per 32 elements: the quantiser, the way back and the products, against the definition in
64 bits."""
import math

import numpy as np
import pytest
import torch

import mxf4_reference as R

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E

FLOATING = (torch.bfloat16, torch.float16, torch.float32)
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}  # half of the least steps


def _id(v):
    return str(v).replace("torch.", "") if isinstance(v, torch.dtype) else None


def _places(rows, cols, q_pad=0, s_pad=0):
    """Codes and scales in wider rows, all bytes 0xFF before."""
    qw, sw = -(-(-(-cols // 2)) // 16) * 16 + q_pad, -(-(-(-cols // 32)) // 4) * 4 + s_pad
    q = torch.full((rows, qw), 255, dtype=torch.uint8, device="cuda")
    s = torch.full((rows, sw), 255, dtype=torch.uint8, device="cuda")
    return q[:, :-(-cols // 2)], s[:, :-(-cols // 32)], q, s


def _hard_rows(rows, cols, dtype, seed):
    """Values over the type's range: middles of two levels among them, blocks of zeros, subnormal and largest numbers."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    # eighths up to 8 times a power of two hit the middles of levels
    grid = torch.randint(-64, 65, (rows, cols), generator=g, device="cuda") / 8
    x = torch.where(torch.rand(rows, 1, generator=g, device="cuda") < 0.6, grid, x)
    e = torch.randint(-20, 12, (rows, -(-cols // 32)), generator=g, device="cuda").repeat_interleave(32, 1)[:, :cols]
    x = (x * torch.exp2(e.float())).clamp(-60000, 60000).to(dtype)
    top, least = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    for r, v in enumerate((0.0, -0.0, top, least, least / 4, -least * 1.5)):
        if r < rows - 1:
            x[r, cols // 3:] = v
    return x


@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 2), (2, 31), (3, 32), (8, 33), (9, 64), (70, 96), (5, 1021), (33, 1024), (300, 160),
                                       (4, 5003), (17, 4096), (2, 70001), (1, 40000)])
def test_quantiser_gives_the_codes_of_the_definition(rows, cols, dtype):
    x = _hard_rows(rows, cols, dtype, rows + cols)
    q, s, qw, sw = _places(rows, cols)
    E.quant_mxf4(x, q, s)
    rq, rs = R.encode(x.double().cpu().numpy())
    assert np.array_equal(s.cpu().numpy(), rs)
    assert np.array_equal(q.cpu().numpy(), rq)
    assert bool((qw[:, q.shape[1]:] == 255).all()) and bool((sw[:, s.shape[1]:] == 255).all())
    back = torch.full_like(x, 7.0)
    E.dequant_mxf4(q, s, back)
    want = torch.from_numpy(R.decode(rq, rs, cols)).cuda()
    assert torch.equal(back, want.to(dtype))


@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
@pytest.mark.parametrize("shift,pad", [(0, 0), (1, 1), (3, 5), (8, 8), (4, 12)])
def test_quantiser_rows_that_start_anywhere(dtype, shift, pad):
    rows, cols = 37, 517
    big = _hard_rows(rows, cols + shift + pad, dtype, 5)
    x = big[:, shift:shift + cols]
    qb = torch.full((rows, 259 + shift + pad), 170, dtype=torch.uint8, device="cuda")
    sb = torch.full((rows, 17 + shift + pad), 170, dtype=torch.uint8, device="cuda")
    q, s = qb[:, shift:shift + 259], sb[:, shift:shift + 17]
    E.quant_mxf4(x, q, s)
    rq, rs = R.encode(x.double().cpu().numpy())
    assert np.array_equal(q.cpu().numpy(), rq) and np.array_equal(s.cpu().numpy(), rs)
    for whole, part in ((qb, q), (sb, s)):
        whole = whole.clone()
        whole[:, shift:shift + part.shape[1]] = 170
        assert bool((whole == 170).all())
    out = torch.full_like(big, 3.0)
    E.dequant_mxf4(q, s, out[:, shift:shift + cols])
    assert torch.equal(out[:, shift:shift + cols], torch.from_numpy(R.decode(rq, rs, cols)).cuda().to(dtype))
    out[:, shift:shift + cols] = 3.0
    assert bool((out == 3.0).all())


@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
def test_quantiser_blocks_that_are_not_finite(dtype):
    x = torch.randn(6, 100, device="cuda").to(dtype)
    x[1, 40], x[2, 99], x[3, 0] = math.nan, math.inf, -math.inf
    q, s, _, _ = _places(6, 100)
    E.quant_mxf4(x, q, s)
    rq, rs = R.encode(x.double().cpu().numpy())
    assert rs[1, 1] == rs[2, 3] == rs[3, 0] == 255 and (rs == 255).sum() == 3
    assert np.array_equal(q.cpu().numpy(), rq) and np.array_equal(s.cpu().numpy(), rs)
    back = torch.zeros_like(x)
    E.dequant_mxf4(q, s, back)
    assert torch.equal(torch.isnan(back).cpu(), torch.from_numpy(np.isnan(R.decode(rq, rs, 100))))


@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
def test_way_back_of_every_code_and_scale(dtype):
    """All 256 bytes under all 256 scales; products above the type's range become infinite, below it they round."""
    q = torch.arange(256, dtype=torch.uint8, device="cuda").repeat_interleave(1).reshape(16, 16)
    q = q.repeat(256, 1)
    s = torch.arange(256, dtype=torch.uint8, device="cuda").repeat_interleave(16)[:, None].contiguous()
    out = torch.zeros(4096, 32, dtype=dtype, device="cuda")
    E.dequant_mxf4(q, s, out)
    want = torch.from_numpy(R.decode(q.cpu().numpy(), s.cpu().numpy(), 32)).cuda().to(dtype)
    assert bool(((out == want) | (torch.isnan(out) & torch.isnan(want))).all())


# ------------------------------------------------------------------------------------------
# products
# ------------------------------------------------------------------------------------------
def _operand(rows, K, seed, spread):
    """Codes of all kinds, scales 2^0 to 2^spread; what lies behind a row is not zero (and the scale NaN)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, s, qw, _ = _places(rows, K)
    qw.copy_(torch.randint(0, 256, qw.shape, generator=g, device="cuda", dtype=torch.uint8))
    s.copy_(127 + torch.randint(0, spread + 1, s.shape, generator=g, device="cuda", dtype=torch.uint8))
    return q, s


def _wide(q, s, K):
    return torch.from_numpy(R.decode(q.cpu().numpy(), s.cpu().numpy(), K)).cuda()


def _check_sums(out, ref, size, K):
    """Products are exact.  A sum of K + 1 terms in fp32, whatever its order, is off by at most K + 1 times a step of the
    sum of magnitudes, 2^-23 where additions truncate; where all terms are multiples of a unit and the sum of magnitudes
    stays below 2^24 units it is exact.  The rounding to the type is off by half a step."""
    half = torch.finfo(out.dtype).eps / 2
    tol = size + half * (ref.abs() + size) + TINY[out.dtype]
    got = out.double()
    if out.dtype == torch.float16:
        over = ref.abs() >= 65520 - tol
        assert bool((got.abs()[over] >= 65504 - tol[over]).all())
        ref, tol, got = ref[~over], tol[~over], got[~over]
    assert bool(torch.isfinite(got).all())
    worst = ((got - ref).abs() / tol).max().item() if got.numel() else 0.0
    assert worst <= 1.0, worst


SHAPES = [(1, 1, 2), (1, 128, 32), (1, 1000, 4096), (2, 7, 30), (15, 129, 64), (16, 8, 126), (17, 300, 130), (31, 128, 1022),
          (33, 513, 640), (64, 256, 256), (65, 100, 66), (100, 1000, 1000), (128, 384, 512), (129, 257, 2050), (200, 96, 96),
          (255, 640, 160), (256, 512, 1024), (257, 1025, 520), (300, 64, 4096), (511, 130, 34), (1000, 777, 1022), (2049, 1024, 256),
          (64, 8192, 512), (300, 5000, 200), (129, 8197, 136), (1000, 3000, 1022), (4500, 700, 128), (260, 40000, 48),
          (8, 64, 20000), (700, 2048, 2304), (5000, 4096, 96)]


@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product_of_exact_sums(M, N, K, dtype):
    """Terms are multiples of 1/4 up to 36 * 4, so |sums| < 144 K: exact in fp32 for 576 K < 2^24."""
    a, sa = _operand(M, K, 1, 1)
    b, sb = _operand(N, K, 2, 1)
    bias = torch.randint(-50, 50, (N,), device="cuda").float() if N % 2 else None
    pitch = N + (0 if M % 2 else 24)
    whole = torch.full((M + 2, pitch), 9.0, dtype=dtype, device="cuda")
    out = whole[1:M + 1, :N]
    E.gemm_mxf4(a, sa, b, sb, out, bias=bias)
    ref = _wide(a, sa, K) @ _wide(b, sb, K).T
    if bias is not None:
        ref = ref + bias.double()
    assert 144 * 4 * K < 2 ** 24
    _check_sums(out, ref, torch.zeros_like(ref), K)
    out.fill_(9.0)
    assert bool((whole == 9.0).all())
    E.ops_status()


@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
@pytest.mark.parametrize("M,N,K", [(3, 200, 3584), (40, 512, 2048), (130, 300, 1000), (600, 1024, 4096), (2000, 1536, 608)])
def test_product_of_quantised_values(M, N, K, dtype):
    x = torch.randn(M, K, device="cuda") * torch.exp2(torch.randint(-8, 9, (M, K), device="cuda").float())
    w = torch.randn(N, K, device="cuda") / 64
    a, sa, _, _ = _places(M, K, 16, 4)
    b, sb, _, _ = _places(N, K)
    E.quant_mxf4(x, a, sa)
    E.quant_mxf4(w, b, sb)
    out = torch.zeros(M, N, dtype=dtype, device="cuda")
    E.gemm_mxf4(a, sa, b, sb, out)
    u, v = _wide(a, sa, K), _wide(b, sb, K)
    _check_sums(out, u @ v.T, (K + 1) * 2.0 ** -23 * (u.abs() @ v.abs().T), K)


@pytest.mark.parametrize("M,N", [(5, 70), (700, 1000)])
def test_product_scales_at_the_ends_and_nan(M, N):
    """Scales of 2^-127 and 2^127, which meet; a NaN scale makes its row or column NaN and nothing else."""
    K = 320
    a, sa = _operand(M, K, 3, 0)
    b, sb = _operand(N, K, 4, 0)
    sa[0, :], sb[:, 3] = 127 - 60, 127 + 10
    sa[2, :] = 0
    sa[3, :] = 254
    a[3] &= 0x11  # 0 or 1/2: in range
    sa[4, 7], sb[1, 0] = 255, 255
    out = torch.zeros(M, N, device="cuda")
    E.gemm_mxf4(a, sa, b, sb, out)
    ref = _wide(a, sa, K) @ _wide(b, sb, K).T
    nan = torch.isnan(ref)
    assert bool(nan[4].all()) and bool(nan[:, 1].all()) and int(nan.sum()) == M + N - 1
    assert torch.equal(torch.isnan(out), nan)
    fine = ~nan & (torch.arange(M, device="cuda") != 3)[:, None]
    u, v = torch.nan_to_num(_wide(a, sa, K)), torch.nan_to_num(_wide(b, sb, K))
    tol = (K + 1) * 2.0 ** -23 * (u.abs() @ v.abs().T) + 2.0 ** -149
    assert bool(((out.double() - ref).abs() <= tol)[fine].all())
    # 2^127 times halves: what passes fp32's range is infinite, the rest as usual
    r, big = ref[3], ref[3].abs() > 3.5e38
    rest = ~big & ~nan[3]
    assert bool(((out[3].double() - r).abs() <= tol[3])[rest & (tol[3] < 1e37)].all())


def _grouped(counts, N, K, dtype, bias, spare, seed=0, first=0, pad=0):
    G, M = len(counts), first + sum(counts) + spare
    a, sa = _operand(M, K, seed + 1, 1)
    bq, bs = _operand(G * (N + pad), K, seed + 2, 1)
    qw, sw = bq.stride(0), bs.stride(0)
    b = bq.as_strided((G, N, bq.shape[1]), ((N + pad) * qw, qw, 1))
    sb = bs.as_strided((G, N, bs.shape[1]), ((N + pad) * sw, sw, 1))
    add = torch.randint(-50, 50, (G, N), device="cuda").float() if bias else None
    offsets = torch.tensor([first + sum(counts[:i]) for i in range(G + 1)], dtype=torch.int32, device="cuda")
    out = torch.full((M, N), 9.0, dtype=dtype, device="cuda")
    E.gemm_mxf4_grouped(a, sa, b, sb, offsets, out, bias=add)
    at = first
    for g, c in enumerate(counts):
        if c:
            ref = _wide(a[at:at + c], sa[at:at + c], K) @ _wide(b[g], sb[g], K).T
            if bias:
                ref = ref + add[g].double()
            _check_sums(out[at:at + c], ref, torch.zeros_like(ref), K)
        at += c
    assert bool((out[:first] == 9.0).all()) and bool((out[at:] == 9.0).all())
    E.ops_status()


@pytest.mark.parametrize("dtype", FLOATING, ids=_id)
@pytest.mark.parametrize("counts,N,K", [((1,), 5, 32), ((0, 3, 0, 0, 9, 1), 300, 96), ((17, 0, 40, 33), 200, 1022), ((130, 5, 257, 0, 64), 520, 256),
                                        ((0, 0, 0), 64, 64), ((3,) * 70, 384, 160), ((300, 1, 700), 1024, 128), ((64, 65, 63, 2), 4096, 512),
                                        ((5, 0, 2, 9) * 20, 2048, 64), ((1500, 900, 0, 2000), 777, 288), ((2,) * 1024, 40, 32)])
def test_grouped_product(counts, N, K, dtype):
    _grouped(counts, N, K, dtype, bias=len(counts) % 2 == 0, spare=7, first=len(counts) % 3, pad=N % 3)


def test_grouped_offsets_out_of_order_or_range_stay_inside():
    M, N, K, G = 200, 300, 128, 5
    a, sa = _operand(M, K, 1, 1)
    b, sb = _operand(G * N, K, 2, 1)
    b, sb = b.unflatten(0, (G, N)), sb.unflatten(0, (G, N))
    whole = torch.full((M + 4, N), 9.0, device="cuda")
    for bad in ([0, 50, 40, 1000, 30, 2000], [-7, -3, 100, 90, 250, 200], [200, 0, 200, 0, 200, 0]):
        E.gemm_mxf4_grouped(a, sa, b, sb, torch.tensor(bad, dtype=torch.int32, device="cuda"), whole[2:-2])
        torch.cuda.synchronize()
        assert bool((whole[:2] == 9.0).all()) and bool((whole[-2:] == 9.0).all())
    E.ops_status()


@pytest.mark.parametrize("M,N", [(16, 1024), (700, 2048)])
def test_product_repeats_bitwise_replays_and_runs_on_other_streams(M, N):
    K = 1056
    a, sa = _operand(M, K, 5, 9)
    b, sb = _operand(N, K, 6, 9)
    out, again, there = (torch.zeros(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    E.gemm_mxf4(a, sa, b, sb, out)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    E.gemm_mxf4(a, sa, b, sb, there, stream=s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        E.gemm_mxf4(a, sa, b, sb, again)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, again) and torch.equal(out, there)
    sa.add_(1)
    graph.replay()
    E.gemm_mxf4(a, sa, b, sb, out)
    torch.cuda.synchronize()
    assert torch.equal(out, again) and not torch.equal(out, there)


def test_no_rows():
    a, sa = _operand(0, 64, 1, 0)
    b, sb = _operand(8, 64, 1, 0)
    E.gemm_mxf4(a, sa, b, sb, torch.zeros(0, 8, device="cuda"))
    E.quant_mxf4(torch.zeros(0, 64, device="cuda"), a, sa)
    E.dequant_mxf4(a, sa, torch.zeros(0, 64, device="cuda"))
    torch.cuda.synchronize()
