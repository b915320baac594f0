"""Row distances that put rows beyond 32 bits of bytes, rows longer than registers hold, and calls on several streams at
once: the 4-bit quantiser, dropout, layer norm and its gradients."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E


@pytest.mark.parametrize("cols,shift", [(1024, 0), (1021, 1)])
def test_rows_beyond_32_bits(cols, shift):
    """Every result of rows 4 GB apart is that of the same rows side by side."""
    ld = (1 << 31) + 8 * shift  # bf16 elements: row 1 begins 4 GB behind row 0
    places = [torch.empty(ld + cols + 16, dtype=torch.bfloat16, device="cuda").as_strided((2, cols), (ld, 1), shift) for _ in range(3)]
    near = [torch.empty(2, cols, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    g = torch.Generator(device="cuda").manual_seed(1)
    for far, n in zip(places, near):
        n.copy_(torch.randn(2, cols, generator=g, device="cuda"))
        far.copy_(n)
    rng, w = torch.tensor([3, 4], device="cuda"), torch.randn(cols, generator=g, device="cuda")
    results = []
    for x, r, out in (places, near):
        got = []
        q, s = torch.zeros(2, (cols + 1) // 2, dtype=torch.uint8, device="cuda"), torch.zeros(2, (cols + 31) // 32, dtype=torch.uint8, device="cuda")
        E.quant_mxf4(x, q, s)
        got += [q, s]
        E.dequant_mxf4(q, s, out)
        got.append(out.clone())
        E.dropout(x, out, 0.2, rng, residual=r)
        got.append(out.clone())
        mean, rstd = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
        E.layer_norm(x, w, None, out, residual=r, p=0.2, rng=rng, mean=mean, rstd=rstd)
        got += [out.clone(), mean, rstd]
        dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        E.layer_norm_bwd(x, r, w, mean, rstd, out, dw, db, torch.empty(E.layer_norm_bwd_work(2, cols), device="cuda"), p=0.2, rng=rng)
        results.append(got + [out.clone(), dw, db])
    # (sums of a row may be added in another order where rows start elsewhere in 16 bytes)
    for a, b in zip(*results):
        if a.dtype == torch.uint8 or shift == 0:
            assert torch.equal(a, b)
        else:
            assert bool(((a.double() - b.double()).abs() <= 2.0 ** -7 * b.double().abs() + 1e-4).all())


def test_codes_of_the_product_beyond_32_bits():
    """The last expert's codes lie 4 GB behind the first's."""
    G, N, K, M = 2, 128, 512, 40
    stride, s_stride = 1 << 32, 1 << 31
    g = torch.Generator(device="cuda").manual_seed(2)
    base = torch.empty(stride + N * K // 2, dtype=torch.uint8, device="cuda")
    s_base = torch.empty(s_stride + N * K // 32, dtype=torch.uint8, device="cuda")
    b, sb = base.as_strided((G, N, K // 2), (stride, K // 2, 1)), s_base.as_strided((G, N, K // 32), (s_stride, K // 32, 1))
    near = [torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8) for _ in range(G)]
    scale = [torch.randint(120, 130, (N, K // 32), generator=g, device="cuda", dtype=torch.uint8) for _ in range(G)]
    for e in range(G):
        b[e].copy_(near[e])
        sb[e].copy_(scale[e])
    a = torch.randint(0, 256, (2 * M, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    sa = torch.randint(120, 130, (2 * M, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    out, want = torch.zeros(2 * M, N, device="cuda"), torch.zeros(2 * M, N, device="cuda")
    E.gemm_mxf4_grouped(a, sa, b, sb, torch.tensor([0, M, 2 * M], dtype=torch.int32, device="cuda"), out)
    for e in range(G):
        E.gemm_mxf4(a[e * M:(e + 1) * M], sa[e * M:(e + 1) * M], near[e], scale[e], want[e * M:(e + 1) * M])
    E.ops_status()
    assert bool(((out - want).abs() <= 1e-5 * want.abs().max()).all())


def test_calls_on_several_streams_at_once():
    """Each with its own workspace; every result is that of the call alone."""
    rows, cols = 600, 2048
    g = torch.Generator(device="cuda").manual_seed(3)
    x, r = (torch.randn(rows, cols, generator=g, device="cuda").half() for _ in range(2))
    w, rng = torch.randn(cols, generator=g, device="cuda"), torch.tensor([1, 2], device="cuda")

    def run(stream, out):
        E.layer_norm(x, w, None, out["y"], mean=out["mean"], rstd=out["rstd"], residual=r, hidden=out["h"], p=0.1, rng=rng, stream=stream)
        E.layer_norm_bwd(x, out["h"], w, out["mean"], out["rstd"], out["dx"], out["dw"], out["db"], out["work"], p=0.1, rng=rng, stream=stream)
        E.quant_mxf4(out["y"], out["q"], out["s"], stream=stream)
        E.gemm_mxf4(out["q"], out["s"], out["q"], out["s"], out["c"], stream=stream)

    def places():
        o = {k: torch.zeros(rows, cols, dtype=torch.float16, device="cuda") for k in ("y", "h", "dx")}
        o |= {k: torch.zeros(rows, device="cuda") for k in ("mean", "rstd")} | {k: torch.zeros(cols, device="cuda") for k in ("dw", "db")}
        return o | {"work": torch.zeros(E.layer_norm_bwd_work(rows, cols), device="cuda"), "c": torch.zeros(rows, rows, device="cuda"),
                    "q": torch.zeros(rows, cols // 2, dtype=torch.uint8, device="cuda"), "s": torch.zeros(rows, cols // 32, dtype=torch.uint8, device="cuda")}

    outs, streams = [places() for _ in range(4)], [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for turn in range(3):
        for s, o in zip(streams, outs[1:]):
            run(s, o)
    torch.cuda.synchronize()
    run(None, outs[0])
    E.ops_status()
    for o in outs[1:]:
        for k in o:
            assert k == "work" or torch.equal(o[k], outs[0][k]), k


def test_gradients_of_no_rows_need_no_pointers_but_the_sums():
    dw, db, work = torch.full((64,), 7.0, device="cuda"), torch.full((64,), 7.0, device="cuda"), torch.zeros(E.layer_norm_bwd_work(0, 64), device="cuda")
    assert E._lib.entwine_layer_norm_bwd(None, E.DTYPE_BF16, 0, 64, 64, None, 64, None, E.DTYPE_FP32, None, None, None, 0, 0.0, None, 0, None, 64, None, 0,
                                         dw.data_ptr(), db.data_ptr(), work.data_ptr(), work.numel(), torch.cuda.current_stream().cuda_stream) == E.OK
    assert bool((dw == 0).all()) and bool((db == 0).all())
