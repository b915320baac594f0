"""Row quantiser, expert sort and weighted return through the C ABI, against numpy in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E

FLOATING = (torch.bfloat16, torch.float16, torch.float32)
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}  # least subnormals


def _name(v):
    return str(v).replace("torch.", "") if isinstance(v, torch.dtype) else None


def _rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    if dtype == torch.int8:
        return torch.randint(-127, 128, shape, generator=g, dtype=torch.int8)
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def _laid_out(t, pitch=None, shift=0, fill=0):
    """The matrix on the device with rows `pitch` elements apart, starting `shift` elements behind an aligned address."""
    rows, cols = t.shape
    pitch = cols if pitch is None else pitch
    store = torch.full((rows * pitch + shift,), fill, dtype=t.dtype, device="cuda")
    view = store[shift:].view(rows, pitch)[:, :cols]
    view.copy_(t)
    return view


def _f64(t):
    return t.detach().double().cpu().numpy()


def _half_step(dtype):
    """Half a rounding step, relative to the value."""
    return torch.finfo(dtype).eps / 2


# ---------------------------------------------------------------------------------------------- quantiser
def _quant_ref(x):
    """127 x is exact in fp64 (24 + 7 bits) and so is every half that the quotient could be near, so the rounded
    quotient lies on the right side of it."""
    x = _f64(x)
    amax = np.abs(x).max(1, keepdims=True)
    bad = ~np.isfinite(amax)
    safe = np.where(bad | (amax == 0), 1.0, amax)
    q = np.rint(np.where(bad, 0.0, x) * 127.0 / safe)
    scale = np.where(bad, np.nan, amax).astype(np.float32)[:, 0] / np.float32(127)
    return np.where(bad, 0, q).astype(np.int8), scale


def _check_quant(x, q, scale):
    rq, rs = _quant_ref(x)
    assert np.array_equal(q.cpu().numpy(), rq)
    assert np.array_equal(scale.cpu().numpy(), rs, equal_nan=True)


@pytest.mark.parametrize("dtype", FLOATING, ids=_name)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (2, 7), (5, 8), (4, 255), (7, 257), (129, 512), (2, 4096), (3, 4099),
                                       (5, 8192), (3, 16384), (2, 28672), (2, 40000)])
def test_quant_matches_the_exact_quotient(rows, cols, dtype):
    x = _rand((rows, cols), dtype, rows * cols, 3.0)
    for pitch, shift, qpitch, qshift in ((cols, 0, cols, 0), (cols + 5, 1, cols + 3, 1), (-(-cols // 16) * 16, 0, -(-cols // 16) * 16, 0),
                                         (-(-cols // 16) * 16 + 16, 0, cols + 1, 3)):
        xd = _laid_out(x, pitch, shift)
        q = _laid_out(torch.full((rows, cols), 99, dtype=torch.int8), qpitch, qshift, fill=77)
        scale = torch.full((rows,), -1.0, device="cuda")
        E.quant_i8(xd, q, scale)
        _check_quant(x, q, scale)
        around = q._base.clone()
        around[qshift:].view(rows, qpitch)[:, :cols] = 77
        assert bool((around == 77).all())  # nothing is written beside the rows


@pytest.mark.parametrize("dtype", FLOATING, ids=_name)
def test_quant_special_rows(dtype):
    big, tiny = torch.finfo(dtype).max, TINY[dtype]
    rows = [torch.zeros(64), torch.full((64,), -0.0), torch.full((64,), big), torch.full((64,), tiny),
            torch.linspace(-big, big, 64, dtype=torch.float64).float(), torch.arange(64) * tiny,
            torch.arange(64) / 2.0 * 4,                       # amax 126: no ties
            torch.cat([torch.tensor([127.0]), torch.arange(63) + 0.5]),   # every other value on a half
            torch.cat([torch.tensor([-254.0]), torch.arange(63) * 2 + 1.0]),
            torch.cat([torch.tensor([0.0, 1.0]), torch.full((62,), 2.0 ** -8)])]
    for bad in (float("nan"), float("inf"), float("-inf")):
        r = torch.randn(64, generator=torch.Generator().manual_seed(3))
        r[17] = bad
        rows.append(r)
    x = torch.stack([r.float() for r in rows]).to(dtype)
    q, scale = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(len(rows), device="cuda")
    E.quant_i8(x.cuda(), q, scale)
    _check_quant(x, q, scale)
    assert bool(torch.isnan(scale[-3:]).all()) and not bool(q[-3:].any())


def test_quant_decides_values_next_to_a_half():
    """fp32 rows built so that many quotients lie within an ulp or two of a half, on either side of it."""
    g = np.random.default_rng(5)
    amax = g.uniform(0.5, 2.0, (64, 1)).astype(np.float32)
    k = g.integers(-126, 126, (64, 1000))
    x = ((k + 0.5) * amax.astype(np.float64) / 127).astype(np.float32)
    x = np.where(g.integers(0, 2, x.shape) > 0, np.nextafter(x, np.float32(9)), x)
    x = torch.from_numpy(np.concatenate([amax, x], 1))
    q, scale = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(64, device="cuda")
    E.quant_i8(x.cuda(), q, scale)
    _check_quant(x, q, scale)


def test_quant_many_rows_and_none():
    x = _rand((70000, 24), torch.bfloat16, 4)
    q, scale = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(x.shape[0], device="cuda")
    E.quant_i8(x.cuda(), q, scale)
    _check_quant(x, q, scale)
    E.quant_i8(x[:0].cuda(), q[:0], scale[:0])


# ---------------------------------------------------------------------------------------------- sort and return
ROUTES = [(1, 1, 1, 1), (1, 8, 8, 64), (3, 2, 5, 7), (16, 8, 64, 256), (33, 4, 16, 72), (100, 1, 2, 40), (257, 8, 60, 136),
          (1000, 6, 1024, 16), (4097, 2, 33, 24), (20000, 4, 128, 8), (40, 3, 1024, 16), (256, 8, 1023, 24), (2049, 1, 1, 16)]


def _ids(T, k, n_experts, seed, drop=0.2):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, n_experts, (T, k), generator=g)       # an expert may come twice for a token
    ids = torch.where(torch.rand(T, k, generator=g) < 0.4, ids // 3, ids)   # uneven loads
    out = torch.tensor([-1, n_experts, n_experts + 5, -7])[torch.randint(0, 4, (T, k), generator=g)]
    return torch.where(torch.rand(T, k, generator=g) < drop, out, ids)


def _sort_ref(ids, n_experts):
    flat = ids.reshape(-1).numpy()
    key = np.where((flat >= 0) & (flat < n_experts), flat, n_experts)
    order = np.argsort(key, kind="stable")
    offsets = np.searchsorted(key[order], np.arange(n_experts + 1))
    row = np.empty(flat.size, np.int64)
    row[order] = np.arange(flat.size)
    return offsets.astype(np.int32), np.where(key < n_experts, row, -1).reshape(ids.shape).astype(np.int32)


def _dispatch(x, ids, n_experts, x_scale=None, fill=-3):
    T, k = ids.shape
    rows = torch.full((T * k, x.shape[1]), fill, dtype=x.dtype, device="cuda")
    offsets = torch.full((n_experts + 1,), -5, dtype=torch.int32, device="cuda")
    row_of = torch.full((T, k), -5, dtype=torch.int32, device="cuda")
    row_scale = None if x_scale is None else torch.full((T * k,), float(fill), device="cuda")
    E.moe_dispatch(x, ids, n_experts, rows, offsets, row_of, x_scale=x_scale, row_scale=row_scale)
    return rows, offsets, row_of, row_scale


def _check_dispatch(x, ids, n_experts, got, x_scale=None, fill=-3):
    rows, offsets, row_of, row_scale = got
    ro, rr = _sort_ref(ids, n_experts)
    assert np.array_equal(offsets.cpu().numpy(), ro) and np.array_equal(row_of.cpu().numpy(), rr)
    want = torch.full(rows.shape, fill, dtype=x.dtype)
    t, j = np.nonzero(rr >= 0)
    want[torch.from_numpy(rr[t, j].astype(np.int64))] = x.cpu()[torch.from_numpy(t)]
    assert torch.equal(rows.cpu(), want)
    if x_scale is not None:
        want = torch.full((rows.shape[0],), float(fill))
        want[torch.from_numpy(rr[t, j].astype(np.int64))] = x_scale.cpu()[torch.from_numpy(t)]
        assert torch.equal(row_scale.cpu(), want)


@pytest.mark.parametrize("T,k,n_experts,H", ROUTES)
def test_dispatch_sorts_and_moves(T, k, n_experts, H):
    for i, dtype in enumerate((torch.bfloat16, torch.float16, torch.float32, torch.int8)):
        ids = _ids(T, k, n_experts, T + i, drop=(0.2, 0.0, 1.0, 0.7)[i])
        ids = ids.to((torch.int64, torch.int32)[i % 2])
        x = _rand((T, H), dtype, i)
        scale = torch.rand(T).cuda() if dtype == torch.int8 else None
        for pitch, shift in ((H, 0), (H + 3, 1), (-(-H // 16) * 16 + 16, 0)):
            xd = _laid_out(x, pitch, shift)
            _check_dispatch(x, ids, n_experts, _dispatch(xd, ids.cuda(), n_experts, scale), scale)


def test_dispatch_far_ids_and_one_crowded_expert():
    x = _rand((300, 32), torch.bfloat16, 1).cuda()
    ids = torch.full((300, 4), 6, dtype=torch.int64)
    _check_dispatch(x, ids, 7, _dispatch(x, ids.cuda(), 7))
    ids[::3, 1], ids[1::3, 2] = (1 << 32) + 2, -(1 << 32) + 3     # wrong ids must not be cut to 32 bits
    _check_dispatch(x, ids, 7, _dispatch(x, ids.cuda(), 7))
    ids = torch.full((300, 4), -1, dtype=torch.int32)
    _check_dispatch(x, ids, 7, _dispatch(x, ids.cuda(), 7))


def test_dispatch_without_tokens_writes_offsets():
    x, ids = torch.zeros(0, 8, device="cuda"), torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    rows, offsets, row_of, _ = _dispatch(x, ids, 5)
    assert not bool(offsets.any())
    E.moe_combine(rows, torch.zeros(0, 2, device="cuda"), row_of, x)
    E.moe_dispatch_bwd(rows, row_of, x)


def _return_case(T, k, n_experts, H, dtype, seed):
    ids = _ids(T, k, n_experts, seed)
    ids[T // 2] = -1                                            # a token that keeps nothing
    _, row_of = _sort_ref(ids, n_experts)
    y = _rand((T * k, H), dtype, seed + 1)
    y[int((row_of >= 0).sum()):] = float("nan")                 # rows that nobody owns must not be read
    w = torch.rand(T, k, generator=torch.Generator().manual_seed(seed)) - 0.2
    w[torch.from_numpy(row_of < 0)] = float("nan")              # nor the weights of what was dropped
    return y, w, torch.from_numpy(row_of), _rand((T, H), dtype, seed + 2)


def _taken(y, row_of):
    """Row of each assignment in 64 bits, zeros where dropped; and where that is."""
    r = row_of.numpy()
    return np.where((r >= 0)[..., None], _f64(y)[np.maximum(r, 0)], 0.0), r >= 0


@pytest.mark.parametrize("dtype", FLOATING, ids=_name)
@pytest.mark.parametrize("T,k,n_experts,H", ROUTES[:8])
def test_return_and_its_gradients(T, k, n_experts, H, dtype):
    y, w, row_of, dout = _return_case(T, k, n_experts, H, dtype, T + H)
    yt, there = _taken(y, row_of)
    w64 = np.where(there, _f64(w), 0.0)
    u, tiny = 2.0 ** -24, TINY[dtype]

    def close(got, ref, mags):
        """k fused multiply-adds in fp32, each off by at most u times a partial sum of magnitudes, and one rounding."""
        got = _f64(got)
        assert np.isfinite(got).all()
        assert (np.abs(got - ref) <= (k + 1) * u * mags * (1 + 2.0 ** -7) + _half_step(dtype) * np.abs(ref) + tiny).all()

    for pitch, shift in ((H, 0), (H + 3, 1), (-(-H // 16) * 16, 0)):
        yd, gd = _laid_out(y, pitch, shift), _laid_out(dout, pitch, shift)
        rd, wd = row_of.cuda(), w.cuda()
        out = _laid_out(torch.full((T, H), 9.0, dtype=dtype), pitch, shift)
        E.moe_combine(yd, wd, rd, out)
        close(out, (yt * w64[..., None]).sum(1), (np.abs(yt) * np.abs(w64)[..., None]).sum(1))
        dx = _laid_out(torch.full((T, H), 9.0, dtype=dtype), pitch, shift)
        E.moe_dispatch_bwd(yd, rd, dx)
        close(dx, yt.sum(1), np.abs(yt).sum(1))
        dy = _laid_out(torch.full((T * k, H), 9.0, dtype=dtype), pitch, shift)
        dw = torch.full((T, k), 9.0, device="cuda")
        E.moe_combine_bwd(gd, yd, wd, rd, dy, dw)
        g = _f64(dout)
        want = np.full((T * k, H), 9.0)
        want[row_of.numpy()[there]] = (w64[..., None] * g[:, None])[there]
        # the fp32 product, then the rounding of the type (none more for fp32)
        assert (np.abs(_f64(dy) - want) <= (u + _half_step(dtype)) * (1 + 2.0 ** -7) * np.abs(want) + tiny).all()
        dot, mag = np.einsum("th,tkh->tk", g, yt), np.einsum("th,tkh->tk", np.abs(g), np.abs(yt))
        assert (np.abs(_f64(dw) - dot) <= H * u * mag * (1 + 2.0 ** -7)).all()   # H additions in any order
        assert not bool(dw[~torch.from_numpy(there)].any())


def test_gradients_agree_with_differences():
    """sum(c * combine(dispatch(x), w)): its gradient by the two backward calls against central differences in 64 bits."""
    T, k, n_experts, H = 6, 3, 4, 16
    ids = _ids(T, k, n_experts, 11)
    _, row_of = _sort_ref(ids, n_experts)
    x, c = _rand((T, H), torch.float32, 1), _rand((T, H), torch.float32, 2)
    w = torch.rand(T, k, generator=torch.Generator().manual_seed(3))
    there = row_of >= 0

    def loss(x, w):   # every assignment's row is its token's row, squared on the way
        return (c.double().numpy()[:, None] * w[..., None] * (x[:, None] ** 2) * there[..., None]).sum()

    rows, _, r, _ = _dispatch(x.cuda(), ids.cuda(), n_experts, fill=0)
    y = rows * rows
    dy, dw = torch.zeros_like(y), torch.empty(T, k, device="cuda")
    E.moe_combine_bwd(c.cuda(), y, w.cuda(), r, dy, dw)
    dx = torch.empty(T, H, device="cuda")
    E.moe_dispatch_bwd(2 * rows * dy, r, dx)
    x64, w64, h = x.double().numpy(), w.double().numpy(), 1e-4
    for t in range(T):
        for i in range(0, H, 5):
            d = np.zeros_like(x64)
            d[t, i] = h
            # quadratic in x: central differences are exact but for fp64 rounding (about 1e-16 * loss / h)
            assert abs((loss(x64 + d, w64) - loss(x64 - d, w64)) / (2 * h) - float(dx[t, i])) <= 1e-5
        for j in range(k):
            d = np.zeros_like(w64)
            d[t, j] = h
            assert abs((loss(x64, w64 + d) - loss(x64, w64 - d)) / (2 * h) - float(dw[t, j])) <= 1e-4


def test_row_numbers_outside_the_rows_count_as_dropped():
    y, out = torch.ones(4, 8, device="cuda"), torch.empty(2, 8, device="cuda")
    row_of = torch.tensor([[0, 4], [1 << 30, -2]], dtype=torch.int32, device="cuda")
    w = torch.full((2, 2), 2.0, device="cuda")
    E.moe_combine(y, w, row_of, out)
    assert out[:, 0].tolist() == [2.0, 0.0]
    dy, dw = torch.zeros_like(y), torch.empty_like(w)
    E.moe_combine_bwd(out, y, w, row_of, dy, dw)
    assert dw.tolist() == [[16.0, 0.0], [0.0, 0.0]] and dy[:, 0].tolist() == [4.0, 0.0, 0.0, 0.0]


def test_offsets_beyond_32_bits():
    """Rows whose first element lies more than 2^32 bytes and 2^31 elements into the matrix."""
    T, k, H = 150000, 2, 8192
    x = torch.randint(-127, 128, (T, H), dtype=torch.int8, device="cuda")
    ids = torch.randint(0, 16, (T, k), dtype=torch.int32, device="cuda")
    rows = torch.empty(T * k, H, dtype=torch.int8, device="cuda")
    offsets, row_of = torch.empty(17, dtype=torch.int32, device="cuda"), torch.empty(T, k, dtype=torch.int32, device="cuda")
    E.moe_dispatch(x, ids, 16, rows, offsets, row_of)
    ro, rr = _sort_ref(ids.cpu(), 16)
    assert np.array_equal(offsets.cpu().numpy(), ro) and np.array_equal(row_of.cpu().numpy(), rr)
    for j in range(k):
        for t0 in range(0, T, 50000):
            assert torch.equal(rows[row_of[t0:t0 + 50000, j].long()], x[t0:t0 + 50000])
    del x
    y = rows.view(torch.bfloat16)                                # [T*k, H/2], 2.4 GB
    y = torch.cat([y, y])                                        # 4.9 GB
    n = y.shape[0]
    at = torch.tensor([[n - 1, 0], [n - 3, n // 2]], dtype=torch.int32, device="cuda")
    y[at.flatten().long()] = torch.arange(1, 5, dtype=torch.bfloat16, device="cuda")[:, None]
    out, w = torch.empty(2, H // 2, dtype=torch.bfloat16, device="cuda"), torch.ones(2, 2, device="cuda")
    E.moe_combine(y, w, at, out)
    assert out[:, 0].tolist() == [3.0, 7.0] and out[:, -1].tolist() == [3.0, 7.0]
    dw = torch.empty(2, 2, device="cuda")
    dy = torch.empty_like(y)
    E.moe_combine_bwd(out, y, w, at, dy, dw)
    assert dw.tolist() == [[3.0 * H / 2, 6.0 * H / 2], [21.0 * H / 2, 28.0 * H / 2]]
    assert dy[at.flatten().long(), -1].tolist() == [3.0, 3.0, 7.0, 7.0]


def test_capture_replay_and_other_streams():
    """The first call of each operator inside a capture, two graphs at once on streams of their own, and eager calls
    beside them: every replay works on what the buffers hold then."""
    T, k, n_experts, H = 96, 4, 8, 128
    side = [torch.cuda.Stream() for _ in range(2)]
    sets, graphs = [], []
    for s in side:
        b = {"x": torch.zeros(T, H, dtype=torch.bfloat16, device="cuda"), "ids": torch.zeros(T, k, dtype=torch.int64, device="cuda"),
             "rows": torch.zeros(T * k, H, dtype=torch.bfloat16, device="cuda"), "offsets": torch.zeros(n_experts + 1, dtype=torch.int32, device="cuda"),
             "row_of": torch.zeros(T, k, dtype=torch.int32, device="cuda"), "w": torch.zeros(T, k, device="cuda"),
             "out": torch.zeros(T, H, dtype=torch.bfloat16, device="cuda"), "q": torch.zeros(T, H, dtype=torch.int8, device="cuda"),
             "scale": torch.zeros(T, device="cuda")}
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            E.moe_dispatch(b["x"], b["ids"], n_experts, b["rows"], b["offsets"], b["row_of"])
            E.moe_combine(b["rows"], b["w"], b["row_of"], b["out"])
            E.quant_i8(b["out"], b["q"], b["scale"])
        sets.append(b)
        graphs.append(g)
    for round_ in range(3):
        for i, b in enumerate(sets):
            b["x"].copy_(_rand((T, H), torch.bfloat16, 10 * round_ + i))
            b["ids"].copy_(_ids(T, k, n_experts, 20 * round_ + i))
            b["w"].copy_(torch.rand(T, k))
            b["rows"].fill_(-3)
        torch.cuda.synchronize()
        for g, s in zip(graphs, side):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for b in sets:
            _check_dispatch(b["x"], b["ids"].cpu(), n_experts, (b["rows"], b["offsets"], b["row_of"], None))
            again = torch.empty_like(b["out"])
            E.moe_combine(b["rows"], b["w"], b["row_of"], again, stream=side[0])
            side[0].synchronize()
            assert torch.equal(again, b["out"])
            _check_quant(b["out"].cpu(), b["q"], b["scale"])


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32, torch.int8), ids=_name)
@pytest.mark.parametrize("H", [1, 5, 15, 16, 17, 31, 33, 47, 100, 523])
def test_rows_at_every_alignment(H, dtype):
    """Matrices that start at every element behind a 16-byte boundary, with NaN (or other levels) around every row: what
    is read beside a row is not used, what lies beside it is not written."""
    T, k, n_experts = 9, 3, 4
    ids = _ids(T, k, n_experts, H)
    _, rr = _sort_ref(ids, n_experts)
    row_of, fill = torch.from_numpy(rr).cuda(), float("nan") if dtype != torch.int8 else 99
    size = torch.empty(0, dtype=dtype).element_size()
    x, y = _rand((T, H), dtype, 1), _rand((T * k, H), dtype, 2)
    w = torch.rand(T, k, generator=torch.Generator().manual_seed(4))
    for shift in range(16 // size):
        for pitch in (H, H + 1, H + 3):
            rows = _laid_out(torch.full((T * k, H), 7, dtype=dtype), pitch, shift, fill=55)
            E.moe_dispatch(_laid_out(x, pitch, 16 // size - 1 - shift, fill=fill), ids.cuda(), n_experts, rows,
                           torch.empty(n_experts + 1, dtype=torch.int32, device="cuda"), torch.empty(T, k, dtype=torch.int32, device="cuda"))
            want = torch.full((T * k, H), 7, dtype=dtype)
            t, j = np.nonzero(rr >= 0)
            want[torch.from_numpy(rr[t, j].astype(np.int64))] = x[torch.from_numpy(t)]
            assert torch.equal(rows.cpu(), want)
            beside = rows._base.clone()
            beside[shift:].view(T * k, pitch)[:, :H] = 55
            assert bool((beside == 55).all())
            if dtype == torch.int8:
                continue
            yd, out = _laid_out(y, pitch, shift, fill=fill), _laid_out(torch.zeros(T, H, dtype=dtype), pitch, (shift + 1) % 4, fill=55)
            E.moe_combine(yd, w.cuda(), row_of, out)
            yt, there = _taken(y, torch.from_numpy(rr))
            w64 = np.where(there, _f64(w), 0.0)
            ref, mag = (yt * w64[..., None]).sum(1), (np.abs(yt) * w64[..., None]).sum(1)
            assert (np.abs(_f64(out) - ref) <= (k + 1) * 2.0 ** -24 * mag * 1.01 + _half_step(dtype) * np.abs(ref) + TINY[dtype]).all()
            g = _rand((T, H), dtype, 3)
            dy, dw = _laid_out(torch.full((T * k, H), 9.0, dtype=dtype), pitch, shift, fill=55), torch.empty(T, k, device="cuda")
            E.moe_combine_bwd(_laid_out(g, pitch, (shift + 2) % 4, fill=fill), yd, w.cuda(), row_of, dy, dw)
            want = np.full((T * k, H), 9.0)
            want[rr[there]] = (w64[..., None] * _f64(g)[:, None])[there]
            assert (np.abs(_f64(dy) - want) <= (2.0 ** -24 + _half_step(dtype)) * 1.01 * np.abs(want) + TINY[dtype]).all()
            dot, mag = np.einsum("th,tkh->tk", _f64(g), yt), np.einsum("th,tkh->tk", np.abs(_f64(g)), np.abs(yt))
            assert (np.abs(_f64(dw) - dot) <= H * 2.0 ** -24 * mag * 1.01).all()
            beside = dy._base.clone()
            beside[shift:].view(T * k, pitch)[:, :H] = 55
            assert bool((beside == 55).all())
