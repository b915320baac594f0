"""The 4-bit product of experts with more rows than 32 bits hold four times."""
import pytest
import torch

import mxf4_reference as R

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E


@pytest.mark.parametrize("rows,G", [((1 << 30) + 70, 2), ((1 << 30) - 70, 2)])
def test_two_experts_of_half_a_billion_rows(rows, G):
    """16 bytes of codes and 4 of scales a row: 17 and 4 GB.  The experts own the last rows only; the others stay as they were."""
    K, N = 32, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    a, sa = torch.empty(rows, 16, dtype=torch.uint8, device="cuda"), torch.empty(rows, 4, dtype=torch.uint8, device="cuda")[:, :1]
    last = 1000
    a[-last:] = torch.randint(0, 256, (last, 16), generator=g, device="cuda", dtype=torch.uint8)
    sa[-last:] = torch.randint(125, 130, (last, 1), generator=g, device="cuda", dtype=torch.uint8)
    b = torch.randint(0, 256, (G, N, 16), generator=g, device="cuda", dtype=torch.uint8)
    sb = torch.full((G, N, 4), 127, device="cuda", dtype=torch.uint8)[:, :, :1]
    out = torch.full((rows, N), 9.0, dtype=torch.bfloat16, device="cuda")
    off = [rows - last + 7, rows - 300, rows]
    E.gemm_mxf4_grouped(a, sa, b, sb, torch.tensor(off, dtype=torch.int32, device="cuda"), out)
    E.ops_status()
    assert bool((out[:off[0]] == 9.0).all())
    for e in range(G):
        at = slice(off[e] - rows, off[e + 1] - rows or None)
        u, v = (torch.from_numpy(R.decode(q.cpu().numpy(), s.cpu().numpy(), K)).cuda() for q, s in ((a[at], sa[at]), (b[e], sb[e])))
        assert torch.equal(out[at], (u @ v.T).bfloat16())  # (multiples of 1/16 below 2^13: exact in fp32)
