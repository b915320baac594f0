"""The parts that the gradients' sums are made of: each CTA writes one, and no more CTAs are launched than the GPU holds at
once, so that none begins its rows when the others end theirs."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2609_11562_b200 import build as B
    B.build()
    from paper_2609_11562_b200 import entwine as E

bf16, fp16, fp32 = torch.bfloat16, torch.float16, torch.float32


# rows that start on 16 bytes' boundaries are copied ahead: three rows of 16-bit elements, two of fp32, and the weights in
# fp32, fit twice into an SM up to 320 threads a row (5120 columns) and 256 (4096); rows that start anywhere are not copied
@pytest.mark.parametrize("dtype,cols,shift,an_sm", [(bf16, 2048, 0, 2), (bf16, 5120, 0, 2), (bf16, 5128, 0, 1), (fp16, 5632, 0, 1), (bf16, 8192, 0, 1),
                                                    (bf16, 12288, 0, 1), (fp32, 1024, 0, 2), (fp32, 4096, 0, 2), (fp32, 4104, 0, 1), (fp32, 5120, 0, 1),
                                                    (fp32, 5632, 0, 1), (fp32, 8192, 0, 1), (fp32, 12288, 0, 1), (bf16, 5121, 1, 2), (fp32, 5120, 1, 2),
                                                    (bf16, 5632, 1, 2), (bf16, 5640, 1, 1)])
def test_as_many_parts_as_ctas_are_resident(dtype, cols, shift, an_sm):
    rows, sms = 1700, torch.cuda.get_device_properties(0).multi_processor_count
    whole = [torch.randn(rows, cols + 8, device="cuda").to(dtype) for _ in range(3)]
    dout, h, dx = (t[:, shift:shift + cols] for t in whole)
    mean, rstd, w = h.float().mean(1), torch.ones(rows, device="cuda"), torch.ones(cols, device="cuda")
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    work = torch.full((E.layer_norm_bwd_work(rows, cols) + 1,), math.nan, device="cuda")
    E.layer_norm_bwd(dout, h, w, mean, rstd, dx, dw, db, work)
    assert math.isnan(float(work[-1]))
    parts = work[:-1].view(-1, 2, cols)
    written = ~torch.isnan(parts).flatten(1).any(1)
    n = int(written.sum())
    assert n == an_sm * sms
    assert bool(written[:n].all()) and bool(torch.isnan(parts[n:]).all())
    assert torch.allclose(parts[:n, 1].double().sum(0), db.double(), rtol=0, atol=rows * 2.0 ** -23 * float(dout.double().abs().sum(0).max()))
