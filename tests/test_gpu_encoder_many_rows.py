"""GPU tests of the norm and the quantizer at more rows than one launch takes threads for."""
import pytest
import torch

import paper_2211_00839_amd as rcd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d", [((1 << 26) + 5, 8), ((1 << 24) + 3, 1032)])
def test_every_row_is_served(rows, d):
    """Rows of a wave each and of a workgroup each: the same bits as the rows a few at a time."""
    free, _ = torch.cuda.mem_get_info()
    if free < 3 * rows * d * 2:
        pytest.skip("the device has no room for three matrices of %d x %d" % (rows, d))
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    step = 1 << 21

    def pieces():
        print(rows, d, flush=True)
        return [(i, min(i + step, rows)) for i in range(0, rows, step)]

    n = rcd.rms_norm(x, want_rstd=True)
    for i, j in pieces():
        few = rcd.rms_norm(x[i:j], want_rstd=True)
        assert torch.equal(n.y[i:j], few.y) and torch.equal(n.rstd[i:j], few.rstd), (i, j)
    del n, few
    q, scale = rcd.quantize_mxfp8(x)
    for i, j in pieces():
        few_q, few_scale = rcd.quantize_mxfp8(x[i:j])
        assert torch.equal(q[i:j].view(torch.uint8), few_q.view(torch.uint8)), (i, j)
        assert torch.equal(scale[i:j].view(torch.uint8), few_scale.view(torch.uint8)), (i, j)
    del x, q, scale
    torch.cuda.empty_cache()
