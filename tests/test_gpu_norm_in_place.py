"""The norm written over its inputs in every allowed way, bit for bit as with buffers of its own."""
import pytest
import torch

import paper_2607_20214_amd as E

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 7), (37, 264), (300, 1001), (2, 16384)])
def test_over_inputs(rows, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r, dy, ds = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(4))
    w = torch.randn(cols, generator=g, device="cuda")
    y, s = E.rms_norm_fwd(x, w, residual=r)
    for over_y, over_s in ((0, None), (1, None), (None, 0), (None, 1), (0, 1), (1, 0)):
        t = [x.clone(), r.clone()]
        a, b = E.rms_norm_fwd(t[0], w, residual=t[1], out=None if over_y is None else t[over_y],
                              out_sum=None if over_s is None else t[over_s])
        assert torch.equal(a, y) and torch.equal(b, s)
    dx, dw = E.rms_norm_bwd(s, w, dy, dsum=ds)
    for over in range(3):
        t = [s.clone(), dy.clone(), ds.clone()]
        a, b = E.rms_norm_bwd(t[0], w, t[1], dsum=t[2], out=t[over])
        assert torch.equal(a, dx) and torch.equal(b, dw)
    with pytest.raises(E.ElsaaError):
        E.rms_norm_fwd(x, w, residual=r, out=s, out_sum=s)
