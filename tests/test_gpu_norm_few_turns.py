"""The norms' backward pass over few rows: every CTA that is launched has rows of its own.  Seen in the workspace, where each CTA leaves its sums of three
vectors' gradients: with inputs that are not zero, sums of zeros are those of a CTA that had nothing to do."""
import ctypes

import pytest
import torch


def sb():
    import __graft_entry__ as ge
    ge.build()
    from paper_2112_15317_b200 import binding as b
    return b


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d,bf16", [(8, 4096, True), (100, 512, True), (100, 512, False), (37, 130, True), (999, 1001, False), (3, 8192, False), (700, 2048, True)])
def test_no_cta_without_rows(rows, d, bf16):
    b = sb()
    dt = torch.bfloat16 if bf16 else torch.float32
    g = torch.Generator().manual_seed(rows)
    x, f, dy, dn = ((0.5 + torch.rand(rows, d, generator=g)).to(dt).cuda() for _ in range(4))
    w_pre, w_post, scale = ((0.5 + torch.rand(d, generator=g)).cuda() for _ in range(3))
    _, _, stats = b.norm_forward(x, w_pre, f, w_post, None, scale, save=True)
    cfg = b.sb_norm_config(rows, 0, d, b.SB_NORM_RMS, b.SB_BF16 if bf16 else b.SB_FP32, 1e-6)
    size = ctypes.c_size_t()
    assert b.sb_norm_bytes(ctypes.byref(cfg), ctypes.byref(size)) == 0
    ws = torch.full((size.value // 4,), 7.0, device="cuda")
    dx, df = torch.empty_like(x), torch.empty_like(x)
    out = [torch.empty(d, device="cuda") for _ in range(3)]
    assert b.sb_norm_backward(ctypes.byref(cfg), *(t.data_ptr() for t in (dy, dn, stats, x, w_pre, f, w_post)), None, scale.data_ptr(), dx.data_ptr(), df.data_ptr(),
                              out[0].data_ptr(), out[1].data_ptr(), None, out[2].data_ptr(), ws.data_ptr(), size.value, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    parts = ws[:ws.numel() // (3 * d) * 3 * d].view(-1, 3, d)
    parts = parts[(parts != 7.0).any(2).all(1)]                          # those of CTAs that were launched
    assert len(parts) > 0 and (parts != 0).any(2).all()
    for k in range(3):                                                   # (and they add up: float sums in another order)
        assert torch.allclose(parts[:, k].double().sum(0), out[k].double(), rtol=1e-5, atol=1e-6 * rows)
