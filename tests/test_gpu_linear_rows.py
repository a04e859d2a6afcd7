"""The mixed-format linear layer and the convolution on the GPU with few rows in the last tile: nothing
is written past Y, and Y is right."""
import pytest
import torch

from paper_2609_33496_amd import cham

pytestmark = pytest.mark.gpu
DEV = "cuda"
FMT = {"int8": cham.A_INT8_ASYM, "e4m3": cham.A_FP8_E4M3, "mxint8": cham.A_MXINT8}


def _x(seed, M, K, scale=1.0):
    return torch.randn(M, K, generator=torch.Generator().manual_seed(seed)) * scale


def _values(q, fmt):
    c = q.codes.cpu()
    if fmt == "int8":
        return (c.double() - q.zero.cpu().double()[:, None]) * q.scale.cpu().double()[:, None]
    if fmt == "e4m3":
        return c.view(torch.float8_e4m3fn).double() * q.scale.cpu().double()[:, None]
    return c.view(torch.int8).double() / 64.0 * torch.exp2(q.e8m0.cpu().double() - 127.0).repeat_interleave(32, 1)


def _into(M, N):
    """Y [M, N] in front of 200 more rows that must stay as they are."""
    buf = torch.full(((M + 200) * N,), 7.0, device=DEV)
    return buf, buf[:M * N].view(M, N)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("M", [1, 2, 5, 27, 28, 33, 65, 92, 97, 129, 130, 257, 1025])
def test_nothing_past_the_last_row(fmt, M):
    for N, K in ((96, 640), (100, 640), (64, 8192), (1283, 320)):
        print(f"[case] rows {fmt} M={M} N={N} K={K} plan={cham.linear_plan(M, N, K, 8)}", flush=True)
        wq = cham.select_weight_formats(_x(N, N, K, 0.02).to(DEV), 1 << cham.W_INT8_SYM)
        q = cham.gated_quantize(_x(M, M, K).to(DEV), None, cham.ACT_NONE, fmt=FMT[fmt])
        buf, Y = _into(M, N)
        cham.mixed_linear(q, wq, Y)
        assert bool((buf[M * N:] == 7.0).all())
        v = _values(q, fmt)
        w = wq.codes.cpu().view(torch.int8).double() * wq.scale.cpu().double()[:, None]
        assert bool(((Y.cpu().double() - v @ w.t()).abs() <= 1e-3 * (v.abs() @ w.abs().t())).all())


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("H,W", [(1, 1), (3, 9), (5, 13), (1, 129)])
def test_nothing_past_the_last_pixel(fmt, H, W):
    C, N = 64, 96
    print(f"[case] pixels {fmt} H={H} W={W}", flush=True)
    wq = cham.select_weight_formats(_x(N, N, 9 * C, 0.02).to(DEV), 1 << cham.W_INT8_SYM)
    q = cham.quantize_act(_x(H * W, H * W, C).to(DEV), FMT[fmt], dynamic=True)
    buf, Y = _into(H * W, N)
    cham.conv3x3_mixed(q, 1, H, W, wq, Y)
    assert bool((buf[H * W * N:] == 7.0).all())
    assert torch.equal(Y, cham.conv3x3_mixed(q, 1, H, W, wq).view(H * W, N))
