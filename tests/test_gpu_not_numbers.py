"""NaN and infinities through the operators in front of 8-bit linear layers and the layers that
read their outputs: what held one is NaN, everything else is untouched."""
import math

import pytest
import torch

from paper_2609_33496_amd import cham

pytestmark = pytest.mark.gpu
DEV = "cuda"
FMT = {"mxfp8": cham.A_MXFP8, "mxint8": cham.A_MXINT8}
BAD = [math.nan, math.inf, -math.inf]


def case(msg):
    print(f"[case] {msg}", flush=True)


def _x(seed, M, K, dt=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(M, K, generator=g).to(dt)


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("M,K", [(6, 640), (3, 2080), (5, 8224)])
def test_mx_blocks_that_hold_one_take_the_scale_nan(fmt, bad, M, K):
    """Byte 255 for that block of 32 (MXFP8: codes that are NaN too), the others as without it."""
    case(f"MX gate {fmt} {bad} M={M} K={K}")
    x = _x(1, M, K, torch.float16)
    clean = cham.gated_quantize(x.to(DEV), None, cham.ACT_NONE, fmt=FMT[fmt])
    x[1, 100], x[2, K - 1] = bad, bad
    q = cham.gated_quantize(x.to(DEV), None, cham.ACT_NONE, fmt=FMT[fmt])
    hit = torch.zeros(M, K // 32, dtype=torch.bool)
    hit[1, 3] = hit[2, -1] = True
    assert torch.equal(q.e8m0.cpu() == 255, hit)
    assert torch.equal(q.e8m0.cpu()[~hit], clean.e8m0.cpu()[~hit])
    keep = ~hit.repeat_interleave(32, 1)
    assert torch.equal(q.codes.cpu()[keep], clean.codes.cpu()[keep])
    if fmt == "mxfp8":
        assert bool(torch.isnan(q.codes.cpu().view(torch.float8_e4m3fn).float())[~keep].all())


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("fmt", FMT)
def test_mx_norm_of_a_row_that_holds_one(fmt, bad):
    """A NaN makes its whole row NaN; beside an infinity, which is NaN itself, the row's elements are
    h / infinity = 0."""
    M, K = 5, 640
    case(f"MX norm {fmt} {bad}")
    x = _x(2, M, K, torch.bfloat16)
    clean, _ = cham.rms_norm_quantize(x.to(DEV), fmt=FMT[fmt])
    x[3, 77] = bad
    q, _ = cham.rms_norm_quantize(x.to(DEV), fmt=FMT[fmt])
    keep = [0, 1, 2, 4]
    assert torch.equal(q.codes[keep], clean.codes[keep]) and torch.equal(q.e8m0[keep], clean.e8m0[keep])
    nan = q.e8m0[3].cpu() == 255
    assert bool(nan.all()) if math.isnan(bad) else nan.tolist() == [i == 2 for i in range(K // 32)]


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("M,N,K", [(5, 96, 640), (77, 200, 2112), (300, 1280, 640), (2, 64, 16384)])
def test_mx_blocks_of_no_numbers_in_the_linear_layer(fmt, M, N, K):
    """Their rows of Y are NaN, whatever the weights; the other rows keep their bits."""
    case(f"MX linear {fmt} M={M} N={N} K={K}")
    x = _x(3, M, K)
    W = _x(4, N, K).to(DEV) * 0.02
    W[3] = 0.0
    wq = cham.select_weight_formats(W, 1 << cham.W_INT8_SYM)
    clean = cham.mixed_linear(cham.gated_quantize(x.to(DEV), None, cham.ACT_NONE, fmt=FMT[fmt]), wq)
    x[1, K - 40] = math.inf
    Y = cham.mixed_linear(cham.gated_quantize(x.to(DEV), None, cham.ACT_NONE, fmt=FMT[fmt]), wq)
    keep = [m for m in range(M) if m != 1]
    assert bool(torch.isnan(Y[1]).all())
    assert torch.equal(Y[keep], clean[keep])


@pytest.mark.parametrize("fmt", FMT)
def test_mx_blocks_of_no_numbers_in_the_convolution(fmt):
    """NaN at the pixel and its neighbours alone; elsewhere the bits of the same layer with zeros in
    that block."""
    B, H, W, C, N = 1, 9, 20, 64, 96
    case(f"MX conv {fmt}")
    x = _x(5, B * H * W, C)
    wq = cham.select_weight_formats(_x(6, N, 9 * C).to(DEV) * 0.02, 1 << cham.W_INT8_SYM)
    at = 4 * W + 7
    zero = x.clone()
    zero[at, 32:] = 0.0
    x[at, 50] = math.nan
    q = [cham.gated_quantize(v.to(DEV), None, cham.ACT_NONE, fmt=FMT[fmt]) for v in (zero, x)]
    for v in q:
        v.nsamples = 1  # the convolution's samples are whole images (MX formats have no scale per sample)
    clean, Y = (cham.conv3x3_mixed(v, B, H, W, wq) for v in q)
    near = torch.zeros(H, W, dtype=torch.bool)
    near[3:6, 6:9] = True
    near = near.flatten().to(DEV)
    Y, clean = Y.reshape(H * W, N), clean.reshape(H * W, N)
    assert bool(torch.isnan(Y[near]).all())
    assert torch.equal(Y[~near], clean[~near])


@pytest.mark.parametrize("fmt", FMT)
def test_the_byte_255_is_nan_whatever_codes_lie_under_it(fmt):
    """As another program may write it: finite codes under the scale NaN, in the linear layer and in
    the convolution, and a split of k that does not hold the block."""
    case(f"byte 255 {fmt}")
    M, N, K = 40, 96, 16384
    x = cham.gated_quantize(_x(7, M, K).to(DEV), None, cham.ACT_NONE, fmt=FMT[fmt])
    wq = cham.select_weight_formats(_x(8, N, K).to(DEV) * 0.02, 1 << cham.W_INT8_SYM)
    clean = cham.mixed_linear(x, wq)
    x.e8m0[9, 3] = 255
    x.codes[9, 96:128] = 0
    Y = cham.mixed_linear(x, wq)
    keep = [m for m in range(M) if m != 9]
    assert bool(torch.isnan(Y[9]).all()) and torch.equal(Y[keep], clean[keep])
    B, H, W, C = 1, 6, 7, 64
    x = cham.gated_quantize(_x(9, B * H * W, C).to(DEV), None, cham.ACT_NONE, fmt=FMT[fmt])
    x.nsamples = 1
    wq = cham.select_weight_formats(_x(10, N, 9 * C).to(DEV) * 0.02, 1 << cham.W_INT8_SYM)
    top = torch.arange(B * H * W, device=DEV)[x.e8m0[:, 1] < x.e8m0.max()][0].item()  # a block that is not the largest
    clean = cham.conv3x3_mixed(x, B, H, W, wq).reshape(H * W, N)
    x.e8m0[top, 1] = 255
    x.codes[top, 32:64] = 0  # a block of nothing but zeros is NaN under it too
    Y = cham.conv3x3_mixed(x, B, H, W, wq).reshape(H * W, N)
    r, c = torch.arange(H * W, device=DEV) // W, torch.arange(H * W, device=DEV) % W
    near = ((r - top // W).abs() <= 1) & ((c - top % W).abs() <= 1)
    assert bool(torch.isnan(Y[near]).all()) and torch.equal(Y[~near], clean[~near])
