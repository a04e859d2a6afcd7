"""The norm and the gate in every activation format straight into the mixed-format linear layer, on the
GPU against 64-bit sums of the decoded codes."""
import math

import pytest
import torch

from paper_2609_33496_amd import cham

pytestmark = pytest.mark.gpu
DEV = "cuda"
FMT = {"int8": cham.A_INT8_ASYM, "e4m3": cham.A_FP8_E4M3, "e5m2": cham.A_FP8_E5M2, "mxfp8": cham.A_MXFP8,
       "mxint8": cham.A_MXINT8}


def _x(seed, M, K, dt=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(M, K, generator=g) * torch.randn(M, K, generator=g).abs().clamp(min=0.3) * scale).to(dt)


def _values(q, fmt):
    """What q's codes stand for, in 64 bits."""
    c = q.codes.cpu()
    if fmt == "int8":
        return (c.double() - q.zero.cpu().double()[:, None]) * q.scale.cpu().double()[:, None]
    if fmt in ("e4m3", "e5m2"):
        return c.view(torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2).double() * q.scale.cpu().double()[:, None]
    s = torch.exp2(q.e8m0.cpu().double() - 127.0).repeat_interleave(32, 1)
    return c.view(torch.float8_e4m3fn).double() * s if fmt == "mxfp8" else c.view(torch.int8).double() / 64.0 * s


def _run(op, x, fmt):
    if op == "norm":
        return cham.rms_norm_quantize(x, fmt=FMT[fmt])[0]
    if op == "gate":
        return cham.gated_quantize(x, None, cham.ACT_GELU_TANH, fmt=FMT[fmt])
    return cham.gated_quantize(x, x, cham.ACT_SILU, fmt=FMT[fmt])


@pytest.mark.parametrize("op", ["norm", "gate", "gated"])
@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("M,N,K", [(1, 96, 640), (77, 130, 1152), (600, 320, 2112)])
def test_each_format_into_the_linear_layer(op, fmt, M, N, K):
    """The layer's own bound: 1e-3 of the sum of magnitudes."""
    print(f"[case] {op} {fmt} M={M} N={N} K={K}", flush=True)
    wq = cham.select_weight_formats(_x(22, N, K, torch.float32, 0.02).to(DEV), 1 << cham.W_INT8_SYM)
    q = _run(op, _x(21, M, K, torch.bfloat16).to(DEV), fmt)
    Y = cham.mixed_linear(q, wq).cpu().double()
    v = _values(q, fmt)
    w = wq.codes.cpu().view(torch.int8).double() * wq.scale.cpu().double()[:, None]
    assert bool(((Y - v @ w.t()).abs() <= 1e-3 * (v.abs() @ w.abs().t())).all())


@pytest.mark.parametrize("op", ["norm", "gate", "gated"])
@pytest.mark.parametrize("fmt", FMT)
def test_a_row_of_no_numbers_stays_a_row(op, fmt):
    """A NaN in a row's input makes that row of Y NaN and leaves the others' bits."""
    M, N, K = 40, 96, 640
    print(f"[case] NaN row {op} {fmt}", flush=True)
    x = _x(31, M, K, torch.float16)
    wq = cham.select_weight_formats(_x(32, N, K, torch.float32, 0.02).to(DEV))
    clean = cham.mixed_linear(_run(op, x.to(DEV), fmt), wq)
    x[17, 333] = math.nan
    Y = cham.mixed_linear(_run(op, x.to(DEV), fmt), wq)
    keep = [m for m in range(M) if m != 17]
    assert bool(torch.isnan(Y[17]).all())
    assert torch.equal(Y[keep], clean[keep])
