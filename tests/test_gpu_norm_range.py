"""The norm over the whole range of its types on the GPU, against 64 bits."""
import pytest
import torch

from paper_2609_33496_amd import cham

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24  # half a binary32 step
# h, the factor, its product with h and the product with g: one rounding each; h's rounding moves
# the mean by as much again
REL = 5 * U


def case(msg):
    print(f"[case] {msg}", flush=True)


def _rows(seed, M, K, dt, size):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K, generator=g).clamp(-3.0, 3.0)
    return (x.double() * size).to(dt)


def _check(q, y):
    """Scales within REL and the two roundings of amax / 448; codes within half a step (2^-4 of a
    value, 2^-10 of the scale below the format's least exponent)."""
    M, K = y.shape
    nb = -(-K // 128)
    p = torch.zeros(M, nb * 128, dtype=torch.float64)
    p[:, :K] = y
    want = (p.view(M, nb, 128).abs().amax(2) / 448.0).clamp(min=2.0 ** -126)
    s = q.scale.cpu().double().t()
    assert float(((s - want).abs() / want).max()) <= REL + 2 * U
    s = s.repeat_interleave(128, 1)[:, :K]
    v = q.codes.cpu().view(torch.float8_e4m3fn).double() * s
    assert bool(((v - y).abs() <= (2.0 ** -4 + 1e-5) * y.abs() + 2.0 ** -10 * s).all())


@pytest.mark.parametrize("dt,size", [(torch.float32, s) for s in (1e19, 3e25, 1e38, 1e-19, 1e-24, 1e-30, 1e-38, 1e-41, 1.0)] +
                         [(torch.bfloat16, s) for s in (1e19, 1e38, 1e-24, 1e-37)] +
                         [(torch.float16, s) for s in (2e4, 1e-4, 1e-7)])
@pytest.mark.parametrize("M,K", [(5, 160), (4, 1152), (3, 2080), (2, 16384), (700, 640)])
def test_rows_of_any_size(dt, size, M, K):
    """With eps = 0 each row comes out with a mean square of 1, from the largest numbers of its type
    to subnormal ones."""
    case(f"norm range {dt} size={size} M={M} K={K}")
    x = _rows(K + M, M, K, dt, size)
    q, _ = cham.rms_norm_quantize(x.to(DEV), None, 0.0)
    h = x.double()
    _check(q, h / torch.sqrt(h.square().mean(1, keepdim=True)))


@pytest.mark.parametrize("size", [1e19, 1e37, 1.0, 1e-24])
@pytest.mark.parametrize("M,K", [(3, 320), (2, 5120), (600, 1152)])
def test_rows_of_any_size_with_residual_and_weights(size, M, K):
    case(f"norm range residual size={size} M={M} K={K}")
    x, r = _rows(1, M, K, torch.bfloat16, size), _rows(2, M, K, torch.float32, size)
    g = 1.0 + 0.2 * _rows(3, 1, K, torch.float32, 1.0)[0]
    q, out = cham.rms_norm_quantize(x.to(DEV), g.to(DEV), 0.0, residual=r.to(DEV))
    assert torch.equal(out.cpu(), x.float() + r)
    h = x.double() + r.double()
    _check(q, h / torch.sqrt(h.square().mean(1, keepdim=True)) * g.double())


def test_one_row_beside_others_of_another_size():
    """A huge row, a tiny one, zeros and an ordinary one in one call, eps = 1e-6."""
    case("norm range mixed rows")
    K = 768
    x = torch.cat([_rows(1, 1, K, torch.float32, s) for s in (1e30, 1e-30, 0.0, 1.0)])
    q, _ = cham.rms_norm_quantize(x.to(DEV), None, 1e-6)
    h = x.double()
    _check(q, h / torch.sqrt(h.square().mean(1, keepdim=True) + float(torch.tensor(1e-6))))
