"""The block product tile by tile on the GPU: small integers, whose sums are exact in any order, so
that Y has to be the integer result bit by bit, at sizes whose plan is asserted."""
import pytest
import torch

from paper_2609_33496_amd import cham

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def case(msg):
    print(f"[case] {msg}", flush=True)


def _integers(M, N, K, pow2):
    """Codes of -2 .. 2, scales of 1/2 .. 2, and the exact Y (float64)."""
    g = torch.Generator(device=DEV).manual_seed(M + 3 * N + 7 * K)
    nb = -(-K // 128)

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi + 1, shape, generator=g, device=DEV)
    x, w = ints(-2, 2, M, K), ints(-2, 2, N, K)
    ex, ew = ints(-1, 1, nb, M), ints(-1, 1, -(-N // 128), nb)

    def codes(v):
        return v.float().to(torch.float8_e4m3fn).view(torch.uint8)

    def held(e):
        return (e + 127).to(torch.uint8) if pow2 else torch.exp2(e.float())
    xs = x.double() * torch.exp2(ex.double()).t().repeat_interleave(128, 1)[:, :K]
    ws = w.double() * torch.exp2(ew.double()).repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    return cham.BQ(M, K, codes(x), held(ex)), cham.BW(N, K, codes(w), held(ew)), xs @ ws.t().contiguous()


def _check(M, N, K, dt, pow2, plan):
    assert cham.block_linear_plan(M, N, K, dt) == plan
    case(f"integers M={M} N={N} K={K} {dt} pow2={pow2} plan={plan}")
    xb, wb, y = _integers(M, N, K, pow2)
    assert torch.equal(cham.block_linear(xb, wb, dtype=dt), y.to(dt))


# one row and one channel in the last tiles, and fewer steps than the pipeline has stages where a
# plan has them: the loads past the last step go furthest past the last tile's end
ENDS = [(BF16, 33, 1409, 32, (32, 64, 1)), (BF16, 33, 8193, 1024, (32, 64, 1)), (BF16, 33, 1409, 1056, (32, 64, 2)),
        (BF16, 4097, 65, 32, (64, 64, 1)), (BF16, 65, 7745, 1024, (64, 64, 1)), (BF16, 4097, 65, 1760, (64, 64, 2)),
        (BF16, 65, 7233, 1280, (64, 64, 2)), (BF16, 257, 9857, 32, (128, 128, 1)), (BF16, 129, 14977, 800, (128, 128, 1)),
        (BF16, 11777, 769, 544, (256, 192, 1)), (BF16, 257, 23041, 800, (256, 192, 1)), (BF16, 769, 15105, 32, (256, 256, 1)),
        (BF16, 257, 24577, 1024, (256, 256, 1)), (F16, 33, 1409, 32, (32, 64, 1)), (F16, 769, 15105, 32, (256, 256, 1)),
        (F32, 33, 1409, 32, (32, 64, 1)), (F32, 33, 1409, 1248, (32, 64, 2)), (F32, 4097, 65, 32, (64, 64, 1)),
        (F32, 4097, 65, 1760, (64, 64, 2)), (F32, 193, 14081, 32, (64, 128, 1)), (F32, 129, 16385, 800, (64, 128, 1))]


@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("dt,M,N,K,plan", ENDS)
def test_last_tiles_of_one_row_and_one_channel(dt, M, N, K, plan, pow2):
    assert M % plan[0] == 1 and N % plan[1] == 1
    _check(M, N, K, dt, pow2, plan)
