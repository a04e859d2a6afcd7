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


# a plan's k-steps, one count after the other: every exit of the six-step loop, whole and ragged last
# blocks, odd and even counts of blocks where two groups of wavefronts share them
STEPS = [(BF16, (32, 64, 1), 33, 1409, range(1, 8)), (BF16, (32, 64, 1), 33, 8193, [8]),
         (BF16, (32, 64, 2), 33, 1409, range(9, 21)), (BF16, (64, 64, 1), 4097, 65, range(1, 6)),
         (BF16, (64, 64, 1), 4801, 65, [6]), (BF16, (64, 64, 1), 3585, 129, [7]), (BF16, (64, 64, 1), 65, 7745, [8]),
         (BF16, (64, 64, 2), 4097, 65, range(15, 28)), (BF16, (128, 128, 1), 257, 9857, range(1, 6)),
         (BF16, (128, 128, 1), 129, 16129, [6]), (BF16, (128, 128, 1), 129, 14977, [7]), (BF16, (128, 128, 1), 129, 13953, [8]),
         (BF16, (256, 192, 1), 11777, 769, [5]), (BF16, (256, 192, 1), 18689, 385, [6]), (BF16, (256, 192, 1), 257, 23041, [7, 8, 9]),
         (BF16, (256, 192, 1), 257, 22273, [10]), (BF16, (256, 192, 1), 257, 21889, [11, 12]),
         (BF16, (256, 256, 1), 769, 15105, [1]), (BF16, (256, 256, 1), 513, 19969, range(2, 6)),
         (BF16, (256, 256, 1), 257, 29441, [6]), (BF16, (256, 256, 1), 257, 26369, [7]), (BF16, (256, 256, 1), 257, 24577, [8]),
         (F32, (32, 64, 1), 33, 1409, range(1, 8)), (F32, (32, 64, 2), 33, 1409, range(11, 23)),
         (F32, (64, 64, 1), 4097, 65, range(1, 6)), (F32, (64, 64, 1), 4929, 257, [6, 7, 8]),
         (F32, (64, 64, 2), 4097, 65, range(19, 31)), (F32, (64, 128, 1), 193, 14081, range(1, 5)),
         (F32, (64, 128, 1), 129, 16385, range(5, 9))]


@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("dt,plan,M,N,blocks", STEPS)
def test_every_count_of_steps(dt, plan, M, N, blocks, pow2):
    for n in blocks:
        K = n * 128 - (96 if n % 2 else 32 if n >= 16 else 0)
        _check(M, N, K, dt, pow2, plan)


CODES = [(BF16, 33, 1409, 160, (32, 64, 1)), (BF16, 33, 1409, 1056, (32, 64, 2)), (BF16, 4097, 65, 160, (64, 64, 1)),
         (BF16, 4097, 65, 1824, (64, 64, 2)), (BF16, 257, 9857, 160, (128, 128, 1)), (BF16, 11777, 769, 544, (256, 192, 1)),
         (BF16, 513, 19713, 288, (256, 256, 1)), (F16, 257, 9857, 160, (128, 128, 1)), (F16, 513, 19713, 288, (256, 256, 1)),
         (F32, 33, 1409, 160, (32, 64, 1)), (F32, 33, 1409, 1248, (32, 64, 2)), (F32, 4097, 65, 160, (64, 64, 1)),
         (F32, 4097, 65, 2336, (64, 64, 2)), (F32, 193, 14081, 160, (64, 128, 1))]


@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("dt,M,N,K,plan", CODES)
def test_every_code_through_every_tile(dt, M, N, K, plan, pow2):
    """A single E4M3 code in each row against ones: Y is the code's value, as activation and (with
    rows and channels of another count, the same tile) as weight; zeros of either sign are equal."""
    assert cham.block_linear_plan(M, N, K, dt) == plan
    case(f"single codes M={M} N={N} K={K} {dt} pow2={pow2} plan={plan}")
    codes = torch.tensor([c for c in range(256) if c & 127 != 127], dtype=torch.uint8, device=DEV)
    nb = -(-K // 128)

    def scale(*shape):
        return torch.full(shape, 127, dtype=torch.uint8, device=DEV) if pow2 else torch.ones(shape, device=DEV)

    def single(rows, first):
        i = torch.arange(rows, device=DEV)
        a = torch.zeros(rows, K, dtype=torch.uint8, device=DEV)
        c = codes[(i + first) % codes.numel()]
        a[i, (i * 7 + i // 254) % K] = c
        return a, c.view(torch.float8_e4m3fn).to(dt)
    for left in (True, False):
        rows = M if left else N
        for first in range(0, codes.numel(), rows):  # few rows: several calls for all codes
            a, v = single(rows, first)
            one = torch.full((N if left else M, K), 0x38, dtype=torch.uint8, device=DEV)
            xb = cham.BQ(M, K, a if left else one, scale(nb, M))
            wb = cham.BW(N, K, one if left else a, scale(-(-N // 128), nb))
            Y = cham.block_linear(xb, wb, dtype=dt)
            assert torch.equal(Y, v[:, None].expand(M, N) if left else v[None, :].expand(M, N)), (left, first)
