"""What the sums of a block product keep: a block's 128 products in 32 bits, and a result's independence of what lies beside it."""
import pytest

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")

from test_gpu_block8 import DT, E4M3, _matmul, _product, _real_case, _up  # noqa: E402

pytestmark = pytest.mark.gpu

# the kernel for few rows; tiles, one and three of 128 rows high, their channels cut among a cluster; pairs
SIZES = [(5, 300), (40, 300), (333, 300), (2500, 2600)]


@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("up,down", [(0, 1), (0, 127), (40, 100), (100, 3), (8, 24), (31, 32), (63, 95), (127, 64)])
def test_a_blocks_sum_has_32_bits(M, N, up, down):
    """In each block the products 448 * 448 and -448 * 448 stand at two places (of one instruction of 32 channels or of two, in either
    order) among whole multiples of 2^-6: every partial sum, in any order, is a multiple of 2^-6 below 448^2 + 126 * 36 < 2^18 in size,
    so that 24 bits hold it, 23 do not, and the small terms are what is left (below 2^13). A result's three blocks have equal scales, of
    1/4 to 1: their sum, below 2^14 in multiples of 2^-8, is exact too, and the result is the exact sum rounded once."""
    gen = torch.Generator(device="cuda").manual_seed(M + up)
    K = 384
    sizes = torch.tensor([0.0, 0.125, -0.125, 0.25, -0.375, 1.0, -1.0, 1.5, 6.0, -6.0], device="cuda")      # products: multiples of 2^-6
    make = lambda R: sizes[torch.randint(0, len(sizes), (R, K), generator=gen, device="cuda")]  # noqa: E731
    x, w = make(M), make(N)
    for b in range(0, K, 128):
        x[:, b + up], x[:, b + down] = 448.0, -448.0
        w[:, b + up] = w[:, b + down] = 448.0
    x, w = x.to(E4M3), w.to(E4M3)
    power = lambda R: torch.exp2(torch.randint(-1, 1, (R, 1), generator=gen, device="cuda").float()).expand(R, K // 128).contiguous()  # noqa: E731
    xs, ws = power(M), power(_up(N, 128))
    want, _ = _product(x, xs, w, ws)
    assert want.abs().max() < 2 ** 14 and (want != 0).any()
    for dtype in ("bf16", "fp16"):
        assert torch.equal(_matmul(x, xs, w, ws, dtype), want.to(DT[dtype]))
    assert cg.get_status() == 0


@pytest.mark.parametrize("M", [3, 60, 300, 2500])
def test_a_column_does_not_depend_on_the_others(M):
    """The same rows of w among others of NaN codes, and blocks of 128 of them among others of NaN scales, give the same bits: at the
    edges of the kernels' tiles (16, 128 and 256 columns) and inside them."""
    N, K = 2600, 528
    x, xs, w, ws = _real_case(M, N, K)
    want = _matmul(x, xs, w, ws)
    n = torch.arange(N, device="cuda")
    for keep in (n % 3 == 0, (n % 128 == 127) | (n % 128 == 0), n % 16 < 2):
        v = w.clone()
        v.view(torch.uint8)[~keep] = 0x7f
        got = _matmul(x, xs, v, ws)
        assert torch.equal(got[:, keep], want[:, keep]) and torch.isnan(got[:, ~keep]).all()
    block = torch.arange(_up(N, 128), device="cuda")
    for keep in (block % 2 == 0, block % 2 == 1, block % 5 == 4):
        vs = ws.clone()
        vs[~keep] = float("nan")
        got, cols = _matmul(x, xs, w, vs), keep[n // 128]
        assert torch.equal(got[:, cols], want[:, cols]) and torch.isnan(got[:, ~cols]).all()


@pytest.mark.parametrize("M", [3, 60, 300, 2500])
def test_a_row_does_not_depend_on_the_others_scales(M):
    """The rows of x that hold a NaN scale among the others, at either end of the warps' and tiles' rows."""
    N, K = 2600, 528
    x, xs, w, ws = _real_case(M, N, K)
    want = _matmul(x, xs, w, ws)
    m = torch.arange(M, device="cuda")
    for keep in (m % 2 == 0, m % 32 == 31 if M > 32 else m == 1, (m % 128 == 0) | (m == M - 1)):
        vs = xs.clone()
        vs[~keep] = float("nan")
        got = _matmul(x, vs, w, ws)
        assert torch.equal(got[keep], want[keep]) and torch.isnan(got[~keep]).all()
