"""8-bit block matrices on the GPU against plain forms: the encoding, whose roundings are given, is equal bit for bit; the
product is equal where every sum is exact, and otherwise within the bound derived at its test."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
cg = pytest.importorskip("paper_2607_20538_gb300")

pytestmark = pytest.mark.gpu

NONFINITE = 1
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3 = torch.float8_e4m3fn


def _up(n, m):
    return -(-n // m)


def _blocks(x, rows):
    """[row blocks][rows][blocks][128] of a matrix, padded with zeros."""
    R, K = x.shape
    y = torch.zeros(_up(R, rows) * rows, _up(K, 128) * 128, dtype=x.dtype)
    y[:R, :K] = x
    return y.view(_up(R, rows), rows, _up(K, 128), 128)


def _wide(scales, rows, R, K):
    return scales.repeat_interleave(rows, 0)[:R].repeat_interleave(128, 1)[:, :K]


# ------------------------------------------------------------------------------------ encoding
def _encoded(x, rows):
    """Codes (bits) and scales by their definition, each step rounded once in fp32 (on the CPU)."""
    scales = _blocks(x.float().abs(), rows).amax((1, 3)) / torch.tensor(448.0)
    wide = _wide(scales, rows, *x.shape)
    codes = torch.where(wide == 0, torch.zeros(()), x.float() / wide).clamp(-448, 448).to(E4M3)
    return codes.view(torch.uint8), scales


def _encode(x, rows, pad=0):
    R, K = x.shape
    store = torch.full((R, K + pad), float("nan"), dtype=x.dtype, device="cuda")
    store[:, :K] = x.cuda()
    codes = torch.full((R, K + 2 * pad), 77, dtype=torch.uint8, device="cuda")
    scales = torch.full((_up(R, rows), _up(K, 128)), 77.0, device="cuda")
    cg.block8_encode(store[:, :K], codes[:, :K].view(E4M3), scales, rows=rows)
    assert (codes[:, K:] == 77).all()
    return codes[:, :K].cpu(), scales.cpu()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("R,K,pad", [(1, 16, 0), (1, 128, 0), (1, 4096, 0), (2, 144, 8), (3, 112, 16), (127, 272, 0), (128, 128, 0), (129, 1040, 24), (300, 2064, 0)])
def test_encode(dtype, rows, R, K, pad):
    gen = torch.Generator().manual_seed(R * K)
    x = torch.randn(R, K, generator=gen) * torch.exp(3 * torch.randn(R, K, generator=gen))      # many codes below the normal ones
    x[torch.rand(R, K, generator=gen) < 0.05] = 0
    x[: R // 2, : K // 3] *= torch.rand(R // 2, K // 3, generator=gen) < 0.02                  # blocks of zeros and a few values
    x = x.clamp(-60000, 60000).to(DT[dtype])
    codes, scales = _encode(x, rows, pad)
    assert cg.get_status() == 0
    want, ws = _encoded(x, rows)
    assert torch.equal(scales, ws)
    assert torch.equal(codes, want)


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("dtype,sizes", [("bf16", [1e-40, 9.2e-41, 3e-38, 2e-26, 2.6e-22, 3.7e-22, 1e-10, 1.0, 1e30, 5e32, 6e32, 3.3e38]), ("fp16", [6e-8, 1e-5, 1.0, 65504.0])])
def test_encode_at_the_ends_of_the_range(rows, dtype, sizes):
    """Scales below the normal numbers and near the largest; a block of zeros has scale 0 and codes 0, also of -0."""
    gen = torch.Generator().manual_seed(1)
    x = torch.cat([(torch.rand(rows, 128, generator=gen) * 2 - 1).to(torch.float64) * s for s in sizes])
    x[::rows, 5] = torch.tensor(sizes, dtype=torch.float64)
    x = torch.cat([x, torch.full((rows, 128), -0.0, dtype=torch.float64)]).float().to(DT[dtype])
    codes, scales = _encode(x, rows)
    assert cg.get_status() == 0
    want, ws = _encoded(x, rows)
    assert torch.equal(scales, ws) and torch.equal(codes, want) and (codes[-1] == 0).all()


@pytest.mark.parametrize("rows", [1, 128])
def test_encode_of_what_is_not_finite(rows):
    x = torch.randn(3 * rows, 256)
    x[rows, 200], x[2 * rows, 3] = float("inf"), float("nan")
    codes, scales = _encode(x.bfloat16(), rows)
    assert cg.get_status() == NONFINITE
    want, ws = _encoded(x.bfloat16(), rows)
    bad = torch.isnan(scales)
    assert bad.tolist() == [[False, False], [False, True], [True, False]]
    assert torch.equal(scales[~bad], ws[~bad])
    wide = _wide(bad, rows, *x.shape)
    assert torch.isnan(codes.view(E4M3).float()[wide]).all() and torch.equal(codes[~wide], want[~wide])


def test_encode_many_rows():
    x = torch.randn(40000, 144).bfloat16()
    codes, scales = _encode(x, 1)
    want, ws = _encoded(x, 1)
    assert torch.equal(scales, ws) and torch.equal(codes, want)


# ------------------------------------------------------------------------------------ product
SIZES = [(1, 1, 16), (1, 8, 128), (1, 6144, 4096), (2, 130, 144), (5, 1000, 272), (16, 128, 128), (17, 257, 640), (31, 96, 1040), (33, 2000, 4096), (64, 129, 384),
         (65, 128, 128), (65, 7, 2048), (100, 1000, 4112), (127, 200, 48), (128, 640, 1280), (129, 384, 256), (333, 1000, 4112), (500, 8, 512), (1000, 3000, 400),
         (2048, 2560, 512), (2049, 2561, 528), (4097, 1153, 144), (300, 20000, 256), (20000, 300, 128), (16, 40000, 128), (40, 60000, 256), (3, 512, 16384),
         (1, 20000, 1040), (8, 9000, 272), (7, 70, 96), (8, 300, 8208), (9, 300, 400), (24, 130, 2064), (100, 40000, 272), (128, 1000, 1152),
         (20000, 2000, 128), (3000, 3000, 384)]


def _exact_case(M, N, K, seed=0):
    """Codes and scales of few bits: whole numbers up to 6 times powers of two, so that every product and every sum is
    exact in fp32 (up to 36 K 2^6 < 2^24 units for a row's whole sum at these sizes; larger K take smaller numbers)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    top = 6 if K <= 4200 else 3
    make = lambda R: torch.randint(-top, top + 1, (R, K), generator=gen, device="cuda").float().to(E4M3)  # noqa: E731
    power = lambda *s: torch.exp2(torch.randint(-2, 2, s, generator=gen, device="cuda").float())  # noqa: E731
    return make(M), power(M, _up(K, 128)), make(N), power(_up(N, 128), _up(K, 128))


def _product(x, xs, w, ws):
    """In 64 bits; and the sum of |x||w| with the scales."""
    (M, K), N = x.shape, w.shape[0]
    out, mag = torch.zeros(M, N, dtype=torch.float64, device="cuda"), torch.zeros(M, N, dtype=torch.float64, device="cuda")
    col = torch.arange(N, device="cuda") // 128
    for b in range(_up(K, 128)):
        k = slice(128 * b, min(K, 128 * b + 128))
        u, v, s = x[:, k].double(), w[:, k].double(), xs[:, b, None].double() * ws[col, b].double()
        out += (u @ v.T) * s
        mag += (u.abs() @ v.abs().T) * s
    return out, mag


def _matmul(x, xs, w, ws, dtype="bf16", pad=0, shift=0):
    M, N = x.shape[0], w.shape[0]
    store = torch.full((M * (N + pad) + 8,), 77.0, dtype=DT[dtype], device="cuda")
    out = store[shift:shift + M * (N + pad)].view(M, N + pad)[:, :N]
    cg.block8_matmul(x, xs, w, ws, out)
    rest = torch.ones_like(store, dtype=torch.bool)
    rest[shift:shift + M * (N + pad)].view(M, N + pad)[:, :N] = False
    assert (store[rest] == 77).all()
    return out


@pytest.mark.parametrize("M,N,K", SIZES)
def test_matmul_of_exact_sums(M, N, K):
    """Every element equal: a row, column or block in a wrong place would show."""
    c = _exact_case(M, N, K)
    want, _ = _product(*c)
    for dtype, pad, shift in (("bf16", 0, 0), ("fp16", 3, 1)):
        got = _matmul(*c, dtype, pad, shift)
        assert torch.equal(got, want.to(DT[dtype]))
    assert cg.get_status() == 0


def _real_case(M, N, K, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(M, K, generator=gen, device="cuda") * torch.exp(0.5 * torch.randn(K, generator=gen, device="cuda"))
    w = torch.randn(N, K, generator=gen, device="cuda") * K ** -0.5
    coded = []
    for t, rows in ((x, 1), (w, 128)):
        t = t.bfloat16()
        codes, scales = torch.empty(t.shape, dtype=E4M3, device="cuda"), torch.empty(_up(t.shape[0], rows), _up(K, 128), device="cuda")
        cg.block8_encode(t, codes, scales, rows=rows)
        coded += [codes, scales]
    return coded


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("M,N,K", [(1, 300, 4096), (7, 1000, 272), (50, 129, 2064), (200, 500, 4112), (333, 1000, 4112), (2100, 2600, 1024)])
def test_matmul(M, N, K, dtype):
    """Products of codes are exact (8 bits); a block's 128 are summed in fp32, a sum off by at most 2^-23 of the terms' sizes each
    (rounded or cut off); the product with the scales (two roundings) and the sum over the blocks add 3 2^-24 a block; the result is
    rounded once (u)."""
    c = _real_case(M, N, K)
    want, mag = _product(*c)
    got = _matmul(*c, dtype).double()
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    bound = (128 + 2 * _up(K, 128)) * 2.0 ** -23 * mag + u * want.abs() + 2.0 ** -25
    assert ((got - want).abs() <= bound).all(), f"worst error / bound {((got - want).abs() / bound).max():.3g}"
    assert torch.equal(got, _matmul(*c, dtype).double()) and cg.get_status() == 0


@pytest.mark.parametrize("M,N,K", [(4, 300, 400), (200, 300, 400), (2200, 2600, 144), (40, 2001, 144), (2200, 2601, 144), (2200, 2567, 272)])
def test_strides(M, N, K):
    """Matrices within wider ones, the last piece of an output's row whole or not."""
    x, xs, w, ws = _exact_case(M, N, K)
    wide = lambda t, pad: torch.cat([t.view(torch.uint8), torch.full((t.shape[0], pad), 0x7f, dtype=torch.uint8, device="cuda")], 1).view(E4M3)[:, :K]  # noqa: E731
    want = _matmul(x, xs, w, ws)
    for pad in (8, -N % 8, -N % 8 + 8):
        assert torch.equal(_matmul(wide(x, 16), xs, wide(w, 240), ws, pad=pad), want)
    assert torch.equal(_matmul(x[:1], xs[:1], wide(w, 16), ws), want[:1])


@pytest.mark.parametrize("M", [5, 40, 200, 2500])
def test_special_values_reach_their_rows(M):
    """A NaN among the codes or the scales, or an infinite scale, shows where it enters and nowhere else."""
    N, K = 2600 if M > 2000 else 300, 400
    x, xs, w, ws = _exact_case(M, N, K)
    want = _matmul(x, xs, w, ws)
    r, c = min(M - 1, 130), 140
    for name in ("x", "xs", "w", "ws"):
        t = dict(x=x.clone(), xs=xs.clone(), w=w.clone(), ws=ws.clone())
        if name == "x":
            t["x"].view(torch.uint8)[r, K - 1] = 0x7f
        elif name == "w":
            t["w"].view(torch.uint8)[c, 0] = 0xff
        elif name == "xs":
            t["xs"][r, 3] = float("nan")
        else:
            t["ws"][1, 1] = float("nan")
        hit = torch.zeros(M, N, dtype=torch.bool, device="cuda")
        if name in ("x", "xs"):
            hit[r] = True
        elif name == "w":
            hit[:, c] = True
        else:
            hit[:, 128:256] = True
        got = _matmul(**t)
        assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit]), name


@pytest.mark.parametrize("M", [1, 3, 60, 300, 2500])
def test_a_row_does_not_depend_on_the_others(M):
    """The same rows of x among others that hold NaN, and rows of w alone, give the same bits in the same kernel."""
    N, K = 2600, 528
    x, xs, w, ws = _real_case(M, N, K)
    want = _matmul(x, xs, w, ws)
    y, ys = x.clone(), xs.clone()
    keep = torch.arange(M, device="cuda") % 3 == 0
    y.view(torch.uint8)[~keep] = 0x7f
    assert torch.equal(_matmul(y, ys, w, ws)[keep], want[keep])


def test_results_beyond_the_type():
    x, xs, w, ws = _exact_case(9, 40, 128)
    want, _ = _product(x, xs * 2.0 ** 10, w, ws)
    got = _matmul(x, xs * 2.0 ** 10, w, ws, "fp16")
    assert torch.equal(got, want.to(torch.float16)) and torch.isinf(got).any()


def test_zeros_and_no_rows():
    x, xs, w, ws = _exact_case(70, 40, 256)
    assert (_matmul(x, xs * 0, w, ws) == 0).all()
    for M, N in ((0, 40), (70, 0)):
        out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        cg.block8_matmul(x[:M], xs[:M], w[:N], ws[:_up(N, 128)], out)
    cg.block8_encode(torch.empty(0, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 128, dtype=E4M3, device="cuda"), torch.empty(0, 1, device="cuda"))
    assert cg.get_status() == 0


@pytest.mark.parametrize("M,N,K", [(300000, 8192, 128), (1100000, 128, 4096), (5, 1100000, 4096), (2, 40, 1 << 20), (300, 200, 1 << 18)])
def test_offsets_past_32_bits_and_long_rows(M, N, K):
    """Results, codes of x and codes of w beyond 2^32 bytes, and rows of a million channels: sampled rows and columns, equal."""
    gen = torch.Generator(device="cuda").manual_seed(K)
    make = lambda R: torch.randint(0, 2, (R, K), generator=gen, device="cuda", dtype=torch.uint8).mul_(0x38).view(E4M3)  # noqa: E731  (0 and 1)
    x, w = make(M), make(N)
    xs, ws = torch.ones(M, _up(K, 128), device="cuda"), torch.ones(_up(N, 128), _up(K, 128), device="cuda")
    xs[::2] *= 2
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    cg.block8_matmul(x, xs, w, ws, out)
    r = torch.unique(torch.cat([torch.tensor([0, M - 1]), torch.randint(0, M, (40,), generator=torch.Generator().manual_seed(1))])).cuda()
    c = torch.unique(torch.cat([torch.tensor([0, N - 1]), torch.randint(0, N, (40,), generator=torch.Generator().manual_seed(2))])).cuda()
    # at most 2 2^20 < 2^24: exact in fp32
    want = (x.view(torch.uint8)[r] > 0).double() @ (w.view(torch.uint8)[c] > 0).double().T * xs[r, :1].double()
    assert torch.equal(out[r][:, c], want.to(torch.bfloat16)) and cg.get_status() == 0


def test_encode_past_32_bits():
    R, K = 1100000, 4096
    x = torch.zeros(R, K, dtype=torch.bfloat16, device="cuda")
    r = torch.tensor([0, 1, 524287, 524288, 1048575, 1048576, R - 1], device="cuda")
    x[r] = torch.randn(len(r), K, device="cuda").bfloat16()
    codes, scales = torch.empty(R, K, dtype=E4M3, device="cuda"), torch.empty(R, K // 128, device="cuda")
    cg.block8_encode(x, codes, scales)
    want, ws = _encoded(x[r].cpu(), 1)
    assert torch.equal(codes.view(torch.uint8)[r].cpu(), want) and torch.equal(scales[r].cpu(), ws)
    assert int((scales != 0).any(1).sum()) == len(r) and cg.get_status() == 0


@pytest.mark.parametrize("M", [1, 100, 2500])
def test_graph_and_streams(M):
    """Encoding and product on a side stream, then captured and replayed on other values."""
    N, K = 2600, 528
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(M, K, generator=gen, device="cuda").bfloat16()
    w, wsc = torch.empty(N, K, dtype=E4M3, device="cuda"), torch.empty(_up(N, 128), _up(K, 128), device="cuda")
    cg.block8_encode(torch.randn(N, K, generator=gen, device="cuda").bfloat16(), w, wsc, rows=128)
    codes, scales, out = torch.empty(M, K, dtype=E4M3, device="cuda"), torch.empty(M, _up(K, 128), device="cuda"), torch.empty(M, N, dtype=torch.bfloat16, device="cuda")

    def run():
        cg.block8_encode(x, codes, scales)
        cg.block8_matmul(codes, scales, w, wsc, out)

    run()
    want = out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    x.copy_(torch.randn(M, K, generator=gen, device="cuda").bfloat16())
    g.replay()
    got = out.clone()
    run()
    assert torch.equal(out, got) and not torch.equal(got, want)
