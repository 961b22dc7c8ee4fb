"""Microscaled 4-bit floating point: codes and scales bit for bit against the definition, products against 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16]
U = 2.0 ** -24
VALUES = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


@pytest.fixture(scope="module")
def mxc():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1512_01274_amd import mxc as m
    return m


def quantize(x):
    """Codes [N, blocks*32] (one each) and scale bytes [N, blocks] of x, by the definition, on the host in 64 bits."""
    N, C = x.shape
    blocks = -(-C // 32)
    b = torch.zeros(N, blocks * 32, dtype=torch.float64)
    b[:, :C] = x.double().cpu()
    b = b.view(N, blocks, 32)
    bad = ~b.isfinite().all(2)
    b = b.masked_fill(bad[:, :, None], 0.0)
    most = b.abs().amax(2)
    byte = torch.where(most > 0, torch.floor(torch.log2(most.clamp(min=1e-300))) - 2 + 127, 0.0).clamp(0)
    a = b.abs() / torch.exp2(byte - 127)[:, :, None]
    dist = (a[..., None] - VALUES[:8]).abs()
    # nearest; of two equally near ones the even code
    code = torch.argmin(dist * 2 + torch.tensor([0.0, 1.0] * 4, dtype=torch.float64) * 1e-9, dim=3)
    code = code + 8 * ((b < 0) | ((b == 0) & torch.signbit(b))).long()
    byte[bad] = 255
    code[bad] = 0
    return code.view(N, -1), byte.long()


def decode(codes, scales, C):
    """[N, C] float64 of the library's codes and scales."""
    codes, scales = codes.cpu().long(), scales.cpu()
    n = torch.stack([codes & 15, codes >> 4], 2).flatten(1)
    s = torch.exp2(scales.double() - 127)
    s[scales == 255] = math.nan
    return (VALUES[n] * s.repeat_interleave(32, 1)[:, :n.shape[1]])[:, :C]


def run_quantize(mxc, x):
    N, C = x.shape
    cb, sb = -(-C // 32) * 16, -(-C // 512) * 16
    codes, scales = torch.full((N * cb + 64,), 0xA5, dtype=torch.uint8, device="cuda"), torch.full((N * sb + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    mxc.mxc_mxfp4_quantize(N, C, mxc.dtype_code(x.dtype), x, codes, scales)
    assert bool((codes[N * cb:] == 0xA5).all()) and bool((scales[N * sb:] == 0xA5).all())
    return codes[:N * cb].view(N, cb).clone(), scales[:N * sb].view(N, sb).clone()


def check_quantize(mxc, x):
    N, C = x.shape
    codes, scales = run_quantize(mxc, x)
    want_c, want_s = quantize(x)
    got = torch.stack([codes & 15, codes >> 4], 2).flatten(1).cpu().long()
    blocks = -(-C // 32)
    assert torch.equal(scales[:, :blocks].cpu().long(), want_s) and not bool(scales[:, blocks:].any())
    # a zero has either sign
    assert torch.equal(torch.where(got == 8, 0, got), torch.where(want_c == 8, 0, want_c))
    assert not bool(got[:, C:].any())
    for dtype in DTYPES:
        y = torch.full((N * C + 32,), 9.0, dtype=dtype, device="cuda")
        mxc.mxc_mxfp4_dequantize(N, C, mxc.dtype_code(dtype), codes, scales, y)
        assert bool((y[N * C:] == 9.0).all())
        want = decode(codes, scales, C).to(dtype)
        y = y[:N * C].view(N, C).cpu()
        assert bool(((y == want) | (y.isnan() & want.isnan())).all())
    return codes, scales


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C", [(1, 1), (3, 2), (2, 31), (5, 32), (4, 33), (7, 63), (3, 64), (2, 100), (3, 511), (2, 512), (3, 513), (1, 4096), (9, 1027),
                                 (130, 96), (2, 16385), (300, 8), (1000, 40)])
def test_quantize(mxc, dtype, N, C):
    g = torch.Generator(device="cuda").manual_seed(N * C)
    x = torch.randn(N, C, generator=g, device="cuda") * torch.exp2(torch.randint(-40, 40, (N, 1), generator=g, device="cuda").float())
    x[torch.rand(N, C, generator=g, device="cuda") < 0.1] = 0
    x[N // 2] = 0
    check_quantize(mxc, x.to(dtype))


@pytest.mark.parametrize("dtype", DTYPES)
def test_borders(mxc, dtype):
    """Every half-way point, its neighbours on both sides, both signs, at every scale there is; subnormal inputs among them."""
    half = torch.tensor([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7], dtype=torch.float64)
    step = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -23
    v = torch.cat([half, half * (1 + step), half * (1 - step)])
    rows = []
    for e in range(-149, 126):
        r = torch.zeros(2, 64, dtype=torch.float64)
        r[0, :48], r[1, :48] = v, -v
        r[:, 31] = 7.0
        r[:, 32] = 4.0
        rows.append(r * 2.0 ** e)
    x = torch.cat(rows).to(dtype)
    check_quantize(mxc, x.cuda())
    check_quantize(mxc, x[:, :63].contiguous().cuda())


@pytest.mark.parametrize("dtype", DTYPES)
def test_not_finite(mxc, dtype):
    x = torch.randn(6, 200, device="cuda").to(dtype)
    x[0, 3], x[1, 40], x[2, 199], x[3, 64] = math.nan, math.inf, -math.inf, -math.nan
    x[4, 0] = float(torch.finfo(dtype).max)
    codes, scales = check_quantize(mxc, x)
    assert bool((scales[[0, 1, 2, 3], [0, 1, 6, 2]] == 255).all())


def filter4(K, C, gen, lo=100, hi=150):
    blocks = -(-C // 32)
    codes = torch.randint(0, 256, (K, blocks * 16), generator=gen, device="cuda", dtype=torch.uint8)
    scales = torch.zeros(K, -(-C // 512) * 16, dtype=torch.uint8, device="cuda")
    scales[:, :blocks] = torch.randint(lo, hi, (K, blocks), generator=gen, device="cuda", dtype=torch.uint8)
    if C % 32:
        tail = codes[:, -16:]
        tail[:, (C % 32 + 1) // 2:] = 0
        if C % 2:
            tail[:, C % 32 // 2] &= 15
    return codes, scales


def check_product(mxc, N, C, K, dtype, bias, relu, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + N + C + K)
    x = (torch.randn(N, C, generator=gen, device="cuda") * torch.exp2(torch.randint(-3, 4, (N, 1), generator=gen, device="cuda").float())).to(dtype)
    codes, scales = filter4(K, C, gen, 117, 123)
    b = torch.randn(K, generator=gen, device="cuda") if bias else None
    y = torch.full((N * K + 32,), 9.0, dtype=dtype, device="cuda")
    code = mxc.dtype_code(dtype)
    ws = mxc.alloc_workspace(mxc.mxc_mxfp4_fc_workspace_bytes(N, C, K, code))
    if ws is not None:
        ws.fill_(0xFF)
    mxc.mxc_mxfp4_fc_fwd(N, C, K, code, x, codes, scales, b, relu, y, ws)
    assert bool((y[N * K:] == 9.0).all())
    xc, xs = run_quantize(mxc, x)
    q, w = decode(xc, xs, C), decode(codes, scales, C)
    q, w = (q.cuda(), w.cuda()) if N * C * K > 1e7 else (q, w)
    want, D = q @ w.t().contiguous(), q.abs() @ w.t().contiguous().abs()
    if bias:
        want, D = want + b.to(want.device).double(), D + b.to(want.device).double().abs()
    if relu:
        want = want.clamp(min=0)
    got = y[:N * K].view(N, K).double().to(want.device)
    tol = 64 * U * D + torch.finfo(dtype).eps / 2 * want.abs() + 1e-37
    bad = (got - want).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4], want[bad][:4])


SHAPES = [(1, 1, 1), (1, 32, 16), (1, 4096, 100), (1, 4097, 1024), (2, 33, 17), (3, 512, 64), (4, 1000, 1000), (5, 77, 3), (8, 2048, 256), (15, 640, 48), (16, 513, 130),
          (17, 1024, 128), (31, 96, 40), (32, 4160, 256), (33, 257, 65), (64, 768, 300), (65, 2000, 129), (100, 9216, 512), (127, 128, 1000), (128, 4096, 512), (129, 544, 257),
          (200, 100, 64), (256, 1024, 256), (257, 1056, 300), (300, 65, 700), (512, 512, 512), (513, 8192, 520), (1000, 1000, 1000), (1030, 260, 2050), (2, 16384, 33)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,C,K", SHAPES)
def test_product(mxc, dtype, N, C, K):
    check_product(mxc, N, C, K, dtype, True, True)
    check_product(mxc, N, C, K, dtype, False, False, seed=1)


@pytest.mark.parametrize("N,C,K", [(128, 9216, 4096), (4096, 4096, 4096), (1, 16384, 16384), (4000, 1001, 5003), (8192, 256, 1000)])
def test_product_large(mxc, N, C, K):
    check_product(mxc, N, C, K, torch.bfloat16, True, False)


@pytest.mark.parametrize("N,C,K", [(1, 4096, 64), (5, 100, 33), (100, 2048, 300), (300, 1000, 520)])
def test_product_exact(mxc, N, C, K):
    """Small whole numbers: sums are exact, so every place has to be right to the last bit; a NaN stays in its row or column."""
    gen = torch.Generator(device="cuda").manual_seed(C)
    x = torch.randint(-3, 4, (N, C), generator=gen, device="cuda").float()
    x[:, ::32] = 4.0        # every block's scale is 1
    codes, scales = filter4(K, C, gen, 127, 128)
    y = torch.empty(N, K, device="cuda")
    ws = mxc.alloc_workspace(mxc.mxc_mxfp4_fc_workspace_bytes(N, C, K, 0))
    mxc.mxc_mxfp4_fc_fwd(N, C, K, 0, x, codes, scales, None, 0, y, ws)
    want = x.cpu().double() @ decode(codes, scales, C).t()
    assert torch.equal(y.cpu().double(), want)
    if N > 2 and K > 3:
        x[2, C // 2] = math.inf
        scales[3, 0] = 255
        mxc.mxc_mxfp4_fc_fwd(N, C, K, 0, x, codes, scales, None, 1, y, ws)
        nan = torch.zeros(N, K, dtype=torch.bool)
        nan[2], nan[:, 3] = True, True
        assert torch.equal(y.cpu().isnan(), nan) and torch.equal(y.cpu()[~nan].double(), want.clamp(min=0)[~nan])


def test_scales(mxc):
    """Large and small scales of both operands meet; results below 2^-126 may be 0."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    N, C, K = 40, 320, 48
    x = torch.randn(N, C, generator=gen, device="cuda").view(N, -1, 32) * torch.exp2(torch.randint(-50, 50, (N, C // 32, 1), generator=gen, device="cuda").float())
    x = x.reshape(N, C)
    codes, scales = filter4(K, C, gen, 77, 177)
    y = torch.empty(N, K, device="cuda")
    mxc.mxc_mxfp4_fc_fwd(N, C, K, 0, x, codes, scales, None, 0, y, mxc.alloc_workspace(mxc.mxc_mxfp4_fc_workspace_bytes(N, C, K, 0)))
    q, w = decode(*run_quantize(mxc, x), C), decode(codes, scales, C)
    want, D = q @ w.t(), q.abs() @ w.t().abs()
    assert bool(((y.cpu().double() - want).abs() <= 64 * U * D + 1e-37).all())


def test_graph(mxc):
    """A captured product, replayed on new inputs with eager calls between."""
    for N, C, K in ((1, 4096, 512), (128, 4096, 512)):
        gen = torch.Generator(device="cuda").manual_seed(N)
        codes, scales = filter4(K, C, gen, 117, 123)
        x, y = torch.randn(N, C, device="cuda").bfloat16(), torch.empty(N, K, device="cuda", dtype=torch.bfloat16)
        ws = mxc.alloc_workspace(mxc.mxc_mxfp4_fc_workspace_bytes(N, C, K, 1))
        call = lambda: mxc.mxc_mxfp4_fc_fwd(N, C, K, 1, x, codes, scales, None, 0, y, ws)  # noqa: E731
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for _ in range(4):
            x.copy_(torch.randn(N, C, device="cuda"))
            call()
            torch.cuda.synchronize()
            want = y.clone()
            y.fill_(0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)


# wide filters' workgroups from 8192 rows; 128 rows of x and more; the sizes of tiles on both sides of 192 of the larger ones
@pytest.mark.parametrize("N,C,K", [(17, 300, 8192), (100, 1000, 8191), (128, 512, 8192), (128, 640, 9001), (129, 512, 8192), (33, 4097, 8200), (64, 96, 16400),
                                   (6144, 256, 2048), (6143, 288, 2047), (6144, 256, 1792), (5000, 100, 2500)])
def test_borders_of_the_paths(mxc, N, C, K):
    for dtype in DTYPES:
        check_product(mxc, N, C, K, dtype, True, True)


@pytest.mark.parametrize("N,C,K,last", [(1, 65504, 140001, 40), (30, 65504, 140001, 40), (200, 65504, 140001, 40), (50000, 64, 50001, 5)])
def test_past_32_bits(mxc, N, C, K, last):
    """A filter of more than 2^32 bytes; more than 2^31 results: the last ones are those of a call of the last filter rows or rows of x."""
    gen = torch.Generator(device="cuda").manual_seed(N)
    x = torch.randn(N, C, generator=gen, device="cuda").bfloat16()
    codes, scales = filter4(K, C, gen, 117, 123)
    y = torch.empty(N, K, dtype=torch.bfloat16, device="cuda")
    ws = lambda n, k: mxc.alloc_workspace(mxc.mxc_mxfp4_fc_workspace_bytes(n, C, k, 1))  # noqa: E731
    mxc.mxc_mxfp4_fc_fwd(N, C, K, 1, x, codes, scales, None, 0, y, ws(N, K))
    rows = N if N <= 200 else last
    xc, xs = run_quantize(mxc, x[N - rows:].contiguous())
    q, w = decode(xc, xs, C).cuda(), decode(codes[K - last:], scales[K - last:], C).cuda()
    want, D = q @ w.t().contiguous(), q.abs() @ w.t().contiguous().abs()
    # (sums: a chain of C/64 partial sums at most)
    assert bool(((y[N - rows:, K - last:].double() - want).abs() <= (C / 64 + 64) * U * D + 2.0 ** -8 * want.abs() + 1e-37).all())


def test_quantize_past_32_bits(mxc):
    """More than 2^31 values, there and back."""
    N, C, last = 70000, 32800, 3
    x = torch.zeros(N, C, dtype=torch.bfloat16, device="cuda")
    x[N - last:] = torch.randn(last, C, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    codes, scales = run_quantize(mxc, x)
    small = run_quantize(mxc, x[N - last:].contiguous())
    assert torch.equal(codes[N - last:], small[0]) and torch.equal(scales[N - last:], small[1]) and not bool(codes[:N - last].any())
    y = torch.empty_like(x)
    mxc.mxc_mxfp4_dequantize(N, C, 1, codes, scales, y)
    assert torch.equal(y[N - last:].cpu().double(), decode(*small, C)) and not bool(y[:N - last].any())


# some rows or few filter rows on one side, tiles on the other; each size of workgroup
@pytest.mark.parametrize("N,C,K", [(300, 640, 4096), (512, 200, 4096), (513, 512, 4096), (1000, 1056, 500), (4000, 130, 65), (9000, 288, 17), (64, 256, 16384), (64, 256, 16400),
                                   (33, 100, 20000), (32, 700, 40000), (128, 1024, 1000), (128, 1024, 2050), (96, 1024, 4100), (128, 1024, 6001), (40, 2048, 8193), (24, 544, 3001), (16, 4096, 4096), (16, 4097, 300), (8, 8192, 1000), (9, 8200, 100), (1, 25088, 1000), (3, 16384, 50),
                                   (1, 2048, 70000), (2, 500, 40000), (16, 700, 4097), (17, 8192, 33), (4, 9216, 5000)])
def test_shapes_of_workgroups(mxc, N, C, K):
    for dtype in DTYPES:
        check_product(mxc, N, C, K, dtype, True, True)


# the single launch and two on both sides of each of its limits
@pytest.mark.parametrize("N,C,K", [(8, 640, 4096), (9, 640, 4096), (8, 640, 4097), (4, 640, 8192), (5, 640, 8192), (4, 640, 8193), (1, 100, 32768), (1, 100, 32769), (2, 100, 20000),
                                   (3, 12320, 33000), (3, 12288, 33000), (4, 12320, 33000), (2, 12289, 40001), (8, 12320, 1000)])
def test_borders_of_the_single_launch(mxc, N, C, K):
    for dtype in DTYPES:
        check_product(mxc, N, C, K, dtype, True, True)
