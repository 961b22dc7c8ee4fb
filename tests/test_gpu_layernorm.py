"""Layer norm and its gradient against the formulas in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def mxc():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1512_01274_amd import mxc as m
    return m


def guarded(shape, dtype, fill=5.0):
    n = math.prod(shape)
    whole = torch.full((n + 64,), fill, dtype=dtype, device="cuda")
    return whole, whole[:n].view(shape)


def intact(whole, part, fill=5.0):
    return bool((whole[part.numel():] == fill).all())


def data(N, C, dtype, seed, offset=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = (r(N, C) * torch.exp(r(N, 1)) + offset * r(N, 1)).to(dtype)
    return x, r(N, C).to(dtype), 1.0 + 0.3 * r(C), 0.5 * r(C)


def chain(C):
    """Roundings that one value meets on its way into a row's sum: a thread's own additions (16 values, or every 1024th piece of a longer
    row), those across the lanes and waves."""
    return 16 + C // 1024 + 12


def forward64(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    var = d.square().mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    return d * rstd * gamma + beta, mean, rstd, d, var


def forward_tolerance(x, gamma, beta, eps, dtype):
    y, mean, rstd, d, var = forward64(x, gamma, beta, eps)
    k = chain(x.shape[1])
    e_mean = (k + 1) * U * x.double().abs().mean(1, keepdim=True)
    e_d = e_mean + U * d.abs()
    e_var = (k + 3) * U * var + 2 * (e_d * d.abs()).mean(1, keepdim=True) + e_d.square().mean(1, keepdim=True)
    e_rstd = rstd * (e_var / (2 * (var + eps)) * 1.1 + 4 * U)          # (1.1: second order, where the mean costs digits of small variances)
    z = d * rstd
    e_z = e_d * rstd + d.abs() * e_rstd + U * z.abs()
    e_y = e_z * gamma.abs() + U * (z * gamma).abs() + U * (y.abs() + beta.abs())
    return 1.01 * (e_y + HALF[dtype] * (y.abs() + e_y)), 1.01 * e_mean, 1.01 * e_rstd


SIZES = [(1, 1), (3, 2), (5, 3), (2, 7), (9, 8), (130, 64), (65, 100), (4, 127), (33, 256), (1, 1000), (128, 1000), (17, 1025), (3, 4096), (300, 4097), (2, 8200), (3, 16384), (2, 16385),
         (2, 32771), (1, 100003), (5000, 16), (70000, 3),
         # on either side of where one launch makes the whole gradient
         (511, 1000), (512, 200), (513, 200), (512, 4097), (513, 4097), (300, 31), (512, 3)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,C", SIZES)
def test_forward(mxc, dtype, N, C):
    x, _, gamma, beta = data(N, C, dtype, N * 7 + C)
    for eps, weights, held in ((1e-5, True, True), (1e-2, False, False), (1.2e-38, True, True)):
        if eps < 1e-30 and C < 3:
            continue        # rows of equal values: no variance is left
        g, b = (gamma, beta) if weights else (None, None)
        whole, y = guarded((N, C), dtype)
        sw, stats = guarded((N, 2), torch.float32)
        mxc.mxc_layernorm_fwd(N, C, mxc.dtype_code(dtype), x, g, b, eps, y, stats if held else None)
        eps = float(torch.tensor(eps, dtype=torch.float32))
        one, zero = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
        G, B = (gamma.double(), beta.double()) if weights else (one.double(), zero.double())
        want, mean, rstd, _, _ = forward64(x, G, B, eps)
        t_y, t_mean, t_rstd = forward_tolerance(x, G, B, eps, dtype)
        bad = ~((y.double() - want).abs() <= t_y)
        assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3])
        if held:
            assert bool(((stats[:, :1].double() - mean).abs() <= t_mean).all())
            assert bool(((stats[:, 1:].double() - rstd).abs() <= t_rstd).all())
        assert intact(whole, y) and intact(sw, stats)
        # in place, the same bits
        again = x.clone()
        mxc.mxc_layernorm_fwd(N, C, mxc.dtype_code(dtype), again, g, b, eps, again, None)
        assert torch.equal(again, y)


@pytest.mark.parametrize("C", [24, 1000, 5000, 20000])
def test_a_large_mean_costs_no_digits(mxc, C):
    """Values 2^12 + k / 16: sums of squares would lose the variance; every difference from the mean is exact to some 2^-12."""
    g = torch.Generator(device="cuda").manual_seed(C)
    x = 4096.0 + torch.randint(-64, 65, (40, C), generator=g, device="cuda") / 16.0
    y, stats = torch.empty_like(x), torch.empty(40, 2, device="cuda")
    mxc.mxc_layernorm_fwd(40, C, 0, x, None, None, 1e-5, y, stats)
    one, zero = torch.ones(C, device="cuda").double(), torch.zeros(C, device="cuda").double()
    want = forward64(x, one, zero, 1e-5)[0]
    t_y, _, _ = forward_tolerance(x, one, zero, 1e-5, torch.float32)
    assert bool(((y.double() - want).abs() <= t_y).all()) and float(t_y.max()) < 0.05


def backward64(x, gamma, stats, dy):
    mean, rstd = stats[:, :1].double(), stats[:, 1:].double()
    z, d = (x.double() - mean) * rstd, dy.double()
    g = d * gamma
    s1, s2 = g.mean(1, keepdim=True), (g * z).mean(1, keepdim=True)
    return rstd * (g - s1 - z * s2), (d * z).sum(0), d.sum(0), (z, d, g, s1, s2, rstd)


def backward_tolerance(parts, dx, dtype):
    z, d, g, s1, s2, rstd = parts
    N, C = z.shape
    k = chain(C)
    # z: two roundings, g: one; the sums' chains; then products, differences and the last factor
    e1, e2 = (k + 3) * U * g.abs().mean(1, keepdim=True), (k + 6) * U * (g * z).abs().mean(1, keepdim=True)
    e = rstd * (e1 + z.abs() * e2 + 6 * U * (g.abs() + s1.abs() + (z * s2).abs()))
    return 1.01 * (e + HALF[dtype] * (dx.abs() + e)), (N + 4) * U * (d * z).abs().sum(0), (N + 1) * U * d.abs().sum(0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,C", SIZES)
def test_gradient(mxc, dtype, N, C):
    x, dy, gamma, beta = data(N, C, dtype, N * 3 + C)
    code = mxc.dtype_code(dtype)
    stats = torch.empty(N, 2, device="cuda")
    mxc.mxc_layernorm_fwd(N, C, code, x, gamma, beta, 1e-3, torch.empty_like(x), stats)
    need = mxc.mxc_layernorm_workspace_bytes(N, C, code)
    ws_whole, ws = guarded((max(need, 256),), torch.uint8, 5)
    for weights in (True, False):
        G = gamma.double() if weights else torch.ones(C, device="cuda").double()
        want, wg, wb, parts = backward64(x, G, stats, dy)
        t_dx, t_g, t_b = backward_tolerance(parts, want, dtype)
        results = []
        for where in ("apart", "apart", "dy", "x"):
            (xw, xx), (dw, dd), (ow, oo) = guarded((N, C), dtype), guarded((N, C), dtype), guarded((N, C), dtype)
            xx.copy_(x)
            dd.copy_(dy)
            gw, dgamma = guarded((C,), torch.float32)
            bw, dbeta = guarded((C,), torch.float32)
            out = {"apart": oo, "dy": dd, "x": xx}[where]
            mxc.mxc_layernorm_bwd(N, C, code, xx, gamma if weights else None, stats, dd, out, dgamma, dbeta, ws)
            results.append((out, dgamma, dbeta))
            assert all(intact(a, b) for a, b in ((xw, xx), (dw, dd), (ow, oo), (gw, dgamma), (bw, dbeta)))
        for out, dgamma, dbeta in results[1:]:
            assert torch.equal(out, results[0][0]) and torch.equal(dgamma, results[0][1]) and torch.equal(dbeta, results[0][2])
        dx, dgamma, dbeta = results[0]
        for got, exact, tol in ((dx, want, t_dx), (dgamma, wg, t_g), (dbeta, wb, t_b)):
            bad = ~((got.double() - exact).abs() <= tol + 1e-42)
            assert not bool(bad.any()), (tuple(got.shape), int(bad.sum()), bad.nonzero()[:3])
    assert intact(ws_whole, ws, 5)
    # each of the weights' gradients may be left out
    dx, dbeta = torch.empty_like(x), torch.empty(C, device="cuda")
    mxc.mxc_layernorm_bwd(N, C, code, x, None, stats, dy, dx, None, dbeta, ws)
    assert torch.equal(dx, results[0][0]) and torch.equal(dbeta, results[0][2])
    dx.zero_()
    mxc.mxc_layernorm_bwd(N, C, code, x, None, stats, dy, dx, None, None, ws)
    assert torch.equal(dx, results[0][0])


# Rows of two and four pieces a lane over more rows than workgroups, with the next row's loads under way (6000) and without (12000), and of 256 MB and more, which go past the caches
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,C", [(600, 6000), (600, 12000), (700, 16383), (4000, 12000), (8000, 6001)])
def test_many_rows_of_several_pieces(mxc, dtype, N, C):
    test_forward(mxc, dtype, N, C)
    test_gradient(mxc, dtype, N, C)


@pytest.mark.parametrize("N,C", [(4, 9), (3, 300), (2, 17000)])
def test_gradient_is_that_of_differences(mxc, N, C):
    """Central differences of the forward formula in 64 bits along random directions of x, gamma and beta."""
    x, dy, gamma, beta = data(N, C, torch.float32, C)
    stats, dx, dgamma, dbeta = torch.empty(N, 2, device="cuda"), torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    mxc.mxc_layernorm_fwd(N, C, 0, x, gamma, beta, 1e-3, torch.empty_like(x), stats)
    mxc.mxc_layernorm_bwd(N, C, 0, x, gamma, stats, dy, dx, dgamma, dbeta, mxc.alloc_workspace(mxc.mxc_layernorm_workspace_bytes(N, C, 0)))
    eps = float(torch.tensor(1e-3, dtype=torch.float32))
    value = lambda a, g, b: (forward64(a, g, b, eps)[0] * dy.double()).sum()  # noqa: E731
    x64, g64, b64 = x.double(), gamma.double(), beta.double()
    want, wg, wb, parts = backward64(x, g64, stats, dy)
    tols = backward_tolerance(parts, want, torch.float32)
    # the stats themselves are rounded: their part of dx's error, relative to rstd and in units of the row's spread
    _, t_mean, t_rstd = forward_tolerance(x, g64, b64, eps, torch.float32)
    rstd = stats[:, 1:].double()
    z, _, g, s1, s2, _ = parts
    spread = g.abs() + s1.abs() + 3 * (z * s2).abs() + (1 + z.abs()) * g.abs().mean(1, keepdim=True)
    extra = (rstd * (t_rstd / rstd * 2 + t_mean * rstd * 2) * spread, (dy.double().abs() * (t_mean * rstd + z.abs() * t_rstd / rstd)).sum(0), 0 * wb)
    h = 1e-4
    for k, (got, at) in enumerate(((dx, x64), (dgamma, g64), (dbeta, b64))):
        direction = torch.randn(at.shape, generator=torch.Generator(device="cuda").manual_seed(k), device="cuda", dtype=torch.float64)
        args = [x64, g64, b64]
        up, down = list(args), list(args)
        up[k], down[k] = at + h * direction, at - h * direction
        change = float((value(*up) - value(*down)) / (2 * h))
        tol = float(((tols[k] + extra[k]) * direction.abs()).sum()) + 1e-5 * float((got.double() * direction).abs().sum())
        assert abs(float((got.double() * direction).sum()) - change) <= tol


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("exponent,eps,C", [(120, 1e-5, 4), (120, 1e-5, 24), (120, 1e-5, 100), (110, 1e-12, 1000), (66, 1.2e-38, 4), (66, 1.2e-38, 24), (66, 1.2e-38, 1000), (66, 1.2e-38, 4097),
                                           (66, 1.2e-38, 12000), (66, 1.2e-38, 17001)])
def test_gradient_where_the_mean_over_the_deviation_is_past_all_numbers(mxc, dtype, exponent, eps, C):
    """Rows of one value, a power of two, beside others: z is zero at every place though |mean| rstd passes the largest number."""
    code = mxc.dtype_code(dtype)
    eps = float(torch.tensor(eps, dtype=torch.float32))
    for N in (5, 513):
        x, dy, gamma, _ = data(N, C, dtype, N + C)
        x[::2] = 2.0 ** exponent
        _, mean, rstd, _, _ = forward64(x, gamma.double(), gamma.double(), eps)
        stats = torch.cat([mean, rstd], 1).float()
        stats[::2, 0], stats[::2, 1] = 2.0 ** exponent, eps ** -0.5
        assert math.log2(float(stats[0, 0])) + math.log2(float(stats[0, 1])) > 128
        want, wg, wb, parts = backward64(x, gamma.double(), stats, dy)
        dx, dgamma, dbeta = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        mxc.mxc_layernorm_bwd(N, C, code, x, gamma, stats, dy, dx, dgamma, dbeta, mxc.alloc_workspace(mxc.mxc_layernorm_workspace_bytes(N, C, code)))
        for got, exact, tol in zip((dx, dgamma, dbeta), (want, wg, wb), backward_tolerance(parts, want, dtype)):
            assert bool(((got.double() - exact).abs() <= tol).all()), (N, tuple(got.shape))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C", [3, 24, 49, 100, 1000, 4097, 5000, 12000, 20001])
def test_rows_whose_values_hardly_differ(mxc, dtype, C):
    """Rows of one value have a variance of 0 whatever the value, and rows of two neighbouring numbers that of half their distance: a rounding of the mean, which is of the
    distance's size, may not enter."""
    code, N = mxc.dtype_code(dtype), 130
    x, _, gamma, beta = data(N, C, dtype, C)
    g = torch.Generator(device="cuda").manual_seed(C)
    value = (torch.exp2(torch.arange(N, device="cuda") % 22 + 3.0) * (1.0 + torch.rand(N, generator=g, device="cuda"))).to(dtype)
    x[:] = value[:, None]
    step = torch.exp2(torch.floor(torch.log2(value.float())) - (23 if dtype == torch.float32 else 7))
    x[1::2, 1::2] = (value.float() + step).to(dtype)[1::2, None]
    assert bool((x[1::2, 1] != x[1::2, 0]).all())
    y, stats = torch.empty_like(x), torch.empty(N, 2, device="cuda")
    mxc.mxc_layernorm_fwd(N, C, code, x, gamma, beta, 1e-5, y, stats)
    eps = float(torch.tensor(1e-5, dtype=torch.float32))
    want, mean, rstd, d, var = forward64(x, gamma.double(), beta.double(), eps)
    k = chain(C)
    # The mean's first rounding is off by `delta` at most; the differences from it are exact (numbers within a factor of two of each other).  Their sum is exact too where they are
    # some hundred units of a last place, so that their mean is off by two roundings of at most delta; where they are a step of bf16 the chain's roundings of them count.
    delta = 1.01 * (k + 2) * U * mean.abs()
    e_c = 1.01 * (k + 2) * U * d.abs().amax(1, keepdim=True) + 2.1 * U * delta
    # (all rows here are ones that the kernels take so: their mean is 16 deviations and more away from zero)
    V = var + eps
    assert bool((mean.abs() > 17 * V.sqrt()).all())
    e_var = (k + 5) * U * var + 2 * var.sqrt() * e_c + 1.1 * e_c * e_c
    e_rstd = rstd * (e_var / (2 * V) * 1.1 + 4 * U)
    assert bool(((stats[:, :1].double() - mean).abs() <= 1.01 * (U * mean.abs() + e_c)).all())
    assert bool(((stats[:, 1:].double() - rstd).abs() <= 1.01 * e_rstd).all())
    z = d * rstd
    e_z = 1.01 * rstd * (e_c + U * delta) + d.abs() * e_rstd + 1.01 * U * z.abs()
    e_y = e_z * gamma.abs() + U * (z * gamma).abs() + U * (want.abs() + beta.abs())
    bad = ~((y.double() - want).abs() <= 1.01 * (e_y + HALF[dtype] * (want.abs() + e_y)))
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3])


def test_rows_that_are_not_finite(mxc):
    """They make NaN of themselves and of what they enter, and leave other rows alone."""
    for C in (24, 5000, 20000):
        x, dy, gamma, beta = data(6, C, torch.bfloat16, C)
        x[1, 3], x[4, C - 1] = math.inf, math.nan
        y, stats = torch.empty_like(x), torch.empty(6, 2, device="cuda")
        mxc.mxc_layernorm_fwd(6, C, 1, x, gamma, beta, 1e-5, y, stats)
        rows = torch.tensor([False, True, False, False, True, False], device="cuda")
        assert torch.equal(y.isnan().all(1), rows) and torch.equal(y.isnan().any(1), rows)
        dx, dgamma, dbeta = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        mxc.mxc_layernorm_bwd(6, C, 1, x, gamma, stats, dy, dx, dgamma, dbeta, mxc.alloc_workspace(mxc.mxc_layernorm_workspace_bytes(6, C, 1)))
        assert torch.equal(dx.isnan().all(1), rows) and torch.equal(dx.isnan().any(1), rows)
        assert bool(dgamma.isnan().all()) and bool(dbeta.isfinite().all())


@pytest.mark.parametrize("N", [6, 600])
def test_gradients_that_are_not_finite(mxc, N):
    """An infinity or a NaN in dy enters its row's dx and its column's sums, one in x its row's dx and all of dgamma; the rest is as without them."""
    for C in (24, 5000, 20000):
        for dtype in (torch.float32, torch.bfloat16):
            x, dy, gamma, beta = data(N, C, dtype, C)
            code, stats, ws = mxc.dtype_code(dtype), torch.empty(N, 2, device="cuda"), mxc.alloc_workspace(mxc.mxc_layernorm_workspace_bytes(N, C, mxc.dtype_code(dtype)))

            def grads():
                mxc.mxc_layernorm_fwd(N, C, code, x, gamma, beta, 1e-5, torch.empty_like(x), stats)
                dx, dgamma, dbeta = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
                mxc.mxc_layernorm_bwd(N, C, code, x, gamma, stats, dy, dx, dgamma, dbeta, ws)
                return dx, dgamma, dbeta

            clean = grads()
            dy[1, 3], dy[4, C - 1], dy[5, 3] = math.inf, math.nan, -math.inf
            rows, columns = torch.zeros(N, dtype=torch.bool, device="cuda"), torch.zeros(C, dtype=torch.bool, device="cuda")
            rows[[1, 4, 5]], columns[[3, C - 1]] = True, True
            dx, dgamma, dbeta = grads()
            assert not bool(dx[rows].isfinite().any()) and torch.equal(dx[~rows], clean[0][~rows])
            for got, was in ((dgamma, clean[1]), (dbeta, clean[2])):
                assert not bool(got[columns].isfinite().any()) and torch.equal(got[~columns], was[~columns])
            x[2, 0] = -math.inf
            rows[2] = True
            dx, dgamma, dbeta = grads()
            assert bool(dx[2].isnan().all()) and torch.equal(dx[~rows], clean[0][~rows])
            assert bool(dgamma.isnan().all()) and torch.equal(dbeta[~columns], clean[2][~columns]) and not bool(stats[2].isfinite().any())


@pytest.mark.parametrize("C", [100, 5000, 20000])
def test_rows_whose_sums_pass_the_largest_number(mxc, C):
    x, _, gamma, beta = data(4, C, torch.float32, C)
    x[1], x[2] = 2.0 ** 125, 2.0 ** 70 * (torch.arange(C, device="cuda") % 2 * 2.0 - 1.0)
    y, stats = torch.empty_like(x), torch.empty(4, 2, device="cuda")
    mxc.mxc_layernorm_fwd(4, C, 0, x, gamma, beta, 1e-5, y, stats)
    assert bool(y[1].isnan().all()) and torch.equal(y[2], beta) and float(stats[2, 1]) == 0.0
    alone, few = torch.empty(2, C, device="cuda"), torch.empty(2, 2, device="cuda")
    mxc.mxc_layernorm_fwd(2, C, 0, x[::3].contiguous(), gamma, beta, 1e-5, alone, few)
    assert torch.equal(y[::3], alone) and torch.equal(stats[::3], few)


def test_offsets_past_32_bits(mxc):
    """More than 2^31 values: the last rows as those of a small call."""
    N, C = 66000, 32768
    for n_c in ((N, C), (N * 32, C // 32)):
        n, c = n_c
        x = torch.zeros(n, c, dtype=torch.bfloat16, device="cuda")
        last, dy, gamma, beta = data(3, c, torch.bfloat16, 1)
        x[-3:] = last
        stats, small = torch.empty(n, 2, device="cuda"), torch.empty(3, 2, device="cuda")
        y = torch.empty_like(last)
        mxc.mxc_layernorm_fwd(3, c, 1, last, gamma, beta, 1e-5, y, small)
        grads = torch.zeros(n, c, dtype=torch.bfloat16, device="cuda")
        mxc.mxc_layernorm_fwd(n, c, 1, x, gamma, beta, 1e-5, grads, stats)
        assert torch.equal(grads[-3:], y) and torch.equal(stats[-3:], small) and torch.equal(grads[0], beta.bfloat16())
        grads.zero_()
        grads[-3:] = dy
        dgamma, dbeta, dg3, db3 = (torch.empty(c, device="cuda") for _ in range(4))
        dx = torch.empty_like(last)
        mxc.mxc_layernorm_bwd(3, c, 1, last, gamma, small, dy, dx, dg3, db3, mxc.alloc_workspace(mxc.mxc_layernorm_workspace_bytes(3, c, 1)))
        mxc.mxc_layernorm_bwd(n, c, 1, x, gamma, stats, grads, grads, dgamma, dbeta, mxc.alloc_workspace(mxc.mxc_layernorm_workspace_bytes(n, c, 1)))
        assert torch.equal(grads[-3:], dx) and not bool(grads[0].any())
        # three values of 32 bits added in either order
        assert torch.allclose(dgamma, dg3, rtol=1e-5, atol=1e-5) and torch.allclose(dbeta, db3, rtol=1e-5, atol=1e-5)
        del x, grads


def test_streams_and_graphs(mxc):
    N, C = 700, 1500
    x, dy, gamma, beta = data(N, C, torch.bfloat16, 9)
    y, dx, stats, dgamma, dbeta = torch.empty_like(x), torch.empty_like(x), torch.empty(N, 2, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = mxc.alloc_workspace(mxc.mxc_layernorm_workspace_bytes(N, C, 1))
    outs = (y, dx, stats, dgamma, dbeta)

    def calls(stream=None):
        mxc.mxc_layernorm_fwd(N, C, 1, x, gamma, beta, 1e-5, y, stats, stream)
        mxc.mxc_layernorm_bwd(N, C, 1, x, gamma, stats, dy, dx, dgamma, dbeta, ws, stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    calls(side)
    torch.cuda.current_stream().wait_stream(side)
    first = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for turn in range(3):
        if turn:
            x.copy_(data(N, C, torch.bfloat16, 20 + turn)[0])
        for t in outs:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        calls()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
        if turn == 0:
            assert all(torch.equal(a, b) for a, b in zip(got, first))


@pytest.mark.parametrize("N,C", [(512, 200), (512, 4097), (3, 12000), (1, 1)])
def test_gradient_of_few_rows_needs_no_workspace(mxc, N, C):
    for dtype in (torch.float32, torch.bfloat16):
        x, dy, gamma, beta = data(N, C, dtype, 5)
        stats, code = torch.empty(N, 2, device="cuda"), mxc.dtype_code(dtype)
        mxc.mxc_layernorm_fwd(N, C, code, x, gamma, beta, 1e-3, torch.empty_like(x), stats)
        want, wg, wb, parts = backward64(x, gamma.double(), stats, dy)
        for in_place in (False, True):
            dx, dgamma, dbeta = dy.clone() if in_place else torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
            mxc.mxc_layernorm_bwd(N, C, code, x, gamma, stats, dx if in_place else dy, dx, dgamma, dbeta)
            for got, exact, tol in zip((dx, dgamma, dbeta), (want, wg, wb), backward_tolerance(parts, want, dtype)):
                assert bool(((got.double() - exact).abs() <= tol + 1e-42).all())
