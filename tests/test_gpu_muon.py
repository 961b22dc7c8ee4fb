"""Orthogonal updates by Newton-Schulz steps, and the optimiser's step with them, against the formulas in 64 bits.

How far off a result may be comes from a model of the roundings that the header names (fp16 operands at fixed powers of two, diagonals apart, X as two
fp16), run in 64 bits: the kernels make the same roundings of values that differ in the order of 32-bit sums, so that some roundings fall the other
way.  Two draws of such errors of one size differ by at most their sum: twice the model's error, with a third time for matrices of few values, whose errors do
not average; and the sums' own."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
A, B, C = 3.4445, -4.7750, 2.0315


@pytest.fixture(scope="module")
def mxc():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1512_01274_amd import mxc as m
    return m


def orthogonal64(x, steps):
    x = x.double()
    norm = x.square().sum().sqrt()
    x = x / norm if norm > 0 else x
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    for _ in range(steps):
        a = x @ x.t().contiguous()
        x = A * x + (B * a + C * (a @ a)) @ x
    return x.t().contiguous() if tall else x


def half(t, up):
    return (t * 2.0 ** up).half().double() / 2.0 ** up


def modelled(x, steps):
    x = x.double()
    norm = x.square().sum().sqrt()
    x = x / norm if norm > 0 else x
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    hi = half(x, 15)
    lo = half(x - hi, 26)
    for k in range(steps):
        a = hi @ hi.t().contiguous()
        d = a.diagonal().float().double()
        o = half(a - torch.diag(a.diagonal()), 14)
        s = o @ o
        p = B * o + C * ((d[:, None] + d[None]) * o + s)
        e = (B * d + C * (d * d + s.diagonal())).float().double()
        p = half(p - torch.diag(p.diagonal()), 14)
        x = (A + e)[:, None] * (hi + lo) + p @ hi
        if k < steps - 1:
            hi = half(x, 15)
            lo = half(x - hi, 26)
    return x.t().contiguous() if tall else x


def tolerance(x, steps, want):
    """Of the norm of the difference, before the result is rounded."""
    model = (modelled(x, steps) - want).norm()
    # 32-bit sums of up to max(sides) products, each step's errors grown at most by A a step (a random walk of roundings)
    sums = math.sqrt(max(x.shape)) * U * A ** steps * 4
    few = 2.0 ** -11 * 4 / math.sqrt(x.numel()) * want.norm()
    return 3 * float(model) + float(few) + sums * float(want.norm()) + 1e-30


def guarded(shape, dtype, fill=5.0):
    n = math.prod(shape)
    whole = torch.full((n + 64,), fill, dtype=dtype, device="cuda")
    return whole, whole[:n].view(shape)


def intact(whole, part, fill=5.0):
    return bool((whole[part.numel():] == fill).all())


def matrix(r, c, kind, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 1009 + r * 7 + c)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float64)  # noqa: E731
    if kind == "random":
        x = rand(r, c)
    elif kind == "few":         # few directions over many weak ones, as gradients are
        k = min(4, r, c)
        x = rand(r, k) @ rand(k, c) + 0.01 * rand(r, c)
    elif kind == "rank1":
        x = rand(r, 1) @ rand(1, c)
    elif kind == "outlier":
        x = rand(r, c)
        x[r // 2] *= 1000
        x[:, c // 3] *= 300
    elif kind == "one":
        x = torch.zeros(r, c, device="cuda", dtype=torch.float64)
        x[r - 1, c // 2] = -3.0
    elif kind == "sparse":
        x = rand(r, c) * (torch.rand(r, c, generator=g, device="cuda") < 0.05)
        x[0, 0] = 1.0
    else:
        x = torch.ones(r, c, device="cuda", dtype=torch.float64)
    return x.float()


def workspace(mxc, shapes):
    n = mxc.mxc_orthogonalize_workspace_bytes([r for r, _ in shapes], [c for _, c in shapes])
    return guarded((n,), torch.uint8, 5)


def check(got, x, steps, rounded=True):
    want = orthogonal64(x, steps)
    off = (got.double() - want)
    tol = tolerance(x, steps, want) + (2.0 ** -8 * float(want.norm()) if rounded else 0.0)
    assert float(off.norm()) <= tol, (tuple(x.shape), float(off.norm()), tol, float(want.norm()))


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (5, 5), (16, 33), (33, 16), (63, 64), (64, 64), (65, 64), (64, 363), (363, 64), (64, 576), (576, 61), (64, 577), (40, 449), (31, 500), (100, 1000), (128, 129), (200, 200), (257, 255), (130, 700), (700, 130),
          (512, 640), (1025, 513), (577, 64), (640, 33), (1, 5000), (7000, 17), (50, 4100)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("r,c", SHAPES)
def test_orthogonalize(mxc, dtype, r, c):
    for kind, steps in (("random", 5), ("few", 5), ("random", 1), ("outlier", 2), ("rank1", 4), ("sparse", 6)):
        x = matrix(r, c, kind, steps).to(dtype)
        whole, y = guarded((r, c), torch.bfloat16)
        ws_whole, ws = workspace(mxc, [(r, c)])
        mxc.mxc_orthogonalize([x], steps, [y], ws)
        first = y.clone()
        check(y, x, steps)
        ws.fill_(255)           # whatever the workspace held
        mxc.mxc_orthogonalize([x], steps, [y], ws)
        assert torch.equal(first, y) and intact(whole, y) and intact(ws_whole, ws, 5)
        # beside one that no compute unit holds: by other kernels, with the same bits
        beside = matrix(65, 600, "random", 9).to(dtype)
        y.zero_()
        mxc.mxc_orthogonalize([x, beside], steps, [y, torch.empty(65, 600, dtype=torch.bfloat16, device="cuda")], workspace(mxc, [(r, c), (65, 600)])[1])
        assert torch.equal(first, y)


@pytest.mark.parametrize("kind", ["one", "ones", "rank1", "outlier", "few"])
def test_orthogonalize_kinds(mxc, kind):
    for r, c in ((3, 4), (64, 64), (300, 190), (40, 2000)):
        x = matrix(r, c, kind, 3)
        y = torch.empty(r, c, dtype=torch.bfloat16, device="cuda")
        mxc.mxc_orthogonalize([x], 5, [y], workspace(mxc, [(r, c)])[1])
        check(y, x, 5)


def test_singular_values(mxc):
    """What the call is for: directions stay, singular values of some hundredths and more come out between 0.68 and 1.2025, the largest value
    of a s + b s^3 + c s^5 below that (and 1 % of roundings)."""
    g = torch.Generator(device="cuda").manual_seed(1)
    u = torch.linalg.qr(torch.randn(300, 300, generator=g, device="cuda", dtype=torch.float64))[0]
    v = torch.linalg.qr(torch.randn(500, 300, generator=g, device="cuda", dtype=torch.float64))[0]
    s = torch.logspace(0, -1.5, 300, device="cuda", dtype=torch.float64)
    x = ((u * s) @ v.t().contiguous()).float()
    y = torch.empty(300, 500, dtype=torch.bfloat16, device="cuda")
    mxc.mxc_orthogonalize([x], 5, [y], workspace(mxc, [(300, 500)])[1])
    core = u.t().contiguous() @ y.double() @ v
    values = torch.linalg.svdvals(core)
    assert 0.67 < float(values.min()) and float(values.max()) < 1.2145
    off = core - torch.diag(core.diagonal())
    assert float(off.norm() / core.norm()) < 0.01


def test_sizes_of_values(mxc):
    """The norm is taken out first: from the least to the largest numbers the same directions."""
    x = matrix(70, 90, "random", 2)
    ws = workspace(mxc, [(70, 90)])[1]
    y = torch.empty(70, 90, dtype=torch.bfloat16, device="cuda")
    for scale in (1.0, 2.0 ** 120, 2.0 ** -110):
        mxc.mxc_orthogonalize([x * scale], 5, [y], ws)
        check(y, x * scale, 5)
    tiny = (x * 2.0 ** -140)            # subnormal numbers of few digits
    mxc.mxc_orthogonalize([tiny], 5, [y], ws)
    check(y, tiny, 5)


def test_zeros_and_values_that_are_not_finite(mxc):
    shapes = [(70, 90), (130, 20), (5, 5)]
    for bad in (0.0, math.nan, math.inf, -math.inf):
        xs = [matrix(r, c, "random", 1) for r, c in shapes]
        if bad == 0.0:
            xs[1].zero_()
        else:
            xs[1][100, 3] = bad
        ys = [torch.full(s, 9.0, dtype=torch.bfloat16, device="cuda") for s in shapes]
        mxc.mxc_orthogonalize(xs, 5, ys, workspace(mxc, shapes)[1])
        check(ys[0], xs[0], 5)
        check(ys[2], xs[2], 5)
        assert bool((ys[1] == 0).all()) if bad == 0.0 else bool(ys[1].isnan().all())


def test_many_matrices_are_each_as_alone(mxc):
    """One call for many of different shapes, more than travel in one launch's arguments: the bits of calls of their own."""
    shapes = [(1 + 37 * i % 150, 1 + 53 * i % 260) for i in range(75)] + [(520, 300), (300, 520), (64, 1000), (33, 3000), (2000, 64), (64, 577)]
    xs = [matrix(r, c, "few", i) for i, (r, c) in enumerate(shapes)]
    ys = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    whole, ws = workspace(mxc, shapes)
    mxc.mxc_orthogonalize(xs, 5, ys, ws)
    assert intact(whole, ws, 5)
    for i in (0, 1, 5, 19, 20, 21, 39, 40, 62, 74, 75, 76, 77, 78, 79, 80):
        alone = torch.empty_like(ys[i])
        mxc.mxc_orthogonalize([xs[i]], 5, [alone], workspace(mxc, [shapes[i]])[1])
        assert torch.equal(alone, ys[i]), shapes[i]
        check(ys[i], xs[i], 5)


@pytest.mark.parametrize("r,c", [(2000, 1300), (1000, 4096), (4096, 1100), (2304, 2304)])
def test_large(mxc, r, c):
    for kind in ("random", "few"):
        x = matrix(r, c, kind, 4).bfloat16()
        y = torch.empty(r, c, dtype=torch.bfloat16, device="cuda")
        mxc.mxc_orthogonalize([x], 5, [y], workspace(mxc, [(r, c)])[1])
        check(y, x, 5)


# Sides at which products have tiles of 128, 192 and 256, whole ones, ones that are split over the reduction, and both beside each other (the tiles of the three products, and into how
# many parts the last ones are split): 128 128 192; 256/5 256/5 256/4; 64/16 64 256; 128/3 64 192; 128/14 64 256; 192 192 256/2; 256 256 256/3; either way round; and first products
# 64/9 of the other kind, 192/9, 256/12, 128/16 and 192/12 beside whole ones, a third 128/4
TILED = [(3000, 2900), (5990, 6010), (6010, 5990), (2048, 8192), (8190, 2050), (1024, 32768), (4100, 9200), (9200, 4100), (4500, 4500),
         (890, 22300), (22900, 1340), (1472, 26560), (4032, 20990), (4416, 23680), (2430, 7550)]


@pytest.mark.parametrize("r,c", TILED)
def test_tiles(mxc, r, c):
    x = matrix(r, c, "few", 6).bfloat16()
    whole, y = guarded((r, c), torch.bfloat16)
    ws_whole, ws = workspace(mxc, [(r, c)])
    mxc.mxc_orthogonalize([x], 5, [y], ws)
    check(y, x, 5)
    # No value by itself is far off, as one of a wrong row or block would be: besides the result's own rounding a value's error is the sum of many roundings, of which none of 2^26 passes
    # six deviations where all have the norm's, and 16 where some rows have more of it.
    want = orthogonal64(x, 5)
    assert bool(((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 16 * tolerance(x, 5, want) / math.sqrt(r * c)).all())
    del want
    assert intact(whole, y) and intact(ws_whole, ws, 5)
    # twice, and beside others, with the same bits
    first = y.clone()
    ws.fill_(255)
    mxc.mxc_orthogonalize([x], 5, [y], ws)
    assert torch.equal(first, y)
    shapes = [(130, 70), (r, c), (1100, 2300), (64, 1000)]
    xs = [x if s == (r, c) else matrix(*s, "random", 7).bfloat16() for s in shapes]
    ys = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    mxc.mxc_orthogonalize(xs, 5, ys, workspace(mxc, shapes)[1])
    assert torch.equal(first, ys[1])


@pytest.mark.parametrize("r,c", [(4100, 9200), (9200, 4100)])
def test_update_by_split_tiles(mxc, r, c):
    """The last step's third product, whose split tiles write the weights when their parts are added."""
    for nesterov, dtype in ((True, torch.float32), (False, torch.bfloat16)):
        lr, momentum, wd, rms = 3e-2, 0.95, 0.1, 0.2
        w, g, m = matrix(r, c, "random", 1) * 0.1, (matrix(r, c, "few", 2) * 1e-3).to(dtype), matrix(r, c, "few", 3) * 1e-2
        whole, wb = guarded((r, c), torch.bfloat16)
        w_whole, now = guarded((r, c), torch.float32)
        now.copy_(w)
        was = m.clone()
        mxc.mxc_muon_update([now], [g], [m], [wb], lr, momentum, nesterov, wd, rms, 0.5, 5, workspace(mxc, [(r, c)])[1])
        mu = float(torch.tensor(momentum, dtype=torch.float32))
        m1 = mu * was.double() + 0.5 * g.double()
        assert bool(((m.double() - m1).abs() <= 2 * U * (mu * was.abs().double() + m1.abs()) + 1e-42).all())
        u = (0.5 * g.double() + mu * m.double() if nesterov else m).float()
        del m1, was
        o = orthogonal64(u, 5)
        step = lr * rms * math.sqrt(max(r, c))
        off = now.double() - ((1.0 - lr * wd) * w.double() - step * o)
        tol = step * tolerance(u, 5, o) + 4 * U * float((w.abs() + step * o.abs()).norm())
        assert float(off.norm()) <= tol, (float(off.norm()), tol)
        assert float(off.abs().max()) <= 16 * tol / math.sqrt(r * c)        # a value by itself, as in test_tiles
        assert torch.equal(wb, now.bfloat16()) and intact(whole, wb) and intact(w_whole, now)


def test_longest_sides(mxc):
    for r, c in ((32768, 3), (70, 32768)):
        x = matrix(r, c, "random", 4)
        y = torch.empty(r, c, dtype=torch.bfloat16, device="cuda")
        mxc.mxc_orthogonalize([x], 5, [y], workspace(mxc, [(r, c)])[1])
        check(y, x, 5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("copy", [False, True])
def test_update(mxc, dtype, nesterov, copy):
    shapes = [(64, 363), (300, 64), (1, 1), (129, 257), (17, 3, 5, 5)]
    for rms, wd, lr, momentum in ((0.2, 0.1, 3e-2, 0.95), (0.0, 0.0, 1e-2, 0.0)):
        held = {k: [] for k in ("w", "g", "m", "wb")}
        for i, s in enumerate(shapes):
            r, c = s[0], math.prod(s[1:])
            for k, t, v in (("w", torch.float32, matrix(r, c, "random", i) * 0.1), ("g", dtype, matrix(r, c, "few", i + 1) * 1e-3), ("m", torch.float32, matrix(r, c, "few", i + 2) * 1e-2),
                            ("wb", torch.bfloat16, torch.zeros(r, c, device="cuda"))):
                whole, part = guarded(s, t)
                part.copy_(v.view(s))
                held[k].append((whole, part))
        was = {k: [p.clone() for _, p in v] for k, v in held.items()}
        now = {k: [p for _, p in v] for k, v in held.items()}
        two = [(s[0], math.prod(s[1:])) for s in shapes]
        ws_whole, ws = workspace(mxc, two)
        mxc.mxc_muon_update(now["w"], now["g"], now["m"], now["wb"] if copy else None, lr, momentum, nesterov, wd, rms, 0.5, 5, ws)
        for i, (r, c) in enumerate(two):
            f32 = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
            g, m, w = (was[k][i].double().view(r, c) for k in ("g", "m", "w"))
            m1 = f32(momentum) * m + 0.5 * g
            got_m = now["m"][i].double().view(r, c)
            assert bool(((got_m - m1).abs() <= 2 * U * (momentum * m.abs() + m1.abs()) + 1e-42).all())
            u = 0.5 * g + f32(momentum) * got_m if nesterov else got_m
            o = orthogonal64(u.float(), 5)
            step = lr * (rms * math.sqrt(max(r, c)) if rms else math.sqrt(max(1.0, r / c)))
            keep = 1.0 - lr * wd
            off = now["w"][i].double().view(r, c) - (keep * w - step * o)
            # u's rounding to 32 bits is one of the sums' errors; then w's own roundings
            tol = step * tolerance(u.float(), 5, o) + 4 * U * float((w.abs() + step * o.abs()).norm())
            assert float(off.norm()) <= tol, (r, c, float(off.norm()), tol)
            assert torch.equal(now["wb"][i], now["w"][i].bfloat16() if copy else torch.zeros_like(now["wb"][i]))
            assert torch.equal(now["g"][i], was["g"][i])
        assert all(intact(whole, part) for v in held.values() for whole, part in v) and intact(ws_whole, ws, 5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("nesterov", [False, True])
def test_update_of_small_matrices(mxc, dtype, nesterov):
    """One launch for 72 of them, without a workspace: the bits of a call that has a larger one too."""
    shapes = [(1 + 17 * i % 64, 1 + 131 * i % 576) if i % 2 else (1 + 131 * i % 576, 1 + 17 * i % 64) for i in range(75)]
    assert mxc.mxc_orthogonalize_workspace_bytes([r for r, _ in shapes], [c for _, c in shapes]) == 0
    def state(more):
        all_shapes = shapes + more
        return [[guarded(s, t) for s in all_shapes] for t in (torch.float32, dtype, torch.float32, torch.bfloat16)]
    results = []
    for more in ([], [(70, 600)]):
        held = state(more)
        for k, (kind, size) in enumerate((("random", 0.1), ("few", 1e-3), ("few", 1e-2))):
            for i, (_, part) in enumerate(held[k]):
                part.copy_(matrix(*part.shape, kind, i + k) * size)
        now = [[p for _, p in v] for v in held]
        ws = workspace(mxc, shapes + more)[1] if more else None
        for _ in range(2):
            mxc.mxc_muon_update(now[0], now[1], now[2], now[3], 1e-2, 0.9, nesterov, 0.1, 0.2, 0.5, 5, ws)
        assert all(intact(whole, part) for v in held for whole, part in v)
        results.append([t.clone() for v in (now[0], now[2], now[3]) for t in v[:len(shapes)]])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_streams_and_graphs(mxc):
    """On a stream of its own, and replayed from a graph: the second step of the same state as in eager calls; two graphs with one workspace, one after the other."""
    shapes = [(96, 200), (300, 40), (513, 130)]
    make = lambda: [[matrix(r, c, "random", i + k) for i, (r, c) in enumerate(shapes)] for k in range(3)]  # noqa: E731
    ws = workspace(mxc, shapes)[1]
    args = (1e-2, 0.9, True, 0.1, 0.2, 1.0, 5, ws)
    eager = make()
    for _ in range(3):
        mxc.mxc_muon_update(eager[0], eager[1], eager[2], None, *args)
    other = make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mxc.mxc_muon_update(other[0], other[1], other[2], None, *args, side)
    torch.cuda.current_stream().wait_stream(side)
    ys = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mxc.mxc_muon_update(other[0], other[1], other[2], None, *args)
    with torch.cuda.graph(second):
        mxc.mxc_orthogonalize(other[1], 5, ys, ws)
    want = [torch.empty_like(y) for y in ys]
    mxc.mxc_orthogonalize(other[1], 5, want, ws)
    for _ in range(2):
        graph.replay()
        for y in ys:
            y.fill_(3.0)
        second.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ys, want))
    for k in (0, 2):
        assert all(torch.equal(a, b) for a, b in zip(eager[k], other[k]))
