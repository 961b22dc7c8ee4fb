"""Log probabilities, entropies, top tokens and gradients against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16]
U = 2.0 ** -24


@pytest.fixture(scope="module")
def mxc():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1512_01274_amd import mxc as m
    return m


def exact(z, labels, scale, dlogp=None, dentropy=None):
    """logp, entropy, log p of every entry and dz of rows z (float64), by the definition."""
    N, K = z.shape
    most = z.amax(1, keepdim=True)
    empty = most == -math.inf
    d = (z - most.masked_fill(empty, 0.0)) * scale
    e = torch.exp(d)
    S = e.sum(1, keepdim=True).masked_fill(empty, 1.0)
    lp, p = d - torch.log(S), e / S
    plp = torch.where(p > 0, p * lp, p * 0.0)       # (a NaN stays)
    H = -plp.sum(1)
    given = (labels >= 0) & (labels < K)
    at = labels.clamp(0, K - 1).long().unsqueeze(1)
    logp = torch.where(given, lp.gather(1, at).squeeze(1), 0.0)
    if dlogp is None:
        return logp, H, lp, p, d
    dl, dh = (dlogp.double() * given)[:, None], dentropy.double()[:, None]
    dz = -dl * p - dh * (plp + p * H[:, None])
    dz.scatter_add_(1, at, dl)
    return logp, H, lp, p, d, torch.where(empty, 0.0, dz * scale)


def near(got, want, tol):
    got, want = got.double(), want.double()
    # (beyond 32 bits a finite value is minus infinity)
    same = (got == want) | (got.isnan() & want.isnan()) | ((got < -3.0e38) & (want < -3.0e38) & (want > -math.inf))
    bad = ~(same | ((got - want).abs() <= tol))
    assert not bool(bad.any()), (int(bad.sum()), got[bad][:4], want[bad][:4])


def row_tol(lp, H):
    """A log probability in 32 bits: d is off by a few roundings of its size; the sum of the exponentials by a rounding for each link of
    a chain of at most 1000, and by its terms' own errors, which are d's (weighted by p, where d is small)."""
    return U * (8 * lp.abs() + 1024), U * 1024 * (1 + H)


def data(N, K, ld, dtype, seed, masked):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(N, ld, generator=g, device="cuda") * 3
    if masked:
        z[torch.rand(N, ld, generator=g, device="cuda") < 0.1] = -math.inf if masked == 1 else float(torch.finfo(dtype).min)
    z = z.to(dtype)
    if ld > K:
        z[:, K:] = float("nan")         # between two rows nothing is read
    labels = torch.randint(0, K, (N,), generator=g, device="cuda", dtype=torch.int32)
    if N > 3:
        labels[1], labels[2] = -1, K
        if masked:
            z[3, :K] = -math.inf if masked == 1 else float(torch.finfo(dtype).min)
    return z, labels, torch.randn(N, generator=g, device="cuda"), torch.randn(N, generator=g, device="cuda")


def check(mxc, N, K, pad, dtype, masked, scale, top, seed=0, offset=0.0):
    ld = K + pad
    z, labels, dlogp, dentropy = data(N, K, ld, dtype, seed + N + K, masked)
    if offset:
        z = (z.float() + offset).to(dtype)
    scale = float(np.float32(scale))
    code = mxc.dtype_code(dtype)
    logp, H, lp, p, d, dz = exact(z[:, :K].double(), labels, scale, dlogp, dentropy)
    tl, th = row_tol(logp, H)
    new = lambda *s, dtype=torch.float32: torch.full((math.prod(s) + 16,), 77, dtype=dtype, device="cuda")  # noqa: E731
    got = {"logp": new(N), "entropy": new(N), "stats": new(N, 2), "tl": new(N, top), "ti": new(N, top, dtype=torch.int32)}
    ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, top))
    if ws is not None:
        ws.fill_(0xFF)
    mxc.mxc_logprob_fwd(N, K, ld, code, z, labels, scale, top, got["logp"], got["entropy"], got["stats"], got["tl"] if top else None,
                        got["ti"] if top else None, ws)
    for k, n in (("logp", N), ("entropy", N), ("stats", 2 * N), ("tl", N * top), ("ti", N * top)):
        assert bool((got[k][n:] == 77).all()), k
    near(got["logp"][:N], logp, tl)
    near(got["entropy"][:N], H, th)
    stats = got["stats"][:2 * N].view(N, 2)
    most = z[:, :K].double().amax(1)
    assert torch.equal(stats[:, 0].double(), most)
    empty = most == -math.inf
    near(stats[:, 1], torch.where(empty, 0.0, torch.log(torch.exp(d).sum(1))), U * 1024)
    if top:
        n = min(top, K)
        ti, tlp = got["ti"][:N * top].view(N, top), got["tl"][:N * top].view(N, top)
        # a stable sort of what the type holds: of equal values the lowest index first
        want = torch.sort(z[:, :K].double() + 0.0, dim=1, descending=True, stable=True).indices[:, :n]
        assert torch.equal(ti[:, :n].long(), want)
        assert bool((ti[:, n:] == -1).all()) and bool((tlp[:, n:] == -math.inf).all())
        wl = lp.gather(1, want)
        over = wl < -3.0e38         # beyond 32 bits: minus infinity or the lowest
        assert bool((tlp[:, :n][over] < -3.0e38).all())
        near(torch.where(over, 0.0, tlp[:, :n].double()), torch.where(over, 0.0, wl), torch.where(over, 0.0, U * (8 * wl.abs() + 1024)))
    # the gradient: a value's own rounding and the errors of its parts
    grow = 8 * d.clamp(min=-200).abs() + 1024
    TS = (p * d.clamp(min=-1e30)).sum(1, keepdim=True).abs()
    dl = dlogp.double()[:, None].abs()
    onehot = torch.zeros_like(p).scatter_(1, labels.clamp(0, K - 1).long()[:, None], 1.0)
    tol = U * scale * (dl * (2 * onehot + p * grow) + dentropy.double()[:, None].abs() * p * (d.clamp(min=-200).abs() + TS + 1) * grow)
    tol = torch.nan_to_num(tol, nan=0.0) + torch.nan_to_num(dz.abs()) * torch.finfo(dtype).eps / 2 + 1e-37
    out = new(N, ld, dtype=dtype)
    l2, h2 = new(N), new(N)
    ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, 0))
    mxc.mxc_logprob_fwd_bwd(N, K, ld, code, z, labels, scale, dlogp, dentropy, l2, h2, out, ws)
    near(l2[:N], logp, tl)
    near(h2[:N], H, th)
    rows = out[:N * ld].view(N, ld)
    near(rows[:, :K], dz, tol)
    assert bool((rows[:, K:] == 77).all()) and bool((out[N * ld:] == 77).all())
    # from the statistics of the forward pass; in place
    buf = z.clone()
    mxc.mxc_logprob_bwd(N, K, ld, code, buf, labels, scale, got["stats"], got["entropy"], dlogp, dentropy, buf)
    near(buf[:, :K], dz, tol)
    assert bool(buf[:, K:].isnan().all())
    buf = z.clone()
    mxc.mxc_logprob_fwd_bwd(N, K, ld, code, buf, labels, scale, dlogp, dentropy, l2, h2, buf, ws)
    assert torch.equal(buf[:, :K], rows[:, :K])


# lengths on both sides of every way of holding a row: one to some values, whole and broken 16-byte pieces, a wave's, a workgroup's, more
LENGTHS = [1, 2, 3, 7, 8, 9, 31, 64, 65, 127, 255, 256, 257, 511, 512, 513, 1000, 1023, 1025, 2047, 2049, 4095, 4097, 8191, 8193, 16385, 32767, 32769]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", LENGTHS)
def test_lengths(mxc, dtype, K):
    check(mxc, 6, K, 0, dtype, 0, 1.0, 5)
    check(mxc, 5, K, 3, dtype, 1, 0.7, 64, seed=1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,K,pad", [(1, 131072, 0), (3, 131071, 1), (2, 131073, 0), (600, 50257, 47), (300, 50257, 0), (2, 300001, 5), (300, 70001, 0),
                                     (2000, 10, 0), (1500, 129, 7), (4099, 33, 0), (1, 1, 0), (700, 1000, 0), (290, 131072, 0), (260, 140000, 1)])
def test_rows(mxc, dtype, N, K, pad):
    if N * K > 2.5e7 and dtype == torch.float32:
        N = 258
    check(mxc, N, K, pad, dtype, 0, 1.0, 20)
    check(mxc, min(N, 280), K, pad, dtype, 2, 1.4, 1, seed=2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset", [1000.0, -30000.0, 1.0e30])
def test_far_from_zero(mxc, dtype, offset):
    """Probabilities do not depend on where the logits lie, but for what the type holds of them."""
    check(mxc, 4, 5000, 3, dtype, 0, 1.0, 8, offset=offset)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [40, 3000, 140001])
def test_ties_and_peaks(mxc, dtype, K):
    """Equal logits, all of them or the largest few; descending, ascending and alternating rows; -0 beside 0."""
    N, top = 7, 64
    z = torch.zeros(N, K, device="cuda")
    z[1] = -torch.arange(K, device="cuda") * 0.25
    z[2] = torch.arange(K, device="cuda") * 0.25
    z[3, ::2] = -0.0
    z[4, K // 2:] = 3.0
    z[5] = -math.inf
    z[6, ::3] = 50.0
    z = z.to(dtype)
    index = torch.empty(N, top, dtype=torch.int32, device="cuda")
    tl, logp, H = torch.empty(N, top, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    labels = torch.zeros(N, dtype=torch.int32, device="cuda")
    code = mxc.dtype_code(dtype)
    ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, top))
    mxc.mxc_logprob_fwd(N, K, K, code, z, labels, 1.0, top, logp, H, None, tl, index, ws)
    n = min(K, top)
    assert torch.equal(index[:, :n].long(), torch.sort(z.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :n])
    w = exact(z.double(), labels, 1.0)
    near(H, w[1], row_tol(w[0], w[1])[1])
    near(logp, w[0], row_tol(w[0], w[1])[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [50, 5000, 140001])
def test_not_finite(mxc, dtype, K):
    """A NaN or plus infinity makes its row NaN and no other one."""
    N = 5
    z, labels, dlogp, dentropy = data(N, K, K, dtype, 3, 0)
    labels.fill_(1)
    z[0, K - 1], z[2, K // 2], z[3, 0] = math.nan, math.inf, -math.nan
    logp, H, dz = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(z)
    code = mxc.dtype_code(dtype)
    mxc.mxc_logprob_fwd_bwd(N, K, K, code, z, labels, 1.0, dlogp, dentropy, logp, H, dz, mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, 0)))
    bad = torch.tensor([True, False, True, True, False], device="cuda")
    for t in (logp, H, dz):
        assert bool(t[bad].isnan().all()) and bool(t[~bad].isfinite().all())


@pytest.mark.parametrize("K", [6, 700])
def test_gradient_by_differences(mxc, K):
    """dz against central differences of the weighted sum of logp and entropy, both in 64 bits but for dz."""
    z, labels, dlogp, dentropy = data(3, K, K, torch.float32, 9, 0)
    dz = torch.empty_like(z)
    mxc.mxc_logprob_fwd_bwd(3, K, K, 0, z, labels, 0.5, dlogp, dentropy, None, None, dz, mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(3, K, 0, 0)))
    h = 2.0 ** -14

    def total(zz):
        logp, H = exact(zz, labels, 0.5)[:2]
        return logp * dlogp.double() + H * dentropy.double()
    for k in list(range(min(K, 6))) + [int(labels[0])]:
        step = torch.zeros(3, K, device="cuda", dtype=torch.float64)
        step[:, k] = h
        slope = (total(z.double() + step) - total(z.double() - step)) / (2 * h)
        # sums of at most 20 links in 32 bits; the third derivative times h^2/6 and 64-bit rounding over 2h are smaller
        assert bool(((dz[:, k].double() - slope).abs() <= 64 * U * (dlogp.abs() + 20 * dentropy.abs())).all()), k


def test_parts_left_out(mxc):
    """NULL outputs and gradients."""
    N, K = 5, 3001
    z, labels, dlogp, dentropy = data(N, K, K, torch.bfloat16, 4, 1)
    zero = torch.zeros(N, device="cuda")
    ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, 1, 64))
    a, b = torch.empty_like(z), torch.empty_like(z)
    for dl, dh in ((dlogp, None), (None, dentropy), (None, None)):
        mxc.mxc_logprob_fwd_bwd(N, K, K, 1, z, labels, 1.0, dl, dh, None, None, a, ws)
        mxc.mxc_logprob_fwd_bwd(N, K, K, 1, z, labels, 1.0, zero if dl is None else dl, zero if dh is None else dh, None, None, b, ws)
        assert torch.equal(a, b)
    full = [torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, 2, device="cuda")]
    mxc.mxc_logprob_fwd(N, K, K, 1, z, labels, 1.0, 0, *full, None, None, ws)
    for i in range(3):
        part = [torch.empty_like(t) if i == j else None for j, t in enumerate(full)]
        mxc.mxc_logprob_fwd(N, K, K, 1, z, labels if i == 0 else None, 1.0, 0, *part, None, None, ws)
        assert torch.equal(part[i], full[i])


def test_graph_and_stream(mxc):
    """Captured on a stream of its own and replayed on new inputs, with eager work between the replays."""
    for N, K in ((1, 140000), (300, 6000)):
        z, labels, dlogp, dentropy = data(N, K, K, torch.bfloat16, 5, 0)
        logp, H, dz = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(z)
        tl, ti = torch.empty(N, 9, device="cuda"), torch.empty(N, 9, device="cuda", dtype=torch.int32)
        ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, 1, 9))

        def both():
            mxc.mxc_logprob_fwd(N, K, K, 1, z, labels, 1.0, 9, logp, H, None, tl, ti, ws)
            mxc.mxc_logprob_fwd_bwd(N, K, K, 1, z, labels, 1.0, dlogp, dentropy, logp, H, dz, ws)
        both()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both()
        for i in range(4):
            z.copy_(data(N, K, K, torch.bfloat16, 50 + i, i % 3)[0])
            both()
            torch.cuda.synchronize()
            want = [t.clone() for t in (logp, H, dz, tl, ti)]
            for t in (logp, H, dz, tl, ti):
                t.fill_(1)
            graph.replay()
            torch.cuda.synchronize()
            for t, w in zip((logp, H, dz, tl, ti), want):
                assert torch.equal(torch.nan_to_num(t.float()), torch.nan_to_num(w.float()))


@pytest.mark.parametrize("N,K,pad,dtype", [(2700, 50257, 0, torch.bfloat16), (5000, 30000, 0, torch.bfloat16), (2300, 30001, 2, torch.float32), (5000, 14000, 0, torch.float32),
                                           (1100, 131072, 0, torch.bfloat16)])
def test_more_than_the_caches(mxc, N, K, pad, dtype):
    """More than 256 MB of logits, which pass the caches by; with top tokens and without."""
    check(mxc, N, K, pad, dtype, 0, 1.0, 20)
    check(mxc, N, K, pad, dtype, 2, 1.4, 0, seed=2)


# rows of 8192, 8193, 16384 and 16385 pieces of 16 bytes; fewer and more than 160 rows; rows that begin at any value
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pieces", [8192, 8193, 16384, 16385])
@pytest.mark.parametrize("N", [159, 160])
def test_borders_of_the_cuts(mxc, dtype, pieces, N):
    V = 16 // dtype.itemsize
    check(mxc, N, pieces * V, 0, dtype, 1, 0.8, 7)
    check(mxc, N, pieces * V - 2 * V + 2, 1, dtype, 0, 1.0, 64, seed=3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,K,pad", [(200, 20000, 3), (300, 20000, 0), (20, 70001, 1)])
def test_rows_of_one_value(mxc, dtype, N, K, pad):
    """Rows whose values are all the same, or all but few: the first indices; few chunks, one, many."""
    top = 64
    z = torch.full((N, K + pad), float("nan"), device="cuda")
    z[:, :K] = torch.arange(N, device="cuda")[:, None] % 9 - 4.0
    z[1::4, K - 3:K] = 9.0
    z[2::4, :K] = -math.inf
    z[2::4, K // 2:K // 2 + 2] = 1.0
    z = z.to(dtype)
    code = mxc.dtype_code(dtype)
    ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, top))
    logp, index = torch.empty(N, top, device="cuda"), torch.empty(N, top, dtype=torch.int32, device="cuda")
    mxc.mxc_logprob_fwd(N, K, K + pad, code, z, None, 1.0, top, None, None, None, logp, index, ws)
    want = torch.sort(z[:, :K].double(), dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(index.long(), want)
    _, _, lp, _, _ = exact(z[:, :K].double(), torch.zeros(N, dtype=torch.int32, device="cuda"), 1.0)
    lp = lp.gather(1, want)
    near(logp, lp, torch.where(lp == -math.inf, 0.0, U * (8 * lp.abs() + 1024)))


@pytest.mark.parametrize("dtype", DTYPES)
def test_past_32_bits(mxc, dtype):
    """More than 2^32 bytes and 2^31 values of logits: the last rows are the ones that a call of these alone gives."""
    N, K, ld, top, last = 43000, 50257, 50261, 9, 5
    z = torch.empty(N, ld, dtype=dtype, device="cuda")
    z[:N - last] = 0
    rows, labels, dlogp, dentropy = data(last, K, ld, dtype, 3, 0)
    z[N - last:] = rows
    wide = lambda t: torch.cat([torch.zeros(N - last, dtype=t.dtype, device="cuda"), t])  # noqa: E731
    code = mxc.dtype_code(dtype)
    got = []
    for n, x, lab, dl, dh in ((N, z, wide(labels), wide(dlogp), wide(dentropy)), (last, rows, labels, dlogp, dentropy)):
        logp, H, stats = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
        tl, ti = torch.empty(n, top, device="cuda"), torch.empty(n, top, dtype=torch.int32, device="cuda")
        mxc.mxc_logprob_fwd(n, K, ld, code, x, lab, 1.0, top, logp, H, stats, tl, ti, mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(n, K, code, top)))
        dz = torch.empty(n, ld, dtype=dtype, device="cuda")
        mxc.mxc_logprob_bwd(n, K, ld, code, x, lab, 1.0, stats, H, dl, dh, dz)
        mxc.mxc_logprob_fwd_bwd(n, K, ld, code, x, lab, 1.0, dl, dh, None, None, x, mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(n, K, code, 0)))
        got.append([t[-last:] for t in (logp, H, stats, tl, ti, dz[:, :K], x[:, :K])])
    for a, b in zip(*got):
        if a.dtype == torch.int32:
            assert torch.equal(a, b)
        else:       # two ways of summing: twice the bound of one, of values of at most some tens
            near(a, b, 2 * U * 1024 * (1 + b.double().abs()) + torch.finfo(a.dtype).eps * b.double().abs())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [3, 70, 250, 511, 700, 1000, 2040])
def test_few_allowed(mxc, dtype, K):
    """Rows in which a few tokens are allowed and the others share one value, the type's lowest or another; crowded and scattered; top of 1 to 64."""
    N = 60
    g = torch.Generator(device="cuda").manual_seed(K)
    z = torch.full((N, K), float(torch.finfo(dtype).min), device="cuda")
    z[1::4] = -2.0
    z[2::4] = 1.5
    for n in range(N):
        many = n * K // N
        at = torch.randperm(K, generator=g, device="cuda")[:many] if n % 3 else torch.arange(K - many, K, device="cuda")
        z[n, at] = (torch.randint(-3, 3, (many,), generator=g, device="cuda") if n % 5 else torch.randn(many, generator=g, device="cuda")).float() - (4.0 if n % 7 == 0 else 0.0)
    z = z.to(dtype)
    code = mxc.dtype_code(dtype)
    order = torch.sort(z.double(), dim=1, descending=True, stable=True).indices
    _, _, lp, _, _ = exact(z.double(), torch.zeros(N, dtype=torch.int32, device="cuda"), 1.0)
    for top in (1, 7, 20, 64):
        ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, top))
        logp, index = torch.empty(N, top, device="cuda"), torch.empty(N, top, dtype=torch.int32, device="cuda")
        mxc.mxc_logprob_fwd(N, K, K, code, z, None, 1.0, top, None, None, None, logp, index, ws)
        n = min(top, K)
        assert torch.equal(index[:, :n].long(), order[:, :n]) and bool((index[:, n:] == -1).all())
        want = lp.gather(1, order[:, :n])
        over = want < -3.0e38
        assert bool((logp[:, :n][over] < -3.0e38).all())
        near(torch.where(over, 0.0, logp[:, :n].double()), torch.where(over, 0.0, want), torch.where(over, 0.0, U * (8 * want.abs() + 1024)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [129, 204, 378, 511, 900])
def test_fewer_pieces_than_top(mxc, dtype, K):
    """More best tokens than the row has 16-byte pieces, or pieces with a value."""
    check(mxc, 9, K, 1, dtype, 0, 1.0, 64, seed=7)
    check(mxc, 9, K, 0, dtype, 1, 1.0, 64, seed=8)
    check(mxc, 9, K, 5, dtype, 2, 0.6, 63, seed=9)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,pieces", [(1, 2048), (1, 2049), (63, 2049), (64, 2049), (63, 8192), (64, 8192), (64, 8193), (2, 7283)])
def test_gradient_of_few_long_rows(mxc, dtype, N, pieces):
    V = 16 // dtype.itemsize
    check(mxc, N, pieces * V, 0, dtype, 2, 0.8, 3)
    check(mxc, N, (pieces - 2) * V + 2, 1, dtype, 1, 1.0, 0, seed=3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,K", [(5, 6), (5, 300), (5, 3000), (1, 70000), (300, 20000)])
def test_far_masked_tokens(mxc, dtype, N, K):
    """The log probability of a masked token is scale times its logit as long as 32 bits hold that: scales around log 2, masks of the lowest value."""
    for scale in (0.25, 0.7, 0.75, 0.95, 1.0):
        z = torch.randn(N, K, generator=torch.Generator(device="cuda").manual_seed(K), device="cuda") + 3
        z[:, K // 2:] = float(torch.finfo(dtype).min) * 0.875
        z[0, 0] = 1e30
        z = z.to(dtype)
        labels = torch.full((N,), K - 1, dtype=torch.int32, device="cuda")
        top = min(64, K)
        code, s = mxc.dtype_code(dtype), float(np.float32(scale))
        want, _, lp, _, _ = exact(z.double(), labels, s)
        logp, tl, ti = torch.empty(N, device="cuda"), torch.empty(N, top, device="cuda"), torch.empty(N, top, dtype=torch.int32, device="cuda")
        mxc.mxc_logprob_fwd(N, K, K, code, z, labels, s, top, logp, None, None, tl, ti, mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, top)))
        near(logp, want, U * (8 * want.abs() + 1024))
        lp = lp.gather(1, ti.long())
        near(tl, lp, U * (8 * lp.abs() + 1024))
        z[0, 1] = math.nan
        mxc.mxc_logprob_fwd(N, K, K, code, z, labels, s, 0, logp, None, None, None, None, mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, top)))
        assert bool(logp[0].isnan()) and bool(logp[1:].isfinite().all())


def gradient_tol(z, labels, scale, dlogp, dentropy, dtype):
    """The definition's logp, H, dz, and how far a gradient may be off: its own rounding and the errors of its parts (as in check);
    exponentials below 2^-126 of the largest are nothing."""
    logp, H, lp, p, d, dz = exact(z.double(), labels, scale, dlogp, dentropy)
    grow = 8 * d.clamp(min=-200).abs() + 1024
    TS = (p * d.clamp(min=-1e30)).sum(1, keepdim=True).abs()
    onehot = torch.zeros_like(p).scatter_(1, labels.clamp(0, z.shape[1] - 1).long()[:, None], 1.0)
    part = U * p * grow + torch.where(p > 0, 2.0 ** -126, 0.0)
    tol = scale * (dlogp.double()[:, None].abs() * (2 * U * onehot + part) + dentropy.double()[:, None].abs() * part * (d.clamp(min=-200).abs() + TS + 1))
    return logp, H, dz, tol + dz.abs() * torch.finfo(dtype).eps / 2 + 1e-37


# rows of eight lanes, of a wave with one and four pieces a lane, of 256, 512 and 1024 threads, in chunks
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,bytes_", [(40, 80), (40, 600), (40, 3000), (40, 7000), (40, 14000), (40, 30000), (200, 60000), (200, 120000), (200, 250000), (3, 120000), (40, 300000)])
def test_gradient_of_masked_tokens(mxc, dtype, N, bytes_):
    """Tokens masked by numbers whose product with a strong weight of the entropy leaves 32 bits: they have no gradient, the others theirs."""
    K = bytes_ // dtype.itemsize - 3
    gen = torch.Generator(device="cuda").manual_seed(K)
    code, lowest = mxc.dtype_code(dtype), float(torch.finfo(dtype).min)
    ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, 0))
    for scale, mask, weight in ((0.5, lowest, 8.0), (0.6, lowest, -3.0), (0.25, lowest, 1e5), (1.0, -2e38, 3.0), (10.0, -2e37, 0.5), (1.0, lowest, -1e5), (1.0, -math.inf, 1e36),
                                (0.5, lowest, -1e36), (0.5, -1e4, 1e36)):
        z = torch.rand(N, K, generator=gen, device="cuda") * 6 - 3
        z[:, ::2] = mask
        z[:, 2] = 9.0           # most of the probability, or (rows below) one allowed token alone
        z[1, 3:] = mask
        z[2, :] = mask
        z[2, K - 1] = -1.5
        z = z.to(dtype)
        labels = torch.randint(0, K, (N,), generator=gen, device="cuda", dtype=torch.int32)
        labels[0] = 2
        s = float(np.float32(scale))
        dlogp = torch.randn(N, generator=gen, device="cuda")
        dentropy = (torch.rand(N, generator=gen, device="cuda") + 0.5) * weight
        logp, H, dz, tol = gradient_tol(z, labels, s, dlogp, dentropy, dtype)
        l, h, out = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(z)
        mxc.mxc_logprob_fwd_bwd(N, K, K, code, z, labels, s, dlogp, dentropy, l, h, out, ws)
        tl, th = row_tol(logp, H)
        near(l, logp, tl)
        near(h, H, th)
        near(out, dz, tol)
        stats = torch.empty(N, 2, device="cuda")
        mxc.mxc_logprob_fwd(N, K, K, code, z, None, s, 0, None, h, stats, None, None, ws)
        mxc.mxc_logprob_bwd(N, K, K, code, z, labels, s, stats, h, dlogp, dentropy, out)
        near(out, dz, tol)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,K,pad", [(5, 13, 0), (5, 300, 5), (6, 5001, 3), (200, 9001, 0), (2, 70001, 1)])
def test_scales_at_the_ends(mxc, dtype, N, K, pad):
    """Temperatures near the ends of what 32 bits hold, with broken 16-byte pieces."""
    for scale in (1e-30, 1.7e-33, 1e-36, 1e-38, 1e-42, 1e37):
        for masked in (0, 1, 2):
            check(mxc, N, K, pad, dtype, masked, scale, 7, seed=masked)


def set_bits(z, row, places, kind):
    """NaN of either sign or plus infinity at places of a row, as bits."""
    bits = {"nan": 0x7FC0, "-nan": 0xFFC0, "inf": 0x7F80}[kind]
    if z.dtype == torch.float32:
        z.view(torch.int32)[row, places] = bits << 16 if bits < 0x8000 else (bits << 16) - (1 << 32)
    else:
        z.view(torch.int16)[row, places] = bits if bits < 0x8000 else bits - (1 << 16)


# rows of a wave, of a workgroup, streamed whole and in chunks
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,K", [(12, 3), (12, 100), (12, 500), (12, 1500), (12, 2900), (12, 7000), (300, 20000), (12, 20000), (12, 140001)])
def test_top_of_rows_that_are_not_finite(mxc, dtype, N, K):
    """Log probabilities are NaN, tokens in the order of their logits, with a NaN past the infinity of its sign; other rows are as ever."""
    z = data(N, K, K, dtype, K, 0)[0]
    gen = torch.Generator(device="cuda").manual_seed(K)
    z[4, 1:] = -math.inf
    for row, share, kind in ((0, 1.0, "nan"), (1, 1.0, "-nan"), (2, 1.0, "inf"), (5, 0.1, "nan"), (6, 0.1, "-nan"), (7, 0.1, "inf"), (10, 0.5, "nan"), (10, 0.5, "-nan")):
        set_bits(z, row, torch.rand(K, generator=gen, device="cuda") < share, kind)
    for row, kind in ((4, "nan"), (5, "nan"), (6, "-nan"), (7, "inf"), (9, "nan"), (9, "inf"), (10, "-nan")):
        set_bits(z, row, torch.randint(0, K, (1,), generator=gen, device="cuda"), kind)
    bad = ~(z.isfinite() | (z == -math.inf)).all(1)
    # the values' bits as whole numbers in the order of the values
    wide = z.view(torch.int32) if dtype == torch.float32 else z.view(torch.int16).int() << 16
    rank = torch.where(wide < 0, wide ^ 0x7FFFFFFF, wide).long()
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices
    code = mxc.dtype_code(dtype)
    _, _, lp, _, _ = exact(z.double(), torch.zeros(N, dtype=torch.int32, device="cuda"), 1.0)
    for top in (1, 20, 64):
        ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, top))
        H, stats = torch.empty(N, device="cuda"), torch.empty(N, 2, device="cuda")
        tl, ti = torch.empty(N, top, device="cuda"), torch.empty(N, top, dtype=torch.int32, device="cuda")
        mxc.mxc_logprob_fwd(N, K, K, code, z, None, 1.0, top, None, H, stats, tl, ti, ws)
        n = min(top, K)
        assert torch.equal(ti[:, :n].long(), order[:, :n])
        assert bool(tl[bad][:, :n].isnan().all())
        assert bool((ti[:, n:] == -1).all()) and bool((tl[:, n:] == -math.inf).all())
        want = lp.gather(1, order[:, :n])[~bad]
        near(tl[~bad][:, :n], want, torch.where(want == -math.inf, 0.0, U * (8 * want.abs() + 1024)))
        assert bool(H[bad].isnan().all()) and bool(stats[bad].isnan().all()) and bool(H[~bad].isfinite().all()) and bool(stats[~bad].isfinite().all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [2, 7, 9, 33, 64, 100, 257, 500, 1000, 1500, 2047, 4000, 8100])
@pytest.mark.parametrize("masked,scale", [(0, 1.0), (2, 0.7), (1, 1.3)])
def test_close(mxc, dtype, K, masked, scale):
    """The bounds of `check` with the chain that a row of K values really has: a thread adds 128 values of its row at most, lanes and waves 22 more.
    Errors of d are 2.5 roundings of its size (of the scale's product, the factor and the difference), an exponential's is two and d's, a sum's one a link
    and the terms' own; twice that, for what is divided, multiplied and put together from them."""
    N = 9
    z, labels, dlogp, dentropy = data(N, K, K, dtype, K + masked, masked)
    s = float(np.float32(scale))
    logp, H, lp, p, d, dz = exact(z.double(), labels, s, dlogp, dentropy)
    a = torch.where(p > 0, d.abs(), 0.0)        # (a token without probability has no part in any sum)
    n = 2 * (min(K, 128) + 22) + 16
    m1, m2 = (p * a).sum(1), (p * a * a).sum(1)
    logS = torch.where(H > 0, H, 0.0) + m1
    tl = U * (n + 8 * torch.where(logp > -math.inf, logp.abs(), 0.0) + 8 * m1 + 8 * logS)
    th = U * (n * (1 + m1) + 8 * m2 + 8 * (logS + m1))
    m1, m2 = m1[:, None], m2[:, None]
    dl, dh = dlogp.double()[:, None].abs(), dentropy.double()[:, None].abs()
    onehot = torch.zeros_like(p).scatter_(1, labels.clamp(0, K - 1).long()[:, None], 1.0)
    tz = U * s * (2 * dl * onehot + p * (dl * (n + 8 * a + 8 * m1) + dh * (n * (1 + a + m1) + 8 * (a * a + a * m1 + m2)))) + dz.abs() * torch.finfo(dtype).eps / 2 + 1e-37
    code, top = mxc.dtype_code(dtype), min(K, 20)
    ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, top))
    l, h, stats, out = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, 2, device="cuda"), torch.empty_like(z)
    t, ti = torch.empty(N, top, device="cuda"), torch.empty(N, top, dtype=torch.int32, device="cuda")
    mxc.mxc_logprob_fwd_bwd(N, K, K, code, z, labels, s, dlogp, dentropy, l, h, out, ws)
    near(l, logp, tl)
    near(h, H, th)
    near(out, dz, tz)
    mxc.mxc_logprob_fwd(N, K, K, code, z, labels, s, top, l, h, stats, t, ti, ws)
    near(l, logp, tl)
    near(h, H, th)
    want = lp.gather(1, ti.long())
    size = torch.where(want > -3e38, want.abs(), 0.0)
    near(torch.where(want > -3e38, t.double(), 0.0), torch.where(want > -3e38, want, 0.0), U * (n + 8 * size + 8 * (m1 + logS[:, None])))
    mxc.mxc_logprob_bwd(N, K, K, code, z, labels, s, stats, h, dlogp, dentropy, out)
    near(out, dz, tz)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pieces", [257, 300, 400, 511, 513, 554, 640, 767, 768, 769, 900, 1023])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_few_tokens_of_no_less_than_zero(mxc, dtype, pieces, top):
    """Rows of which fewer logits than `top` are 0 or more, or one is: the others are negative, or one masked value; of lengths that fill some of a
    thread's pieces."""
    N, K = 24, pieces * 16 // dtype.itemsize - 3
    gen = torch.Generator(device="cuda").manual_seed(pieces)
    z = -torch.rand(N, K, generator=gen, device="cuda") * 5 - 0.5
    z[1::3] = torch.where(torch.rand(N, K, generator=gen, device="cuda") < 0.03, z, torch.tensor(-1e4, device="cuda"))[1::3]
    z[2::3] = -1e20
    for n in range(N):
        at = torch.randperm(K, generator=gen, device="cuda")[:n * top // N + 1]
        z[n, at] = torch.randint(0, 4, (len(at),), generator=gen, device="cuda").float()
    z = z.to(dtype)
    code = mxc.dtype_code(dtype)
    ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, top))
    logp, index = torch.empty(N, top, device="cuda"), torch.empty(N, top, dtype=torch.int32, device="cuda")
    mxc.mxc_logprob_fwd(N, K, K, code, z, None, 1.0, top, None, None, None, logp, index, ws)
    order = torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(index.long(), order)
    want = exact(z.double(), torch.zeros(N, dtype=torch.int32, device="cuda"), 1.0)[2].gather(1, order)
    near(logp, want, U * (8 * want.abs() + 1024))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,K", [(5, 30), (9, 3001), (70, 27974), (3, 70001)])
def test_small_scales_with_large_weights(mxc, dtype, N, K):
    """A scale that is hardly a normal number, divided by a large sum, under weights that bring the gradient back into range."""
    for scale, weight in ((2.5e-38, 1e13), (1e-36, 1e30), (3e36, 1e-30)):
        s = float(np.float32(scale))
        z, labels, dlogp, dentropy = data(N, K, K, dtype, K, 0)
        z[1] *= 2.0 / s if s < 1 else 1.0       # (within what either type holds)
        z[1].clamp_(-1e38, 1e38)
        dlogp, dentropy = dlogp * weight, dentropy * weight
        logp, H, dz, tol = gradient_tol(z, labels, s, dlogp, dentropy, dtype)
        code = mxc.dtype_code(dtype)
        ws = mxc.alloc_workspace(mxc.mxc_logprob_workspace_bytes(N, K, code, 0))
        out, h, stats = torch.empty_like(z), torch.empty(N, device="cuda"), torch.empty(N, 2, device="cuda")
        mxc.mxc_logprob_fwd_bwd(N, K, K, code, z, labels, s, dlogp, dentropy, None, None, out, ws)
        near(out, dz, tol)
        mxc.mxc_logprob_fwd(N, K, K, code, z, None, s, 0, None, h, stats, None, None, ws)
        mxc.mxc_logprob_bwd(N, K, K, code, z, labels, s, stats, h, dlogp, dentropy, out)
        near(out, dz, tol)
