"""AdamW over many tensors against the formula in 64 bits; states of 8 bits against the neighbours they may take."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
H = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, wd=0.1, grad_scale=0.5)


@pytest.fixture(scope="module")
def mxc():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1512_01274_amd import mxc as m
    return m


def make(n, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + n)
    r = lambda: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    size = torch.exp2(torch.randint(-20, 3, (n // 32 + 1, 1), generator=g, device="cuda").float()).expand(-1, 32).reshape(-1)[:n]
    grad = r() * size
    grad[torch.rand(n, generator=g, device="cuda") < 0.1] = 0
    return r(), grad.to(dtype), r() * size * 0.3, (r() * size) ** 2


def guarded(t):
    """A copy of t with sentinels behind it; the whole and the part that holds t."""
    whole = torch.full((t.numel() + 64,), 5, dtype=t.dtype, device="cuda")
    whole[:t.numel()] = t
    return whole, whole[:t.numel()]


def exact_step(w, g, m, v, step, h=H):
    w, g, m, v = (t.double() for t in (w, g, m, v))
    g = g * h["grad_scale"]
    part = h["beta1"] * m.abs() + (1 - h["beta1"]) * g.abs()
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g * g
    denominator = torch.sqrt(v / (1 - h["beta2"] ** step)) + h["eps"]
    rate = h["lr"] / (1 - h["beta1"] ** step)
    new = w - h["lr"] * h["wd"] * w - rate * m / denominator
    # roundings: four in m and its parts, in v and its parts; w's two; the quotient's, of m's parts and of the denominator
    return new, m, v, 4 * U * w.abs() + 2 * U * new.abs() + 24 * U * rate * part / denominator, 8 * U * part, 8 * U * v


def near(got, want, tol):
    bad = ~((got.double() - want).abs() <= tol + 1e-42)
    assert not bool(bad.any()), (int(bad.sum()), got[bad][:4], want[bad][:4])


SIZES = [[1], [5, 0, 7], [255, 256, 257], [1023, 1024, 1025, 4095, 4096, 4097], [i % 97 + 1 for i in range(200)], [100000, 3, 65536 * 3 + 1], [0, 0, 9, 0], [2000001]]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("copy", [True, False])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_adamw(mxc, dtype, copy, sizes):
    data = [make(n, dtype, i) for i, n in enumerate(sizes)]
    for step in (1, 1000):
        held = [[guarded(t) for t in d] for d in data]
        w, g, m, v = ([h[k][1] for h in held] for k in range(4))
        wb = [guarded(torch.zeros(n, dtype=torch.bfloat16, device="cuda")) for n in sizes]
        mxc.mxc_adamw_update(w, g, m, v, [b[1] for b in wb] if copy else None, **H, step=step)
        for i, d in enumerate(data):
            new, mm, vv, tw, tm, tv = exact_step(*d, step)
            near(w[i], new, tw)
            near(m[i], mm, tm)
            near(v[i], vv, tv)
            assert torch.equal(g[i], d[1])
            assert torch.equal(wb[i][1], w[i].bfloat16() if copy else torch.zeros_like(wb[i][1]))
            for whole, part in held[i] + [wb[i]]:
                assert bool((whole[part.numel():] == 5).all())


def values8(state, n):
    """m, r of n values and what one step between codes is at each (float64)."""
    out = []
    rec = state.view(-1, 528)
    for base, sc in ((0, 512), (256, 520)):
        codes = rec[:, base:base + 256].contiguous().view(torch.float8_e4m3fn).double()
        scale = torch.exp2(rec[:, sc:sc + 8].double() - 127).repeat_interleave(32, 1)
        step = torch.exp2(torch.floor(torch.log2(codes.abs().clamp(min=2.0 ** -6))) - 3)
        out += [(codes * scale).reshape(-1)[:n], (step * scale).reshape(-1)[:n]]
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_adamw8(mxc, dtype, sizes):
    """Four steps: weights by the formula from the states as they were; states the neighbours of the formula's; the scale's rule."""
    data = [make(n, dtype, i) for i, n in enumerate(sizes)]
    w = [guarded(d[0]) for d in data]
    state = [guarded(torch.zeros(mxc.mxc_adamw8_state_bytes(n), dtype=torch.uint8, device="cuda")) for n in sizes]
    wb = [guarded(torch.zeros(n, dtype=torch.bfloat16, device="cuda")) for n in sizes]
    for step in (1, 2, 3, 4):
        grads = [make(n, dtype, i + 31 * step)[1] for i, n in enumerate(sizes)]
        before = [(a[1].clone(), s[1].clone()) for a, s in zip(w, state)]
        mxc.mxc_adamw8_update([a[1] for a in w], grads, [s[1] for s in state], [b[1] for b in wb], **H, step=step, seed=step * 12345)
        for i, n in enumerate(sizes):
            if n == 0:
                continue
            m0, _, r0, _ = values8(before[i][1], n)
            new, m, v, tw, tm, tv = exact_step(before[i][0], grads[i], m0, r0 * r0, step)
            near(w[i][1], new, tw)
            assert torch.equal(wb[i][1], w[i][1].bfloat16())
            m1, sm, r1, sr = values8(state[i][1], n)
            r = torch.sqrt(v)
            # a neighbour: less than the larger of the two steps that meet at it away, and the 32-bit value's own error
            assert bool(((m1 - m).abs() <= sm * (1 + 2.0 ** -15) + tm).all()) and bool(((r1 - r).abs() <= sr * (1 + 2.0 ** -15) + 16 * U * r).all())
            assert bool((r1[r > 1e-40] > 0).all())
            rec = state[i][1].view(-1, 528)
            for x, at in ((m, 512), (r, 520)):
                block = torch.nn.functional.pad(x.abs(), (0, rec.shape[0] * 256 - n)).view(-1, 8, 32).amax(2)
                scale = torch.exp2(rec[:, at:at + 8].double() - 127)
                live = block > 1e-34
                assert bool((block <= 448.0001 * scale)[live].all()) and bool((block * 1.0001 > 224 * scale)[live].all())
                assert not bool(rec[:, at:at + 8][block == 0].any())
            codes = rec[:, :512].reshape(-1, 2, 256).transpose(0, 1).reshape(2, -1)
            assert not bool(codes[:, n:].any())       # places past the last value
            for whole, part in (w[i], state[i], wb[i]):
                assert bool((whole[part.numel():] == 5).all())


def test_adamw8_mean_and_seed(mxc):
    """The same call gives the same codes, another seed or tensor number others; over many seeds a code's mean is the value."""
    n = 4096
    w, g, _, _ = make(n, torch.float32, 5)
    bytes_ = mxc.mxc_adamw8_state_bytes(n)

    def run(seed, tensors=1):
        state = [torch.zeros(bytes_, dtype=torch.uint8, device="cuda") for _ in range(tensors)]
        mxc.mxc_adamw8_update([w.clone() for _ in state], [g] * tensors, state, None, **H, step=1, seed=seed)
        return state
    a, b = run(7, 95), run(7, 95)       # more than one launch
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert len({bytes(x.cpu().numpy().tobytes()) for x in a}) == 95
    assert not torch.equal(a[0], a[1]) and not torch.equal(a[0], a[72]) and not torch.equal(a[1], a[73]) and not torch.equal(a[0], run(8)[0])
    _, m, v, _, _, _ = exact_step(w, g, torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), 1)
    total_m, total_r, rounds = 0.0, 0.0, 400
    for seed in range(rounds):
        m1, sm, r1, sr = values8(run(seed * 977)[0], n)
        total_m, total_r = total_m + m1, total_r + r1
    # a mean of 400 choices between two neighbours: deviation at most step / 2 / 20; six of them, over 4096 values
    assert bool(((total_m / rounds - m).abs() <= 6 * sm / 40 + 1e-40).all())
    big = torch.sqrt(v) > sr            # (a small r that would be 0 half of the time is kept above it)
    assert bool(((total_r / rounds - torch.sqrt(v)).abs() <= 6 * sr / 40)[big].all())
    assert abs(float(((total_m / rounds - m) / sm).mean())) <= 6 / 40 / math.sqrt(n) * 1.5


def test_not_finite(mxc):
    """A gradient that is not finite reaches its own weight; in 8 bits its block of 32 reads as NaN from then on."""
    n = 600
    w, g, m, v = make(n, torch.float32, 1)
    g[3], g[300], g[599] = math.inf, math.nan, -math.inf
    at = torch.zeros(n, dtype=torch.bool, device="cuda")
    at[[3, 300, 599]] = True
    w1, m1, v1 = w.clone(), m.clone(), v.clone()
    mxc.mxc_adamw_update([w1], [g], [m1], [v1], None, **H, step=2)
    assert torch.equal(~v1.isfinite(), at) and torch.equal(~m1.isfinite(), at) and torch.equal(w1.isnan(), at)
    w1, state = w.clone(), torch.zeros(mxc.mxc_adamw8_state_bytes(n), dtype=torch.uint8, device="cuda")
    mxc.mxc_adamw8_update([w1], [g], [state], None, **H, step=2, seed=3)
    assert torch.equal(w1.isnan(), at)
    rec = state.view(-1, 528)
    bad = torch.nn.functional.pad(at, (0, 768 - n)).view(3, 8, 32).any(2)
    assert torch.equal(rec[:, 512:520] == 255, bad) and torch.equal(rec[:, 520:] == 255, bad)
    mxc.mxc_adamw8_update([w1], [torch.zeros_like(g)], [state], None, **H, step=3, seed=4)
    assert torch.equal(w1.isnan(), bad.repeat_interleave(32, 1).reshape(-1)[:n])


def test_graph(mxc):
    """A captured step: the factors are the call's, the data the replay's."""
    sizes = [300, 5000, 17]
    data = [make(n, torch.bfloat16, i) for i, n in enumerate(sizes)]
    w, g, m, v = ([d[k].clone() for d in data] for k in range(4))
    state = [torch.zeros(mxc.mxc_adamw8_state_bytes(n), dtype=torch.uint8, device="cuda") for n in sizes]
    w8 = [t.clone() for t in w]

    def both():
        mxc.mxc_adamw_update(w, g, m, v, None, **H, step=5)
        mxc.mxc_adamw8_update(w8, g, state, None, **H, step=5, seed=9)
    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    everything = w + m + v + w8 + state
    for i in range(4):
        start = [t.clone() for t in everything]
        both()
        torch.cuda.synchronize()
        want = [t.clone() for t in everything]
        for t, s in zip(everything, start):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(everything, want))
        for t in g:
            t.copy_(torch.randn(t.numel(), device="cuda"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_more_than_the_caches(mxc, dtype, bits):
    """More than 256 MB, which pass the caches by."""
    sizes = [34000003, 5, 2999]
    if bits == 32:
        test_adamw(mxc, dtype, True, sizes)
    else:
        test_adamw8(mxc, dtype, sizes)


@pytest.mark.parametrize("bits", [32, 8])
def test_past_32_bits(mxc, bits):
    """A tensor of more than 2^31 values: its last ones are those of a tensor of these alone (8 bits: the weights, after one step)."""
    n, last = (1 << 31) + 256 * 4 + 77, 256 * 3 + 77
    w, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(4)
    w[n - last:], g[n - last:] = torch.randn(last, generator=gen, device="cuda"), torch.randn(last, generator=gen, device="cuda").bfloat16()
    small = w[n - last:].clone(), g[n - last:].clone()
    copy = torch.empty(n, device="cuda", dtype=torch.bfloat16)
    if bits == 32:
        m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        sm, sv = torch.zeros(last, device="cuda"), torch.zeros(last, device="cuda")
        mxc.mxc_adamw_update([w], [g], [m], [v], [copy], **H, step=1)
        mxc.mxc_adamw_update([small[0]], [small[1]], [sm], [sv], None, **H, step=1)
        assert torch.equal(m[n - last:], sm) and torch.equal(v[n - last:], sv)
    else:
        state = torch.zeros(mxc.mxc_adamw8_state_bytes(n), dtype=torch.uint8, device="cuda")
        ss = torch.zeros(mxc.mxc_adamw8_state_bytes(last), dtype=torch.uint8, device="cuda")
        mxc.mxc_adamw8_update([w], [g], [state], [copy], **H, step=1, seed=1)
        mxc.mxc_adamw8_update([small[0]], [small[1]], [ss], None, **H, step=1, seed=1)
        assert torch.equal(state.view(-1, 528)[-4:, 512:], ss.view(-1, 528)[:, 512:])
    assert torch.equal(w[n - last:], small[0]) and torch.equal(copy[n - last:], small[0].bfloat16()) and not bool(w[:n - last].any())
