"""Embedding and its table's gradient against the formulas in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}       # half a step of a rounding, relative


@pytest.fixture(scope="module")
def mxc():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1512_01274_amd import mxc as m
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def guarded(shape, dtype, fill=5.0):
    """A tensor with sentinels behind it, and the whole."""
    n = math.prod(shape)
    whole = torch.full((n + 64,), fill, dtype=dtype, device="cuda")
    return whole, whole[:n].view(shape)


def intact(whole, part, fill=5.0):
    return bool((whole[part.numel():] == fill).all())


def some_tokens(N, V, kind, g):
    if kind == "uniform":
        t = torch.randint(0, V, (N,), generator=g, device="cuda")
    elif kind == "common":
        t = (torch.exp(torch.rand(N, generator=g, device="cuda") * math.log(V + 1.0)).long() - 1).clamp_(0, V - 1)
    elif kind == "one":
        t = torch.full((N,), V - 1, device="cuda")
    elif kind == "none":
        t = torch.full((N,), -1, device="cuda")
    elif kind == "two":
        t = torch.where(torch.arange(N, device="cuda") % 3 == 0, 0, V - 1)
    else:       # runs of 129 and of 128 equal tokens, either side of where a token's places are cut into parts
        t = torch.arange(N, device="cuda") // (129 if kind == "runs129" else 128) % V
    t[torch.rand(N, generator=g, device="cuda") < 0.05] = -1
    if N > 3:
        t[2] = V            # outside as well
        t[3] = -2 ** 31
    return t.int()


def exact_rows(tokens, V, w, scale):
    there = (tokens >= 0) & (tokens < V)
    return torch.where(there[:, None], w.double()[tokens.clamp(0, V - 1).long()] * scale, 0.0)


def exact_grad(tokens, V, dy, scale):
    """The gradient, and the bound that its tolerance counts in: places of a row, and the sum of its sizes."""
    there = (tokens >= 0) & (tokens < V)
    at, d = tokens[there].long(), dy[there].double()
    zero = torch.zeros(V, dy.shape[1], dtype=torch.float64, device="cuda")
    return zero.index_add(0, at, d) * scale, zero.index_add(0, at, d.abs()) * abs(scale), torch.bincount(at, minlength=V)[:, None]


SIZES = [(1, 1, 1), (1, 5, 3), (7, 3, 8), (64, 1000, 37), (257, 50, 264), (300, 100, 1031), (5, 9, 4096), (2000, 333, 2056)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V,C", SIZES)
def test_forward(mxc, dtype, N, V, C):
    g = gen(N * 31 + C)
    w = torch.randn(V, C, generator=g, device="cuda").to(dtype)
    tokens = some_tokens(N, V, "uniform", g)
    for scale in (1.0, -0.37, 0.0):
        whole, y = guarded((N, C), dtype)
        mxc.mxc_embedding_fwd(N, V, C, mxc.dtype_code(dtype), tokens, w, scale, y)
        want = exact_rows(tokens, V, w, torch.tensor(scale).item() if scale != -0.37 else float(torch.tensor(-0.37, dtype=torch.float32)))
        # the product's rounding to 32 bits and that to the type
        assert bool(((y.double() - want).abs() <= (HALF[dtype] + U) * 1.01 * want.abs()).all())
        assert intact(whole, y)


def test_forward_values_that_are_not_finite(mxc):
    w = torch.tensor([[math.inf, 1.0, math.nan], [-math.inf, 0.0, 2.0]], device="cuda")
    tokens = torch.tensor([1, -1, 0, 2], dtype=torch.int32, device="cuda")
    y = torch.full((4, 3), 9.0, device="cuda")
    mxc.mxc_embedding_fwd(4, 2, 3, 0, tokens, w, 2.0, y)
    want = torch.tensor([[-math.inf, 0.0, 4.0], [0, 0, 0], [math.inf, 2.0, math.nan], [0, 0, 0]], device="cuda")
    assert torch.equal(y.nan_to_num(nan=77.0), want.nan_to_num(nan=77.0))


GRADS = [(1, 1, 1, "uniform"), (3, 7, 5, "uniform"), (500, 100, 64, "common"), (1000, 1000, 33, "uniform"), (1024, 3, 520, "one"), (1024, 70, 8, "none"),
         (1025, 3, 520, "one"), (1025, 70, 8, "none"), (1500, 64, 1, "common"), (3000, 1, 3, "uniform"), (5000, 257, 1031, "common"), (4096, 4000, 24, "runs129"),
         (4100, 4000, 136, "runs128"), (9999, 2, 2056, "two"), (20000, 50257, 8, "common"), (2049, 300000, 4, "uniform"), (70001, 999, 16, "common"),
         # on either side of where one launch does it
         (2048, 256, 40, "common"), (2049, 256, 40, "common"), (2048, 255, 33, "common"), (2048, 300, 2048, "common"), (2048, 300, 2049, "common"), (1500, 400, 2100, "one"),
         (1100, 257, 65, "one"), (1024, 3, 129, "two")]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("N,V,C,kind", GRADS)
def test_gradient(mxc, dtype, add, N, V, C, kind):
    g = gen(N + V * 7 + C)
    tokens = some_tokens(N, V, kind, g)
    dy = torch.randn(N, C, generator=g, device="cuda").to(dtype)
    was = torch.randn(V, C, generator=g, device="cuda")
    whole, dw = guarded((V, C), torch.float32)
    need = mxc.mxc_embedding_workspace_bytes(N, V, C, mxc.dtype_code(dtype))
    assert need % 256 == 0
    ws_whole, ws = guarded((max(need, 256),), torch.uint8, 5)
    results = []
    for _ in range(2):
        dw.copy_(was)
        mxc.mxc_embedding_bwd(N, V, C, mxc.dtype_code(dtype), tokens, dy, 0.5, add, dw, ws)
        results.append(dw.clone())
    want, size, places = exact_grad(tokens, V, dy, 0.5)
    tol = (places + 2) * U * size
    if add:
        want = want + was.double()
        tol = tol + U * want.abs()
        assert torch.equal(results[0][places[:, 0] == 0], was[places[:, 0] == 0])
    else:
        assert not bool(results[0][places[:, 0] == 0].any())
    bad = ~((results[0].double() - want).abs() <= tol + 1e-42)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4])
    assert torch.equal(results[0], results[1])
    assert intact(whole, dw) and intact(ws_whole, ws, 5)


# More places of a segment than a wave holds in registers (over 16384 a segment), up to a million; tables of 256 MB and more, whose rows go past the caches, with more places than one
# launch takes
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("N,V,C,kind", [(100000, 50257, 8, "common"), (20000, 300000, 4, "uniform"), (99999, 1000, 3, "runs129"), (300000, 7, 4, "one"), (1000001, 50257, 4, "common"),
                                        (3000, 33000, 2048, "common"), (5000, 70000, 1001, "uniform")])
def test_gradient_of_many_places_and_rows(mxc, dtype, add, N, V, C, kind):
    test_gradient(mxc, dtype, add, N, V, C, kind)


def test_gradient_is_that_of_differences(mxc):
    """Along a direction of the table: the change of a weighted sum of the forward formula, which is linear in it."""
    g = gen(3)
    N, V, C = 1500, 40, 20
    tokens, weight = some_tokens(N, V, "common", g), torch.randn(N, C, generator=g, device="cuda")
    w, direction = (torch.randn(V, C, generator=g, device="cuda", dtype=torch.float64) for _ in range(2))
    dw = torch.empty(V, C, device="cuda")
    mxc.mxc_embedding_bwd(N, V, C, 0, tokens, weight, 0.5, False, dw, mxc.alloc_workspace(mxc.mxc_embedding_workspace_bytes(N, V, C, 0)))
    value = lambda t: (exact_rows(tokens, V, t, 0.5) * weight.double()).sum()  # noqa: E731
    change = (value(w + direction) - value(w - direction)) / 2
    _, size, places = exact_grad(tokens, V, weight, 0.5)
    tol = ((places + 2) * U * size * direction.abs()).sum() + 1e-9 * change.abs()
    assert abs(float((dw.double() * direction).sum() - change)) <= float(tol)


def test_gradient_rows_with_infinities_touch_their_token_alone(mxc):
    N, V, C = 2000, 50, 24
    g = gen(5)
    tokens = (torch.arange(N, device="cuda") % V).int()
    dy = torch.randn(N, C, generator=g, device="cuda")
    dy[7, 3], dy[8, 0], dy[V + 8, 0] = math.nan, math.inf, -math.inf
    dw = torch.empty(V, C, device="cuda")
    mxc.mxc_embedding_bwd(N, V, C, 0, tokens, dy, 1.0, False, dw, mxc.alloc_workspace(mxc.mxc_embedding_workspace_bytes(N, V, C, 0)))
    want = torch.zeros(V, C, dtype=torch.bool, device="cuda")
    want[7, 3] = want[8, 0] = True
    assert torch.equal(dw.isnan(), want) and bool(dw[~want].isfinite().all())


def test_offsets_past_32_bits(mxc):
    """Tables, inputs and gradients of more than 2^32 bytes and 2^31 values."""
    V, C = 66000, 32768
    w = torch.zeros(V, C, dtype=torch.bfloat16, device="cuda")
    tokens = torch.tensor([V - 1, 0, 65536, -1, V - 1], dtype=torch.int32, device="cuda")
    for i, v in enumerate((V - 1, 0, 65536)):
        w[v] = i + 1
    y = torch.empty(5, C, dtype=torch.bfloat16, device="cuda")
    mxc.mxc_embedding_fwd(5, V, C, 1, tokens, w, 2.0, y)
    assert torch.equal(y, torch.tensor([2, 4, 6, 0, 2], dtype=torch.bfloat16, device="cuda")[:, None].expand(5, C))
    # the gradient of as many places, all rows of w as dy
    many = (torch.arange(V, device="cuda") % 3).int()
    dw = torch.empty(3, C, device="cuda")
    mxc.mxc_embedding_bwd(V, 3, C, 1, many, w, 1.0, False, dw, mxc.alloc_workspace(mxc.mxc_embedding_workspace_bytes(V, 3, C, 1)))
    want = torch.zeros(3, device="cuda")
    for i, v in enumerate((V - 1, 0, 65536)):
        want[v % 3] += i + 1
    assert torch.equal(dw, want[:, None].expand(3, C))
    del w, y
    dw = torch.full((V, C), 3.0, device="cuda")
    dy = torch.ones(5, C, device="cuda")
    mxc.mxc_embedding_bwd(5, V, C, 0, tokens, dy, 1.0, True, dw)
    assert bool((dw[V - 1] == 5).all()) and bool((dw[65536] == 4).all()) and bool((dw[0] == 4).all()) and bool((dw[V - 2] == 3).all())
    mxc.mxc_embedding_bwd(5, V, C, 0, tokens, dy, 1.0, False, dw)
    assert float(dw.sum(dtype=torch.float64)) == 4 * C


def test_streams_and_graphs(mxc):
    """On a stream of its own, and replayed from a graph with other tokens in the same places."""
    g = gen(11)
    N, V, C = 3000, 500, 72
    tokens, dy = some_tokens(N, V, "common", g), torch.randn(N, C, generator=g, device="cuda").bfloat16()
    w, y, dw = torch.randn(V, C, generator=g, device="cuda").bfloat16(), torch.empty(N, C, device="cuda", dtype=torch.bfloat16), torch.empty(V, C, device="cuda")
    ws = mxc.alloc_workspace(mxc.mxc_embedding_workspace_bytes(N, V, C, 1))
    few = tokens[:200].clone()
    dw_few = torch.zeros(V, C, device="cuda")

    def calls(stream=None):
        mxc.mxc_embedding_fwd(N, V, C, 1, tokens, w, 1.5, y, stream)
        mxc.mxc_embedding_bwd(N, V, C, 1, tokens, y, 1.5, False, dw, ws, stream)
        mxc.mxc_embedding_bwd(200, V, C, 1, few, y, 1.5, False, dw_few, None, stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    calls(side)
    torch.cuda.current_stream().wait_stream(side)
    first = [t.clone() for t in (y, dw, dw_few)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for turn in range(4):
        if turn:
            tokens.copy_(some_tokens(N, V, ("common", "one", "uniform")[turn - 1], g))
            few.copy_(tokens[:200])
        for t in (y, dw, dw_few):
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dw, dw_few)]
        for t in (y, dw, dw_few):
            t.fill_(9.0)
        calls()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, dw, dw_few)))
        if turn == 0:
            assert all(torch.equal(a, b) for a, b in zip(got, first))
