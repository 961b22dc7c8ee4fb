"""The embedding, layer norm, layers, loss and both optimisers as a next-token model uses them: gradients of a whole step against the same network in 64 bits,
steps against the formulas, steps from a captured graph against eager ones."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tokens():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1512_01274_amd import tokens as t
    return t


# vocabulary, channels, hidden, window, rows
SIZES = [(37, 24, 40, 3, 20), (1000, 512, 1024, 4, 256), (5, 9, 7, 1, 1), (50257, 72, 136, 2, 130), (300, 257, 100, 5, 64)]


def plain(tokens, model, rows, labels):
    """(log probabilities, gradients) of the mean of -logp in 64 bits, from the weights that the layers read."""
    w = [(c if c.dim() == 2 else p).double().cpu().requires_grad_() for c, p in zip(model.copy, model.w)]
    rows, labels = rows.cpu().long(), labels.cpu().long()
    N, T = rows.shape
    inside = (rows >= 0) & (rows < w[0].shape[0])
    e = torch.where(inside[..., None], w[0][rows.clamp(0, w[0].shape[0] - 1)], torch.zeros((), dtype=torch.float64))
    norm = lambda x, g, b: torch.nn.functional.layer_norm(x, x.shape[-1:], g, b, tokens.EPS)  # noqa: E731
    a = norm(e, w[1], w[2]).reshape(N, -1)
    u = torch.relu(a @ w[3].t() + w[4]) @ w[5].t() + w[6]
    logits = norm(u, w[7], w[8]) @ w[0].t()
    has = labels >= 0
    logp = torch.where(has, torch.log_softmax(logits, 1).gather(1, labels.clamp(min=0)[:, None])[:, 0], torch.zeros((), dtype=torch.float64))
    return logp.detach(), torch.autograd.grad(-logp.sum() / N, w)


def trained(tokens, sizes, steps):
    """A model some steps after its start, so that biases and norms' weights are not what they began with, and a batch of it."""
    V, C, H, T, N = sizes
    model, batch = tokens.Model(V, C, H, T), tokens.text(V, T)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for i in (tokens.G0, tokens.B0, tokens.C1, tokens.C2, tokens.G1, tokens.B1):
        model.w[i].add_(0.1 * torch.randn(model.w[i].shape, generator=gen, device="cuda"))
    for _ in range(steps):
        model.train_step(*batch(N))
    rows, labels = batch(N)
    if N > 2:
        labels[1] = -1
        rows[2, 0] = V                      # outside of the table: as padding
    return model, batch, rows, labels


def by_steps(tokens, model, rows, labels, rounded):
    """(log probabilities, gradients) by the formulas in 64 bits; `rounded`: what a tensor between the calls goes through."""
    table, g0, b0, w1, c1, w2, c2, g1, b1 = [(c if c.dim() == 2 else p).double().cpu() for c, p in zip(model.copy, model.w)]
    rows, labels = rows.cpu().long(), labels.cpu().long()
    (N, T), (V, C) = rows.shape, table.shape
    inside = ((rows >= 0) & (rows < V)).reshape(-1, 1)
    at = rows.reshape(-1).clamp(0, V - 1)

    def norm(x, g, b):
        mean, var = x.mean(1, keepdim=True), x.var(1, unbiased=False, keepdim=True)
        rstd = (var + tokens.EPS).rsqrt()
        return (x - mean) * rstd, rstd, rounded((x - mean) * rstd * g + b)

    def norm_back(z, rstd, g, dy):
        q = dy * g
        return rounded(rstd * (q - q.mean(1, keepdim=True) - z * (q * z).mean(1, keepdim=True))), (dy * z).sum(0), dy.sum(0)

    z0, rstd0, a = norm(torch.where(inside, table[at], 0.0), g0, b0)
    a = a.reshape(N, T * C)
    h = rounded(torch.relu(a @ w1.t() + c1))
    z1, rstd1, o = norm(rounded(h @ w2.t() + c2), g1, b1)
    logits = rounded(o @ table.t())
    has, label = ((labels >= 0) & (labels < V))[:, None], labels.clamp(0, V - 1)[:, None]
    logs = torch.log_softmax(logits, 1)
    logp = torch.where(has, logs.gather(1, label), 0.0)[:, 0]
    dz = rounded(torch.where(has, logs.exp().scatter_add(1, label, torch.full((N, 1), -1.0, dtype=torch.float64)), 0.0) / N)
    do = rounded(dz @ table)
    du, dg1, db1 = norm_back(z1, rstd1, g1, do)
    dh = rounded((du @ w2) * (h > 0))
    da = rounded(dh @ w1).reshape(N * T, C)
    de, dg0, db0 = norm_back(z0, rstd0, g0, da)
    dtable = (dz.t() @ o).index_add(0, at, torch.where(inside, de, 0.0))
    return logp, [dtable, dg0, db0, dh.t() @ a, dh.sum(0), du.t() @ h, du.sum(0), dg1, db1]


@pytest.mark.parametrize("sizes", SIZES)
def test_gradients(tokens, sizes):
    """Against the formulas with what lies between the calls rounded to bf16 as there (which by itself is up to a tenth of a norm's weights' gradients, whose terms
    cancel), the formulas themselves against autograd.  Sums of up to 2048 fp32 terms are off by 2^-18 or so of their terms' norm, by which one value in some hundreds is
    rounded to the other side, by a step of 2^-7: in the norm 2^-11, for ten such tensors 2^-9, and eight times that where terms cancel."""
    model, _, rows, labels = trained(tokens, sizes, 2)
    auto_logp, auto = plain(tokens, model, rows, labels)
    exact_logp, exact = by_steps(tokens, model, rows, labels, lambda x: x)
    assert float((exact_logp - auto_logp).abs().max()) <= 1e-12 * (1 + float(auto_logp.abs().max()))
    for i, (g, r) in enumerate(zip(exact, auto)):
        assert float((g - r).norm()) <= 1e-9 * float(r.norm()) + 1e-12, i
    want_logp, want = by_steps(tokens, model, rows, labels, lambda x: x.bfloat16().double())
    logp = torch.full((rows.shape[0],), 7.0, device="cuda")
    for g in model.grad:
        g.fill_(float("nan"))
    model.gradients(rows, labels, logp)
    assert float((logp.cpu().double() - want_logp).abs().max()) <= 2.0 ** -6 * (1.0 + float(want_logp.abs().max()))
    for i, (g, r) in enumerate(zip(model.grad, want)):
        assert bool(g.isfinite().all()), i
        off = float((g.cpu().double() - r).norm())
        assert off <= 2.0 ** -6 * float(r.norm()) + 1e-12, i


def test_gradient_is_the_difference(tokens):
    """The loss's change along a direction of all tensors, by differences of the network in 64 bits, against the gradients' product with it, which the roundings between the
    calls change: ten of 2^-8 of what is summed, 2^-4.6 of the product of the norms."""
    model, _, rows, labels = trained(tokens, SIZES[0], 2)
    logp = torch.empty(rows.shape[0], device="cuda")
    model.gradients(rows, labels, logp)
    gen = torch.Generator().manual_seed(5)
    along = [torch.randn(w.shape, generator=gen, dtype=torch.float64) for w in model.w]
    copies, weights, losses, h = model.copy, model.w, [], 1e-5
    for sign in (1, -1):
        model.w = [w.double().cpu() + sign * h * d for w, d in zip(weights, along)]
        model.copy = [c.double().cpu() + sign * h * d for c, d in zip(copies, along)]
        losses.append(-float(plain(tokens, model, rows, labels)[0].mean()))
    got = sum(float((g.cpu().double() * d).sum()) for g, d in zip(model.grad, along))
    norm = sum(float(g.double().square().sum()) for g in model.grad) ** 0.5
    size = sum(float(d.square().sum()) for d in along) ** 0.5
    assert abs(got - (losses[0] - losses[1]) / (2 * h)) <= 2.0 ** -4.6 * norm * size


@pytest.mark.parametrize("which", range(9))
def test_gradient_of_each_tensor_is_the_difference(tokens, which):
    """The loss's change along one tensor's own gradient g, by differences of the network in 64 bits, against |g|: a gradient that is missing is off by all of it, one of the other sign by
    twice that.  A rounding to bf16 is off by 2^-9.8 of a tensor's norm (a half step of 2^-8, evenly spread over values between two powers of two); ten of them between the
    calls make 2^-8.1, eight times that where terms cancel (2^-5.1), and 2^-3 leaves four times that."""
    model, _, rows, labels = trained(tokens, SIZES[0], 2)
    logp = torch.empty(rows.shape[0], device="cuda")
    model.gradients(rows, labels, logp)
    g = model.grad[which].double().cpu()
    size = float(g.norm())
    assert size > 0
    copies, weights, losses, h = model.copy, model.w, [], 1e-5
    for sign in (1, -1):
        model.w, model.copy = [w.double().cpu() for w in weights], [c.double().cpu() for c in copies]
        for tensors in (model.w, model.copy):
            tensors[which] = tensors[which] + sign * h * g / size
        losses.append(-float(plain(tokens, model, rows, labels)[0].mean()))
    change = (losses[0] - losses[1]) / (2 * h)
    assert abs(change - size) <= 2.0 ** -3 * size


@pytest.mark.parametrize("sizes", SIZES[:3])
def test_updates(tokens, sizes):
    """What a step changes, by the gradients that it leaves.  Filters: the momentum is fp32 arithmetic of two operations; the step has singular values of 0.68 to 1.21
    times lr 0.2 sqrt(longest side) for those of the direction that are not small, and 1.21 bounds all.  The others: AdamW's first step is lr of either sign, eps 1e-8
    beside the gradient's root apart, and the decay.  Copies are the weights, rounded once."""
    V, C, H, T, N = sizes
    model, batch = tokens.Model(V, C, H, T), tokens.text(V, T)
    before = [w.clone() for w in model.w]
    model.train_step(*batch(N), lr=1e-2, wd=0.1)
    for i in range(9):
        g, w, old = model.grad[i].double(), model.w[i].double(), before[i].double()
        assert torch.equal(model.copy[i], model.w[i].bfloat16()), i
        rest = (old * (1 - 1e-3) - w) / 1e-2
        assert bool(rest.isfinite().all())
        if i in tokens.FILTERS:
            assert float((model.m[i].double() - g).abs().max()) <= 2.0 ** -23 * float(g.abs().max())
            s = torch.linalg.svdvals(rest.cpu()) / (0.2 * max(g.shape) ** 0.5)
            lead = float(((rest * g).sum() / rest.norm() / g.norm().clamp(min=1e-30)))
            assert float(s[0]) <= 1.21 + 2.0 ** -9 and (float(g.norm()) == 0 or (float(s[0]) >= 0.67 and lead > 0)), i
        else:
            # fp32: old and w are of the size of the weights, their difference is divided by lr
            off = (rest - g / (g.abs() + 1e-8)).abs().max()
            assert float(off) <= 2.0 ** -22 * float(old.abs().max() + 1) / 1e-2 + 2.0 ** -18, i


def test_captured(tokens):
    """Gradients and filters' steps captured once and replayed, with eager work of other sizes between: the bits of the eager steps."""
    V, C, H, T, N = SIZES[1]
    model, batch, rows, labels = trained(tokens, SIZES[1], 1)
    logp = torch.empty(N, device="cuda")
    other, other_batch = tokens.Model(37, 24, 40, 3), tokens.text(37, 3)
    from paper_1512_01274_amd import mxc

    def steps():
        model.gradients(rows, labels, logp)
        pick = lambda tensors: [tensors[i] for i in tokens.FILTERS]  # noqa: E731
        mxc.mxc_muon_update(pick(model.w), pick(model.grad), pick(model.m), pick(model.copy), 1e-3, 0.95, True, 0.01, 0.2, 1.0, 5, model._update)

    kept = [model.w, model.copy, model.m]
    start = [[t.clone() for t in ts] for ts in kept]
    batches = [batch(N) for _ in range(4)]

    def reset():
        for ts, olds in zip(kept, start):
            for t, old in zip(ts, olds):
                t.copy_(old)

    results = []
    for r, l in batches:
        rows.copy_(r)
        labels.copy_(l)
        steps()
        results.append([t.clone() for t in model.grad + model.w + [logp]])
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps()
    reset()
    for (r, l), want in zip(batches, results):
        rows.copy_(r)
        labels.copy_(l)
        graph.replay()
        other.train_step(*other_batch(50))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(model.grad + model.w + [logp], want))


def test_captured_among_other_batch_sizes(tokens):
    """A captured batch's gradients keep their bits when eager batches of more and of fewer rows come between."""
    V, C, H, T = 300, 72, 100, 3
    model, batch = tokens.Model(V, C, H, T), tokens.text(V, T)
    rows, labels = batch(100)
    logp = torch.empty(100, device="cuda")
    model.gradients(rows, labels, logp)
    want = [t.clone() for t in model.grad + [logp]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        model.gradients(rows, labels, logp)
    for N in (120, 65, 7, 400, 100):
        other = torch.empty(N, device="cuda")
        model.gradients(*batch(N), other)
        model.predict(batch(N)[0])
        for t in model.grad + [logp]:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(model.grad + [logp], want)), N


def test_on_another_stream(tokens):
    """The same model's steps on a stream of their own have the bits of the first stream's."""
    runs = []
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream()):
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            model, batch = tokens.Model(300, 72, 100, 3), tokens.text(300, 3)
            for _ in range(3):
                model.train_step(*batch(90))
        torch.cuda.synchronize()
        runs.append([w.clone() for w in model.w])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_asked(tokens):
    """The most probable next tokens of single rows are those of a batch's, ordered, and their log probabilities those of the network in 64 bits."""
    model, batch, rows, labels = trained(tokens, SIZES[0], 3)
    logp, index = model.predict(rows)
    assert logp.shape == index.shape == (20, 5) and bool((logp[:, :-1] >= logp[:, 1:]).all())
    for k in range(5):
        want = plain(tokens, model, rows, index[:, k])[0]
        assert float((logp[:, k].cpu() - want).abs().max()) <= 2.0 ** -5 * (1.0 + float(want.abs().max()))
    one = model.predict(rows[3:4].contiguous())
    assert float((one[0] - logp[3:4]).abs().max()) <= 2.0 ** -5 * (1.0 + float(logp[3].abs().max()))


def test_command(tokens, capsys):
    tokens.main("--vocabulary 50 --channels 32 --hidden 48 --window 2 --batch 96 --steps 3".split())
    assert "step    2  loss" in capsys.readouterr().out
