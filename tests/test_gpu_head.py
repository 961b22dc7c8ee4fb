"""The operators together: a head that is trained and then served in 4 bits, against the same steps in plain fp32."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def head():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1512_01274_amd import head as h
    return h


def plain_training(net, batches, lr, wd):
    """The same steps by autograd and the formula in fp32; the losses."""
    w = [p.clone().requires_grad_() for p in net.w]
    m, v = [torch.zeros_like(p) for p in w], [torch.zeros_like(p) for p in w]
    losses = []
    for t, (x, labels) in enumerate(batches, 1):
        z = torch.relu(x.float() @ w[0].t() + w[1]) @ w[2].t() + w[3]
        loss = torch.nn.functional.cross_entropy(z, labels.long())
        grads = torch.autograd.grad(loss, w)
        losses.append(float(loss.detach()))
        with torch.no_grad():
            for p, g, a, b in zip(w, grads, m, v):
                a.mul_(0.9).add_(g, alpha=0.1)
                b.mul_(0.999).add_(g * g, alpha=0.001)
                p.mul_(1 - lr * wd).sub_(lr / (1 - 0.9 ** t) * a / ((b / (1 - 0.999 ** t)).sqrt() + 1e-8))
    return losses


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("features,hidden,classes,N", [(64, 96, 37, 48), (512, 1024, 1000, 256)])
def test_trained_and_served(head, bits, features, hidden, classes, N):
    """Losses follow those of the same steps in fp32: bf16 rounds activations and gradients by 2^-9 each and 8-bit states their moments by 2^-4
    without bias, far less than the batches differ among each other.  Served in 4 bits most answers stay."""
    net, batch = head.Head(features, hidden, classes, bits), head.clusters(features, classes)
    batches = [batch(N) for _ in range(150)]
    plain = plain_training(net, batches, 1e-3, 0.01)
    ours = [-float(net.train_step(*b).mean()) for b in batches]
    assert abs(ours[0] - plain[0]) <= 2.0 ** -6 * plain[0]
    assert ours[-1] < 0.5 * ours[0]
    for i in range(0, 150, 25):
        assert abs(sum(ours[i:i + 25]) - sum(plain[i:i + 25])) <= 0.1 * sum(plain[i:i + 25]) + 0.25, i
    x, labels = batch(N)
    z = torch.relu(x.float() @ net.copy[0].float().t() + net.w[1]) @ net.copy[2].float().t() + net.w[3]
    logp, entropy, top_logp, top = net.served().score(x, labels, top=3)
    assert float((top[:, 0] == z.argmax(1)).float().mean()) > 0.5
    assert bool((top_logp[:, 0] >= top_logp[:, 1]).all()) and bool((entropy >= 0).all()) and bool((logp <= 0).all())


def test_first_gradients(head):
    """One step's gradients against autograd of the same network in fp32 (bf16 activations and gradients between the layers: a rounding
    each, 2^-8 of what is summed)."""
    net, batch = head.Head(128, 160, 50), head.clusters(128, 50)
    w = [c.float().requires_grad_() if c.dim() == 2 else p.clone().requires_grad_() for c, p in zip(net.copy, net.w)]
    x, labels = batch(64)
    net.train_step(x, labels)
    h = torch.relu(x.float() @ w[0].t() + w[1])
    logits = h @ w[2].t() + w[3]
    torch.nn.functional.cross_entropy(logits, labels.long()).backward()
    for ours, theirs in zip(net.grad, w):
        assert float((ours - theirs.grad).abs().max()) <= 2.0 ** -5 * float(theirs.grad.abs().max())


@pytest.mark.parametrize("bits", [32, 8])
def test_results_of_a_step_stay(head, bits):
    """A step's log probabilities are the caller's: the next steps of the same batch size leave them as they are."""
    net, batch = head.Head(64, 96, 37, bits), head.clusters(64, 37)
    kept = [net.train_step(*batch(48)) for _ in range(3)]
    first = [k.clone() for k in kept]
    net.train_step(*batch(48))
    assert all(torch.equal(a, b) for a, b in zip(kept, first)) and not torch.equal(kept[0], kept[1]) and not torch.equal(kept[1], kept[2])
