"""A next-token model of a fixed window, trained and asked: the library's embedding, layer norm, layers, loss and optimisers together.

A row is the `window` tokens before a place, -1 where the text has none.  Their rows of the table, normalised, are the first layer's input; two
FullyConnected layers bring them to one row, which is normalised and multiplied with the same table: the logits.  A training step is that, the log
probabilities of the labels with the gradient of their mean, the gradients backwards - the table's is the last product's and the places' added -
and the updates: the two filters' by Muon, the table, biases and layer norms' weights by AdamW.  No label (-1): no loss and no gradient.

Usage: python -m paper_1512_01274_amd.tokens [--vocabulary 1000] [--steps 200]
"""
import argparse

import torch

from paper_1512_01274_amd import mxc

BF16, EPS = mxc.MXC_BF16, 1e-5
TABLE, G0, B0, W1, C1, W2, C2, G1, B1 = range(9)
FILTERS, OTHERS = (W1, W2), (TABLE, G0, B0, C1, C2, G1, B1)


class Model:
    """Master weights in fp32 (table, first norm, two layers, last norm), copies of those that the layers read in bf16."""

    def __init__(self, vocabulary, channels, hidden, window, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        V, C, H, T = self.dims = vocabulary, channels, hidden, window
        shapes = [(V, C), (C,), (C,), (H, T * C), (H,), (C, H), (C,), (C,), (C,)]
        scale = {TABLE: C ** -0.5, W1: (2.0 / (T * C)) ** 0.5, W2: (2.0 / H) ** 0.5}
        self.w = [torch.randn(s, generator=gen, device=device) * scale[i] if i in scale else torch.full(s, 1.0 if i in (G0, G1) else 0.0, device=device)
                  for i, s in enumerate(shapes)]
        self.copy = [w.bfloat16() for w in self.w]
        self.grad, self.m, self.v = ([torch.zeros_like(w) for w in self.w] for _ in range(3))
        self.step, self._buffers, self._workspaces, self._need = 0, {}, {}, {}
        self._update = mxc.alloc_workspace(mxc.mxc_orthogonalize_workspace_bytes(*zip(*(shapes[i] for i in FILTERS))), device=device)

    def _of_batch(self, N):
        """Activations, gradients and workspace for batches of N.  Rows of a buffer and bytes of a workspace are a power of two, each made once and kept, for a captured step goes on using
        them: all together are less than twice the largest of each."""
        V, C, H, T = self.dims
        device, rows = self.w[0].device, 1 << (N - 1).bit_length()
        if N not in self._need:
            need = [mxc.mxc_conv2d_workspace_bytes(op, N, c, 1, 1, k, 1, 1, 1, 0, BF16, mxc.MXC_NHWC) for c, k in ((T * C, H), (H, C), (C, V))
                    for op in (mxc.MXC_FWD, mxc.MXC_BWD_DATA, mxc.MXC_BWD_DATA_RELU, mxc.MXC_BWD_WEIGHT, mxc.MXC_BIAS_GRAD)]
            need += [mxc.mxc_logprob_workspace_bytes(N, V, BF16, top) for top in (0, min(V, 5))]
            need += [mxc.mxc_embedding_workspace_bytes(N * T, V, C, BF16), mxc.mxc_layernorm_workspace_bytes(N * T, C, BF16), mxc.mxc_layernorm_workspace_bytes(N, C, BF16)]
            self._need[N] = 1 << max(max(need) - 1, 0).bit_length()
        if rows not in self._buffers:
            new = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device=device)  # noqa: E731
            self._buffers[rows] = {"e": new(rows * T, C), "a": new(rows * T, C), "s0": new(rows * T, 2, dtype=torch.float32), "h": new(rows, H), "u": new(rows, C), "o": new(rows, C),
                                   "s1": new(rows, 2, dtype=torch.float32), "z": new(rows, V), "da": new(rows * T, C), "dh": new(rows, H), "du": new(rows, C),
                                   "weight": new(rows, dtype=torch.float32)}
        if self._need[N] not in self._workspaces:
            self._workspaces[self._need[N]] = mxc.alloc_workspace(self._need[N], device=device)
        return {**self._buffers[rows], "workspace": self._workspaces[self._need[N]]}

    def _rows(self, tokens):
        V, C, H, T = self.dims
        if tokens.dim() != 2 or tokens.shape[1] != T or tokens.dtype != torch.int32 or not tokens.is_contiguous():
            raise ValueError(f"expected dense int32 rows of {T} tokens, got {tokens.dtype} of shape {tuple(tokens.shape)}")
        if tokens.shape[0] == 0:
            raise ValueError("expected rows of tokens, got none")
        return tokens.shape[0]

    def _forward(self, N, tokens, b):
        V, C, H, T = self.dims
        w, copy, ws = self.w, self.copy, b["workspace"]
        mxc.mxc_embedding_fwd(N * T, V, C, BF16, tokens, copy[TABLE], 1.0, b["e"])
        mxc.mxc_layernorm_fwd(N * T, C, BF16, b["e"], w[G0], w[B0], EPS, b["a"], b["s0"])
        mxc.mxc_fc_fwd(N, T * C, H, BF16, b["a"], copy[W1], w[C1], True, b["h"], ws)
        mxc.mxc_fc_fwd(N, H, C, BF16, b["h"], copy[W2], w[C2], False, b["u"], ws)
        mxc.mxc_layernorm_fwd(N, C, BF16, b["u"], w[G1], w[B1], EPS, b["o"], b["s1"])
        mxc.mxc_fc_fwd(N, C, V, BF16, b["o"], copy[TABLE], None, False, b["z"], ws)

    def gradients(self, tokens, labels, logp):
        """The gradients of the mean of -logp, in `grad`; logp: N fp32 values, the labels' log probabilities."""
        V, C, H, T = self.dims
        N = self._rows(tokens)
        b = self._of_batch(N)
        copy, grad, ws = self.copy, self.grad, b["workspace"]
        self._forward(N, tokens, b)
        b["weight"].fill_(-1.0 / N)         # (batches of other sizes have the same buffers)
        mxc.mxc_logprob_fwd_bwd(N, V, V, BF16, b["z"], labels, 1.0, b["weight"], None, logp, None, b["z"], ws)
        mxc.mxc_fc_bwd_weight(N, C, V, BF16, b["o"], b["z"], grad[TABLE], ws)
        mxc.mxc_fc_bwd_data(N, C, V, BF16, b["z"], copy[TABLE], None, b["du"], ws)
        mxc.mxc_layernorm_bwd(N, C, BF16, b["u"], self.w[G1], b["s1"], b["du"], b["du"], grad[G1], grad[B1], ws)
        mxc.mxc_fc_bwd_weight(N, H, C, BF16, b["h"], b["du"], grad[W2], ws)
        mxc.mxc_bias_grad(N, C, 1, 1, BF16, mxc.MXC_NHWC, b["du"], grad[C2], ws)
        mxc.mxc_fc_bwd_data(N, H, C, BF16, b["du"], copy[W2], b["h"], b["dh"], ws)
        mxc.mxc_fc_bwd_weight(N, T * C, H, BF16, b["a"], b["dh"], grad[W1], ws)
        mxc.mxc_bias_grad(N, H, 1, 1, BF16, mxc.MXC_NHWC, b["dh"], grad[C1], ws)
        mxc.mxc_fc_bwd_data(N, T * C, H, BF16, b["dh"], copy[W1], None, b["da"], ws)
        mxc.mxc_layernorm_bwd(N * T, C, BF16, b["e"], self.w[G0], b["s0"], b["da"], b["da"], grad[G0], grad[B0], ws)
        mxc.mxc_embedding_bwd(N * T, V, C, BF16, tokens, b["da"], 1.0, 1, grad[TABLE], ws)

    def update(self, lr=1e-3, wd=0.01):
        self.step += 1
        of = lambda which, tensors: [tensors[i] for i in which]  # noqa: E731
        mxc.mxc_muon_update(of(FILTERS, self.w), of(FILTERS, self.grad), of(FILTERS, self.m), of(FILTERS, self.copy), lr, 0.95, True, wd, 0.2, 1.0, 5, self._update)
        mxc.mxc_adamw_update(of(OTHERS, self.w), of(OTHERS, self.grad), of(OTHERS, self.m), of(OTHERS, self.v), of(OTHERS, self.copy), lr, 0.9, 0.999, 1e-8, wd, 1.0, self.step)

    def train_step(self, tokens, labels, lr=1e-3, wd=0.01):
        """One step on int32 rows of tokens and labels; returns the log probabilities of the labels (before the step), a new tensor."""
        logp = torch.empty(self._rows(tokens), dtype=torch.float32, device=tokens.device)
        self.gradients(tokens, labels, logp)
        self.update(lr, wd)
        return logp

    def predict(self, tokens, top=5):
        """(log probabilities, tokens) of the `top` (5 at most) most probable next ones for each row."""
        V = self.dims[0]
        N = self._rows(tokens)
        b, top = self._of_batch(N), min(top, V, 5)
        self._forward(N, tokens, b)
        logp, index = torch.empty(N, top, device=tokens.device), torch.empty(N, top, dtype=torch.int32, device=tokens.device)
        mxc.mxc_logprob_fwd(N, V, V, BF16, b["z"], None, 1.0, top, None, None, None, logp, index, b["workspace"])
        return logp, index


def text(vocabulary, window, seed=1, device="cuda"):
    """Synthetic text: the token before has two followers, of which the one before that decides, but for one place in eight; batches of places of sequences of 64, whose first rows are not full."""
    gen = torch.Generator().manual_seed(seed)
    followers = torch.randint(0, vocabulary, (vocabulary, 2), generator=gen)

    def batch(N):
        length, rows = 64, -(-N // 64)
        t = torch.full((rows, window + length), -1, dtype=torch.int64)
        noise, any_token = torch.rand(rows, length, generator=gen) < 0.125, torch.randint(0, vocabulary, (rows, length), generator=gen)
        for i in range(length):
            before = t[:, max(0, window + i - 2):window + i].clamp(min=0)
            t[:, window + i] = torch.where(noise[:, i] | (i == 0), any_token[:, i], followers[before[:, -1], before[:, 0] % 2])
        windows = t.unfold(1, window + 1, 1)[:, :length].reshape(-1, window + 1)[:N]
        return windows[:, :window].int().contiguous().to(device), windows[:, window].int().contiguous().to(device)
    return batch


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--vocabulary", type=int, default=1000)
    ap.add_argument("--channels", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--window", type=int, default=4)
    ap.add_argument("--batch", type=int, default=512)
    ap.add_argument("--steps", type=int, default=200)
    a = ap.parse_args(argv)
    model, batch = Model(a.vocabulary, a.channels, a.hidden, a.window), text(a.vocabulary, a.window)
    for i in range(a.steps):
        loss = -model.train_step(*batch(a.batch))
        if i % 50 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {float(loss.mean()):.4f}", flush=True)
    tokens, labels = batch(a.batch)
    right = model.predict(tokens)[1] == labels[:, None]
    print(f"asked: first {float(right[:, 0].float().mean()):.3f}, first five {float(right.any(1).float().mean()):.3f}")


if __name__ == "__main__":
    main()
