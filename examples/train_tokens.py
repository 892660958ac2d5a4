"""Data-parallel training of a small token model on one GPU, every heavy step by the library's calls: k ranks' gradients as separate buffers.

A token's row of the table (zc_embedding), a layer norm (zc_layer_norm), two layers in 4-bit blocks as in train_layers.py, and a score for every token: the model learns which token follows.
Backward: the layers' products, the norm's gradients (zc_layer_norm_backward, with the residual's added on the way), the table's (zc_embedding_backward).  Then the collective's local work on the
buffers of gradients (train_layers.average_by_streams), and two optimisers: matrices by zc_muon, the table, the norm and the biases by zc_adamw.

    python examples/train_tokens.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2502_18554_amd as zc  # noqa: E402
from train_layers import DEV, Layer, average_by_streams, backward, check, forward  # noqa: E402


class Model:
    """vocab tokens, rows of d values, a layer d -> hidden, a layer hidden -> d added to the row, and a layer d -> vocab for the scores."""

    def __init__(self, vocab, d, hidden, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.vocab, self.d = vocab, d
        matrices = [(hidden, d), (d, hidden), (vocab, d)]
        self.matrices = [torch.randn(s, generator=g, device=DEV) / s[1] ** 0.5 for s in matrices]
        # the table, the two norms' weights and biases, the layers' biases
        self.others = [torch.randn(vocab, d, generator=g, device=DEV)] + [torch.full((d,), v, device=DEV) for v in (1.0, 0.0, 1.0, 0.0)] + [torch.zeros(s[0], device=DEV) for s in matrices]
        self.shapes = [tuple(p.shape) for p in self.matrices + self.others]
        self.layers = [Layer(p) for p in self.matrices]


def gradients(model, tokens, targets, grads, scale=1.0):
    """Mean loss of the batch, its gradients into `grads` (views of a rank's buffer, in the order of model.shapes), and what stands between the calls."""
    table, w0, b0, w1, b1, *biases = model.others
    n, d = tokens.numel(), model.d
    sizes = max(n, model.vocab, *(max(p.shape) for p in model.matrices))
    ws = torch.empty(zc.zc_mx_workspace_bytes(sizes, sizes, sizes), dtype=torch.uint8, device=DEV)
    norm_ws = torch.empty(zc.zc_layer_norm_workspace_bytes(n, d), dtype=torch.uint8, device=DEV)
    table_ws = torch.empty(zc.zc_embedding_workspace_bytes(n, model.vocab, d), dtype=torch.uint8, device=DEV)

    def norm(x, w, b):
        out, stats = torch.empty_like(x), torch.empty(2, n, device=DEV)
        check(zc.zc_layer_norm(x, w, b, out, stats))
        return out, stats

    x0 = torch.empty(n, d, device=DEV)
    check(zc.zc_embedding(table, tokens, x0, scale=scale))
    y0, stats0 = norm(x0, w0, b0)
    mid = torch.relu(forward(model.layers[0], y0, biases[0], ws))
    x1 = x0.clone()
    check(zc.zc_mx_linear(mid, *model.layers[1].held, x1, ws, d_bias=biases[1], add=True))              # the residual stream
    y1, stats1 = norm(x1, w1, b1)
    scores = forward(model.layers[2], y1, biases[2], ws)
    logs = torch.log_softmax(scores, dim=1)
    loss = -logs[torch.arange(n, device=DEV), targets].mean()

    dscores = torch.exp(logs)
    dscores[torch.arange(n, device=DEV), targets] -= 1
    dscores /= n
    g0, g1, g2, gtable, gw0, gb0, gw1, gb1, *gbiases = grads
    dy1 = backward(model.layers[2], y1, dscores, g2, ws)
    dx = torch.empty(n, d, device=DEV)                                                                   # of the residual stream
    check(zc.zc_layer_norm_backward(dy1, x1, stats1, w1, dx, gw1, gb1, norm_ws))
    dx1 = dx.clone()
    dmid = backward(model.layers[1], mid, dx, g1, ws) * (mid > 0)
    dy0 = backward(model.layers[0], y0, dmid, g0, ws)
    check(zc.zc_layer_norm_backward(dy0, x0, stats0, w0, dx, gw0, gb0, norm_ws, add=True))
    check(zc.zc_embedding_backward(dx, tokens, gtable, table_ws, scale=scale))
    for g, of in zip(gbiases, (dmid, dx1, dscores)):
        g.copy_(of.sum(0))
    return loss, dict(x0=x0, x1=x1, dy0=dy0, dy1=dy1, dx1=dx1, dx=dx)


def train(steps=60, ranks=4, rows=256, vocab=199, d=96, hidden=160, seed=0, verbose=True):
    """The model learns a fixed successor of every token.  Returns the mean loss of every step."""
    model = Model(vocab, d, hidden, seed)
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    successor = torch.randperm(vocab, generator=g, device=DEV)
    counts = [torch.Size(s).numel() for s in model.shapes]
    buffers = [torch.zeros(sum(counts), device=DEV) for _ in range(ranks)]
    average = torch.empty(sum(counts), device=DEV)
    shapes = [tuple(p.shape) for p in model.matrices]
    momentum = torch.zeros(zc.zc_muon_state_bytes(shapes), dtype=torch.uint8, device=DEV)
    muon_ws = torch.empty(zc.zc_muon_workspace_bytes(shapes), dtype=torch.uint8, device=DEV)
    moments = torch.zeros(zc.zc_adamw_state_bytes([p.numel() for p in model.others], 32), dtype=torch.uint8, device=DEV)
    losses = []
    for step in range(1, steps + 1):
        loss = 0.0
        for buffer in buffers:
            tokens = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
            grads = [v.view(s) for v, s in zip(buffer.split(counts), model.shapes)]
            loss += float(gradients(model, tokens, successor[tokens], grads)[0]) / ranks
        average_by_streams(buffers, average)
        grads = [v.view(s) for v, s in zip(average.split(counts), model.shapes)]
        check(zc.zc_muon(model.matrices, grads[:3], momentum, muon_ws, 0.01, match_rms=True))
        check(zc.zc_adamw([p.view(-1) for p in model.others], [v.reshape(-1) for v in grads[3:]], moments, step, 3e-3, 0.9, 0.98, 1e-8, 0.0))
        for layer in model.layers:
            layer.requantise()
        losses.append(loss)
        if verbose and (step == 1 or step % 10 == 0):
            print(f"step {step:4d}  loss {loss:.4f}", flush=True)
    return losses


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
