"""Data-parallel training of two layers on one GPU, every heavy step by the library's calls: k ranks' gradients as separate buffers.

A step of each rank: the layers' products with weights and activations in 4-bit blocks (zc_mx_linear), their gradients by products
of operands quantised along the other axis (zc_mx_quantize, zc_mx_product), into one buffer of gradients.  Then the collective's local work: the buffers
are compressed (zc_compress), summed as streams (zc_reduce_compressed) and come back as their average (zc_decompress_average).  Then the
optimiser's step over all tensors, states in 8 bits (zc_adamw), and the new weights into blocks along both axes.

    python examples/train_layers.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2502_18554_amd as zc  # noqa: E402

DEV = "cuda:0"


def check(status):
    if status:
        raise zc.ZcError(status, "train_layers")


class Layer:
    """Weights (n, k) as a view of the ranks' common buffer, and what the products take: blocks along k, and along n."""

    def __init__(self, weights):
        self.weights = weights
        n, k = weights.shape
        self.held, self.held_t = blocks_for(n, k), blocks_for(k, n)
        self.requantise()

    def requantise(self):
        check(zc.zc_mx_quantize(self.weights, *self.held, *self.held_t))


def blocks_for(rows, cols):
    return (torch.empty((rows, zc.zc_mx_codes_stride(cols)), dtype=torch.uint8, device=DEV),
            torch.empty((rows, zc.zc_mx_scales_stride(cols)), dtype=torch.uint8, device=DEV))


def forward(layer, x, bias, ws):
    out = torch.empty((x.shape[0], layer.weights.shape[0]), dtype=torch.float32, device=DEV)
    check(zc.zc_mx_linear(x, *layer.held, out, ws, d_bias=bias))
    return out


def backward(layer, x, dy, grad_w, ws, want_dx=True):
    """grad_w = dy^T x, and dx = dy w."""
    rows, n = dy.shape
    k = x.shape[1]
    dy_held, dy_held_t, x_held_t = blocks_for(rows, n), blocks_for(n, rows), blocks_for(k, rows)
    check(zc.zc_mx_quantize(dy, *dy_held, *dy_held_t))
    check(zc.zc_mx_quantize(x, None, None, *x_held_t))
    check(zc.zc_mx_product(*dy_held_t, *x_held_t, rows, grad_w, ws))
    if not want_dx:
        return None
    dx = torch.empty((rows, k), dtype=torch.float32, device=DEV)
    check(zc.zc_mx_product(*dy_held, *layer.held_t, n, dx, ws))
    return dx


def average_by_streams(buffers, out, relative_bound=1e-4):
    """The average of the ranks' buffers, as a compressed Allreduce leaves it: streams, their sum, the sum's average."""
    n, k = out.numel(), len(buffers)
    bound = relative_bound * max(float(b.abs().max()) for b in buffers) + 1e-20
    ws = torch.empty(zc.zc_workspace_bytes(n, k), dtype=torch.uint8, device=DEV)
    streams = [torch.empty(zc.zc_compress_bound(n), dtype=torch.uint8, device=DEV) for _ in range(k + 1)]
    sizes = []
    for b, s in zip(buffers, streams):
        status, size = zc.zc_compress(b, n, bound, s, ws)
        check(status)
        sizes.append(size)
    status, size = zc.zc_reduce_compressed(streams[:k], sizes, streams[k], ws)
    check(status)
    status, _ = zc.zc_decompress_average(streams[k], size, out, ws)
    check(status)
    return sum(sizes) / (4 * n * k)


def train(steps=60, ranks=4, rows=256, sizes=(192, 512, 96), seed=0, verbose=True):
    """Two layers learn what two other layers do.  Returns the mean loss of every step."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    d_in, d_mid, d_out = sizes
    shapes = [(d_mid, d_in), (d_mid,), (d_out, d_mid), (d_out,)]
    counts = [torch.Size(s).numel() for s in shapes]
    teacher = [torch.randn(s, generator=g, device=DEV) / s[-1] ** 0.5 for s in shapes]
    params = [torch.randn(s, generator=g, device=DEV) / s[-1] ** 0.5 if len(s) == 2 else torch.zeros(s, device=DEV) for s in shapes]
    state = torch.zeros(zc.zc_adamw_state_bytes(counts, 8), dtype=torch.uint8, device=DEV)
    first, second = Layer(params[0]), Layer(params[2])
    largest = max(rows, *sizes)
    ws = torch.empty(zc.zc_mx_workspace_bytes(largest, largest, largest), dtype=torch.uint8, device=DEV)
    buffers = [torch.zeros(sum(counts), device=DEV) for _ in range(ranks)]
    average = torch.empty(sum(counts), device=DEV)
    losses = []
    for step in range(1, steps + 1):
        loss = 0.0
        for buffer in buffers:
            grads = [v.view(s) for v, s in zip(buffer.split(counts), shapes)]
            x = torch.randn((rows, d_in), generator=g, device=DEV)
            want = torch.relu(x @ teacher[0].t() + teacher[1]) @ teacher[2].t() + teacher[3]
            mid = torch.relu(forward(first, x, params[1], ws))
            off = forward(second, mid, params[3], ws) - want
            loss += float((off * off).mean()) / ranks
            dy = off * (2.0 / off.numel())
            dmid = backward(second, mid, dy, grads[2], ws) * (mid > 0)
            backward(first, x, dmid, grads[0], ws, want_dx=False)
            grads[1].copy_(dmid.sum(0))
            grads[3].copy_(dy.sum(0))
        share = average_by_streams(buffers, average)
        grads = [v.view(s) for v, s in zip(average.split(counts), shapes)]
        check(zc.zc_adamw(params, grads, state, step, 3e-3, 0.9, 0.98, 1e-8, 0.0, state_bits=8, seed=seed + 1))
        first.requantise()
        second.requantise()
        losses.append(loss)
        if verbose and (step == 1 or step % 10 == 0):
            print(f"step {step:4d}  loss {loss:.4f}  streams {100 * share:.1f} % of the buffers", flush=True)
    return losses


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
