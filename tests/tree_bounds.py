"""What kvq_tree_attention may be off by, for tests whose caches are so long that a bound on the sum of all roundings hides a lost tile.

Rounded to fp16 are the weights and the cached values, 2^-11 of each at the most and of either sign: with roundings that are even between their bounds
a sum over keys has a standard deviation of 2^-11 / sqrt(3) times the root of the sum of its squared terms, and six of them hold for
some 10^8 outputs.  Scores have 32 bits: a sum of 128 products and of zero points in two halves, 64 steps of 2^-24 of the sum of their sizes
at the most, of either sign from key to key.  Sums of weights and of products take T / 8 additions of 32 bits."""
import math

import torch


def weights(scores):
    """softmax of [rows, keys] in 64 bits; rows of nothing but -inf give zeros."""
    m = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total)


def bounded(p, v, reach, half_out):
    """Outputs of weights p [rows, keys] and values v [keys, 128] and their bound; reach [rows]: the largest sum of the sizes of a score's products."""
    want = p @ v
    each = math.sqrt(2) * 2.0 ** -11 / math.sqrt(3) + 64 * 2.0 ** -24 * reach[:, None]
    spread = (p * p) @ (v * v)
    own = (p * p).sum(-1, keepdim=True)
    tol = 6 * each * (spread.sqrt() + want.abs() * own.sqrt())
    tol = tol + 2 * 2.0 ** -24 * (1 + p.shape[1] / 8) * (spread.sqrt() + want.abs())
    if half_out:
        tol = tol + 2.0 ** -11 * want.abs() + 2.0 ** -25
    return want, tol


def tree(K, V, q, k, v, sees, lam, scale, half_out):
    """Outputs and bounds [batch, heads, n, 128] for cached K, V (64 bits) and the nodes' q, k, v."""
    B, H, n, _ = q.shape
    g = H // K.shape[1]
    want = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    tol = torch.empty_like(want)
    sees = sees.to(q.device).expand(B, n, n)
    for b in range(B):
        for h in range(H):
            u = h // g
            qc = (q[b, h] if lam is None else (q[b, h].float() * lam[u]).half()).double()
            parts = [(qc, K[b, u]), (q[b, h].double(), k[b, u].double())]
            s = torch.cat([x @ y.t() for x, y in parts], 1) * scale
            reach = torch.cat([x.abs() @ y.abs().t() for x, y in parts], 1).amax(1) * abs(scale)
            s[:, K.shape[2]:][~sees[b]] = -math.inf
            want[b, h], tol[b, h] = bounded(weights(s), torch.cat([V[b, u], v[b, u].double()]), reach, half_out)
    return want, tol
