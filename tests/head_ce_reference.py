"""Next-token cross entropy from hidden states and its gradient, written out in 64 bits."""
import torch


def forward(h, W, targets, scale):
    """loss and lse of every row (loss 0 without a target)."""
    x = (h.double() @ W.double().T) * scale
    lse = torch.logsumexp(x, -1)
    t = targets.long()
    rest = x.clone()
    rest[t >= 0] = rest[t >= 0].scatter(1, t[t >= 0, None], float("-inf"))
    # log(1 + sum of the others relative to the target)
    own = x.gather(1, t.clamp(min=0)[:, None])[:, 0]
    loss = torch.log1p(torch.exp(torch.logsumexp(rest, -1) - own))
    loss = torch.where(torch.isinf(loss) | (loss > 30), lse - own, loss)
    return torch.where(t >= 0, loss, 0.0), lse


def backward(h, W, targets, lse, d_loss, d_lse, scale):
    """dh, dW and G for upstream gradients d_loss and d_lse (or None), with p = exp(x - lse) for the given lse."""
    h, W, V = h.double(), W.double(), W.shape[0]
    t = targets.long()
    there = (t >= 0) & (t < V)
    a = torch.where(there, d_loss.double(), 0.0)
    b = torch.zeros_like(a) if d_lse is None else d_lse.double()
    p = torch.exp((h @ W.T) * scale - lse.double()[:, None])
    hit = torch.zeros_like(p)
    hit[there] = hit[there].scatter(1, t[there, None], 1.0)
    G = scale * ((a + b)[:, None] * p - a[:, None] * hit)
    live = (a != 0) | (b != 0)
    G = torch.where((live & ~torch.isneginf(lse.double()))[:, None], G, 0.0)
    return G @ W, G.T @ torch.where(live[:, None], h, 0.0), G
