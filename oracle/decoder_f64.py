"""float64 oracle of what a decoder has around its attention: the definitions of
include/decoder_mi355x.h on CPU tensors, elementary operations only."""
import torch


def linear_nll(x, weight, labels, ignore=-100, dloss=None):
    """(loss, lse), and with ``dloss`` also (dx, dweight) and the probabilities and
    gradients of the logits (zeros for ignored rows)."""
    x, weight = x.double(), weight.double()
    live = labels != ignore
    bad = live & ((labels < 0) | (labels >= len(weight)))
    at = torch.where(live & ~bad, labels, 0)[:, None]
    logits = torch.where(live[:, None], x, 0.0) @ weight.t()
    top = logits.amax(1, keepdim=True)
    lse = top + (logits - top).exp().sum(1, keepdim=True).log()
    loss = torch.where(bad, torch.nan, (lse - logits.gather(1, at))[:, 0])
    out = [torch.where(live, loss, 0.0), torch.where(live, lse[:, 0], 0.0)]
    if dloss is None:
        return out
    p = (logits - lse).exp()
    g = p.clone()
    g.scatter_add_(1, at, torch.full_like(lse, -1.0))
    scale = torch.where(bad, torch.nan, dloss.double())
    p, g = (torch.where(live[:, None], y * scale[:, None], 0.0) for y in (p, g))
    dx = torch.where(live[:, None], g @ weight, 0.0)
    return [*out, dx, g.t() @ torch.where(live[:, None], x, 0.0), p, g]


def embedding(ids, table, scale=1.0):
    keep = (ids >= 0) & (ids < len(table))
    out = torch.zeros(len(ids), table.shape[1], dtype=torch.float64)
    out[keep] = table.double()[ids[keep]] * scale
    return out


def embedding_grad(dout, ids, rows, scale=1.0):
    keep = (ids >= 0) & (ids < rows)
    out = torch.zeros(rows, dout.shape[1], dtype=torch.float64)
    return out.index_put_((ids[keep],), dout.double()[keep] * scale, accumulate=True)


def layer_norm(x, weight=None, bias=None, eps=1e-5, center=True, dy=None):
    """(y, mean, rstd), and with ``dy`` also (dx, dweight, dbias)."""
    x = x.double()
    d = x.shape[1]
    mean = x.mean(1, keepdim=True) if center else torch.zeros(len(x), 1, dtype=torch.float64)
    var = (x - mean).square().sum(1, keepdim=True) / d
    rstd = (var + eps) ** -0.5
    h = (x - mean) * rstd
    w = torch.ones(d, dtype=torch.float64) if weight is None else weight.double()
    y = h * w + (0.0 if bias is None else bias.double())
    out = [y, mean[:, 0], rstd[:, 0]]
    if dy is None:
        return out
    dy = dy.double()
    g = dy * w
    dx = g - h * (g * h).mean(1, keepdim=True)
    if center:
        dx = dx - g.mean(1, keepdim=True)
    return [*out, dx * rstd, (dy * h).sum(0), dy.sum(0)]
