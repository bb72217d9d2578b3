"""The operators around a language model's attention, as cases to time and compare.

A case is one pass through the entry points that a training step or a serving
step calls:

    op "nll"    softmax_linear_nll_fwd / _bwd   the loss of hidden states against
                a vocabulary's rows, its logits never kept; with the gradients of
                both where "train"
    op "embed"  softmax_embedding_fwd / _bwd    rows of a table by token, and the
                table's gradient where "train"
    op "norm"   softmax_layer_norm_fwd / _bwd   rows brought to mean 0 and
                variance 1 ("center") or to mean square 1, with the gradients of
                input, weight and bias where "train"

The plain forms below compute the same in elementary torch operations, in 32
bits: all logits at once, one addition into the table for each token, sums over
columns and rows.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
IGNORE = -100  # the label of a token that has no loss
EPS = 1e-5


# ---------------------------------------------------------------------------
# The cases

def _nll(name, rows, vocab, d, dtype, ignored, weighted, apart, train):
    """``ignored``: share of tokens without a loss; ``weighted``: tokens have
    weights of their own; ``apart``: rows of x lie that many rows apart."""
    return {"name": name, "op": "nll", "rows": rows, "vocab": vocab, "d": d, "dtype": dtype,
            "ignored": ignored, "weighted": weighted, "apart": apart, "train": train}


def _embed(name, tokens, vocab, d, dtype, scale, padding, train):
    """``padding``: share of tokens that are padding (id -1)."""
    return {"name": name, "op": "embed", "tokens": tokens, "vocab": vocab, "d": d,
            "dtype": dtype, "scale": scale, "padding": padding, "train": train}


def _norm(name, rows, d, dtype, center, train):
    return {"name": name, "op": "norm", "rows": rows, "d": d, "dtype": dtype, "center": center,
            "train": train}


def listed():
    return [
        # One candidate token's likelihood: the whole vocabulary is read for
        # one row.
        _nll("nll_score_1x50001", 1, 50001, 2048, "bf16", 0.0, False, 1, False),
        # A batch of continuations to rank, the hidden states of their last
        # positions taken out of the sequences.
        _nll("nll_score_33x32768", 33, 32768, 1160, "f16", 0.0, False, 8, False),
        # A training step of the example decoder: 24 short documents, float32.
        _nll("nll_train_1496x256", 1496, 256, 256, "f32", 0.1, False, 1, True),
        # Fine-tuning on answers: half of the tokens are prompt, and tokens
        # have weights; odd sizes.
        _nll("nll_train_701x10007", 701, 10007, 520, "f16", 0.5, True, 1, True),
        # A training step of a mid-sized model on packed documents.
        _nll("nll_train_8192x50001", 8192, 50001, 2048, "bf16", 0.05, False, 1, True),
        # A wide model with a large vocabulary: the largest call.
        _nll("nll_train_4096x131072", 4096, 131072, 4096, "bf16", 0.0, False, 1, True),
        # The tokens of a decode step of 64 requests: the smallest call.
        _embed("embed_decode_64", 64, 50001, 4096, "bf16", 1.0, 0.0, False),
        # The example decoder's table in a training step: every row is hit
        # several times, and the sums are float32.
        _embed("embed_train_1496x256", 1496, 256, 256, "f32", 1.0, 0.0, True),
        # Packed documents with padding at the end, scaled by sqrt(d).
        _embed("embed_train_16384x50001", 16384, 50001, 2048, "bf16", 2048 ** 0.5, 0.1, True),
        # The norm in front of a layer in a decode step.
        _norm("norm_decode_64x4096", 64, 4096, "bf16", True, False),
        # The same in a training step.
        _norm("norm_train_16384x4096", 16384, 4096, "bf16", True, True),
        # Many short rows, without the mean: the norm of each head's queries.
        _norm("norm_train_115200x200", 115200, 200, "f16", False, True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# The multiply-adds of the largest listed product, and the elements of the
# largest listed rows.
MOST_PRODUCT = 4096 * 131072 * 4096
MOST_ELEMENTS = 16384 * 4096


def draw(rng):
    op = rng.choice(["nll", "nll", "nll", "embed", "embed", "norm", "norm"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    train = rng.random() < 0.7
    d = 8 * _log_uniform(rng, 8, 512)
    if op == "norm":
        rows = min(_log_uniform(rng, 1, 131072), MOST_ELEMENTS // d // SIZE[dtype] * 2)
        return {"op": op, "rows": rows, "d": d, "dtype": dtype, "center": rng.random() < 0.6,
                "train": train}
    vocab = _log_uniform(rng, 256, 131072)
    if op == "embed":
        vocab = min(vocab, MOST_ELEMENTS // d // SIZE[dtype] * 2)
        return {"op": op, "tokens": _log_uniform(rng, 1, 16384), "vocab": vocab, "d": d,
                "dtype": dtype, "scale": rng.choice([1.0, d ** 0.5]),
                "padding": rng.choice([0.0, 0.1, 0.4]), "train": train}
    rows = _log_uniform(rng, 1, 8192)
    # A float32 product has no matrix operations as fast as 16-bit ones.
    most = MOST_PRODUCT // 16 if dtype == "f32" else MOST_PRODUCT // 2
    rows = max(1, min(rows, most // (vocab * d)))
    return {"op": op, "rows": rows, "vocab": vocab, "d": d, "dtype": dtype,
            "ignored": rng.choice([0.0, 0.0, 0.1, 0.6]), "weighted": rng.random() < 0.3,
            "apart": rng.choice([1, 1, 1, 3]), "train": train}


# ---------------------------------------------------------------------------
# Inputs

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, device=DEVICE, generator=g)


def _tokens(g, count, vocab):
    """Tokens as a text has them: the first of the vocabulary often, the last
    ones seldom."""
    u = torch.rand(count, device=DEVICE, generator=g, dtype=torch.float64)
    return (vocab ** u - 1).floor().long().clamp(0, vocab - 1)


def _prepare_nll(case, g):
    rows, vocab, d = case["rows"], case["vocab"], case["d"]
    kind = TYPES[case["dtype"]]
    # Rows of the vocabulary of length 1.5 or so; a hidden state is a normed
    # row that leans towards its label's, some far and some not at all, so that
    # likelihoods of all sizes are met.
    weight = (_normal(g, vocab, d) * (1.5 / d ** 0.5)).to(kind)
    labels = _tokens(g, rows, vocab)
    lean = 10.0 * torch.rand(rows, 1, device=DEVICE, generator=g)
    x = _normal(g, rows * case["apart"], d)
    x[::case["apart"]] += lean * weight[labels].float() / 1.5
    x = x.to(kind)[::case["apart"]]
    none = int(rows * case["ignored"])
    labels[torch.randperm(rows, device=DEVICE, generator=g)[:none]] = IGNORE
    # The gradient of a mean over the tokens that have a loss.
    dloss = torch.full((rows,), 1.0 / (rows - none), device=DEVICE)
    if case["weighted"]:
        dloss *= 0.1 + 1.8 * torch.rand(rows, device=DEVICE, generator=g)
    return {"x": x, "weight": weight, "labels": labels, "dloss": dloss}


def _prepare_embed(case, g):
    tokens, vocab, d, kind = case["tokens"], case["vocab"], case["d"], TYPES[case["dtype"]]
    ids = _tokens(g, tokens, vocab)
    pad = int(tokens * case["padding"])
    if pad:
        ids[-pad:] = -1
    return {"ids": ids, "table": _normal(g, vocab, d).to(kind), "scale": case["scale"],
            "dout": _normal(g, tokens, d).to(kind)}


def _prepare_norm(case, g):
    rows, d, kind = case["rows"], case["d"], TYPES[case["dtype"]]
    # A residual stream: columns of different means and rows of different sizes.
    x = _normal(g, rows, d) + 0.5 * _normal(g, d) + 0.3
    x *= 0.5 + 2.0 * torch.rand(rows, 1, device=DEVICE, generator=g)
    return {"x": x.to(kind), "weight": (1.0 + 0.2 * _normal(g, d)).to(kind),
            "bias": (0.1 * _normal(g, d)).to(kind) if case["center"] else None,
            "dy": _normal(g, rows, d).to(kind), "center": case["center"]}


def prepare(case, seed):
    make = {"nll": _prepare_nll, "embed": _prepare_embed, "norm": _prepare_norm}[case["op"]]
    return {"op": case["op"], "train": case["train"], **make(case, _generator(seed))}


# ---------------------------------------------------------------------------
# The plain forms

def _plain_nll(s):
    x, weight = s["x"].float(), s["weight"].float()
    keep = s["labels"] != IGNORE
    at = torch.where(keep, s["labels"], 0)[:, None]
    logits = x @ weight.t()
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    log = torch.log(total)
    out = {"loss": torch.where(keep, (top - logits.gather(1, at) + log)[:, 0], 0.0),
           "lse": torch.where(keep, (top + log)[:, 0], 0.0)}
    if s["train"]:
        g = e / total
        g.scatter_add_(1, at, torch.full_like(total, -1.0))
        g *= torch.where(keep, s["dloss"], 0.0)[:, None]
        out["dx"] = (g @ weight).to(s["x"].dtype)
        out["dweight"] = (g.t() @ x).to(s["x"].dtype)
    return out


def _plain_embed(s):
    ids, table, scale = s["ids"], s["table"], s["scale"]
    rows = len(table)
    keep = (ids >= 0) & (ids < rows)
    taken = table[torch.where(keep, ids, 0)].float()
    out = {"out": torch.where(keep[:, None], taken * scale, 0.0).to(table.dtype)}
    if s["train"]:
        # One row more, for the tokens that have none.
        sums = torch.zeros(rows + 1, table.shape[1], device=table.device)
        sums.index_add_(0, torch.where(keep, ids, rows), s["dout"].float())
        out["dtable"] = (sums[:rows] * scale).to(table.dtype)
    return out


def _plain_norm(s):
    kind = s["x"].dtype
    x, weight = s["x"].float(), s["weight"].float()
    mean = x.mean(1, keepdim=True) if s["center"] else torch.zeros_like(x[:, :1])
    x = x - mean
    rstd = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
    x = x * rstd
    y = x * weight
    if s["bias"] is not None:
        y = y + s["bias"].float()
    out = {"y": y.to(kind), "rstd": rstd[:, 0]}
    if s["center"]:
        out["mean"] = mean[:, 0]
    if s["train"]:
        dy = s["dy"].float()
        out["dweight"] = (dy * x).sum(0).to(kind)
        if s["bias"] is not None:
            out["dbias"] = dy.sum(0).to(kind)
        g = dy * weight
        dx = g - x * (g * x).mean(1, keepdim=True)
        if s["center"]:
            dx = dx - g.mean(1, keepdim=True)
        out["dx"] = (dx * rstd).to(kind)
    return out


# ---------------------------------------------------------------------------
# The framework's

def _own_nll(sm, s):
    loss, lse = sm.softmax_linear_nll_fwd(s["x"], s["weight"], s["labels"], ignore=IGNORE)
    out = {"loss": loss, "lse": lse}
    if s["train"]:
        out["dx"], out["dweight"] = sm.softmax_linear_nll_bwd(
            s["dloss"], s["x"], s["weight"], s["labels"], loss, lse, ignore=IGNORE)
    return out


def _own_embed(sm, s):
    out = {"out": sm.softmax_embedding_fwd(s["ids"], s["table"], scale=s["scale"])}
    if s["train"]:
        out["dtable"] = sm.softmax_embedding_bwd(s["dout"], s["ids"], len(s["table"]),
                                                 scale=s["scale"])
    return out


def _own_norm(sm, s):
    y, mean, rstd = sm.softmax_layer_norm_fwd(s["x"], s["weight"], s["bias"], eps=EPS,
                                              center=s["center"])
    out = {"y": y, "rstd": rstd}
    if s["center"]:
        out["mean"] = mean
    if s["train"]:
        out["dx"], out["dweight"], dbias = sm.softmax_layer_norm_bwd(
            s["dy"], s["x"], s["weight"], mean, rstd, bias=s["bias"] is not None)
        if s["bias"] is not None:
            out["dbias"] = dbias
    return out


def run(state):
    if own:
        import paper_1904_12380_amd as sm
        return {"nll": _own_nll, "embed": _own_embed, "norm": _own_norm}[state["op"]](sm, state)
    return {"nll": _plain_nll, "embed": _plain_embed, "norm": _plain_norm}[state["op"]](state)


# ---------------------------------------------------------------------------
# What a pass cannot do without

def work(case):
    size, d = SIZE[case["dtype"]], case["d"]
    if case["op"] == "nll":
        rows, vocab = case["rows"], case["vocab"]
        live = rows - int(rows * case["ignored"])
        moved = (live + vocab) * d * size + rows * 16
        products = 1
        if case["train"]:  # dloss is read, both gradients are written
            moved += (rows + vocab) * d * size + rows * 4
            products = 3
        return {"bytes": moved, "flops": 2 * products * live * vocab * d}
    if case["op"] == "embed":
        tokens, vocab = case["tokens"], case["vocab"]
        live = tokens - int(tokens * case["padding"])
        moved = tokens * 8 + (live + tokens) * d * size
        if case["train"]:
            moved += (live + vocab) * d * size
        return {"bytes": moved, "flops": (2 if case["train"] else 1) * live * d}
    rows = case["rows"]
    moved = 2 * rows * d * size + rows * 8 + 2 * d * size
    if case["train"]:  # dy is read, dx and the columns' gradients are written
        moved += 2 * rows * d * size + 2 * d * size
    return {"bytes": moved, "flops": (20 if case["train"] else 8) * rows * d}


# ---------------------------------------------------------------------------
# The definitions in 64 bits

def _exact_nll(s):
    x, weight, labels = s["x"].double(), s["weight"].double(), s["labels"]
    live = (labels != IGNORE).nonzero()[:, 0]
    x, at = x[live], labels[live]
    logp = torch.mm(x, weight.t())
    lse = logp.logsumexp(1)
    logp -= lse[:, None]
    here = torch.arange(len(live), device=x.device)
    out = {"loss": x.new_zeros(len(labels)).index_copy(0, live, -logp[here, at]),
           "lse": x.new_zeros(len(labels)).index_copy(0, live, lse)}
    if s["train"]:
        p = logp.exp_()
        p[here, at] -= 1.0
        p *= s["dloss"].double()[live, None]
        out["dx"] = torch.zeros(s["x"].shape, dtype=torch.float64, device=x.device)
        out["dx"][live] = torch.mm(p, weight)
        out["dweight"] = torch.mm(p.t(), x)
    return out


def _exact_embed(s):
    ids, table = s["ids"], s["table"].double()
    live = (ids >= 0).nonzero()[:, 0]
    out = {"out": table.new_zeros(len(ids), table.shape[1])}
    out["out"][live] = table[ids[live]] * s["scale"]
    if s["train"]:
        out["dtable"] = torch.zeros_like(table).index_put_(
            (ids[live],), s["dout"][live].double() * s["scale"], accumulate=True)
    return out


def _exact_norm(s):
    x = s["x"].double()
    weight = s["weight"].double()
    if s["train"]:
        x.requires_grad_()
        weight.requires_grad_()
    bias = s["bias"].double() if s["bias"] is not None else torch.zeros_like(weight)
    mean = x.sum(1) / x.shape[1] if s["center"] else x.detach().new_zeros(len(x))
    off = x - mean[:, None]
    rstd = ((off * off).sum(1) / x.shape[1] + EPS) ** -0.5
    y = off * rstd[:, None] * weight + bias
    out = {"y": y.detach(), "rstd": rstd.detach()}
    if s["center"]:
        out["mean"] = mean.detach()
    if s["train"]:
        out["dx"], out["dweight"] = torch.autograd.grad(y, (x, weight), s["dy"].double())
        if s["bias"] is not None:
            out["dbias"] = s["dy"].double().sum(0)
    return out


def exact(case, seed):
    state = prepare(case, seed)
    return {"nll": _exact_nll, "embed": _exact_embed, "norm": _exact_norm}[case["op"]](state)
