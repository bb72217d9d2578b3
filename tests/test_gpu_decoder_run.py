"""A decoder's two ends together, as a training step uses them: tokens to rows of a
table, a norm, the loss against the same table, and all gradients."""
import pytest
import torch

import paper_1904_12380_amd as sm
from oracle import decoder_f64 as oracle
from tests import decoder_data as data

pytestmark = pytest.mark.gpu


def leaves(dtype, vocab=300, d=64, seed=1):
    g = torch.Generator().manual_seed(seed)
    kind = data.TYPES[dtype]
    table = (torch.randn(vocab, d, generator=g) * 0.3).to(kind)
    weight = (1 + 0.2 * torch.randn(d, generator=g)).to(kind)
    bias = (0.1 * torch.randn(d, generator=g)).to(kind)
    ids = torch.randint(vocab, (150,), generator=g)
    labels = ids.roll(-1)
    labels[::9] = -100
    ids[-5:] = -1
    return [t.cuda() for t in (ids, labels, table, weight, bias)]


def step(ids, labels, table, weight, bias, scale=8.0):
    """Forward and backward by the functions that record nothing."""
    x = sm.softmax_embedding_fwd(ids, table, scale=scale)
    y, mean, rstd = sm.softmax_layer_norm_fwd(x, weight, bias)
    loss, lse = sm.softmax_linear_nll_fwd(y, table, labels)
    dloss = torch.where(labels == -100, 0.0, 1.0 / 128)
    dy, dtable = sm.softmax_linear_nll_bwd(dloss, y, table, labels, loss, lse)
    dx, dweight, dbias = sm.softmax_layer_norm_bwd(dy, x, weight, mean, rstd, bias=True)
    return [loss, dtable + sm.softmax_embedding_bwd(dx, ids, len(table), scale=scale), dweight,
            dbias]


def autograd(ids, labels, table, weight, bias):
    leaf = [t.detach().clone().requires_grad_() for t in (table, weight, bias)]
    y = sm.softmax_layer_norm(sm.softmax_embedding(ids, leaf[0], scale=8.0), *leaf[1:])
    loss = sm.softmax_linear_nll(y, leaf[0], labels)
    (loss.sum() / 128).backward()
    return [loss.detach(), *(t.grad for t in leaf)]


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_tied_table_against_the_oracle(dtype):
    ids, labels, table, weight, bias = leaves(dtype)
    got = autograd(ids, labels, table, weight, bias)
    cpu = [t.double().cpu().requires_grad_() for t in (table, weight, bias)]
    i, l = ids.cpu(), labels.cpu()
    x = torch.where((i >= 0)[:, None], cpu[0][i.clamp(min=0)] * 8.0, 0.0)
    y = torch.nn.functional.layer_norm(x, (64,), cpu[1], cpu[2], 1e-5)
    loss = torch.nn.functional.cross_entropy(y @ cpu[0].t(), l, reduction="none")
    want = [loss.detach(), *torch.autograd.grad(loss.sum() / 128, cpu)]
    # Four tensors between the steps are rounded to the type (x, y, dy, dx), and the
    # gradients once or twice more: eight half steps in the norm, with errors of the
    # logits (64 terms of up to 3) as large as those of y.
    for name, a, b in zip(("loss", "table", "weight", "bias"), got, want):
        off = float((a.double().cpu() - b).norm() / b.norm())
        assert off < 8 * data.HALF[dtype] + 1e-5, (name, off)


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_recorded_and_direct_calls_agree(dtype):
    args = leaves(dtype)
    assert all(torch.equal(a, b) for a, b in zip(step(*args), autograd(*args)))


@pytest.mark.parametrize("dtype", list(data.TYPES))
def test_replayed_steps(dtype):
    """A step captured and replayed with other inputs in the same tensors, with eager
    steps between the replays."""
    args = leaves(dtype)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(*args)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*args)
    for seed in (1, 2, 3, 1):
        for t, new in zip(args, leaves(dtype, seed=seed)):
            t.copy_(new)
        args[1][:40 * (seed - 1)] = -100  # and another number of tokens with a loss
        graph.replay()
        eager = step(*args)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager)), seed
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager)), seed


def test_two_graphs_at_once():
    """Their workspaces are their own."""
    sets = [leaves("bf16", seed=s) for s in (1, 2)]
    want = [step(*s) for s in sets]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in sets]
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(*s))
        graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(5):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_calls_on_a_side_stream_beside_a_busy_one():
    sets = [leaves("bf16", seed=s) for s in (1, 2)]

    def run(ids, labels, table, weight, bias, stream=None):
        x = sm.softmax_embedding_fwd(ids, table, stream=stream)
        y, mean, rstd = sm.softmax_layer_norm_fwd(x, weight, bias, stream=stream)
        loss, lse = sm.softmax_linear_nll_fwd(y, table, labels, stream=stream)
        dy, dw = sm.softmax_linear_nll_bwd(loss, y, table, labels, loss, lse, stream=stream)
        grads = sm.softmax_layer_norm_bwd(dy, x, weight, mean, rstd, bias=True, stream=stream)
        return [loss, dw, *grads, sm.softmax_embedding_bwd(grads[0], ids, len(table),
                                                           stream=stream)]

    want = [run(*s) for s in sets]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda._sleep(10_000_000)
        here = run(*sets[0])
        there = run(*sets[1], side)
        torch.cuda.synchronize()
        for got, ref in ((here, want[0]), (there, want[1])):
            assert all(torch.equal(x, y) for x, y in zip(got, ref))
        del here, there


def test_outputs_that_are_given():
    """Written in place, counted as written, and refused on another device's or of
    another shape."""
    ids, labels, table, weight, bias = leaves("f32")
    x = torch.empty(150, 64, device="cuda")
    assert sm.softmax_embedding_fwd(ids, table, out=x) is x
    loss, lse = torch.empty(150, device="cuda"), torch.empty(150, device="cuda")
    got = sm.softmax_linear_nll_fwd(x, table, labels, loss=loss, lse=lse)
    assert got[0] is loss and got[1] is lse
    want = oracle.linear_nll(x.cpu(), table.cpu(), labels.cpu())
    assert float((loss.double().cpu() - want[0]).abs().max()) < 1e-4
    with pytest.raises(sm.SoftmaxError):        # the output is an input
        sm.softmax_embedding_fwd(ids, table[:150], out=table[:150])


def test_example_losses_and_gradients():
    """The example decoder's loss, against its own logits taken by elementary
    operations."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "decoder.py")
    spec = importlib.util.spec_from_file_location("example_decoder", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    torch.manual_seed(3)
    model = example.Decoder()
    g = torch.Generator().manual_seed(4)
    tokens, cu, lens = example.documents(g, torch.randperm(example.VOCAB, generator=g), 9, 60)
    labels = tokens.roll(-1)
    labels[cu[1:].long() - 1] = -100
    got = model.losses(tokens, cu, labels)
    got.sum().backward()
    grads = [p.grad.clone() for p in model.parameters()]
    model.zero_grad()
    logp = torch.log_softmax(model.packed(tokens, cu).double(), 1)
    keep = labels != -100
    want = torch.where(keep, -logp.gather(1, torch.where(keep, labels, 0)[:, None])[:, 0], 0.0)
    want.sum().backward()
    # fp32 throughout but for the attention, which both go through with the same
    # inputs: 256 terms in a logit, each with a factor up to 64 of sizes.
    assert float((got.double() - want).detach().abs().max()) < 64 * 256 * 2.0 ** -24
    # The gradients pass through the attention's in bf16: half a step, twice over.
    for p, grad in zip(model.parameters(), grads):
        assert float((p.grad - grad).norm()) <= 2.0 ** -8 * float(p.grad.norm())
