"""Inputs of the tests of what a decoder has around its attention, and bounds on
the kernels' errors, by counting roundings.

Half a step of a type is eps / 2 of the value: HALF.  Sums of n terms in fp32, in
whatever order and whether a matrix operation rounds or cuts off, are within n *
2^-23 of the sum of the terms' sizes."""
import torch

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}  # half a denormal step
CUT = 2.0 ** -23


def matrix(g, rows, cols, dtype, scale=1.0):
    return (torch.randn(rows, cols, generator=g) * scale).to(TYPES[dtype])


def strided(t, pad, lead=0):
    """The same values with rows further apart, inside a larger tensor of NaN."""
    wide = torch.full((t.shape[0], lead + t.shape[1] + pad), torch.nan, dtype=t.dtype,
                      device=t.device)
    out = wide[:, lead:lead + t.shape[1]]
    out.copy_(t)
    return out


def close(name, got, want, bound):
    """got within bound of want (float64 tensors on the CPU), NaN and infinities
    where want has them."""
    got = got.double().cpu()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), name
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), name
    off = torch.where(fine, (got - want).abs(), 0.0)
    bound = torch.as_tensor(bound, dtype=torch.float64).expand_as(want)
    worst = torch.where(fine, off - bound, -1.0)
    if worst.numel() and worst.max() > 0:
        i = int(worst.argmax())
        raise AssertionError(f"{name}: {got.flatten()[i]} against {want.flatten()[i]}, "
                             f"off by {off.flatten()[i]}, bound {bound.flatten()[i]}, at {i} of "
                             f"{tuple(want.shape)}; {int((worst > 0).sum())} outside")


def nll_bounds(x, weight, labels, ignore, dloss, dtype, exact):
    """Bounds of (loss, lse, dx, dweight) from what oracle.decoder_f64.linear_nll
    gives with ``dloss``.

    A logit is off by d cut sums.  An exponential relative to the maximum is off by
    that, by its argument's two roundings (|argument| <= 2 max|logit|) and the
    instruction's own (2 half steps), as is the label's logit; the sum of
    exponentials by its sums (at most 64 in a row and 9 levels, then binary64)."""
    loss, lse, dx, dweight, p, g = exact
    live = (labels != ignore)[:, None]
    x = torch.where(live, x.double(), 0.0).nan_to_num()
    w = weight.double()
    size = x.abs() @ w.abs().t()
    d = x.shape[1]
    logit = d * CUT * size.amax(1) + TINY["f32"]
    most = (x @ w.t()).abs().amax(1)
    term = logit + 2.0 ** -24 * (4 * most + 2)
    total = term + 80 * 2.0 ** -24
    b_lse = total + 2.0 ** -24 * lse.abs()
    b_loss = logit + total + 2.0 ** -24 * loss.abs()
    # Of g: the exponential of logit - lse (lse off by its bound), its product with
    # the token's weight (two roundings), and the rounding to the type.
    rel = (logit + b_lse + 2.0 ** -24 * (4 * most + 6))[:, None]
    b_g = p.abs() * (torch.expm1(rel) + b_loss[:, None]) + g.abs() * (4 * 2.0 ** -24)
    # Exponentials below the normal numbers, 2^-126, are taken as 0 by the
    # instruction, and what the largest dloss leaves of g below them by the matrix
    # operations.
    b_g = b_g + 2.0 ** -125 * dloss.abs().max()
    rounding = torch.zeros_like(b_g)
    if dtype != "f32":
        # Up to 256 tokens g is held in two parts of the type.
        few = int(live.sum()) <= 256
        rounding = (g.abs() + b_g) * (HALF[dtype] ** 2 if few else HALF[dtype])
        if dtype == "f16":
            # Relative to the largest dloss, times 2^14: half a step of denormal numbers.
            rounding = rounding + 2.0 ** -25 * 2.0 ** -14 * dloss.abs().max()
    b_g, rounding = torch.where(live, b_g, 0.0), torch.where(live, rounding, 0.0)
    b_gw = b_g + rounding
    # dx takes in what the rounding left at the label, in fp32.
    at = torch.where(live[:, 0] & (labels >= 0) & (labels < len(w)), labels, 0)[:, None]
    rest = rounding.gather(1, at) * 2.0 ** -22 if dtype != "f32" else torch.zeros(len(at), 1)
    b_gx = b_g + rounding.scatter(1, at, rest.to(rounding.dtype))
    gs, v, t = g.abs() + b_gw, w.shape[0], x.shape[0]
    # Products are summed in up to 64 splits, and g's two parts one after the other.
    b_dx = b_gx @ w.abs() + (2 * v + 64) * CUT * (gs @ w.abs())
    b_dw = b_gw.t() @ x.abs() + (2 * t + 64) * CUT * (gs.t() @ x.abs())
    out = [b_loss, b_lse, b_dx, b_dw]
    for i, want in ((2, dx), (3, dweight)):
        out[i] = out[i] + (want.abs() + out[i]) * (HALF[dtype] + 2.0 ** -24) + TINY[dtype]
    return [torch.where(live[:, 0], b, 0.0) if b.dim() == 1 else b for b in out]
