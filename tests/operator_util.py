"""Plain implementations in 64 bits of the operators around the time-step loop, and the bounds that a float32 evaluation of them keeps.

U is half a unit in the last place of float32, relative.  A sum of n terms, added in any tree whose longest chain has `chain` additions, is off by at
most chain * U * sum|term|; `CHAIN` covers the trees of the kernels (a lane's own chain, then lanes, waves and workgroups).  Rounding to
bfloat16 (8 bits, as U is for 24) adds 2^-8 of the value."""
import torch

U = 2.0 ** -24
CHAIN = 64
CHAIN_ROWS = 512      # sums over rows: a workgroup's rows one after the other, then the workgroups
BF16 = 2.0 ** -8


def rounding(dtype, value):
    return (BF16 if dtype == torch.bfloat16 else U) * value.abs()


def check(got, want, bound, what):
    got, want, bound = got.double().cpu(), want.double().cpu(), torch.as_tensor(bound, dtype=torch.float64).cpu().expand(want.shape)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaN in other places"
    special = want.isinf()
    assert torch.equal(got[special], want[special]), f"{what}: infinities"
    off = (got - want).abs()
    bad = ~(off <= bound) & ~special & ~want.isnan()
    assert not bad.any(), f"{what}: {int(bad.sum())} of {want.numel()} values off, the worst {float((off / bound.clamp(min=1e-300))[bad].max()):.3g} times its bound"


def layer_norm(x, weight, bias, eps):
    """(y, mean, rstd) and y's bound: the mean is off by CHAIN U E|x|, the deviation relative to that and to itself."""
    x = x.double()
    w = 1.0 if weight is None else weight.double()
    b = 0.0 if bias is None else bias.double()
    mean = x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    xhat = (x - mean) * rstd
    y = xhat * w + b
    off = CHAIN * U * (x.abs().mean(-1, keepdim=True) * rstd + 1) * (1 + xhat.abs())
    bound = off * (w.abs() if weight is not None else 1.0) + 4 * U * y.abs() + (U * 4 * b.abs() if bias is not None else 0.0)
    return y, mean[..., 0], rstd[..., 0], bound


def layer_norm_grad(dy, x, mean, rstd, weight):
    """(dx, dweight, dbias) from the statistics given, and their bounds."""
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[..., None], rstd.double()[..., None]
    g = dy * (1.0 if weight is None else weight.double())
    xhat = (x - mean) * rstd
    dx = rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
    # xhat itself: one rounding of the difference, one of the product
    size = rstd * (g.abs() + g.abs().mean(-1, keepdim=True) + xhat.abs() * (g * xhat).abs().mean(-1, keepdim=True))
    dims = tuple(range(x.dim() - (1 if weight is None else weight.dim())))
    terms, rows = dy * xhat, dy
    total = (lambda t: t.sum(dims)) if dims else (lambda t: t)
    return (dx, total(terms), total(rows)), (CHAIN * U * size, CHAIN_ROWS * U * total(terms.abs()), CHAIN_ROWS * U * total(rows.abs()))


def embedding(table, tokens, scale):
    V = table.shape[0]
    there = (tokens >= 0) & (tokens < V)
    rows = table.double()[torch.where(there, tokens, 0).long()] * scale
    return torch.where(there[..., None], rows, 0.0)


def embedding_grad(tokens, dout, vocab, scale):
    """(dtable, bound): a word's sum chains at most as many additions as it has places."""
    tokens, dout = tokens.reshape(-1).long().cpu(), dout.reshape(-1, dout.shape[-1]).double().cpu()
    there = (tokens >= 0) & (tokens < vocab)
    total, size = (torch.zeros(vocab, dout.shape[1], dtype=torch.float64).index_add_(0, tokens[there], d[there]) for d in (dout, dout.abs()))
    count = torch.bincount(tokens[there], minlength=vocab)[:, None]
    return total * scale, (count + 2) * U * size * abs(scale)


def cross_entropy(logits, targets, dloss, scale):
    """(loss, lse, dlogits) and their bounds: exp(x - lse) is off by a few U and by U of its argument's parts."""
    x = logits.double().cpu()
    N, V = x.shape
    t, dloss = targets.long().cpu(), torch.ones(N, dtype=torch.float64) if dloss is None else dloss.double().cpu()
    there = (t >= 0) & (t < V)
    at = torch.where(there, t, 0)[:, None]
    top = x.max(1, keepdim=True).values
    empty = (x == float("-inf")).all(1)
    top = torch.where(empty[:, None], 0.0, top)
    lse = torch.log(torch.exp(x - top).sum(1)) + top[:, 0]
    loss = torch.where(there, torch.where(empty, float("inf"), lse - x.gather(1, at)[:, 0]), 0.0)
    p = torch.where(empty[:, None], 0.0, torch.exp(x - lse[:, None]))
    hot = torch.zeros_like(x).scatter_(1, at, 1.0)
    use = there & ~empty
    grad = torch.where(use[:, None], scale * dloss[:, None] * (p - hot), 0.0)
    finite = torch.where(x.isfinite(), x, 0.0)
    off = CHAIN * U * (4 + lse.nan_to_num(posinf=0, neginf=0).abs() + top[:, 0].nan_to_num(posinf=0, neginf=0).abs())
    pbound = p * (off[:, None] + 4 * U * (finite - top).abs()) + 2.0 ** -126
    gbound = torch.where(use[:, None], abs(scale) * dloss[:, None].abs() * (pbound + 4 * U * (p + hot)), 0.0)
    return (loss, lse, grad), (off + 4 * U * x.gather(1, at)[:, 0].nan_to_num(posinf=0, neginf=0).abs(), off, gbound)
