"""What cross entropy keeps of a row's digits, against 64 bits: the loss whatever offset all logits of the row share, the gradient of
classes far below the largest."""
import pytest
import torch

from operator_util import U, check, rounding
from paper_2412_07752_amd import api

pytestmark = pytest.mark.gpu

CLASSES = [3, 7, 100, 2048, 9000, 70_000, 150_001]   # rows of one value a lane, in the registers of a few lanes to a workgroup, and read twice


def chain(classes):
    """Roundings one behind the other in a row's sum: a thread's values (at most 32 up to 16384 classes, then those that 1024 threads leave each, whole chunks of 8 at the ends), lanes, waves; and where a
    row is read twice, three for each of a thread's chunks of 4 at which its maximum may rise (what the exponents lose there is part of |d|)."""
    return max(32, classes // 1024 + 16) + 6 + 16 + (3 * (classes // 4096 + 2) if classes > 65536 else 0)


def sum_and_bound(x):
    """(top, s, relative bound of s) of float64 rows, for loss_and_bound and the gradient."""
    top = x.max(1, keepdim=True).values
    d = x - top
    e = torch.exp(d)
    s = e.sum(1, keepdim=True)
    return top, s, U * (chain(x.shape[1]) + 2 + 3 * (e / s * d.abs()).sum(1, keepdim=True))


def loss_and_bound(x, t):
    """(loss, bound).  loss = log s + (top - x_t), s = sum e_j, e_j = exp(d_j), d_j = x_j - top.  The difference is off by U |d|, the product with log2 e and that constant by as much each, the
    exponential by 2 U: e_j by (2 + 3 |d_j|) U, relative; s by chain U more, which is what log s is off by, beside 4 U of itself (two units in the last place).  Then U of the target's difference and of the sum."""
    top, s, off = sum_and_bound(x.double())
    log_s, down = torch.log(s)[:, 0], (top - x.double().gather(1, t[:, None]))[:, 0]
    return log_s + down, off[:, 0] + U * (4 * log_s + 2 * down + log_s)


@pytest.mark.parametrize("classes", CLASSES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_loss_does_not_lose_digits_to_the_offset_of_a_row(classes, dtype):
    gen = torch.Generator().manual_seed(classes)
    offsets = torch.tensor([0.0, 100.0, -100.0, 1000.0, -30_000.0, 30_000.0, 1e6, 0.0])
    x = torch.randn(len(offsets), classes, generator=gen) + offsets[:, None]
    t = torch.randint(classes, (len(offsets),), generator=gen)
    t[0], t[1] = classes - 1, 0
    x[torch.arange(len(offsets)), t] += torch.log(torch.tensor(float(classes))) + 6   # (a target that has nearly all of the probability)
    x = x.to(dtype).cuda()
    t = t.cuda()
    want, bound = loss_and_bound(x, t)
    loss, _ = api.flashrnn_cross_entropy(x, t)
    check(loss, want, bound, "loss")
    alone, _ = api.flashrnn_cross_entropy(x, t, gradient=False)
    check(alone, want, bound, "loss alone")


@pytest.mark.parametrize("classes", CLASSES)
def test_float32_gradients_of_classes_far_below_the_largest(classes):
    """The largest logit is 0 and every other 30 to 80 below: the differences are exact and the sum is 1 but for less than U.  What is left is the exponential (4 U: two units in the last place) and a
    handful of roundings: the sum, its quotient, the product (2 U each)."""
    gen = torch.Generator().manual_seed(classes)
    x = -(30 + 50 * torch.rand(5, classes, generator=gen))
    top, t = torch.randint(classes, (5,), generator=gen), torch.randint(classes, (5,), generator=gen)
    t[0] = top[0]
    x[torch.arange(5), top] = 0.0
    e = torch.exp(x.double())   # (on the host, from its parts: the library's softmax of float64 rows on the GPU is itself off by 60 units of 2^-24 beyond 1024 classes)
    p = e / e.sum(1, keepdim=True)
    want = p.scatter_add(1, t[:, None], torch.full((5, 1), -1.0, dtype=torch.float64))
    _, grad = api.flashrnn_cross_entropy(x.cuda(), t.cuda())
    check(grad, want, 10 * U * p + rounding(torch.float32, want), "dlogits")


@pytest.mark.parametrize("classes", [3, 40, 256, 1000, 9000, 65_536, 131_072, 150_001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_and_lse_to_the_bounds_of_a_row_of_their_length(classes, dtype):
    """p = f e / s: s as loss_and_bound has it, e in the gradient by 4 U (bf16 logits: by (2 + 3 |d|) U), the quotient, the product and the difference by U each."""
    gen = torch.Generator().manual_seed(classes + 1)
    x = (torch.randn(7, classes, generator=gen) * 3).to(dtype)
    t = torch.randint(classes, (7,), generator=gen)
    top, s, off = sum_and_bound(x.double())
    d = x.double() - top
    p = torch.exp(d) / s
    hot = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    bound = p * (off + U * (4 if dtype == torch.float32 else 2 + 3 * d.abs()) + 2 * U) + U * (p - hot).abs() + 2.0 ** -126
    want_lse = (torch.log(s) + top)[:, 0]
    lse = torch.empty(7, device="cuda")
    _, grad = api.flashrnn_cross_entropy(x.cuda(), t.cuda(), lse=lse)
    check(grad, p - hot, bound + (rounding(dtype, p - hot) if dtype == torch.bfloat16 else 0), "dlogits")
    check(lse, want_lse, off[:, 0] + U * (4 * torch.log(s)[:, 0] + want_lse.abs()), "lse")
