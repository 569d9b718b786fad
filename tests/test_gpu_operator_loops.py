"""The operators around the time-step loop beyond one round of workgroups: rows, places and chunks that a group of threads comes to on its second turn and later, on data of which no two parts are alike."""
import pytest
import torch

import operator_util as ou
from paper_2412_07752_amd import api

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, *shape, dtype=F32):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _words(gen, n, vocab, index=torch.int64):
    """Words whose frequency falls with their rank, and places outside the vocabulary on both sides."""
    t = (float(vocab) ** torch.rand(n, generator=gen, device="cuda") - 1).long().clamp(max=vocab - 1)
    mask = torch.rand(n, generator=gen, device="cuda")
    return torch.where(mask < 0.02, -1, torch.where(mask > 0.98, vocab, t)).to(index)


def _some_rows(gen, rows, turn):
    """Rows around every turn's beginning, the last ones, and some at random."""
    at = torch.arange(0, rows, turn, device="cuda")
    at = (at[:, None] + torch.arange(-40, 40, device="cuda")).reshape(-1)
    at = torch.cat([at, torch.arange(rows - 70, rows, device="cuda"), torch.randint(rows, (4000,), generator=gen, device="cuda")])
    return at[(at >= 0) & (at < rows)].unique()


# (rows per turn of a forward call: 8192 workgroups of 256 threads over the threads that share a row)
@pytest.mark.parametrize("tokens,heads,width,x_dtype,dtype,turn", [
    (37_500, 8, 256, F32, BF16, 131_072), (140_000, 3, 80, F32, F32, 262_080), (20_001, 0, 1111, F32, F32, 16_384), (66_001, 0, 768, BF16, BF16, 65_536),
    (34_003, 0, 2048, BF16, F32, 32_768), (2_501, 0, 12_001, F32, BF16, 2_048), (1_100_001, 0, 5, BF16, F32, 1 << 20), (263_001, 0, 33, BF16, BF16, 262_144)])
def test_layer_norm_of_more_rows_than_one_turn(tokens, heads, width, x_dtype, dtype, turn):
    gen = _gen(tokens)
    shape = (heads, width) if heads else (width,)
    rows = tokens * max(1, heads)
    if heads:   # hidden states inside the loop's states: dense but for the time axis
        x = _normal(gen, tokens // 20 + 1, 2, 20, *shape, dtype=x_dtype)[1:, 0]
    else:
        x = _normal(gen, tokens, *shape, dtype=x_dtype) * torch.exp(_normal(gen, tokens, 1) * 0.5).to(x_dtype)
    w, b = 1 + 0.2 * _normal(gen, *shape), _normal(gen, *shape)
    y, mean, rstd = api.flashrnn_layer_norm_fwd(x, w, b, dtype=dtype)
    dy = _normal(gen, *x.shape, dtype=dtype)
    dx, dw, db = api.flashrnn_layer_norm_bwd(dy, x, mean, rstd, w)
    at = _some_rows(gen, rows, turn)
    take = lambda t: t.reshape(rows, width)[at]
    group = at % max(1, heads)
    xs, ws, bs = take(x), w.view(-1, width)[group], b.view(-1, width)[group]
    want_y, want_mean, want_rstd, bound = ou.layer_norm(xs, ws, bs, 1e-5)
    ou.check(take(y), want_y, bound + ou.rounding(dtype, want_y), "y")
    size = xs.double().abs().mean(-1)
    ou.check(mean.view(-1)[at], want_mean, ou.CHAIN * ou.U * size, "mean")
    ou.check(rstd.view(-1)[at], want_rstd, ou.CHAIN * ou.U * want_rstd * (1 + size * want_rstd), "rstd")
    want, bounds = ou.layer_norm_grad(take(dy), xs, mean.view(-1)[at], rstd.view(-1)[at], ws)
    ou.check(take(dx), want[0], bounds[0] + ou.rounding(dtype, want[0]), "dx")
    (_, want_dw, want_db), (_, dw_bound, db_bound) = ou.layer_norm_grad(dy.reshape(tokens, *shape), x.reshape(tokens, *shape), mean.view(tokens, *shape[:-1]), rstd.view(tokens, *shape[:-1]), w)
    # (rows below 8 values: 256 strips of rows, each added up one behind the other)
    chain = ou.CHAIN_ROWS if width >= 8 else tokens // 256 + 1 + 256
    ou.check(dw, want_dw, dw_bound * (chain / ou.CHAIN_ROWS), "dweight")
    ou.check(db, want_db, db_bound * (chain / ou.CHAIN_ROWS), "dbias")


@pytest.mark.parametrize("n,vocab,width,table_dtype,dtype", [(17_001, 5000, 1024, BF16, BF16), (40_003, 700, 2048, F32, BF16), (70_001, 300, 100, BF16, F32), (66_002, 50_304, 1111, F32, F32), (9_001, 40, 4099, BF16, BF16)])
@pytest.mark.parametrize("index", [torch.int64, torch.int32])
def test_embedding_of_several_places_at_a_time(n, vocab, width, table_dtype, dtype, index):
    gen = _gen(n)
    table, tokens = _normal(gen, vocab, width, dtype=table_dtype), _words(gen, n, vocab, index)
    out = api.flashrnn_embedding_fwd(table, tokens, scale=1.7, dtype=dtype)
    there = (tokens >= 0) & (tokens < vocab)
    want = torch.where(there[:, None], table[torch.where(there, tokens, 0).long()].float() * torch.tensor(1.7, device="cuda"), 0.0).to(dtype)   # (one product, rounded as the kernel's)
    assert torch.equal(out, want)


def test_embedding_of_more_places_than_one_turn():
    """A million workgroups of 32 groups of lanes with four places each, and a few more."""
    n, gen = (1 << 20) * 128 + 70_001, _gen(1)
    table = _normal(gen, 1000, 2, dtype=BF16)
    tokens = torch.randint(1000, (n,), generator=gen, device="cuda", dtype=torch.int32)
    out = api.flashrnn_embedding_fwd(table, tokens)
    for i in range(0, n, 1 << 25):
        assert torch.equal(out[i:i + (1 << 25)], table[tokens[i:i + (1 << 25)].long()])


@pytest.mark.parametrize("n,vocab,width,frequent", [(20_000, 50_304, 2048, 0), (24_001, 300, 1408, 11), (600_000, 70_000, 80, 3), (66_003, 999, 516, 998)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_embedding_gradient_in_the_longest_runs(n, vocab, width, frequent, dtype):
    """Runs of 64 places, among them whole runs of one word; tables beyond what one round of workgroups fills with zeros."""
    gen = _gen(n)
    tokens, dout = _words(gen, n, vocab), _normal(gen, n, width, dtype=dtype)
    tokens[torch.rand(n, generator=gen, device="cuda") < 0.2] = frequent
    there = (tokens >= 0) & (tokens < vocab)
    want, size = (torch.zeros(vocab, width, dtype=torch.float64, device="cuda").index_add_(0, tokens[there], d[there].double()) * 1.7 for d in (dout, dout.abs()))
    count = torch.bincount(tokens[there], minlength=vocab)[:, None]
    bound = (count + 2) * ou.U * size
    dtable = torch.full((vocab, width), float("nan"), device="cuda")
    api.flashrnn_embedding_bwd(tokens, dout, vocab, scale=1.7, dtable=dtable)
    ou.check(dtable, want, bound, "dtable")
    base = torch.where(count > 0, _normal(gen, vocab, width), float("nan"))
    got = api.flashrnn_embedding_bwd(tokens, dout, vocab, scale=1.7, dtable=base.clone(), accumulate=True)
    total = torch.where(count > 0, base.double() + want, float("nan"))
    ou.check(got, total, bound + ou.U * (total.abs() + base.double().abs()), "accumulated")


@pytest.mark.parametrize("rows,classes,dtype", [(1_100_003, 3, F32), (1_050_001, 7, BF16), ((1 << 25) + 5_003, 8, BF16)])
def test_cross_entropy_of_more_rows_than_one_turn(rows, classes, dtype):
    gen = _gen(rows)
    logits, targets = _normal(gen, rows, classes, dtype=dtype), torch.randint(-1, classes, (rows,), generator=gen, device="cuda")
    loss, grad = api.flashrnn_cross_entropy(logits, targets, grad_scale=0.25)
    at = _some_rows(gen, rows, 1 << 20 if classes < 8 else 1 << 25)
    want, bounds = ou.cross_entropy(logits[at], targets[at], None, 0.25)
    ou.check(loss[at], want[0], bounds[0], "loss")
    ou.check(grad[at], want[2], bounds[2] + ou.rounding(dtype, want[2]), "dlogits")


@pytest.mark.parametrize("sizes", [[20_000_003], [9_000_001, 11, 8_500_000, 7], [300_000] * 130])
@pytest.mark.parametrize("types", [[F32], [BF16], [F32, BF16]])
@pytest.mark.parametrize("in_place", [False, True])
def test_clip_of_more_chunks_than_one_turn(sizes, types, in_place):
    """More than 1024 chunks of a table of tensors, and outputs beyond the second-level caches."""
    gen = _gen(len(sizes))
    grads = [_normal(gen, n, dtype=types[k % len(types)]) for k, n in enumerate(sizes)]
    want = sum((g.double() ** 2).sum().item() for g in grads) ** 0.5
    given = [g.clone() for g in grads]
    out = given if in_place else [torch.full_like(g, 7.0) for g in grads]
    norm = api.flashrnn_grad_clip(given, 0.5, out=None if in_place else out)
    assert abs(norm.item() - want) <= 2 * ou.U * want
    for i, (g, o) in enumerate(zip(grads, out)):
        scaled = g.double() * (0.5 / want)
        off = (o.double() - scaled).abs()
        assert (off <= 4 * ou.U * scaled.abs() + ou.rounding(g.dtype, scaled)).all(), (i, off.max().item())
        assert in_place or torch.equal(given[i], g)


@pytest.mark.parametrize("width", [20_011, 32_768, 40_000])
def test_layer_norm_of_long_rows_to_the_bounds_of_their_own_chain(width):
    """Rows that the registers do not hold: a thread adds up every 256th value, then 64 lanes and four waves meet.  The bounds scale with that chain."""
    gen = _gen(width)
    more = (-(-width // 256) + 6 + 4) / ou.CHAIN
    x, w, b = _normal(gen, 9, width), 1 + 0.2 * _normal(gen, width), _normal(gen, width)
    y, mean, rstd = api.flashrnn_layer_norm_fwd(x, w, b)
    want_y, want_mean, want_rstd, bound = ou.layer_norm(x, w, b, 1e-5)
    size = x.double().abs().mean(-1)
    ou.check(y, want_y, more * bound, "y")
    ou.check(mean, want_mean, more * ou.CHAIN * ou.U * size, "mean")
    ou.check(rstd, want_rstd, more * ou.CHAIN * ou.U * want_rstd * (1 + size * want_rstd), "rstd")
    dy = _normal(gen, 9, width)
    dx, _, _ = api.flashrnn_layer_norm_bwd(dy, x, mean, rstd, w)
    want, bounds = ou.layer_norm_grad(dy, x, mean, rstd, w)
    ou.check(dx, want[0], more * bounds[0], "dx")
