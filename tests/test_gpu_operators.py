"""The operators around the time-step loop against plain implementations in 64 bits: sizes, types, strides and masks where they can go wrong."""
import itertools

import pytest
import torch

import operator_util as ou
from paper_2412_07752_amd import api

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TYPES = [F32, BF16]


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _normal(gen, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype).cuda()


def _odd_place(t):
    """The same tensor, its memory starting at an address that only the element's own size divides."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    flat[1:] = t.reshape(-1)
    return flat[1:].view(t.shape)


# ---- embedding -------------------------------------------------------------------------------------------------------------------------------
EMBEDDINGS = [(1, 1, 1), (1, 30, 768), (3, 7, 5), (64, 2, 64), (65, 129, 33), (257, 1000, 100), (1000, 65, 256), (2049, 3, 24), (4096, 32000, 96), (5000, 131072, 17), (300, 50, 4099)]


def _tokens(gen, n, vocab, index, skew=True):
    """Words whose frequency falls with their rank, with places outside the vocabulary on both sides."""
    u = torch.rand(n, generator=gen)
    t = (vocab ** u - 1).long().clamp(max=vocab - 1) if skew else (u * vocab).long().clamp(max=vocab - 1)
    mask = torch.rand(n, generator=gen)
    t = torch.where(mask < 0.05, -1, t)
    t = torch.where(mask > 0.97, vocab, t)
    t = torch.where((mask > 0.05) & (mask < 0.07), torch.iinfo(index).min, t)
    return t.to(index).cuda()


@pytest.mark.parametrize("n,vocab,width", EMBEDDINGS)
@pytest.mark.parametrize("table_dtype,dtype", itertools.product(TYPES, TYPES))
@pytest.mark.parametrize("index", [torch.int64, torch.int32])
def test_embedding(n, vocab, width, table_dtype, dtype, index):
    gen = _gen(n + width)
    table, tokens = _normal(gen, vocab, width, dtype=table_dtype), _tokens(gen, n, vocab, index)
    out = api.flashrnn_embedding_fwd(table, tokens, scale=1.7, dtype=dtype)
    want = ou.embedding(table, tokens, 1.7)
    ou.check(out, want, 2 * ou.U * want.abs() + ou.rounding(dtype, want), "out")
    there = ((tokens >= 0) & (tokens < vocab)).cpu()
    assert not out.cpu()[~there].any()


@pytest.mark.parametrize("n,vocab,width", EMBEDDINGS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("index", [torch.int64, torch.int32])
def test_embedding_gradient(n, vocab, width, dtype, index):
    gen = _gen(n + width)
    tokens, dout = _tokens(gen, n, vocab, index), _normal(gen, n, width, dtype=dtype)
    want, bound = ou.embedding_grad(tokens, dout, vocab, 1.7)
    dtable = torch.full((vocab, width), float("nan"), device="cuda")
    ws = torch.full((api.flashrnn_embedding_workspace_bytes(n, vocab, width),), 0xAB, dtype=torch.uint8, device="cuda")
    api.flashrnn_embedding_bwd(tokens, dout, vocab, scale=1.7, dtable=dtable, workspace=ws)
    ou.check(dtable, want, bound, "dtable")
    again = api.flashrnn_embedding_bwd(tokens, dout, vocab, scale=1.7)
    assert torch.equal(dtable, again), "another result on the same inputs"
    # added to what is there; other rows stay as they are, whatever they hold
    there = torch.bincount(tokens[(tokens >= 0) & (tokens < vocab)].long().cpu(), minlength=vocab) > 0
    base = torch.where(there[:, None], torch.randn(vocab, width, generator=gen), float("nan")).cuda()
    got = api.flashrnn_embedding_bwd(tokens, dout, vocab, scale=1.7, dtable=base.clone(), accumulate=True)
    total = torch.where(there[:, None], base.double().cpu() + want, float("nan"))
    ou.check(got, total, bound + ou.U * (total.abs() + base.double().cpu().abs()), "accumulated")


@pytest.mark.parametrize("n,vocab,width,words", [(3000, 40, 64, [7]), (4097, 70000, 40, [69999, 0]), (70000, 300, 8, [299]), (20000, 65536, 72, [65535]), (9000, 65535, 16, [65534, 65533, 0])])
@pytest.mark.parametrize("dtype", TYPES)
def test_embedding_gradient_of_very_frequent_words(n, vocab, width, words, dtype):
    """One word, or a few, over thousands of places that no tile of any kernel holds."""
    gen = _gen(n)
    tokens = torch.tensor(words)[torch.randint(len(words), (n,), generator=gen)]
    tokens[::97] = torch.randint(vocab, (len(tokens[::97]),), generator=gen)
    tokens, dout = tokens.cuda(), _normal(gen, n, width, dtype=dtype)
    want, bound = ou.embedding_grad(tokens, dout, vocab, 1.0)
    got = api.flashrnn_embedding_bwd(tokens, dout, vocab)
    ou.check(got, want, bound, "dtable")
    assert torch.equal(got, api.flashrnn_embedding_bwd(tokens, dout, vocab))


@pytest.mark.parametrize("n,vocab,width", [(300, 300_000, 8), (12288, 262_143, 24), (12289, 262_143, 24), (12000, 262_144, 24), (20_000, 2_000_000, 4), (300_001, 70_000, 16), (600_000, 513, 12)])
@pytest.mark.parametrize("index", [torch.int64, torch.int32])
def test_embedding_gradient_of_every_way_to_sort(n, vocab, width, index):
    """Few and many places, words of one to three digits, tiles of several steps; with padding on both sides of the vocabulary."""
    gen = _gen(n)
    tokens, dout = _tokens(gen, n, vocab, index), _normal(gen, n, width)
    want, bound = ou.embedding_grad(tokens, dout, vocab, 0.5)
    got = api.flashrnn_embedding_bwd(tokens, dout, vocab, scale=0.5)
    ou.check(got, want, bound, "dtable")
    assert torch.equal(got, api.flashrnn_embedding_bwd(tokens, dout, vocab, scale=0.5))
    again = api.flashrnn_embedding_bwd(tokens, dout, vocab, scale=0.5, dtable=got.clone(), accumulate=True)
    ou.check(again, 2 * want, 2 * bound + 2 * ou.U * want.abs(), "accumulated")


@pytest.mark.parametrize("n,vocab,width", [(1, 1, 1), (64, 65, 3), (65, 64, 2), (1024, 300, 40), (1025, 300, 40), (1023, 100_000, 7), (1024, 2000, 1100), (900, 7, 2048), (1024, 40, 2050), (3, 5, 70_000)])
@pytest.mark.parametrize("dtype,index", [(F32, torch.int32), (BF16, torch.int64)])
def test_embedding_gradient_of_few_places(n, vocab, width, dtype, index):
    """Around the largest number of places, and of places times columns, that one launch takes; words all different, all the same, and in between."""
    gen = _gen(n + width)
    words = _tokens(gen, n, vocab, index)
    dout = _normal(gen, n, width, dtype=dtype)
    for tokens in (words, torch.full_like(words, vocab - 1), torch.arange(n, dtype=index, device="cuda") * 2 - 1):
        want, bound = ou.embedding_grad(tokens, dout, vocab, 1.5)
        got = api.flashrnn_embedding_bwd(tokens, dout, vocab, scale=1.5, dtable=torch.full((vocab, width), float("nan"), device="cuda"))
        ou.check(got, want, bound, "dtable")
        assert torch.equal(got, api.flashrnn_embedding_bwd(tokens, dout, vocab, scale=1.5))
        again = api.flashrnn_embedding_bwd(tokens, dout, vocab, scale=1.5, dtable=got.clone(), accumulate=True)
        ou.check(again, 2 * want, 2 * bound + 2 * ou.U * want.abs(), "accumulated")


@pytest.mark.parametrize("n,vocab,width", [(512, 300, 768), (513, 300, 768), (256, 9, 4096), (257, 9, 4096), (1024, 33, 128), (1024, 33, 129)])
@pytest.mark.parametrize("dtype,index", [(F32, torch.int64), (BF16, torch.int32)])
def test_embedding_gradient_of_the_most_places_that_one_launch_takes(n, vocab, width, dtype, index):
    test_embedding_gradient_of_few_places(n, vocab, width, dtype, index)


def test_embedding_of_places_beyond_32_bit_offsets():
    n, width = (1 << 31) // 4096 + 5000, 4096
    tokens = torch.zeros(n, dtype=torch.int32, device="cuda")
    tokens[-3:] = torch.tensor([7, 5, 7], dtype=torch.int32)
    table = torch.arange(9, device="cuda", dtype=BF16)[:, None].expand(9, width).contiguous()
    out = api.flashrnn_embedding_fwd(table, tokens)
    assert out[-3:].float().mean(1).tolist() == [7.0, 5.0, 7.0] and not out[:-3].any()
    dtable = api.flashrnn_embedding_bwd(tokens, out, 9)
    assert (dtable[7] == 14).all() and (dtable[5] == 5).all() and not dtable[[0, 1, 2, 3, 4, 6, 8]].any()


def test_embedding_of_no_tokens_and_of_padding_alone():
    table = torch.randn(9, 12, device="cuda")
    none = torch.empty((0, 4), dtype=torch.int64, device="cuda")
    assert api.flashrnn_embedding_fwd(table, none).shape == (0, 4, 12)
    assert not api.flashrnn_embedding_bwd(none, torch.empty(0, 4, 12, device="cuda"), 9, dtable=torch.ones(9, 12, device="cuda")).any()
    padding = torch.full((5,), -1, device="cuda")
    assert not api.flashrnn_embedding_fwd(table, padding).any()
    assert not api.flashrnn_embedding_bwd(padding, torch.full((5, 12), float("nan"), device="cuda"), 9).any()
    kept = torch.full((9, 12), 3.0, device="cuda")
    api.flashrnn_embedding_bwd(padding, torch.ones(5, 12, device="cuda"), 9, dtable=kept, accumulate=True)
    assert (kept == 3.0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_embedding_of_memory_that_starts_anywhere(dtype):
    gen = _gen(5)
    table, tokens = _odd_place(_normal(gen, 50, 48, dtype=dtype)), _tokens(gen, 200, 50, torch.int64)
    out = _odd_place(torch.empty(200, 48, dtype=dtype, device="cuda"))
    api.flashrnn_embedding_fwd(table, tokens, out=out)
    assert torch.equal(out, api.flashrnn_embedding_fwd(table.clone(), tokens))
    dout, dtable = _odd_place(_normal(gen, 200, 48, dtype=dtype)), _odd_place(torch.empty(50, 48, device="cuda"))
    api.flashrnn_embedding_bwd(tokens, dout, 50, dtable=dtable)
    assert torch.equal(dtable, api.flashrnn_embedding_bwd(tokens, dout.clone(), 50))


def test_embedding_of_a_table_beyond_32_bit_offsets():
    V, H = (1 << 31) // 4096 + 3, 4096
    table = torch.zeros(V, H, dtype=BF16, device="cuda")
    table[-2:] = 1.5
    tokens = torch.tensor([V - 1, 0, V - 2, V - 3], device="cuda")
    out = api.flashrnn_embedding_fwd(table, tokens)
    assert out.float().mean(1).tolist() == [1.5, 0.0, 1.5, 0.0]
    del table
    dtable = api.flashrnn_embedding_bwd(tokens, torch.ones(4, H, device="cuda"), V)
    assert (dtable[-3:] == 1).all() and (dtable[0] == 1).all() and not dtable[1:-3].any()


# ---- layer norm --------------------------------------------------------------------------------------------------------------------------------
WIDTHS = [1, 2, 7, 8, 16, 33, 64, 80, 127, 192, 256, 500, 512, 513, 768, 1000, 1024, 1111, 2048, 2052, 3000, 4096, 5001, 8192, 8200, 16384, 20011, 32768, 40000]


def _rows(gen, rows, width, dtype):
    return ((torch.randn(rows, width, generator=gen) + torch.randn(rows, 1, generator=gen)) * torch.exp(torch.randn(rows, 1, generator=gen))).to(dtype).cuda()


def _check_norm(x, weight, bias, dtype, dx_dtype, gen, eps=1e-5):
    y, mean, rstd = api.flashrnn_layer_norm_fwd(x, weight, bias, eps=eps, dtype=dtype)
    want_y, want_mean, want_rstd, bound = ou.layer_norm(x, weight, bias, eps)
    ou.check(y, want_y, bound + ou.rounding(dtype, want_y), "y")
    ou.check(mean, want_mean, ou.CHAIN * ou.U * x.double().abs().mean(-1), "mean")
    ou.check(rstd, want_rstd, ou.CHAIN * ou.U * want_rstd * (1 + (x.double().abs().mean(-1) * want_rstd)), "rstd")
    bare = api.flashrnn_layer_norm_fwd(x, weight, bias, eps=eps, dtype=dtype, save_for_backward=False)
    assert torch.equal(bare[0], y) and bare[1] is None and bare[2] is None
    dy = _normal(gen, *x.shape, dtype=dtype)
    dx, dw, db = api.flashrnn_layer_norm_bwd(dy, x, mean, rstd, weight, dtype=dx_dtype)
    want, bounds = ou.layer_norm_grad(dy, x, mean, rstd, weight)
    ou.check(dx, want[0], bounds[0] + ou.rounding(dx_dtype, want[0]), "dx")
    ou.check(dw, want[1], bounds[1], "dweight")
    ou.check(db, want[2], bounds[2], "dbias")
    again = api.flashrnn_layer_norm_bwd(dy, x, mean, rstd, weight, dtype=dx_dtype)
    assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), again)), "another result on the same inputs"
    alone = api.flashrnn_layer_norm_bwd(dy, x, mean, rstd, weight, dtype=dx_dtype, param_grads=False)
    assert torch.equal(alone[0], dx) and alone[1] is None and alone[2] is None


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_of_every_width(width, dtype):
    gen = _gen(width)
    w, b = (1 + 0.2 * torch.randn(width, generator=gen)).cuda(), _normal(gen, width)
    _check_norm(_rows(gen, 37, width, dtype), w, b, dtype, dtype, gen)


@pytest.mark.parametrize("rows", [1, 2, 3, 64, 65, 1023, 5000])
@pytest.mark.parametrize("width", [48, 77, 768, 3000])
def test_layer_norm_of_few_and_many_rows(rows, width):
    gen = _gen(rows)
    _check_norm(_rows(gen, rows, width, BF16), (1 + 0.2 * torch.randn(width, generator=gen)).cuda(), _normal(gen, width), BF16, BF16, gen)


@pytest.mark.parametrize("rows", [512, 513, 700])
@pytest.mark.parametrize("shape", [(9,), (40,), (100,), (260,), (520,), (1001,), (1500,), (2100,), (5000,), (9000,), (12001,), (5, 48), (3, 80), (257, 16), (16, 256)])
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_gradient_on_both_sides_of_one_launch(rows, shape, dtype):
    """dweight and dbias of few rows are added up beside dx, those of more from partial sums."""
    gen = _gen(rows + shape[0])
    wide = _normal(gen, rows, 2, *shape, dtype=dtype)
    _check_norm(wide[:, 1], (1 + 0.2 * torch.randn(*shape, generator=gen)).to(dtype).cuda(), _normal(gen, *shape, dtype=dtype), dtype, dtype, gen)


@pytest.mark.parametrize("x_dtype,dtype,dx_dtype,param_dtype", itertools.product(TYPES, TYPES, TYPES, TYPES))
@pytest.mark.parametrize("width", [96, 1111])
def test_layer_norm_of_every_mix_of_types(x_dtype, dtype, dx_dtype, param_dtype, width):
    gen = _gen(3)
    _check_norm(_rows(gen, 50, width, x_dtype), (1 + 0.2 * torch.randn(width, generator=gen)).to(param_dtype).cuda(), _normal(gen, width, dtype=param_dtype), dtype, dx_dtype, gen)


@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("heads", [0, 3])
def test_layer_norm_without_weight_or_bias(weight, bias, heads):
    gen = _gen(4)
    shape = (heads, 40) if heads else (40,)
    x = _normal(gen, 21, *shape)
    _check_norm(x, _normal(gen, *shape) if weight else None, _normal(gen, *shape) if bias else None, F32, BF16, gen)


@pytest.mark.parametrize("T,B,NH,D", [(1, 1, 1, 16), (1, 16, 4, 192), (5, 3, 3, 80), (7, 2, 12, 64), (33, 4, 8, 128), (3, 5, 48, 16), (2, 3, 2, 1024), (9, 1, 1, 768), (64, 16, 1, 2048), (3, 2, 257, 16), (50, 7, 5, 48)])
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_of_hidden_states_head_by_head(T, B, NH, D, dtype):
    """x = the hidden states inside the states of a call of the loop: dense but for the time axis."""
    gen = _gen(T + D)
    states = _normal(gen, T + 1, 4, B, NH, D)
    _check_norm(states[1:, 0], (1 + 0.2 * torch.randn(NH, D, generator=gen)).cuda(), _normal(gen, NH, D), dtype, dtype, gen)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [64, 100, 768])
def test_layer_norm_of_memory_that_starts_anywhere(dtype, width):
    gen = _gen(6)
    x, dy, w, b = (_odd_place(t) for t in (_rows(gen, 30, width, dtype), _normal(gen, 30, width, dtype=dtype), _normal(gen, width), _normal(gen, width)))
    y, mean, rstd = api.flashrnn_layer_norm_fwd(x, w, b, y=_odd_place(torch.empty_like(x)))
    want = api.flashrnn_layer_norm_fwd(x.clone(), w.clone(), b.clone())
    assert torch.equal(y, want[0]) and torch.equal(mean, want[1]) and torch.equal(rstd, want[2])
    out = tuple(_odd_place(t) for t in (torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)))
    api.flashrnn_layer_norm_bwd(dy, x, mean, rstd, w, out=out)
    assert all(torch.equal(a, b) for a, b in zip(out, api.flashrnn_layer_norm_bwd(dy.clone(), x.clone(), mean, rstd, w.clone())))


@pytest.mark.parametrize("view", ["last of three", "every other block", "expanded"])
def test_layer_norm_of_strided_inputs(view):
    gen = _gen(8)
    base = _normal(gen, 6, 3, 5, 72)
    x = {"last of three": base[:, 2], "every other block": base[::2], "expanded": base[0, 0, :1].expand(4, 72)}[view]
    _check_norm(x, _normal(gen, 72), _normal(gen, 72), F32, F32, gen)


@pytest.mark.parametrize("rows,width", [(1, 8), (40, 100), (40, 3000), (512, 768), (700, 768), (600, 9000), (5, 30000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_gradient_in_place(rows, width, dtype):
    """dx in dy's or in x's memory: the same bits, dweight and dbias too where the sums run in the same order."""
    gen = _gen(rows)
    x, dy, w = _rows(gen, rows, width, dtype), _normal(gen, rows, width, dtype=dtype), _normal(gen, width)
    _, mean, rstd = api.flashrnn_layer_norm_fwd(x, w)
    want = api.flashrnn_layer_norm_bwd(dy, x, mean, rstd, w)
    _, (_, wbound, bbound) = ou.layer_norm_grad(dy, x, mean, rstd, w)
    for own in range(2):
        a, b = dy.clone(), x.clone()
        dx, dw, db = api.flashrnn_layer_norm_bwd(a, b, mean, rstd, w, out=((b, a)[own], torch.empty_like(w), torch.empty_like(w)))
        assert torch.equal(dx, want[0])
        ou.check(dw, want[1], 2 * wbound, "dweight")
        ou.check(db, want[2], 2 * bbound, "dbias")


def test_layer_norm_of_no_rows():
    w, b = torch.ones(24, device="cuda"), torch.ones(24, device="cuda")
    x = torch.empty(0, 3, 24, device="cuda")
    y, mean, rstd = api.flashrnn_layer_norm_fwd(x, w, b)
    assert y.shape == x.shape and mean.shape == (0, 3)
    out = (torch.empty_like(x), torch.full_like(w, 5.0), torch.full_like(w, 5.0))
    dx, dw, db = api.flashrnn_layer_norm_bwd(x, x, mean, rstd, w, out=out)
    assert not dw.any() and not db.any()


@pytest.mark.parametrize("width", [40, 768, 3000, 20000])
def test_layer_norm_keeps_constant_and_offset_rows_exact(width):
    """Equal values give y = bias; a large offset costs the variance nothing but what the mean's own rounding does."""
    x = torch.full((3, width), 7.25, device="cuda")
    bias = torch.randn(width, device="cuda")
    y, mean, rstd = api.flashrnn_layer_norm_fwd(x, torch.ones(width, device="cuda"), bias, eps=1e-5)
    assert torch.equal(y, bias.expand(3, width)) and (mean == 7.25).all()
    gen = _gen(9)
    _check_norm(_normal(gen, 5, width) + 1000.0, None, None, F32, F32, gen)


@pytest.mark.parametrize("width", [40, 3000])
def test_layer_norm_keeps_nan_and_infinities_in_their_row(width):
    x = torch.randn(6, width, device="cuda")
    clean = api.flashrnn_layer_norm_fwd(x)[0].clone()
    x[1, 3], x[4, 0] = float("nan"), float("inf")
    y, mean, rstd = api.flashrnn_layer_norm_fwd(x)
    assert y[1].isnan().all() and y[4].isnan().all()
    for r in (0, 2, 3, 5):
        assert torch.equal(y[r], clean[r])


def test_layer_norm_beyond_32_bit_offsets():
    base = torch.empty((1 << 31) + 4096, dtype=BF16, device="cuda")
    x = base.as_strided((2, 64), ((1 << 31) + 8, 1))
    x.copy_(torch.randn(2, 64))
    _check_norm(x, None, None, F32, F32, _gen(1))
    del base, x
    rows = (1 << 31) // 8 + 5
    x = torch.randn(64, 8, device="cuda", dtype=BF16).repeat(rows // 64 + 1, 1)[:rows]
    y = api.flashrnn_layer_norm_fwd(x, save_for_backward=False)[0]
    assert torch.equal(y[-128:], api.flashrnn_layer_norm_fwd(x[-128:].clone(), save_for_backward=False)[0])


@pytest.mark.parametrize("heads,width", [(0, 12), (0, 700), (2, 16)])
def test_layer_norm_gradient_against_differences(heads, width):
    """Central differences of the plain forward pass in 64 bits; a step of h = 1e-4 leaves h^2 times third derivatives of order rstd^3 = O(1)."""
    gen = _gen(width)
    params = (heads, width) if heads else (width,)
    x, dy, w, b = (torch.randn(*s, generator=gen, dtype=torch.float64).float() for s in ((3, *params), (3, *params), params, params))
    _, mean, rstd = api.flashrnn_layer_norm_fwd(x.cuda(), w.cuda(), b.cuda())
    got = api.flashrnn_layer_norm_bwd(dy.cuda(), x.cuda(), mean, rstd, w.cuda())
    f = lambda x, w, b: float((ou.layer_norm(x, w, b, 1e-5)[0] * dy.double()).sum())
    args = [t.double() for t in (x, w, b)]
    for k, (a, g) in enumerate(zip(args, got)):
        flat = a.view(-1)
        for i in torch.randperm(flat.numel(), generator=gen)[:25].tolist():
            v, h = flat[i].item(), 1e-4
            flat[i] = v + h
            up = f(*args)
            flat[i] = v - h
            down = f(*args)
            flat[i] = v
            assert abs((up - down) / (2 * h) - g.reshape(-1)[i].item()) < 2e-5 * (1 + float(dy.abs().sum()) / width), (k, i)


# ---- cross entropy ---------------------------------------------------------------------------------------------------------------------------------
CLASSES = [1, 2, 5, 30, 64, 100, 256, 257, 1000, 2047, 2048, 4100, 8192, 10001, 16384, 32000, 50304, 65537, 100000, 131072, 150001]


def _logits(gen, rows, classes, dtype):
    return (torch.randn(rows, classes, generator=gen) * 3).to(dtype).cuda()


def _check_loss(logits, targets, dloss=None, scale=0.25, **kw):
    lse = torch.empty(logits.shape[0], device="cuda")
    (want_loss, want_lse, want_grad), (bl, bs, bg) = ou.cross_entropy(logits, targets, dloss, scale)
    loss, grad = api.flashrnn_cross_entropy(logits, targets, dloss, scale, lse=lse, **kw)
    assert grad.dtype == logits.dtype
    ou.check(loss, want_loss, bl, "loss")
    ou.check(lse, want_lse, bs, "lse")
    ou.check(grad, want_grad, bg + ou.rounding(grad.dtype, want_grad), "dlogits")
    return loss, grad


@pytest.mark.parametrize("classes", CLASSES)
@pytest.mark.parametrize("dtype", TYPES)
def test_cross_entropy_of_every_number_of_classes(classes, dtype):
    gen = _gen(classes)
    logits, targets = _logits(gen, 9, classes, dtype), torch.randint(classes, (9,), generator=gen).cuda()
    targets[0], targets[1], targets[2] = 0, classes - 1, -100
    loss, grad = _check_loss(logits, targets)
    alone, none = api.flashrnn_cross_entropy(logits, targets, gradient=False)
    assert none is None and torch.equal(alone, loss)
    kept = logits.clone()
    _check_in_place = api.flashrnn_cross_entropy(kept, targets, None, 0.25, dlogits=kept)
    assert torch.equal(_check_in_place[0], loss) and torch.equal(kept, grad)


@pytest.mark.parametrize("rows", [1, 2, 63, 300, 3000])
@pytest.mark.parametrize("classes", [33, 1000, 12000])
@pytest.mark.parametrize("index", [torch.int64, torch.int32])
def test_cross_entropy_of_few_and_many_rows(rows, classes, index):
    gen = _gen(rows)
    targets = torch.randint(-1, classes + 1, (rows,), generator=gen).to(index).cuda()
    targets[0] = torch.iinfo(index).min
    _check_loss(_logits(gen, rows, classes, BF16), targets, torch.randn(rows, generator=gen).cuda())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [61, 1024, 9000, 40000])
def test_cross_entropy_of_strided_rows(classes, dtype):
    """Logits in the columns of a wider matrix, the gradient into another one; what lies beside them stays."""
    gen = _gen(classes)
    wide, to = _logits(gen, 7, classes + 13, dtype), torch.full((7, classes + 6), 9.0, dtype=dtype, device="cuda")
    logits, targets = wide[:, 5:5 + classes], torch.randint(classes, (7,), generator=gen).cuda()
    _check_loss(logits, targets, dlogits=to[:, 3:3 + classes])
    assert (to[:, :3] == 9).all() and (to[:, 3 + classes:] == 9).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [40, 1000, 9000, 140000])
def test_cross_entropy_with_masked_classes(classes, dtype):
    gen = _gen(classes)
    logits, targets = _logits(gen, 8, classes, dtype), torch.randint(classes // 2, (8,), generator=gen).cuda()
    logits[:, classes // 2:] = float("-inf")                   # masked classes, targets among the others
    logits[1, :classes // 2] = torch.finfo(dtype).min          # the type's lowest value is a value: all that are left share the probability
    logits[2] = float("-inf")                                  # nothing left
    logits[3, :] = float("-inf")
    logits[3, targets[3]] = -5.0                               # one class left, the target: loss 0
    logits[4, targets[4]] = float("-inf")                      # the target itself is masked: loss inf, the gradient of the others as ever
    logits[5] = torch.finfo(dtype).max
    targets[6] = -1
    logits[6] = float("nan")                                   # ignored, whatever it holds: loss 0, gradient 0
    loss, grad = _check_loss_ignoring(logits, targets, 6)
    assert loss[2].isinf() and not grad[2].any() and loss[3] == 0 and loss[4].isinf() and loss[6] == 0 and not grad[6].any()


def _check_loss_ignoring(logits, targets, row):
    loss, grad = api.flashrnn_cross_entropy(logits, targets, None, 0.25)
    rest = [r for r in range(len(targets)) if r != row]
    want, bounds = ou.cross_entropy(logits[rest], targets[rest], None, 0.25)
    ou.check(loss[rest], want[0], bounds[0], "loss")
    ou.check(grad[rest], want[2], bounds[2] + ou.rounding(grad.dtype, want[2]), "dlogits")
    return loss, grad


@pytest.mark.parametrize("classes", [40, 9000])
def test_cross_entropy_keeps_nan_and_infinities_in_their_row(classes):
    gen = _gen(1)
    logits, targets = _logits(gen, 5, classes, F32), torch.randint(classes, (5,), generator=gen).cuda()
    clean = [t.clone() for t in api.flashrnn_cross_entropy(logits, targets)]
    logits[1, 7], logits[3, 2] = float("nan"), float("inf")
    loss, grad = api.flashrnn_cross_entropy(logits, targets)
    for r in (1, 3):
        assert loss[r].isnan() and grad[r].isnan().all()
    logits[1] = float("nan")
    loss, grad = api.flashrnn_cross_entropy(logits, targets)
    assert loss[1].isnan() and grad[1].isnan().all()
    for r in (0, 2, 4):
        assert torch.equal(loss[r], clean[0][r]) and torch.equal(grad[r], clean[1][r])


def test_cross_entropy_of_no_rows():
    loss, grad = api.flashrnn_cross_entropy(torch.empty(0, 30, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"))
    assert loss.shape == (0,) and grad.shape == (0, 30)


def test_cross_entropy_beyond_32_bit_offsets():
    classes = 50304
    rows = (1 << 32) // classes // 2 + 40
    gen = _gen(2)
    last = _logits(gen, 16, classes, BF16)
    logits = torch.zeros(rows, classes, dtype=BF16, device="cuda")
    logits[-16:] = last
    targets = torch.arange(rows, device="cuda") % classes
    loss, grad = api.flashrnn_cross_entropy(logits, targets, dlogits=logits)
    want = api.flashrnn_cross_entropy(last, targets[-16:].clone())
    assert torch.equal(loss[-16:], want[0]) and torch.equal(grad[-16:], want[1])


def test_cross_entropy_gradient_against_differences():
    gen = _gen(3)
    x, t, dl = torch.randn(4, 11, generator=gen).double(), torch.tensor([0, 10, -1, 5]), torch.randn(4, generator=gen)
    grad = api.flashrnn_cross_entropy(x.float().cuda(), t.cuda(), dl.cuda(), 0.7)[1]
    f = lambda: float((ou.cross_entropy(x, t, None, 1.0)[0][0] * dl.double()).sum() * 0.7)
    x = x.float().double()
    for i in range(4):
        for j in range(11):
            v, h = x[i, j].item(), 1e-4
            x[i, j] = v + h
            up = f()
            x[i, j] = v - h
            down = f()
            x[i, j] = v
            assert abs((up - down) / (2 * h) - grad[i, j].item()) < 2e-6


# ---- clipping ----------------------------------------------------------------------------------------------------------------------------------
def _grads(gen, sizes, types, scale=1.0):
    return [_normal(gen, *(s if isinstance(s, tuple) else (s,)), dtype=t, scale=scale) for s, t in zip(sizes, itertools.cycle(types))]


def _check_clip(grads, max_norm, in_place):
    want = sum(float((g.double() ** 2).sum()) for g in grads) ** 0.5
    factor = 1.0 if want <= max_norm else max_norm / want
    given = [g.clone() for g in grads]
    out = given if in_place else [torch.full_like(g, 7.0) for g in grads]
    norm = api.flashrnn_grad_clip(given, max_norm, out=None if in_place else out)
    assert abs(norm.item() - want) <= 2 * ou.U * want
    for i, (g, o) in enumerate(zip(grads, out)):
        scaled = g.double() * factor
        if factor == 1.0:
            assert torch.equal(o, g)
        else:
            ou.check(o, scaled, 4 * ou.U * scaled.abs() + ou.rounding(g.dtype, scaled) + (2.0 ** -133 if g.dtype == BF16 else 2.0 ** -149), f"tensor {i}")
        if not in_place:
            assert torch.equal(given[i], g)


@pytest.mark.parametrize("sizes", [[1], [5], [8192], [8193, 1], [0, 3, 0], [100000], [1, 2, 3, 4, 5, 6, 7, 8, 9], [(300, 70), 64, (3, 5, 7)], [33] * 127, [33] * 128, [17] * 129, [9] * 1000, [3_000_001, 11]])
@pytest.mark.parametrize("types", [[F32], [BF16], [F32, BF16]])
@pytest.mark.parametrize("in_place", [False, True])
def test_clip(sizes, types, in_place):
    gen = _gen(len(sizes))
    grads = _grads(gen, sizes, types)
    _check_clip(grads, 0.5, in_place)
    _check_clip(grads, 1e6, in_place)


@pytest.mark.parametrize("in_place", [False, True])
def test_clip_of_memory_that_starts_anywhere(in_place):
    gen = _gen(1)
    flat = _normal(gen, 20000)
    half = _normal(gen, 20000).to(BF16)
    grads = [flat[1:4], flat[5:5], flat[7:9000], flat[9001:20000], half[3:4], half[5:11111], half[11114:]]
    want = sum(float((g.double() ** 2).sum()) for g in grads) ** 0.5
    keep = [flat.clone(), half.clone()]
    norm = api.flashrnn_grad_clip(grads, 0.25, out=None if in_place else [torch.empty_like(g) for g in grads])
    assert abs(norm.item() - want) <= 2 * ou.U * want
    if not in_place:
        assert torch.equal(flat, keep[0]) and torch.equal(half, keep[1])
    else:
        inside = torch.zeros(20000, dtype=torch.bool)
        for a, b in ((1, 4), (7, 9000), (9001, 20000)):
            inside[a:b] = True
        assert torch.equal(flat.cpu()[~inside], keep[0].cpu()[~inside])
        ou.check(flat[7:9000], keep[0][7:9000].double() * (0.25 / want), 4 * ou.U * keep[0][7:9000].double().abs() * (0.25 / want), "flat")


def test_clip_norm_alone_and_of_nothing():
    gen = _gen(2)
    grads = _grads(gen, [1000, 77], [F32, BF16])
    keep = [g.clone() for g in grads]
    norm = api.flashrnn_grad_clip(grads, float("inf"))
    want = sum(float((g.double() ** 2).sum()) for g in grads) ** 0.5
    assert abs(norm.item() - want) <= 2 * ou.U * want and all(torch.equal(a, b) for a, b in zip(grads, keep))
    zero = torch.full((1,), 5.0, device="cuda")
    assert api.flashrnn_grad_clip([], 1.0, norm=zero).item() == 0.0
    zeros = torch.zeros(300, device="cuda")
    assert api.flashrnn_grad_clip([zeros], 0.0).item() == 0.0 and not zeros.any()
    ones = torch.ones(300, device="cuda")
    api.flashrnn_grad_clip([ones], 0.0)
    assert not ones.any()


def test_clip_of_values_whose_squares_leave_float32():
    for scale in (1e30, 1e-30):
        grads = [torch.full((5000,), scale, device="cuda"), torch.full((7,), -scale, device="cuda", dtype=BF16)]
        want = sum(float((g.double() ** 2).sum()) for g in grads) ** 0.5
        norm = api.flashrnn_grad_clip(grads, scale)
        assert abs(norm.item() - want) <= 2 * ou.U * want
        assert abs(grads[0][0].item() - scale * scale / want) <= 4 * ou.U * scale


def test_clip_of_nan_and_infinity():
    a = torch.ones(10, device="cuda")
    b = torch.tensor([1.0, float("nan")], device="cuda")
    assert api.flashrnn_grad_clip([a, b], 1.0).isnan().all() and a.isnan().all() and b.isnan().all()
    a = torch.ones(10, device="cuda")
    b = torch.tensor([1.0, float("inf")], device="cuda")
    assert api.flashrnn_grad_clip([a, b], 1.0).isinf().all() and not a.any() and b[1].isnan()


# ---- streams and graphs ---------------------------------------------------------------------------------------------------------------------------
def _all_of_them(s):
    """One call of each operator on the buffers of s."""
    api.flashrnn_embedding_fwd(s["table"], s["tokens"], out=s["x"])
    api.flashrnn_layer_norm_fwd(s["x"], s["weight"], s["bias"], y=s["y"], mean=s["mean"], rstd=s["rstd"])
    api.flashrnn_cross_entropy(s["y"], s["tokens"], loss=s["loss"], dlogits=s["dy"])
    api.flashrnn_layer_norm_bwd(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"], out=(s["dx"], s["dweight"], s["dbias"]), workspace=s["ws_norm"])
    api.flashrnn_embedding_bwd(s["tokens"], s["dx"], len(s["table"]), dtable=s["dtable"], workspace=s["ws_embed"])
    api.flashrnn_grad_clip([s["dtable"], s["dweight"], s["dbias"]], 0.1, norm=s["norm"], workspace=s["ws_clip"])
    return [s[k] for k in ("x", "y", "loss", "dy", "dx", "dweight", "dbias", "dtable", "norm")]


def _buffers(seed, n=300, vocab=500, width=64):
    gen = _gen(seed)
    s = {"table": _normal(gen, vocab, width), "tokens": _tokens(gen, n, vocab, torch.int64), "weight": _normal(gen, width), "bias": _normal(gen, width)}
    for k in ("x", "y", "dx", "dy"):
        s[k] = torch.zeros(n, width, device="cuda")
    for k, shape in (("mean", n), ("rstd", n), ("loss", n), ("dweight", width), ("dbias", width), ("norm", 1)):
        s[k] = torch.zeros(shape, device="cuda")
    s["dtable"] = torch.zeros(vocab, width, device="cuda")
    for k in ("ws_norm", "ws_embed", "ws_clip"):
        s[k] = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    return s


def test_operators_run_on_the_current_stream_and_on_the_one_passed():
    s = _buffers(1)
    want = [t.clone() for t in _all_of_them(s)]
    late, stream = s["table"].clone(), torch.cuda.Stream()
    s["table"].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)   # (clocks: ten milliseconds)
        s["table"].copy_(late)
        got = _all_of_them(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out = torch.zeros_like(want[0])
    torch.cuda.synchronize()
    api.flashrnn_embedding_fwd(s["table"], s["tokens"], out=out, stream=stream)
    stream.synchronize()
    assert torch.equal(out, want[0])


def test_what_a_call_on_another_stream_allocates_belongs_to_that_stream():
    """Behind a wait on the stream passed, while the current stream takes and fills all memory that the allocator hands out again."""
    s = _buffers(1)
    want = [t.clone() for t in _all_of_them(s)]
    stream = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            torch.cuda._sleep(10_000_000)
        x = api.flashrnn_embedding_fwd(s["table"], s["tokens"], stream=stream)
        y, mean, rstd = api.flashrnn_layer_norm_fwd(x, s["weight"], s["bias"], stream=stream)
        loss, dy = api.flashrnn_cross_entropy(y, s["tokens"], stream=stream)
        dx, dweight, dbias = api.flashrnn_layer_norm_bwd(dy, x, mean, rstd, s["weight"], stream=stream)
        dtable = api.flashrnn_embedding_bwd(s["tokens"], dx, len(s["table"]), stream=stream)
        norm = api.flashrnn_grad_clip([dtable, dweight, dbias], 0.1, stream=stream)
        junk = [torch.full((1 << k,), 123, dtype=torch.uint8, device="cuda") for k in range(9, 23)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((x, y, loss, dy, dx, dweight, dbias, dtable, norm), want)), len(junk)


def test_operators_in_a_graph():
    """Captured once and replayed on new inputs, with eager work between the replays."""
    s = _buffers(2)
    _all_of_them(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _all_of_them(s)
    for seed in (3, 4, 5):
        new = _buffers(seed)
        for k in ("table", "tokens", "weight", "bias"):
            s[k].copy_(new[k])
        graph.replay()
        got = [s[k].clone() for k in ("x", "y", "loss", "dy", "dx", "dweight", "dbias", "dtable", "norm")]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, _all_of_them(new)))


# ---- the native part of the binding ------------------------------------------------------------------------------------------------------------
def _calls():
    """Calls with every buffer passed, so that the native module may take them, and changes to them that it hands back."""
    gen = _gen(11)
    w, b = _normal(gen, 5, 16), _normal(gen, 5, 16)
    states = _normal(gen, 4, 2, 3, 5, 16)
    lead = (3, 3, 5)
    tokens, table, logits = torch.tensor([[1, 5, -1], [9, 1, 3]]).cuda(), _normal(gen, 9, 16), _normal(gen, 6, 9)
    z = lambda *shape, dtype=F32: torch.zeros(shape, dtype=dtype, device="cuda")
    h, t6 = states[1:, 0], tokens.reshape(-1)
    norm = dict(x=h, weight=w, bias=b, y=z(3, 3, 5, 16, dtype=BF16), mean=z(*lead), rstd=z(*lead))
    _, mean, rstd = api.flashrnn_layer_norm_fwd(h, w, b)
    grad = dict(dy=_normal(gen, 3, 3, 5, 16, dtype=BF16), x=h, mean=mean, rstd=rstd, weight=w, out=(z(3, 3, 5, 16, dtype=BF16), z(5, 16), z(5, 16)))
    loss = dict(logits=logits, targets=t6, dloss=_normal(gen, 6), grad_scale=0.5, loss=z(6), lse=z(6), dlogits=z(6, 9))
    wide = _normal(gen, 6, 14)
    embed = dict(table=table, tokens=tokens, scale=2.0, out=z(2, 3, 16))
    dembed = dict(tokens=tokens, dout=_normal(gen, 2, 3, 16), vocab=9, scale=2, dtable=z(9, 16))
    clip = dict(grads=[_normal(gen, 7), _normal(gen, 3, 4, dtype=BF16)], max_norm=0.5, out=[z(7), z(3, 4, dtype=BF16)], norm=z(1))
    strided = lambda t: t.transpose(0, -1).contiguous().transpose(0, -1)
    return [
        (api.flashrnn_embedding_fwd, embed, [dict(out=z(2, 3, 16, dtype=BF16)), dict(tokens=tokens.int()), dict(table=torch.nn.Parameter(table)), dict(scale=3), dict(out=None), dict(scale=True), dict(scale=torch.tensor(2.0))],
         [dict(tokens=tokens.float()), dict(tokens=tokens.t()), dict(out=z(3, 2, 16)), dict(out=z(2, 3, 15)), dict(table=strided(table)), dict(table=table.double()), dict(table=table[0]),
          dict(tokens=tokens.cpu()), dict(table=table[:0])]),
        (api.flashrnn_embedding_bwd, dembed, [dict(accumulate=True), dict(tokens=tokens.int()), dict(workspace=z(100000)), dict(dtable=None), dict(vocab=torch.tensor(9))],
         [dict(vocab=8), dict(vocab=2 ** 70), dict(vocab=-1), dict(dtable=z(9, 15)), dict(dout=z(3, 2, 16)), dict(workspace=z(1)), dict(dtable=z(9, 16, dtype=BF16)), dict(dout=dembed["dout"].double())]),
        (api.flashrnn_layer_norm_fwd, norm, [dict(weight=None), dict(bias=None), dict(weight=None, bias=None), dict(x=h.contiguous()), dict(save_for_backward=False), dict(eps=1), dict(y=None), dict(mean=None),
                                             dict(x=states[::2, 1], y=z(2, 3, 5, 16), mean=z(2, 3, 5), rstd=z(2, 3, 5))],
         [dict(x=strided(h)), dict(weight=w[:4]), dict(bias=b.bfloat16()), dict(weight=w[0], bias=b), dict(y=z(3, 3, 5, 15)), dict(mean=z(3, 3)), dict(eps=-1.0), dict(eps=float("nan")),
          dict(x=h.half()), dict(weight=w.t()), dict(x=h.cpu()), dict(rstd=z(*lead, dtype=BF16))]),
        (api.flashrnn_layer_norm_bwd, grad, [dict(weight=None, out=(z(3, 3, 5, 16), z(16), z(16))), dict(param_grads=False), dict(out=(z(3, 3, 5, 16), None, z(5, 16))), dict(workspace=z(100000)), dict(out=None),
                                             dict(x=h.contiguous())],
         [dict(dy=grad["dy"][:2]), dict(mean=mean[:2]), dict(rstd=rstd.double()), dict(workspace=z(1)), dict(out=(z(3, 3, 5, 16), z(16), z(5, 16))), dict(weight=w[:4]), dict(x=strided(h))]),
        (api.flashrnn_cross_entropy, loss, [dict(dloss=None), dict(lse=None), dict(gradient=False), dict(dlogits=None), dict(targets=t6.int()), dict(logits=wide[:, 2:11]), dict(dlogits=z(6, 12)[:, 1:10]), dict(grad_scale=2)],
         [dict(targets=t6[:5]), dict(targets=t6.float()), dict(logits=strided(logits)), dict(dlogits=z(6, 9, dtype=BF16)), dict(dlogits=z(1, 9).expand(6, 9)), dict(loss=z(5)), dict(lse=z(6, dtype=BF16)),
          dict(dloss=z(6).double()), dict(logits=logits[0]), dict(logits=logits.half())]),
        (api.flashrnn_grad_clip, clip, [dict(max_norm=1e9), dict(max_norm=float("inf")), dict(grads=tuple(clip["grads"])), dict(workspace=z(100000)), dict(max_norm=1), dict(norm=None),
                                        dict(grads=[clip["out"][0], clip["out"][1]], out=None)],
         [dict(out=clip["out"][:1]), dict(out=[clip["out"][0], z(3, 4)]), dict(grads=[z(7), z(3, 4).t()]), dict(grads=[z(7), z(3, 4).double()]), dict(norm=z(2)), dict(max_norm=-1.0), dict(workspace=z(1)),
          dict(max_norm=float("nan"))]),
    ]


def _outcome(fn, kw):
    """What a call returns and leaves in its buffers, or what it raises."""
    flat = lambda v: [v] if torch.is_tensor(v) else [t for x in v for t in flat(x)] if isinstance(v, (list, tuple)) else []
    kw = {k: (v.clone() if torch.is_tensor(v) and k in ("out", "dtable", "y", "mean", "rstd", "loss", "lse", "dlogits", "norm") and v.is_contiguous() and fn is not api.flashrnn_layer_norm_bwd else v)
          for k, v in kw.items()}
    if fn is api.flashrnn_grad_clip and kw["out"] is None:
        kw["grads"] = [g.clone() for g in kw["grads"]]
    try:
        result = fn(**kw)
    except Exception as e:
        return type(e).__name__, str(e)
    torch.cuda.synchronize()
    return [t.clone().cpu() for t in flat(result) + flat([kw.get(k) for k in ("out", "lse", "grads") if kw.get(k) is not None])]


def test_native_calls_and_calls_through_python_give_and_refuse_the_same(monkeypatch):
    api.lib()
    assert api._native is not None
    results = {}
    for native in (True, False):
        if not native:
            monkeypatch.setattr(api, "_native", None)
        results[native] = []
        for fn, base, fine, refused in _calls():
            for i, change in enumerate([{}] + fine + refused):
                got = _outcome(fn, dict(base, **change))
                assert isinstance(got, tuple) == (i > len(fine)), (fn.__name__, change, got)
                results[native].append((fn.__name__, i, got))
    for (name, i, a), (_, _, b) in zip(results[True], results[False]):
        assert type(a) is type(b), (name, i, a, b)
        assert a == b if isinstance(a, tuple) else len(a) == len(b) and all(torch.equal(p, q) for p, q in zip(a, b)), (name, i)


def test_plain_calls_are_made_by_the_native_module():
    api.lib()
    (_, embed, *_), (_, dembed, *_), (_, norm, *_), (_, grad, *_), (_, loss, *_), (_, clip, *_) = _calls()
    n = api._native
    assert n.embedding_fwd(embed["table"], embed["tokens"], 2.0, embed["out"]) == 0
    assert n.embedding_bwd(dembed["tokens"], dembed["dout"], 9, 2, dembed["dtable"], False, None) == 0
    assert n.layer_norm_fwd(norm["x"], norm["weight"], norm["bias"], 1e-5, norm["y"], norm["mean"], norm["rstd"]) == 0
    assert n.layer_norm_bwd(grad["dy"], grad["x"], grad["mean"], grad["rstd"], grad["weight"], *grad["out"], None) == 0
    assert n.cross_entropy(loss["logits"], loss["targets"], None, 0.5, loss["loss"], None, loss["dlogits"]) == 0
    assert n.grad_clip(clip["grads"], 0.5, clip["out"], clip["norm"], None, True) == 0
    for f in (n.embedding_fwd, n.embedding_bwd, n.layer_norm_fwd, n.layer_norm_bwd, n.cross_entropy, n.grad_clip):
        assert f() == 1 and f(*range(9)) == 1
    torch.cuda.synchronize()
