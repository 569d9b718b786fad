"""The cases that the operators around a recurrent layer are measured on: what a language model does before and after the time-step loop.

Embedding lookup and its gradient, layer norm (over a row, or head by head over the states that the loop leaves) and its gradient, cross
entropy with its gradient, and clipping by the global gradient norm.  Each case is one call of a public entry point on buffers that a user's
program has in hand; where `own` is false the same is computed from elementary torch operations in float32, rounded once at the end.

op  "embed"       out[i] = scale * table[token i]; a token outside the vocabulary (padding) gives zeros
    "embed_grad"  its gradient: one float32 row per word of the vocabulary
    "norm"        layer norm; heads > 0: head by head, x = the hidden states inside states[T+1,S,B,NH,D] (float32)
    "norm_grad"   its gradient, from the saved statistics: dx, dweight, dbias
    "loss"        cross entropy per row and the gradient of its mean; targets outside the classes are ignored
    "clip"        the norm over all gradients of a stack of layers, and the gradients scaled down to it
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-5
PADDING = 0.03     # share of tokens that are padding, and of targets that are ignored
STATES = 4         # states of the cell whose hidden states are normalised (sLSTM)


def _embed(name, op, tokens, vocab, width, dtype):
    return {"name": name, "op": op, "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype}


def _norm(name, op, steps, rows, heads, width, xdtype, dtype):
    return {"name": name, "op": op, "steps": steps, "rows": rows, "heads": heads, "width": width, "xdtype": xdtype, "dtype": dtype}


def _loss(name, rows, classes, dtype):
    return {"name": name, "op": "loss", "rows": rows, "classes": classes, "dtype": dtype}


def _clip(name, layers, heads, width, vocab, dtype, packed):
    return {"name": name, "op": "clip", "layers": layers, "heads": heads, "width": width, "vocab": vocab, "dtype": dtype, "packed": packed}


def listed():
    return [
        # token-by-token generation for 16 sequences: one embedding row each, the layer's output normalised head by head
        _embed("embed_b16_768", "embed", 16, 32000, 768, "bf16"),
        _norm("norm_heads_4x192_b16_t1", "norm", 1, 16, 4, 192, "f32", "bf16"),
        # the loss of a small byte model, float32
        _loss("loss_16x256_f32", 16, 256, "f32"),
        # gradients of one small layer and its tables (gradient checks, small models)
        _clip("clip_1x64_1_layer_f32", 1, 1, 64, 256, "f32", False),
        # the embedding's gradient of one ordinary step: 16 sequences of 256 tokens
        _embed("embed_grad_4096_768", "embed_grad", 4096, 32000, 768, "bf16"),
        # odd width, float32
        _norm("norm_grad_3663_1111_f32", "norm_grad", 333, 11, 0, 1111, "f32", "f32"),
        # pre-norm of an ordinary layer: 16 sequences of 1024 tokens
        _norm("norm_grad_16384_768", "norm_grad", 1024, 16, 0, 768, "bf16", "bf16"),
        # long context, wide layer: 32 sequences of 2048 tokens, eight heads of 256 units
        _embed("embed_65536_2048", "embed", 65536, 50304, 2048, "bf16"),
        _embed("embed_grad_65536_2048", "embed_grad", 65536, 50304, 2048, "bf16"),
        _norm("norm_heads_8x256_b32_t2048", "norm", 2048, 32, 8, 256, "f32", "bf16"),
        # the loss of 16 sequences of 1024 tokens over a full vocabulary
        _loss("loss_16384x50304", 16384, 50304, "bf16"),
        # gradients of twelve wide layers with their tables, packed one behind the other in flat buffers
        _clip("clip_8x256_12_layers_f32", 12, 8, 256, 50304, "f32", True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: one token to 65536, rows of 16 to 8192 values, odd widths among them, heads of 16 to 1024 units, vocabularies and
    classes from 30 to 131072, one layer to 48; at most as much work as the largest listed case."""
    most = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "loss", "clip"])
        dtype = "bf16" if rng.random() < 0.65 else "f32"
        if op in ("embed", "embed_grad"):
            width = _log_int(rng, 16, 4096) if rng.random() < 0.3 else 8 * _log_int(rng, 2, 512)
            case = _embed("", op, _log_int(rng, 1, 65536), _log_int(rng, 30, 131072), width, dtype)
        elif op in ("norm", "norm_grad"):
            heads = rng.choice([0, 0, _log_int(rng, 1, 48)])
            if heads:
                width, xdtype = 16 * _log_int(rng, 1, 64), "f32"
            else:
                width = _log_int(rng, 16, 8192) if rng.random() < 0.4 else 8 * _log_int(rng, 2, 1024)
                xdtype = "f32" if dtype == "f32" or rng.random() < 0.3 else "bf16"
            if max(1, heads) * width > 8192:
                continue
            case = _norm("", op, _log_int(rng, 1, 2048), _log_int(rng, 1, 64), heads, width, xdtype, dtype)
        elif op == "loss":
            case = _loss("", _log_int(rng, 1, 32768), _log_int(rng, 30, 131072), dtype)
        else:
            case = _clip("", _log_int(rng, 1, 48), _log_int(rng, 1, 16), 16 * _log_int(rng, 1, 32), _log_int(rng, 30, 131072),
                         rng.choice(["f32", "bf16", "mixed"]), rng.random() < 0.5)
            if case["heads"] * case["width"] > 4096:
                continue
        del case["name"]
        if work(case)["bytes"] <= most:
            return case


def _layer_tensors(case):
    """(shape, dtype) of every gradient of the stack: the table, then per layer the input projection, the recurrent weights (float32, as the
    time-step loop returns them), the bias and the two vectors of a layer norm."""
    NH, D = case["heads"], case["width"]
    H = NH * D
    io = "f32" if case["dtype"] == "f32" else "bf16"
    loop = "bf16" if case["dtype"] == "bf16" else "f32"
    out = [((case["vocab"], H), io)]
    for _ in range(case["layers"]):
        out += [((4 * H, H), io), ((NH, D, 4, D), loop), ((NH, 4, D), loop), ((H,), loop), ((H,), loop)]
    return out


def _places(case):
    """Offset of every gradient in the flat buffer of its type, and the buffers' lengths; packed: one behind the other, else on 256 bytes."""
    at, end = [], {"f32": 0, "bf16": 0}
    for shape, dtype in _layer_tensors(case):
        step = 1 if case["packed"] else 256 // SIZE[dtype]
        first = -(-end[dtype] // step) * step
        at.append(first)
        end[dtype] = first + math.prod(shape)
    return at, end


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, st = case["op"], {"case": case}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    def indices(count, kinds):
        """Words of a text: frequency falls with the rank (about as 1 / rank), a few places are padding (-1)."""
        weight = torch.arange(kinds, device="cuda", dtype=torch.float64).add_(2.7).reciprocal_().cumsum_(0)
        picks = torch.searchsorted(weight, uniform(count).double() * weight[-1]).clamp_(max=kinds - 1)
        return torch.where(uniform(count) < PADDING, -1, picks)

    if op in ("embed", "embed_grad"):
        N, V, H, io = case["tokens"], case["vocab"], case["width"], DTYPES[case["dtype"]]
        st["tokens"], st["scale"] = indices(N, V), H ** 0.5
        if op == "embed":
            st["table"] = (normal(V, H) * H ** -0.5).to(io)
            st["out"] = torch.empty((N, H), dtype=io, device="cuda")
        else:
            st["dout"] = (normal(N, H) * 0.01).to(io)
            st["out"] = torch.empty((V, H), dtype=torch.float32, device="cuda")
    elif op in ("norm", "norm_grad"):
        T, B, NH, D, io = case["steps"], case["rows"], case["heads"], case["width"], DTYPES[case["dtype"]]
        if NH:   # hidden states of a loop: slots 1 to T of state 0
            st["x"] = torch.tanh(normal(T + 1, STATES, B, NH, D))[1:, 0]
        else:    # a residual stream: rows of different scale and offset
            st["x"] = ((normal(T, B, D) + normal(T, B, 1)) * torch.exp(normal(T, B, 1) * 0.5)).to(DTYPES[case["xdtype"]])
        params = (NH, D) if NH else (D,)
        st["weight"], st["bias"] = (1 + 0.1 * normal(*params)), 0.1 * normal(*params)
        lead = tuple(st["x"].shape[:-1])
        if op == "norm":
            st["y"], st["mean"], st["rstd"] = torch.empty(tuple(st["x"].shape), dtype=io, device="cuda"), torch.empty(lead, device="cuda"), torch.empty(lead, device="cuda")
        else:
            x = st["x"].float()
            st["mean"] = x.mean(-1)
            st["rstd"] = (x - st["mean"][..., None]).square().mean(-1).add(EPS).rsqrt()
            st["dy"] = (normal(*st["x"].shape) * 0.1).to(io)
            st["out"] = (torch.empty_like(st["dy"]), torch.empty(params, device="cuda"), torch.empty(params, device="cuda"))
    elif op == "loss":
        N, V, io = case["rows"], case["classes"], DTYPES[case["dtype"]]
        st["targets"] = indices(N, V)
        logits = torch.empty((N, V), dtype=io, device="cuda")
        step = max(1, (1 << 28) // V)
        for i in range(0, N, step):   # (the float32 draw of a whole batch would be twice its size)
            logits[i:i + step] = normal(min(step, N - i), V) * 2
        seen = st["targets"] >= 0
        logits[seen.nonzero()[:, 0], st["targets"][seen]] += 6     # a model that has learned something
        if V % 64 > 1:
            logits[:, V - 1] = float("-inf")                       # a class that only fills up the vocabulary
            st["targets"][st["targets"] == V - 1] = 0
        st["logits"], st["grad_scale"] = logits, 1.0 / N
        st["out"] = (torch.empty(N, device="cuda"), torch.empty_like(logits))
    else:
        at, end = _places(case)
        flat = {d: torch.zeros(n, dtype=DTYPES[d], device="cuda") for d, n in end.items() if n}
        st["flat"] = {d: torch.zeros_like(f) for d, f in flat.items()}
        st["grads"], st["out"] = [], []
        for (shape, dtype), first in zip(_layer_tensors(case), at):
            n = math.prod(shape)
            g = flat[dtype][first:first + n].view(shape)
            g.normal_(std=2e-3, generator=gen)
            st["grads"].append(g)
            st["out"].append(st["flat"][dtype][first:first + n].view(shape))
        st["max_norm"], st["norm"] = 0.25, torch.empty(1, device="cuda")
    return st


def _run_own(st):
    from paper_2412_07752_amd import api
    op = st["case"]["op"]
    if op == "embed":
        return api.flashrnn_embedding_fwd(st["table"], st["tokens"], scale=st["scale"], out=st["out"])
    if op == "embed_grad":
        return api.flashrnn_embedding_bwd(st["tokens"], st["dout"], st["case"]["vocab"], scale=st["scale"], dtable=st["out"])
    if op == "norm":
        return api.flashrnn_layer_norm_fwd(st["x"], st["weight"], st["bias"], eps=EPS, y=st["y"], mean=st["mean"], rstd=st["rstd"])
    if op == "norm_grad":
        return api.flashrnn_layer_norm_bwd(st["dy"], st["x"], st["mean"], st["rstd"], st["weight"], out=st["out"])
    if op == "loss":
        return api.flashrnn_cross_entropy(st["logits"], st["targets"], grad_scale=st["grad_scale"], loss=st["out"][0], dlogits=st["out"][1])
    norm = api.flashrnn_grad_clip(st["grads"], st["max_norm"], out=st["out"], norm=st["norm"])
    return norm, st["flat"]


def run(st):
    if own:
        return _run_own(st)
    op = st["case"]["op"]
    if op == "embed":
        there = st["tokens"] >= 0
        rows = st["table"][st["tokens"].clamp(min=0)].float() * st["scale"]
        return torch.where(there[:, None], rows, 0.0).to(st["table"].dtype)
    if op == "embed_grad":
        there = st["tokens"] >= 0
        rows = torch.where(there[:, None], st["dout"].float() * st["scale"], 0.0)
        return torch.zeros(st["out"].shape, device="cuda").index_add_(0, st["tokens"].clamp(min=0), rows)
    if op == "norm":
        x = st["x"].float()
        mean = x.mean(-1)
        xc = x - mean[..., None]
        rstd = (xc.square().mean(-1) + EPS).rsqrt()
        return (xc * rstd[..., None] * st["weight"] + st["bias"]).to(st["y"].dtype), mean, rstd
    if op == "norm_grad":
        dy, rstd = st["dy"].float(), st["rstd"][..., None]
        xhat = (st["x"].float() - st["mean"][..., None]) * rstd
        g = dy * st["weight"]
        dx = rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
        lead = (0, 1)
        return dx.to(st["dy"].dtype), (dy * xhat).sum(lead), dy.sum(lead)
    if op == "loss":
        x, t = st["logits"].float(), st["targets"]
        there, at = t >= 0, t.clamp(min=0)[:, None]
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - top)
        total = e.sum(1, keepdim=True)
        loss = torch.log(total[:, 0]) + top[:, 0] - x.gather(1, at)[:, 0]
        e *= st["grad_scale"] / total
        e.scatter_add_(1, at, torch.full_like(total, -st["grad_scale"]))
        e *= there[:, None]
        return torch.where(there, loss, 0.0), e.to(st["logits"].dtype)
    norm = torch.stack([g.float().square().sum() for g in st["grads"]]).sum().sqrt()
    factor = torch.where(norm <= st["max_norm"], 1.0, st["max_norm"] / norm)
    for g, o in zip(st["grads"], st["out"]):
        o.copy_(g.float() * factor)
    return norm.reshape(1), st["flat"]


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        padded = torch.cat([st["table"].double() * st["scale"], torch.zeros((1, case["width"]), dtype=torch.float64, device="cuda")])
        return padded[st["tokens"]]    # (-1 is the last row)
    if op == "embed_grad":
        keep = st["tokens"] >= 0
        out = torch.zeros((case["vocab"], case["width"]), dtype=torch.float64, device="cuda")
        return out.index_put_((st["tokens"][keep],), st["dout"][keep].double(), accumulate=True) * st["scale"]
    if op == "norm":
        x = st["x"].double()
        variance, mean = torch.var_mean(x, -1, unbiased=False)
        rstd = 1 / torch.sqrt(variance + EPS)
        return (x - mean[..., None]) / torch.sqrt(variance + EPS)[..., None] * st["weight"].double() + st["bias"].double(), mean, rstd
    if op == "norm_grad":
        x = st["x"].double().contiguous().requires_grad_()
        weight, bias = st["weight"].double().requires_grad_(), st["bias"].double().requires_grad_()
        centred = x - x.mean(-1, keepdim=True)
        y = centred / torch.sqrt((centred * centred).mean(-1, keepdim=True) + EPS) * weight + bias
        return torch.autograd.grad(y, (x, weight, bias), st["dy"].double())
    if op == "loss":
        N, V = st["logits"].shape
        loss, grad = torch.zeros(N, dtype=torch.float64, device="cuda"), torch.zeros((N, V), dtype=torch.float64, device="cuda")
        step = max(1, (1 << 27) // V)
        for i in range(0, N, step):
            x, t = st["logits"][i:i + step].double(), st["targets"][i:i + step]
            logp = x - torch.logsumexp(x, 1, keepdim=True)
            r = torch.nonzero(t >= 0)[:, 0]
            loss[i + r] = -logp[r, t[r]]
            p = torch.exp(logp[r])
            p[torch.arange(len(r), device="cuda"), t[r]] -= 1
            grad[i + r] = p * st["grad_scale"]
        return loss, grad
    total = sum(float((g.double() ** 2).sum()) for g in st["grads"])
    factor = min(1.0, st["max_norm"] / math.sqrt(total))
    at, end = _places(case)
    flat = {d: torch.zeros(n, dtype=torch.float64, device="cuda") for d, n in end.items() if n}
    for g, first, (shape, dtype) in zip(st["grads"], at, _layer_tensors(case)):
        flat[dtype][first:first + math.prod(shape)] = g.reshape(-1).double() * factor
    return torch.tensor([math.sqrt(total)], dtype=torch.float64), flat


def _distinct(count, kinds):
    """How many different words `count` places of a text hold, as prepare() draws them (expected)."""
    p = (torch.arange(kinds, dtype=torch.float64) + 2.7).reciprocal()
    return float((1 - (1 - p / p.sum()) ** (count * (1 - PADDING))).sum())


def work(case):
    op = case["op"]
    if op in ("embed", "embed_grad"):
        N, H, e = case["tokens"], case["width"], SIZE[case["dtype"]]
        if op == "embed":   # a row of the table is read once, however often its word comes
            return {"bytes": int((N + _distinct(N, case["vocab"])) * H * e) + N * 8, "flops": N * H}
        return {"bytes": N * (H * e + 8) + case["vocab"] * H * 4, "flops": 2 * N * H}
    if op in ("norm", "norm_grad"):
        rows, D, heads = case["steps"] * case["rows"] * max(1, case["heads"]), case["width"], max(1, case["heads"])
        x, y = SIZE[case["xdtype"]], SIZE[case["dtype"]]
        if op == "norm":
            return {"bytes": rows * (D * (x + y) + 8) + 8 * heads * D, "flops": 8 * rows * D}
        return {"bytes": rows * (D * (x + 2 * y) + 8) + 12 * heads * D, "flops": 14 * rows * D}
    if op == "loss":
        return {"bytes": case["rows"] * (2 * case["classes"] * SIZE[case["dtype"]] + 12), "flops": 6 * case["rows"] * case["classes"]}
    sizes = [(math.prod(s), SIZE[d]) for s, d in _layer_tensors(case)]
    return {"bytes": sum(2 * n * e for n, e in sizes) + 4, "flops": sum(3 * n for n, _ in sizes)}
