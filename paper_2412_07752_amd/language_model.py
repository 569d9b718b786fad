"""A small language model around the recurrent layer: everything the library offers, run together.

    python -m paper_2412_07752_amd.language_model [--steps N] [--cell slstm] [--layers L] [--heads NH] [--width D] [--vocab V] [--batch B] [--seqlen T]

trains on a synthetic text (a fixed random chain of words) and then continues it token by token.  A layer is
x + norm_heads(RNN(W norm(x))): layer norm, input projection, the time-step loop, layer norm head by head on the hidden states where they lie
inside the loop's states; the logits use the embedding's table.  Every step is explicit, forward and backward: torch supplies memory, the two
dense products around the loop and the update of the weights.  Weights are float32; `dtype` is the type of what the loop and its neighbours
read and write.
"""
import argparse
import time

import torch

from . import api

CELLS = {"lstm": api.FLASHRNN_LSTM, "gru": api.FLASHRNN_GRU, "slstm": api.FLASHRNN_SLSTM, "elman": api.FLASHRNN_ELMAN, "gru4": api.FLASHRNN_GRU4}


class LanguageModel:
    def __init__(self, vocab, heads, width, layers=1, cell="slstm", dtype=torch.bfloat16, device="cuda", seed=0):
        self.cell, self.dtype, self.vocab, self.layers = CELLS[cell], dtype, vocab, layers
        self.NH, self.D, self.H, self.G, self.S = heads, width, heads * width, api.flashrnn_num_gates(CELLS[cell]), api.flashrnn_num_states(CELLS[cell])
        gen = torch.Generator(device=device).manual_seed(seed)
        normal = lambda *shape: torch.randn(shape, generator=gen, device=device)
        H, G, NH, D = self.H, self.G, self.NH, self.D
        self.scale = H ** 0.5
        p = {"table": normal(vocab, H) / H ** 0.5, "norm.weight": torch.ones(H, device=device), "norm.bias": torch.zeros(H, device=device)}
        for k in range(layers):
            p[f"{k}.norm.weight"], p[f"{k}.norm.bias"] = torch.ones(H, device=device), torch.zeros(H, device=device)
            p[f"{k}.W"], p[f"{k}.R"], p[f"{k}.b"] = normal(G * H, H) / H ** 0.5, normal(NH, D, G, D) / D ** 0.5, torch.zeros(NH, G, D, device=device)
            if cell in ("lstm", "slstm"):
                p[f"{k}.b"][:, 1] = 3.0   # forget gate
            p[f"{k}.head_norm.weight"], p[f"{k}.head_norm.bias"] = torch.ones(NH, D, device=device), torch.zeros(NH, D, device=device)
        self.params = p

    def _io(self, name):
        return self.params[name].to(self.dtype)

    def _project(self, k, x):
        """The loop's inputs for rows x[T, B, H]."""
        T, B, H = x.shape
        return (x.view(T * B, H) @ self._io(f"{k}.W").t()).view(T, B, self.G, self.NH, self.D)

    def loss_and_gradients(self, tokens):
        """tokens[T + 1, B] (padding: -1): mean loss over the places that have a next word, and the gradient of every parameter."""
        p, NH, D, H = self.params, self.NH, self.D, self.H
        words, targets = tokens[:-1].contiguous(), tokens[1:].contiguous()
        T, B = words.shape
        table = self._io("table")
        x = api.flashrnn_embedding_fwd(table, words, scale=self.scale)
        saved = []
        for k in range(self.layers):
            n, mean, rstd = api.flashrnn_layer_norm_fwd(x, p[f"{k}.norm.weight"], p[f"{k}.norm.bias"])
            R, b = self._io(f"{k}.R"), self._io(f"{k}.b")
            states, cache, ws = api.flashrnn_fwd(self.cell, self._project(k, n), R, b)
            h = states[1:, 0]
            y, hmean, hrstd = api.flashrnn_layer_norm_fwd(h, p[f"{k}.head_norm.weight"], p[f"{k}.head_norm.bias"], dtype=self.dtype)
            saved.append((x, n, mean, rstd, R, b, states, cache, ws, h, hmean, hrstd))
            x = x + y.view(T, B, H)
        n, mean, rstd = api.flashrnn_layer_norm_fwd(x, p["norm.weight"], p["norm.bias"])
        n2 = n.view(T * B, H)
        logits = n2 @ table.t()
        count = (targets >= 0).sum()
        per_row = (1.0 / count.clamp(min=1)).expand(T * B).float().contiguous()
        loss, dlogits = api.flashrnn_cross_entropy(logits, targets.view(-1), per_row, dlogits=logits)   # (in place)
        g = {"table": (dlogits.t() @ n2).float()}
        dx, g["norm.weight"], g["norm.bias"] = api.flashrnn_layer_norm_bwd((dlogits @ table).view(T, B, H), x, mean, rstd, p["norm.weight"])
        for k in reversed(range(self.layers)):
            x, n, mean, rstd, R, b, states, cache, ws, h, hmean, hrstd = saved.pop()
            dH, g[f"{k}.head_norm.weight"], g[f"{k}.head_norm.bias"] = api.flashrnn_layer_norm_bwd(dx.view(T, B, NH, D), h, hmean, hrstd, p[f"{k}.head_norm.weight"])
            dWx, g[f"{k}.R"], g[f"{k}.b"], _ = api.flashrnn_bwd(self.cell, R, b, states, cache, dH, workspace=ws)
            dWx = dWx.view(T * B, self.G * H)
            g[f"{k}.W"] = (dWx.t() @ n.view(T * B, H)).float()
            dn = (dWx @ self._io(f"{k}.W")).view(T, B, H)
            dx2, g[f"{k}.norm.weight"], g[f"{k}.norm.bias"] = api.flashrnn_layer_norm_bwd(dn, x, mean, rstd, p[f"{k}.norm.weight"])
            dx = dx + dx2
        api.flashrnn_embedding_bwd(words, dx, self.vocab, scale=self.scale, dtable=g["table"], accumulate=True)   # (tied to the logits' weights)
        return loss.sum() / count.clamp(min=1), g

    def train_step(self, tokens, lr=0.1, max_norm=1.0):
        """One step of gradient descent, clipped by the global norm.  Returns (loss, norm before clipping), both on the device."""
        loss, g = self.loss_and_gradients(tokens)
        names = list(self.params)
        norm = api.flashrnn_grad_clip([g[n] for n in names], max_norm)
        for n in names:
            self.params[n].add_(g[n], alpha=-lr)
        return loss, norm

    def start(self, batch):
        """States of a text that has not begun, one tensor [2, S, B, NH, D] per layer: slot 0 before a step, slot 1 behind it."""
        return [torch.zeros((2, self.S, batch, self.NH, self.D), dtype=torch.float32, device=self.params["table"].device) for _ in range(self.layers)]

    def step(self, words, states):
        """One word per sequence: words[B] -> logits[B, vocab]; the states move on in place."""
        p, B = self.params, words.shape[0]
        table = self._io("table")
        x = api.flashrnn_embedding_fwd(table, words.view(1, B), scale=self.scale)
        for k, s in enumerate(states):
            n, _, _ = api.flashrnn_layer_norm_fwd(x, p[f"{k}.norm.weight"], p[f"{k}.norm.bias"], save_for_backward=False)
            api.flashrnn_fwd_static_scratch(self.cell, self._project(k, n), self._io(f"{k}.R"), self._io(f"{k}.b"), s[1], save_for_backward=False, states=s)
            y, _, _ = api.flashrnn_layer_norm_fwd(s[1:, 0], p[f"{k}.head_norm.weight"], p[f"{k}.head_norm.bias"], dtype=self.dtype, save_for_backward=False)
            x = x + y.view(1, B, self.H)
        n, _, _ = api.flashrnn_layer_norm_fwd(x, p["norm.weight"], p["norm.bias"], save_for_backward=False)
        return n.view(B, self.H) @ table.t()

    def generate(self, prompt, count):
        """prompt[T, B] of at least one word -> the `count` most likely next words, [count, B]."""
        if prompt.shape[0] == 0 or count < 0:
            raise ValueError(f"a prompt of {prompt.shape[0]} words cannot be continued by {count}")
        states, out = self.start(prompt.shape[1]), prompt.new_empty((count, prompt.shape[1]), dtype=torch.int64)
        for words in prompt if count else ():
            logits = self.step(words, states)
        for i in range(count):
            torch.argmax(logits, 1, out=out[i])
            if i + 1 < count:
                logits = self.step(out[i], states)
        return out


def chain_text(vocab, length, batch, seed=0, device="cuda"):
    """tokens[length, batch] of a chain in which every word has four possible successors, one of them in three quarters of all cases."""
    gen = torch.Generator(device=device).manual_seed(seed)
    successors = torch.randint(vocab, (vocab, 4), generator=gen, device=device)
    words = [torch.randint(vocab, (batch,), generator=gen, device=device)]
    for _ in range(length - 1):
        u = torch.rand(batch, generator=gen, device=device)
        words.append(successors[words[-1], torch.where(u < 0.75, 0, (u * 12 - 8).long().clamp(1, 3))])
    return torch.stack(words), successors


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in (("steps", 60), ("layers", 2), ("heads", 4), ("width", 64), ("vocab", 500), ("batch", 16), ("seqlen", 128)):
        ap.add_argument(f"--{name}", type=int, default=default)
    ap.add_argument("--cell", choices=sorted(CELLS), default="slstm")
    ap.add_argument("--lr", type=float, default=2.0)
    a = ap.parse_args(argv)
    model = LanguageModel(a.vocab, a.heads, a.width, a.layers, a.cell)
    text, successors = chain_text(a.vocab, a.seqlen + 1 + a.steps * a.seqlen, a.batch)
    began = time.time()
    for i in range(a.steps):
        loss, norm = model.train_step(text[i * a.seqlen:(i + 1) * a.seqlen + 1], lr=a.lr)
        if i % max(1, a.steps // 10) == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {loss.item():.3f}  gradient norm {norm.item():.3f}  {(time.time() - began) / (i + 1) * 1e3:.1f} ms a step", flush=True)
    prompt = text[-32:]
    out = model.generate(prompt, 16)
    likely = torch.cat([prompt[-1:], out[:-1]])
    print(f"continued by {out.shape[0]} words: {(successors[likely, 0] == out).float().mean().item():.0%} are the chain's likeliest successor")
    return loss.item()


if __name__ == "__main__":
    main()
