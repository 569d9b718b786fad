"""The model that runs all operators together: gradients against automatic differentiation in 64 bits, steps one by one against whole sequences."""
import pytest
import torch

from paper_2412_07752_amd import language_model as lm

pytestmark = pytest.mark.gpu


def _norm(x, w, b, eps=1e-5):
    c = x - x.mean(-1, keepdim=True)
    return c / torch.sqrt((c * c).mean(-1, keepdim=True) + eps) * w + b


def _plain_loss(model, p, tokens):
    """The same model on the CPU, the sLSTM in its form without stabilizer (equal where no exponential leaves the range)."""
    words, targets = tokens[:-1], tokens[1:]
    T, B = words.shape
    NH, D, H, G = model.NH, model.D, model.H, model.G
    x = torch.where((words >= 0)[..., None], p["table"][words.clamp(min=0)], torch.zeros(())) * model.scale
    for k in range(model.layers):
        Wx = (_norm(x, p[f"{k}.norm.weight"], p[f"{k}.norm.bias"]) @ p[f"{k}.W"].t()).view(T, B, G, NH, D)
        h = c = n = torch.zeros(B, NH, D, dtype=torch.float64)
        hs = []
        for t in range(T):
            g = Wx[t] + torch.stack([torch.stack([h[:, i] @ p[f"{k}.R"][i, :, j] for i in range(NH)], 1) for j in range(G)], 1) + p[f"{k}.b"].transpose(0, 1)
            i, f, z, o = g[:, 0].exp(), torch.sigmoid(g[:, 1]), torch.tanh(g[:, 2]), torch.sigmoid(g[:, 3])
            c, n = f * c + i * z, f * n + i
            h = o * c / n
            hs.append(h)
        x = x + _norm(torch.stack(hs), p[f"{k}.head_norm.weight"], p[f"{k}.head_norm.bias"]).reshape(T, B, H)
    logits = _norm(x, p["norm.weight"], p["norm.bias"]) @ p["table"].t()
    there = targets >= 0
    lse = torch.logsumexp(logits, -1)
    return ((lse - logits.gather(-1, targets.clamp(min=0)[..., None])[..., 0]) * there).sum() / there.sum()


@pytest.mark.parametrize("dtype,tolerance", [(torch.float32, 2e-5), (torch.bfloat16, 6e-2)])
def test_gradients_against_automatic_differentiation(dtype, tolerance):
    """float32: the loop's own bound of 1e-5 per output, twice in a row; bfloat16: 2e-2 per loop and 2^-8 at each of about ten roundings in between."""
    model = lm.LanguageModel(50, 2, 16, layers=2, dtype=dtype, seed=3)
    tokens = lm.chain_text(50, 13, 5, seed=1)[0]
    tokens[9:, 1] = -1
    tokens[0, 2] = -1
    loss, grads = model.loss_and_gradients(tokens)
    p = {n: v.double().cpu().requires_grad_() for n, v in model.params.items()}
    want = _plain_loss(model, p, tokens.cpu())
    want.backward()
    assert abs(loss.item() - want.item()) < tolerance * want.item()
    assert set(grads) == set(p)
    for n, g in grads.items():
        off = (g.double().cpu() - p[n].grad).norm() / p[n].grad.norm()
        assert off < tolerance, (n, float(off))


@pytest.mark.parametrize("cell", sorted(lm.CELLS))
def test_single_words_follow_the_whole_sequence(cell):
    """The logits of step-by-step calls give the loss that the whole sequence gave."""
    model = lm.LanguageModel(40, 2, 32, layers=2, cell=cell, dtype=torch.float32, seed=5)
    tokens = lm.chain_text(40, 9, 3, seed=2)[0]
    loss, _ = model.loss_and_gradients(tokens)
    states, total = model.start(3), 0.0
    for t in range(8):
        logits = model.step(tokens[t], states).double()
        total += (torch.logsumexp(logits, 1) - logits.gather(1, tokens[t + 1][:, None])[:, 0]).sum().item()
    assert abs(total / 24 - loss.item()) < 1e-5 * loss.item()


def test_training_learns_the_chain_and_continues_it():
    """Words with four successors, one of them in three quarters of all cases: 1.0 nat a word is to be reached from log(vocab)."""
    torch.manual_seed(0)
    assert lm.main(["--steps", "150", "--vocab", "40", "--layers", "1", "--heads", "2", "--width", "32", "--seqlen", "64", "--lr", "1.0"]) < 2.0
