"""The example that runs the operators together: its gradients against 64-bit formulas, and that it learns."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_gradients_of_the_example():
    """Relative bounds in the Frobenius norm.  A held value is off by h = 2^-4 of itself at most (those near a block's least are nothing in
    a sum of squares), a bf16 one by u = 2^-8.  dWo: h for h1, u each for h0, gate, up, a, h1, the logits and d_logits.  silu's relative
    slope is below 2 for the gates there are (|g| < 1 of size), its derivative's slope below 1: dWd gets h of a's checkpoint, 3 h of
    its factors', dWg and dWu h of h0's checkpoint and 3 h of the factors'.  Roundings of one matrix add up at random, so that
    amplification by products with the weights is no more than these worst cases leave room for."""
    from paper_2502_11034_amd.example_training import Chain, Model
    model, chain = Model(300, 96, 160, 777, entropy_weight=0.1, seed=3), Chain(300)
    t, target = chain.pairs(777)
    target[::50] = -1
    logprob = model.gradients(t, target).cpu().double()
    w = [c.cpu().double().requires_grad_() for c in model.copies]
    t, target = t.cpu(), target.cpu()
    h0 = w[0][t]
    a = torch.nn.functional.silu(h0 @ w[1].t()) * (h0 @ w[2].t())
    logp = torch.log_softmax((h0 + a @ w[3].t()) @ w[4].t(), 1)
    lp = torch.where(target >= 0, logp.gather(1, target.clamp(min=0)[:, None])[:, 0], 0.0)
    entropy = -(logp.exp() * logp).sum(1)
    (-lp.mean() - 0.1 * entropy.mean()).backward()
    h, u = 2.0 ** -4, 2.0 ** -8
    assert (logprob - lp).abs().max() < 40 * u           # six roundings of values of size up to 5
    for got, want, bound in zip(model.grads, w, (4 * h, 4 * h, 4 * h, 4 * h, h + 7 * u)):
        got, want = got.cpu().double(), want.grad
        assert (got - want).norm() <= bound * want.norm()


def test_the_example_learns():
    from paper_2502_11034_amd.example_training import main
    # the chain's own entropy is 1.06, the first loss above ln 128 = 4.85
    assert main(["--steps", "150", "--vocab", "128", "--dim", "64", "--hidden", "96", "--tokens", "1024"]) < 1.6
