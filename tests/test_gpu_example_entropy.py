"""The example's bonus for entropy: its share of the gradients alone, of which the loss as a whole has too little to show a wrong sign."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_gradient_of_the_entropy_alone():
    """Relative bounds in the Frobenius norm, for d_logits = -w p (log p + H) / n.  A held value is off by h = 2^-4 of itself at most, a bf16 one by
    u = 2^-8.  Logits of size 1 carry six roundings (of h0, gate, up, a, h1, their own), 6 u, which enter once through p and once through
    log p, whose distance to -H is of size 1 too: 12 u, with 2 u for d_logits' own rounding and the entropy's.  Then as for the whole
    loss: dWo has h of h1's checkpoint and 7 u, the others 4 h.  No gradient, or one of the other sign, is off by 1 and by 2."""
    from paper_2502_11034_amd.example_training import Chain, Model
    weight = 0.7
    model, chain = Model(300, 96, 160, 777, entropy_weight=weight, seed=5), Chain(300)
    model.d_logprob.zero_()
    t, target = chain.pairs(777)
    target[::50] = -1                                  # entropy counts without a target too
    model.gradients(t, target)
    w = [c.cpu().double().requires_grad_() for c in model.copies]
    t = t.cpu()
    h0 = w[0][t]
    a = torch.nn.functional.silu(h0 @ w[1].t()) * (h0 @ w[2].t())
    logp = torch.log_softmax((h0 + a @ w[3].t()) @ w[4].t(), 1)
    (weight * (logp.exp() * logp).sum(1).mean()).backward()              # a loss of less entropy
    h, u = 2.0 ** -4, 2.0 ** -8
    for got, want, bound in zip(model.grads, w, 4 * (4 * h + 14 * u,) + (h + 21 * u,)):
        got, want = got.cpu().double(), want.grad
        assert (got - want).norm() <= bound * want.norm()
        assert (got + want).norm() > bound * want.norm() and want.norm() > bound * want.norm() > 0
