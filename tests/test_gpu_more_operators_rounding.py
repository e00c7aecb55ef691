"""What gradients from bf16 data lose: the one rounding of d_z, or of d_g and d_u, to bf16 that is documented, and nothing beside it.

With weight gradients in fp32 the products of the rounded numbers, taken in 64 bits, are met but for the numbers that round the other way because they
were off before: by a relative e at most, 2^-17 here (the logits' sums, the exponential of an argument below 2^5, a dozen roundings of 2^-24), so that up to
2 e / 2^-8 = 2^-8 of them differ, by one step, 2^-7 of a number's power of two: 2^-7 sqrt(2^-8) = 2^-11 in the root of the mean square, if all of them were
next to a power of two from above.  The rounding itself is 2^-9 to 2^-10: what a second one would add shows."""
import pytest
import torch

from paper_2502_11034_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SAME = 2.0 ** -11


def space(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


def apart(a, b):
    return float((a.double() - b).norm() / b.norm())


def check(got, rounded, plain):
    """got: fp32; products of the rounded numbers and of those before in 64 bits."""
    assert apart(got, rounded) <= SAME
    assert 2.0 ** -10 <= apart(got, plain) <= 2.0 ** -8


@pytest.mark.parametrize("rows, vocab, dim", [(512, 9000, 264), (700, 3000, 1000)])
def test_gradients_of_log_probabilities(rows, vocab, dim):
    g = torch.Generator(device=DEV).manual_seed(1)
    x, w = torch.randn(rows, dim, generator=g, device=DEV).bfloat16(), (torch.randn(vocab, dim, generator=g, device=DEV) * dim ** -0.5).bfloat16()
    t, d = torch.randint(0, vocab, (rows,), generator=g, device=DEV), torch.randn(rows, generator=g, device=DEV)
    logprob, stats = torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
    d_x, d_w = torch.empty_like(x), torch.empty(vocab, dim, device=DEV)
    B.adagc_linear_logprobs(x, w, t, logprob, stats, workspace=space(B.adagc_linear_logprobs_workspace_bytes(rows, vocab, dim, B.ADAGC_BF16)))
    B.adagc_linear_logprobs_backward(x, w, t, stats, d, d_x, d_w, workspace=space(B.adagc_linear_logprobs_backward_workspace_bytes(rows, vocab, dim, B.ADAGC_BF16)))
    d_z = -torch.softmax(x.double() @ w.double().t(), 1)
    d_z[torch.arange(rows, device=DEV), t] += 1.0
    d_z *= d.double()[:, None]
    rounded = d_z.float().bfloat16().double()
    check(d_w, rounded.t() @ x.double(), d_z.t() @ x.double())
    assert apart(d_x, (rounded @ w.double()).float().bfloat16().double()) <= 2 * SAME            # (d_x is bf16: it rounds the other way too)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("rows, dim, hidden", [(512, 264, 3000), (700, 1000, 520)])
def test_gradients_of_gated_projections(rows, dim, hidden, kept):
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(rows, dim, generator=gen, device=DEV).bfloat16()
    w_gate, w_up = ((torch.randn(hidden, dim, generator=gen, device=DEV) * dim ** -0.5).bfloat16() for _ in range(2))
    d_out = torch.randn(rows, hidden, generator=gen, device=DEV).bfloat16()
    out, gate, up = (torch.empty_like(d_out) for _ in range(3))
    B.adagc_gated_linear(x, w_gate, w_up, out, gate, up, workspace=space(B.adagc_gated_linear_workspace_bytes(rows, dim, hidden, B.ADAGC_BF16)))
    d_x, d_w_gate, d_w_up = torch.empty_like(x), *(torch.empty(hidden, dim, device=DEV) for _ in range(2))
    B.adagc_gated_linear_backward(d_out, x, w_gate, w_up, d_x, d_w_gate, d_w_up, **({"gate": gate, "up": up} if kept else {}),
                                  workspace=space(B.adagc_gated_linear_backward_workspace_bytes(rows, dim, hidden, B.ADAGC_BF16)))
    g, u = (gate.double(), up.double()) if kept else (x.double() @ w_gate.double().t(), x.double() @ w_up.double().t())
    s = torch.sigmoid(g)
    d_g, d_u = d_out.double() * u * s * (1 + g * torch.sigmoid(-g)), d_out.double() * g * s
    rounded = [v.float().bfloat16().double() for v in (d_g, d_u)]
    check(d_w_gate, rounded[0].t() @ x.double(), d_g.t() @ x.double())
    check(d_w_up, rounded[1].t() @ x.double(), d_u.t() @ x.double())
    want = rounded[0] @ w_gate.double() + rounded[1] @ w_up.double()
    assert apart(d_x, want.float().bfloat16().double()) <= 2 * SAME
