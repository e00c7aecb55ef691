"""Corners of the operators around the step: results next to the ends of fp32's range, and instantiations that ordinary sizes seldom reach."""
import math

import pytest
import torch

import operators_oracle as O
from paper_2502_11034_amd import binding as B
from test_gpu_operators import DEV, FILL, Framed, check_logprobs, gen, near, run_wgrad

pytestmark = pytest.mark.gpu
U = O.U32


# ------------------------------------------------------------------------------------------------ gated activation

def gate_off(g, dtype):
    """What t = 1 / (1 + exp(-g)) may be off by, in half steps of fp32 of itself.  The same number for every g in fp32: the exponential's
    instruction a step (2) and its correction 1, the sum 1, the reciprocal's instruction a step (2); 1 - t has a product more.  For
    bf16 values the argument g log2 e is one rounded number times a rounded constant: 2 |g| more."""
    return 8.0 if dtype == torch.float32 else 9.0 + 2.0 * g.abs()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1.5, 2.0 ** 100])
def test_gates_far_from_zero(dtype, size):
    """Relative error independent of the gate, and no zeros where the product is a normal number: silu(-88) = -5.3e-37."""
    dtype = torch.float32 if dtype == "f32" else torch.bfloat16
    step = torch.linspace(-160, 90, 64 * 100).view(64, 100)
    step[0, :8] = torch.tensor([-88.0, -87.5, -88.7, -89.0, -91.0, -1.2784645, -0.0, 1e-30])
    gate = step.to(dtype)
    up = torch.full_like(gate, size)
    out = Framed(64, 100, dtype)
    ckpts = [torch.empty(B.adagc_act8_bytes(64, 100), dtype=torch.uint8, device=DEV) for _ in range(2)]
    B.adagc_swiglu(gate.to(DEV), up.to(DEV), out.t, *ckpts)
    g, u = gate.double(), up.double()
    want = g * torch.sigmoid(g) * u
    near(out.result(), want, want.abs() * (gate_off(g, dtype) + 4) * U + 2.0 ** -126, dtype)        # three more products

    g, u = (O.values(c.cpu(), 64, 100) for c in ckpts)
    t = torch.sigmoid(g)
    d_out = torch.randn(64, 100, generator=gen(50)).to(dtype)
    d = d_out.double()
    d_gate, d_up, again = (Framed(64, 100, dtype) for _ in range(3))
    B.adagc_swiglu_backward(d_out.to(DEV), *ckpts, d_gate.t, d_up.t, again.t)
    rest = torch.sigmoid(-g)                                                                  # 1 - t
    slope = 1 + g * rest
    near(again.result(), g * t * u, (g * t * u).abs() * (gate_off(g, dtype) + 4) * U + 2.0 ** -126, dtype)
    near(d_up.result(), d * g * t, (d * g * t).abs() * (gate_off(g, dtype) + 4) * U + 2.0 ** -126, dtype)
    # d and u times t times the slope, in which g rest is off by as much as t and one product
    off = (d * u).abs() * t * U * (slope.abs() * (gate_off(g, dtype) + 5) + (g * rest).abs() * (gate_off(g, dtype) + 1))
    near(d_gate.result(), d * u * t * slope, off + 2.0 ** -126, dtype)


# ------------------------------------------------------------------------------------------------ gradient of the logits

def gradient(z, t, scale, d_logprob, d_entropy, in_place=False):
    rows, vocab = z.shape
    zd = Framed(rows, vocab, z.dtype, data=z)
    logprob, entropy, stats = (torch.empty(s, device=DEV) for s in ((rows,), (rows,), (rows, 2)))
    B.adagc_token_logprobs(zd.t, t.to(DEV), logprob, entropy, stats, scale=scale)
    d = zd if in_place else Framed(rows, vocab, z.dtype)
    B.adagc_token_logprobs_backward(zd.t, t.to(DEV), stats, entropy, d_logprob.to(DEV), d_entropy.to(DEV), d.t, scale=scale)
    return d.result()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale, size", [(1.0, 3.5e34), (1.0, 3e38), (0.5, 1e37), (2.0 ** 100, 3e4), (2.0 ** 100, 1e36), (2.0 ** 100, 1e-30),
                                         (2.0 ** -100, 3e38), (2.0 ** -100, 1.0)])
def test_gradients_of_any_size(dtype, scale, size):
    """Wherever scale and gradients are numbers: masked and vanishing tokens get 0, the others what the formula gives, infinite only
    where that is."""
    dtype, g = torch.float32 if dtype == "f32" else torch.bfloat16, gen(51)
    z = torch.randn(6, 300, generator=g).to(dtype)
    z[:, ::3] = -math.inf
    z[1, 5:] = -math.inf
    z[2, 7] = 100.0
    t = torch.tensor([1, 2, 7, -1, 4, 299])
    dl, dh = ((torch.rand(6, generator=g) / 2 + 0.5) * size * torch.randn(6, generator=g).sign() for _ in range(2))
    got = gradient(z, t, scale, dl, dh)
    assert not got[z == -math.inf].any()
    want, off = O.logprobs_backward(z, t, scale, dl, dh)
    most = torch.finfo(dtype).max
    want = torch.where(want.abs() > most, want.sign() * math.inf, want)
    near(got, want, off, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("odd", [math.nan, math.inf, -math.inf])
def test_rows_of_nothing_get_no_gradient(dtype, odd):
    """All of a masked row's gradient is 0, also where the gradients asked for are no numbers; the other rows do not notice."""
    z = torch.randn(3, 1030, generator=gen(52)).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    z[1] = -math.inf
    t, dl, dh = torch.tensor([5, 6, -1]), torch.tensor([1.0, odd, odd]), torch.tensor([0.5, odd, -0.5])
    want, off = O.logprobs_backward(z, t, 1.0, torch.tensor([1.0, 0.0, 0.0]), torch.tensor([0.5, 0.0, -0.5]))
    for in_place in (False, True):
        got = gradient(z, t, 1.0, dl, dh, in_place)
        near(got, want, off, z.dtype)
        assert not got[1].any()


# ------------------------------------------------------------------------------------------------ log-probabilities

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [9, 20011])                     # a row in one part and in several
@pytest.mark.parametrize("scale", [2.0 ** -100, 1e-20, 0.25])
def test_differences_beyond_the_range(dtype, vocab, scale):
    """A token of the type's lowest value beside one of its largest: the difference is no fp32 number, scale times it may be one."""
    dtype = torch.float32 if dtype == "f32" else torch.bfloat16
    z = torch.full((2, vocab), -math.inf, dtype=dtype)
    z[:, 3:7] = torch.tensor([torch.finfo(dtype).min, 1.0, torch.finfo(dtype).max, -2.0 ** 127], dtype=dtype)
    t = torch.tensor([3, 6])
    check_logprobs(z, t, scale, 4)


# ------------------------------------------------------------------------------------------------ weight gradient

@pytest.mark.parametrize("thin", ["n_in", "n_out"])
def test_wgrad_of_more_tiles_than_two_to_22(thin):
    """One token, so that dW is the product itself: 2^29 + 1 outputs of one input, and one output of as many inputs."""
    n = 2 ** 29 + 1
    long = (torch.arange(n, dtype=torch.int32, device=DEV) % 15 - 7).to(torch.bfloat16)       # exact next to a block's 7
    n_out, n_in = (n, 1) if thin == "n_in" else (1, n)
    d_out, x = (long[None], torch.full((1, 1), 2.0, dtype=torch.bfloat16, device=DEV))
    if thin == "n_out":
        d_out, x = x, d_out
    ckpt = torch.empty(B.adagc_act8_bytes(1, n_in), dtype=torch.uint8, device=DEV)
    B.adagc_act8_pack(x, ckpt)
    w = torch.full((n_out, n_in), FILL, dtype=torch.bfloat16, device=DEV)
    size = B.adagc_act8_wgrad_workspace_bytes(1, n_out, n_in, B.ADAGC_BF16)
    B.adagc_act8_wgrad(d_out, ckpt, w, workspace=torch.empty(max(1, size), dtype=torch.uint8, device=DEV))
    assert all(torch.equal(a, 2 * b) for a, b in zip(w.view(-1).split(2 ** 27), long.split(2 ** 27)))


@pytest.mark.parametrize("dw", ["f32", "bf16"])
@pytest.mark.parametrize("rows, n_out, n_in, ld_d, offset, ld_w, accumulate", [
    (96, 128, 128, None, 0, None, False),              # three steps: one that the loop itself has staged
    (165, 200, 200, 203, 1, 201, True),                # five, and tokens after them
    (480, 129, 97, None, 0, None, False),              # fifteen, not split
    (1000, 130, 150, 131, 3, 151, True),               # 31 in seven parts
    (4097, 300, 224, None, 0, 229, False),             # 128 in 32 parts, and a token after them
    (2200, 700, 255, 701, 0, None, True),
])
def test_wgrad_of_fp32_gradients_and_narrow_inputs(dw, rows, n_out, n_in, ld_d, offset, ld_w, accumulate):
    """fp32 gradients of layers with 97 to 255 inputs have tiles, a main loop and a joining kernel of their own."""
    g = gen(rows + n_out)
    d_out = torch.randn(rows, n_out, generator=g) * torch.exp(2 * torch.randn(rows, 1, generator=g))
    x = (torch.randn(rows, n_in, generator=g) * torch.exp(torch.randn(1, n_in, generator=g))).to(torch.bfloat16)
    dw = torch.float32 if dw == "f32" else torch.bfloat16
    start = torch.randn(n_out, n_in, generator=g).to(dw) if accumulate else None
    got, held = run_wgrad(d_out, x, dw, ld_d, offset, ld_w, start)
    want, off = O.wgrad(d_out, held)
    if accumulate:
        want = want + start.double()
        off = off + 2 * U * (want.abs() + off)
    near(got, want, off, dw)


@pytest.mark.parametrize("rows", [31, 32, 64, 97, 160, 224, 511, 512, 2085])
def test_wgrad_of_fp32_gradients_and_narrow_inputs_is_exact(rows):
    """Whole numbers, every sum of which is one in fp32: no token is lost or taken twice, whatever the number of steps and parts."""
    g = gen(rows)
    d_out = torch.randint(-2 ** 9, 2 ** 9 + 1, (rows, 333), generator=g).float() * 2.0 ** -3        # two bf16 terms
    x = torch.randint(-8, 9, (rows, 200), generator=g).to(torch.bfloat16)
    x[:, ::32] = 8                                     # blocks of one scale hold these exactly
    got, held = run_wgrad(d_out, x, torch.float32)
    assert torch.equal(held, x.double())
    assert torch.equal(got.double(), d_out.double().t() @ x.double())
