"""The activation of the gated projections at gates of every size, against 64 bits: its relative error does not grow with the gate, and what is
left of a sigmoid far below 0 counts where the other factors bring it back."""
import math

import pytest
import torch

from paper_2502_11034_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODES = {torch.float32: B.ADAGC_F32, torch.bfloat16: B.ADAGC_BF16}
FEW, TILES, LARGE = (16, 8, 5), (300, 8, 70), (256, 1024, 2100)          # fp32: the last one's operands are taken in parts
FAR = -167.0                   # below, a sigmoid may be 0


def gates(rows, seed):
    """-170 .. 100: the ends, both sides of where the arithmetic changes, and numbers in between."""
    g = torch.empty(rows, dtype=torch.float64)
    special = [-170.0, -160.0, -120.0, -104.0, -103.0, -90.0, -89.0, -88.75, -88.5, -87.25, -87.0, -86.75, -1.28125, 0.0, 87.0, 100.0]
    g.uniform_(-165, 100, generator=torch.Generator().manual_seed(seed))
    g[:len(special)] = torch.tensor(special, dtype=torch.float64)
    return g


def within(got, want, relative, absolute, dtype):
    """|got - want| <= relative half steps of fp32 of |want|, and absolute, and half a step of dtype."""
    got, half = got.double().cpu(), torch.finfo(dtype).eps / 2
    off = relative * U32 * want.abs() + absolute
    bound = off + (half * (want.abs() + off) if dtype == torch.bfloat16 else 0.0)
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), float(((got - want).abs() / bound)[bad].max()))


def inputs(rows, dim, hidden, dtype, up, seed):
    """x whose first two numbers are the gate and up of every column: both products are these numbers."""
    g = gates(rows, seed).to(dtype)
    x = torch.zeros(rows, dim, dtype=dtype)
    x[:, 0], x[:, 1] = g, up
    w_gate, w_up = torch.zeros(hidden, dim, dtype=dtype), torch.zeros(hidden, dim, dtype=dtype)
    w_gate[:, 0], w_up[:, 1] = 1.0, 1.0
    return g.double(), x.to(DEV), w_gate.to(DEV), w_up.to(DEV)


def space(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)


# What a sigmoid may be off by in half steps of fp32: an exponential of one step, its correction and 1 + e rounded, a reciprocal of one step, 8 in all; with bf16
# data, where the exponent g / ln 2 is rounded, up to half a step of it and ln 2 times that of the result, 2 |g| more.
def sigmoid_off(g, dtype):
    return 8 + (0 if dtype == torch.float32 else 2 * g.abs())


def least(dtype):
    """Half of a type's steps below its normal numbers (2^-149 in fp32, 2^-133 in bf16, which has been an fp32 number before)."""
    info = torch.finfo(dtype)
    return info.smallest_normal * info.eps / 2 + (2.0 ** -150 if dtype == torch.bfloat16 else 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, dim, hidden", [FEW, TILES, LARGE])
def test_results(dtype, rows, dim, hidden):
    dtype = TYPES[dtype]
    for up in (1.5, -2.0 ** 90):
        g, x, w_gate, w_up = inputs(rows, dim, hidden, dtype, up, 1)
        out = torch.empty(rows, hidden, dtype=dtype, device=DEV)
        B.adagc_gated_linear(x, w_gate, w_up, out, workspace=space(B.adagc_gated_linear_workspace_bytes(rows, dim, hidden, CODES[dtype])))
        want = g * torch.sigmoid(g) * up
        # three products more
        absolute = least(dtype) + torch.where(g < FAR, want.abs(), 0.0)
        for column in (0, hidden - 1):
            within(out[:, column], want, sigmoid_off(g, dtype) + 3, absolute, dtype)
        assert (out == out[:, :1]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("rows, dim, hidden", [FEW, TILES, LARGE])
def test_gradients(dtype, kept, rows, dim, hidden):
    """One column has a gradient: d_x is d_g and d_u, each times 1."""
    dtype = TYPES[dtype]
    for up, d in ((1.5, 1.0), (2.0 ** 40, 2.0 ** 60), (1.0, -2.0 ** 100)):
        g, x, w_gate, w_up = inputs(rows, dim, hidden, dtype, up, 2)
        d_out, d_x, again = torch.zeros(rows, hidden, dtype=dtype, device=DEV), torch.empty_like(x), torch.empty(rows, hidden, dtype=dtype, device=DEV)
        d_out[:, hidden // 2] = d
        held = {"gate": x[:, :1].expand(rows, hidden).contiguous(), "up": x[:, 1:2].expand(rows, hidden).contiguous()} if kept else {}
        B.adagc_gated_linear_backward(d_out, x, w_gate, w_up, d_x, out=again, **held,
                                      workspace=space(B.adagc_gated_linear_backward_workspace_bytes(rows, dim, hidden, CODES[dtype])))
        t, rest = torch.sigmoid(g), torch.sigmoid(-g)
        far = torch.where(g < FAR, 1.0, 0.0)
        bf16 = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0                     # d_g and d_u are rounded too
        # a normal number is left of a product with numbers that are: below 2^-125 it may be 0
        want = d * g * t
        within(d_x[:, 1], want, sigmoid_off(g, dtype) + 3, 2.0 ** -125 + far * want.abs() + bf16 * want.abs(), dtype)
        want = d * up * t * (1 + g * rest)
        parts = (d * up * t).abs() * (1 + g.abs() * rest)                        # what the sum's roundings are relative to; 1 - t is off as t is
        within(d_x[:, 0], want, 0, (2 * sigmoid_off(g, dtype) + 6) * U32 * parts + 2.0 ** -125 + abs(d * up) * 2.0 ** -125 * g.clamp(min=0) + far * want.abs() + bf16 * want.abs(), dtype)
        want = g * t * up
        within(again[:, 0], want, sigmoid_off(g, dtype) + 3, least(dtype) + far * want.abs(), dtype)


def test_gates_without_a_number():
    """-inf as every gate far below 0, inf as every one far above, NaN as itself; kept, so that no product has them."""
    rows, dim, hidden = 5, 8, 3
    for dtype in TYPES.values():
        g = torch.tensor([-math.inf, -1e30, math.inf, 1e30, math.nan]).to(dtype)
        x, w = torch.zeros(rows, dim, dtype=dtype, device=DEV), torch.zeros(hidden, dim, dtype=dtype, device=DEV)
        w[:, 0] = 1.0
        gate, up = g.to(DEV)[:, None].expand(rows, hidden).contiguous(), torch.full((rows, hidden), 2.0, dtype=dtype, device=DEV)
        d_x, out = torch.empty_like(x), torch.empty(rows, hidden, dtype=dtype, device=DEV)
        zero = torch.zeros_like(w)
        for w_gate, w_up in ((w, zero), (zero, w)):
            d_out = torch.ones_like(out)
            if w_gate is zero:
                d_out[2:] = 0.0                           # (d_u of the others is no number that a product with 0 leaves alone)
            B.adagc_gated_linear_backward(d_out, x, w_gate, w_up, d_x, gate=gate, up=up, out=out,
                                          workspace=space(B.adagc_gated_linear_backward_workspace_bytes(rows, dim, hidden, CODES[dtype])))
            assert (out[:2] == 0).all() and (out[2] == math.inf).all() and (out[3] == 2 * g[3].to(DEV)).all() and torch.isnan(out[4]).all()
            assert (d_x[:2, 0] == 0).all()
            if w_up is zero:
                assert d_x[3, 0] == 6.0 and torch.isnan(d_x[4, 0])               # the sigmoid's slope is 0: d u, three times


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("rows, dim, hidden", [FEW, TILES, LARGE])
def test_factors_whose_product_leaves_the_range_before_a_far_gate_brings_it_back(dtype, kept, rows, dim, hidden):
    """d_g of gates below -87: d u is 2^190 and the like, d u t a normal number."""
    dtype = TYPES[dtype]
    for up, d in ((2.0 ** 90, 2.0 ** 100), (-2.0 ** 100, 2.0 ** 90), (2.0 ** 120, 1.0), (2.0 ** -20, 2.0 ** 120), (2.0 ** 120, 2.0 ** -20)):
        g, x, w_gate, w_up = inputs(rows, dim, hidden, dtype, up, 3)
        g = g.clamp(max=-87.5).to(dtype).double()
        x[:, 0] = g.to(dtype)
        d_out, d_x = torch.zeros(rows, hidden, dtype=dtype, device=DEV), torch.empty_like(x)
        d_out[:, hidden // 2] = d
        held = {"gate": x[:, :1].expand(rows, hidden).contiguous(), "up": x[:, 1:2].expand(rows, hidden).contiguous()} if kept else {}
        B.adagc_gated_linear_backward(d_out, x, w_gate, w_up, d_x, **held,
                                      workspace=space(B.adagc_gated_linear_backward_workspace_bytes(rows, dim, hidden, CODES[dtype])))
        want = d * up * torch.sigmoid(g) * (1 + g)
        assert (want.abs() < 2.0 ** 100).all()
        bf16 = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
        # the sigmoid, 1 + g and three products
        within(d_x[:, 0], want, sigmoid_off(g, dtype) + 6, 2.0 ** -125 + torch.where(g < FAR, 1.0, 0.0) * want.abs() + bf16 * want.abs(), dtype)
