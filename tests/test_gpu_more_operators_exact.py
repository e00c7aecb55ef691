"""Products of the operators that keep nothing between the passes, bit for bit: operands whose sums are exact in fp32 in any order, with numbers
of so many bits that every part of a product counts that is taken as three bf16 numbers."""
import pytest
import torch

from paper_2502_11034_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODES = {torch.float32: B.ADAGC_F32, torch.bfloat16: B.ADAGC_BF16}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def workspace(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)


def numbers(rows, cols, bits, g):
    """Whole numbers of exactly so many bits, of both signs; of one bit: powers of two from 1 to 8."""
    shape = (rows, cols)
    if bits == 1:
        n = 2 ** torch.randint(0, 4, shape, generator=g, device=DEV)
    else:
        n = torch.randint(2 ** (bits - 1), 2 ** bits, shape, generator=g, device=DEV) | 1
    return (n * (2 * torch.randint(0, 2, shape, generator=g, device=DEV) - 1)).float()


# Bits of the operand and of the gradient that it is multiplied with: 24 bits are all three parts of a number, one bit the first alone, 12 bits the first
# two; and 24 are what a product may have, for fp32 to hold it.
BITS = {"f32": [(24, 1), (1, 24), (12, 12)], "bf16": [(8, 1), (1, 8), (4, 4)]}


class Certain:
    """Log-probabilities with all but no doubt: 64 of the dimensions have a code of +1 and -1 for every token, and a row of x is 16 times that of one
    token, whose logit is so far above the others that its probability is 1 and theirs 0.  So d_z is d at the target (another token), -d at
    that one and 0 elsewhere, and with no token twice every gradient is a single product."""

    CODE, SIZE = 64, 16.0

    def __init__(self, rows, vocab, dim, dtype, seed):
        g = gen(seed)
        self.rows, self.vocab, self.dim, self.dtype, self.g = rows, vocab, dim, dtype, g
        code = 2.0 * torch.randint(0, 2, (vocab, self.CODE), generator=g, device=DEV) - 1
        self.with_target = min(rows, vocab // 2)
        order = torch.randperm(rows, generator=g, device=DEV)[:self.with_target]
        i = torch.arange(self.with_target, device=DEV)
        self.own = torch.zeros(rows, dtype=torch.int64, device=DEV)              # the certain token: from the first one up
        self.t = torch.full((rows,), -1, dtype=torch.int64, device=DEV)          # the target: from the last one down
        self.own[order], self.t[order] = i, vocab - 1 - i
        self.has = self.t >= 0
        self.x, self.w = (torch.zeros(n, dim, device=DEV) for n in (rows, vocab))
        self.x[:, :self.CODE], self.w[:, :self.CODE] = code[self.own] * self.SIZE, code
        z = self.x[:, :self.CODE] @ self.w[:, :self.CODE].t()                     # whole numbers
        self.most, self.target_logit = z.amax(1), z.gather(1, self.t.clamp(min=0)[:, None])[:, 0]
        z.scatter_(1, self.own[:, None], -1e30)
        assert (z.amax(1) <= self.most - 200).all()

    def gradients(self, d, d_x, d_w, accumulate=False):
        code = CODES[self.dtype]
        x, w = self.x.to(self.dtype), self.w.to(self.dtype)
        assert torch.equal(x.float(), self.x) and torch.equal(w.float(), self.w)
        logprob, stats = torch.empty(self.rows, device=DEV), torch.empty(self.rows, 2, device=DEV)
        B.adagc_linear_logprobs(x, w, self.t, logprob, stats, workspace=workspace(B.adagc_linear_logprobs_workspace_bytes(self.rows, self.vocab, self.dim, code)))
        assert torch.equal(stats[:, 0], self.most) and (stats[:, 1] == 0).all()
        assert torch.equal(logprob, torch.where(self.has, self.target_logit - self.most, 0.0))
        B.adagc_linear_logprobs_backward(x, w, self.t, stats, d, d_x, d_w, accumulate=accumulate,
                                         workspace=workspace(B.adagc_linear_logprobs_backward_workspace_bytes(self.rows, self.vocab, self.dim, code)))


def check_certain(rows, vocab, dim, name, seed=1):
    dtype = TYPES[name]
    for bits, bits_d in BITS[name]:
        for payload in ("x", "w"):
            c = Certain(rows, vocab, dim, dtype, seed)
            of = c.x if payload == "x" else c.w
            of[:, c.CODE:] = numbers(of.shape[0], dim - c.CODE, bits, c.g)
            if payload == "w":
                c.w[:c.with_target, c.CODE:] = 0.0                               # the certain tokens': a difference of two would not be exact
            d = numbers(1, rows, bits_d, c.g)[0]
            d_x, d_w = torch.full((rows, dim), 77.0, dtype=dtype, device=DEV), torch.full((vocab, dim), 77.0, dtype=dtype, device=DEV)
            c.gradients(d, d_x, d_w)
            d = torch.where(c.has, d, 0.0).double()[:, None]
            want = d * (c.w.double()[c.t] - c.w.double()[c.own])
            assert torch.equal(d_x.double(), want), (bits, bits_d, payload, "d_x", float((d_x.double() - want).abs().max()))
            want = torch.zeros(vocab, dim, dtype=torch.float64, device=DEV)
            dx = d * c.x.double()
            want[c.t[c.has]] = dx[c.has]
            want[c.own[c.has]] = -dx[c.has]
            assert torch.equal(d_w.double(), want), (bits, bits_d, payload, "d_w", float((d_w.double() - want).abs().max()))
            del want, dx


@pytest.mark.parametrize("rows, vocab, dim", [(4096, 8193, 256), (4096, 8200, 256), (4096, 8312, 256), (4096, 8313, 256), (16500, 2049, 200), (16500, 2100, 130),
                                              (512, 65600, 1024), (2650, 50257, 512), (300, 32770, 1024)])
def test_gradients_of_a_short_last_piece_of_the_vocabulary(rows, vocab, dim):
    """fp32 operands in parts, the last piece of 1 to 121 tokens: fewer than a tile has, and a few more than its products have to have."""
    check_certain(rows, vocab, dim, "f32")


def test_input_gradient_from_very_many_gated_columns():
    """fp32, rows of d_g and d_u 2^23 numbers apart and more, beyond the 32-bit offsets of the tiles that take parts.  Gates of 64, whose sigmoid is 1:
    d_u = 64 d_out; ups of 0: d_g = 0."""
    rows, dim, hidden = 128, 128, 2 ** 23 + 5
    g = gen(3)
    x = torch.randn(rows, dim, generator=g, device=DEV)
    w_gate, w_up = (torch.randn(hidden, dim, generator=g, device=DEV) for _ in range(2))
    own = torch.randint(0, hidden, (rows,), generator=g, device=DEV)
    own[:2] = torch.tensor([0, hidden - 1], device=DEV)
    w_up[own] = numbers(rows, dim, 24, g)
    d, d_out = numbers(1, rows, 1, g)[0], torch.zeros(rows, hidden, device=DEV)
    d_out[torch.arange(rows, device=DEV), own] = d
    gate, up = torch.full((rows, hidden), 64.0, device=DEV), torch.zeros(rows, hidden, device=DEV)
    d_x = torch.empty_like(x)
    B.adagc_gated_linear_backward(d_out, x, w_gate, w_up, d_x, gate=gate, up=up,
                                  workspace=torch.empty(B.adagc_gated_linear_backward_workspace_bytes(rows, dim, hidden, B.ADAGC_F32), dtype=torch.uint8, device=DEV))
    assert torch.equal(d_x.double(), 64 * d.double()[:, None] * w_up[own].double())
