"""Products of the operators that keep nothing between the passes, bit for bit: operands whose sums are exact in fp32 in any order, with numbers
of so many bits that every part of a product counts that is taken as three bf16 numbers (test_exact_products_host.py shows that they tell)."""
import math

import pytest
import torch

from exact_products import BITS, numbers, one_place
from paper_2502_11034_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODES = {torch.float32: B.ADAGC_F32, torch.bfloat16: B.ADAGC_BF16}
U32 = 2.0 ** -24


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def workspace(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)


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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, dim", [(1, 3, 65), (8, 700, 768), (9, 700, 93), (16, 17000, 200), (17, 600, 4100), (33, 129, 100), (40, 300, 2051), (127, 259, 765),
                                              (130, 127, 72), (300, 1024, 1000), (300, 515, 2090), (300, 9000, 2100), (600, 700, 4128), (513, 22116, 130), (4100, 300, 4200),
                                              (4100, 5000, 136), (2100, 4100, 264), (16500, 3900, 130)])
def test_gradients_of_certain_tokens(dtype, rows, vocab, dim):
    check_certain(rows, vocab, dim, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, dim", [(2, 257, 8), (5, 20011, 136), (16, 17000, 200), (20, 5003, 40), (64, 50257, 33), (300, 1024, 1000), (300, 9000, 2100), (513, 22116, 64),
                                              (2100, 4100, 264)])
def test_every_logit_is_counted_once(dtype, rows, vocab, dim):
    """All logits of a row are equal, in the odd rows 0: L = ln vocab, and one logit more or less would change it by 1 / vocab."""
    g = gen(5)
    x, w = torch.randint(-3, 4, (rows, dim), generator=g, device=DEV).to(TYPES[dtype]), torch.randint(-3, 4, (1, dim), generator=g, device=DEV).to(TYPES[dtype])
    x[1::2] = 0
    z = (x.double() * w.double()).sum(1)
    w = w.expand(vocab, dim).contiguous()
    t = torch.arange(rows, device=DEV) * 7 % vocab
    logprob, stats = torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
    B.adagc_linear_logprobs(x, w, t, logprob, stats, workspace=workspace(B.adagc_linear_logprobs_workspace_bytes(rows, vocab, dim, CODES[x.dtype])))
    assert torch.equal(stats[:, 0].double(), z)
    want = math.log(vocab)
    # zeros: sums of ones, which are exact, and a logarithm of two steps; others: exponentials of two half steps and what puts them right, four more, and
    # sums of equal numbers: vocab / 256 + 24 additions one after another
    off = torch.full((rows,), 4 * U32 * want, device=DEV, dtype=torch.float64)
    off[0::2] += (vocab / 256 + 24 + 6) * U32
    assert (off < 0.9 / vocab).all()
    assert ((stats[:, 1].double() - want).abs() <= off).all() and ((logprob.double() + want).abs() <= off).all()


# rows, dim, hidden; fp32: from 193 rows (backward 128) and 2^29 multiplications on in parts
GATED = [(8, 768, 512), (16, 61, 700), (24, 264, 96), (33, 40, 130), (129, 765, 333), (300, 72, 64), (300, 1000, 264), (200, 1001, 2700), (193, 130, 22000), (200, 4128, 700),
         (600, 4104, 300), (1100, 1000, 600), (4097, 72, 1031), (4100, 136, 2600), (2060, 264, 2056), (1030, 4096, 4096)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, dim, hidden", GATED)
def test_gated_projections(dtype, rows, dim, hidden):
    """Rows of x, or of the weights, have one number: both products, which are left in gate and up, are single products."""
    code, kind, g = CODES[TYPES[dtype]], TYPES[dtype], gen(6)
    for one in ("x", "w"):
        for bits, other in BITS[dtype]:
            if one == "x":
                at, x = one_place(rows, dim, bits, g)
                weights = [numbers(hidden, dim, other, g) for _ in range(2)]
                want = [x.double().gather(1, at[:, None]) * w.double()[:, at].t() for w in weights]
            else:
                x = numbers(rows, dim, bits, g)
                placed = [one_place(hidden, dim, other, g) for _ in range(2)]
                placed[1] = ((placed[1][0] + 1) % dim, placed[1][1].roll(1, 1))            # other places than the gate's
                weights = [w for _, w in placed]
                want = [x.double()[:, at] * w.double().gather(1, at[:, None])[:, 0] for at, w in placed]
            out, gate, up = (torch.full((rows, hidden), 77.0, dtype=kind, device=DEV) for _ in range(3))
            B.adagc_gated_linear(x.to(kind), weights[0].to(kind), weights[1].to(kind), out, gate, up,
                                 workspace=workspace(B.adagc_gated_linear_workspace_bytes(rows, dim, hidden, code)))
            assert torch.equal(gate.double(), want[0]) and torch.equal(up.double(), want[1]), (one, bits, other)


def gated_backward(d_out, x, w_gate, w_up, d_x, d_w_gate, d_w_up, up):
    """Gates of 64, whose sigmoid is 1 and slope 1, kept: d_u = 64 d_out, and d_g = up d_out."""
    rows, hidden = d_out.shape
    gate, up = torch.full_like(d_out, 64.0), torch.full_like(d_out, up)
    B.adagc_gated_linear_backward(d_out, x, w_gate, w_up, d_x, d_w_gate, d_w_up, gate=gate, up=up,
                                  workspace=workspace(B.adagc_gated_linear_backward_workspace_bytes(rows, x.shape[1], hidden, CODES[x.dtype])))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, dim, hidden", GATED)
def test_gated_gradients(dtype, rows, dim, hidden):
    kind, g = TYPES[dtype], gen(7)
    for bits, other in BITS[dtype]:
        w_gate, w_up = (numbers(hidden, dim, bits, g) for _ in range(2))
        # d_x: a row has a gradient in one column ...
        at, d = one_place(rows, hidden, other, g)
        own = d.double().gather(1, at[:, None])
        for up, a, b, want in ((0.0, w_gate, w_up, 64 * own * w_up.double()[at]), (1.0, w_gate, torch.zeros_like(w_up), own * w_gate.double()[at])):
            d_x = torch.full((rows, dim), 77.0, dtype=kind, device=DEV)
            gated_backward(d.to(kind), torch.zeros_like(d_x), a.to(kind), b.to(kind), d_x, None, None, up)
            assert torch.equal(d_x.double(), want), (bits, other, up)
        # ... or in all, and a column of a weight one number
        at, of_column = one_place(dim, hidden, bits, g)
        w = of_column.t().contiguous()
        d = numbers(rows, hidden, other, g)
        d_x = torch.full((rows, dim), 77.0, dtype=kind, device=DEV)
        gated_backward(d.to(kind), torch.zeros_like(d_x), w_gate.to(kind), w.to(kind), d_x, None, None, 0.0)
        assert torch.equal(d_x.double(), 64 * d.double()[:, at] * of_column.double().gather(1, at[:, None])[:, 0]), (bits, other)
        # the weights' gradients: a column's gradient is in one row ...
        x, w = numbers(rows, dim, bits, g), torch.zeros(hidden, dim, dtype=kind, device=DEV)
        at, of_column = one_place(hidden, rows, other, g)
        d_gate, d_up = (torch.full((hidden, dim), 77.0, dtype=kind, device=DEV) for _ in range(2))
        gated_backward(of_column.t().contiguous().to(kind), x.to(kind), w, w, None, d_gate, d_up, 1.0)
        want = of_column.double().gather(1, at[:, None]) * x.double()[at]
        assert torch.equal(d_gate.double(), want) and torch.equal(d_up.double(), 64 * want), (bits, other)
        # ... or in all, and a column of x one number
        at, of_column = one_place(dim, rows, bits, g)
        d = numbers(rows, hidden, other, g)
        gated_backward(d.to(kind), of_column.t().contiguous().to(kind), w, w, None, d_gate, d_up, 1.0)
        want = d.double()[at].t() * of_column.double().gather(1, at[:, None])[:, 0]
        assert torch.equal(d_gate.double(), want) and torch.equal(d_up.double(), 64 * want), (bits, other)


def root_mean_square(got, want, k):
    """fp32 sums of k products in six parts: 6 k additions at most, each off by up to half a step of what has been summed so far, all directions alike: sqrt(1 / 3) of
    half a step in the root of the mean square, of a sum whose square grows evenly: sqrt(6 k / 3 / 2) half steps of the whole.  The products of parts that
    are left out are 2^-26 of it, and the result is rounded: 4 half steps more than cover both."""
    assert (got.double() - want).norm() <= (math.sqrt(k) + 4) * U32 * want.norm()


def test_random_products_in_parts():
    """Dense random operands, where parts of one tile with another's would show everywhere: less than a product of parts left out."""
    g = gen(8)
    rows, dim, hidden = 300, 256, 7100
    x, w_gate, w_up = (torch.randn(*s, generator=g, device=DEV) for s in ((rows, dim), (hidden, dim), (hidden, dim)))
    out, gate, up = (torch.empty(rows, hidden, device=DEV) for _ in range(3))
    B.adagc_gated_linear(x, w_gate, w_up, out, gate, up, workspace=workspace(B.adagc_gated_linear_workspace_bytes(rows, dim, hidden, B.ADAGC_F32)))
    for got, w in ((gate, w_gate), (up, w_up)):
        root_mean_square(got, x.double() @ w.double().t(), dim)
    d, d_w_gate, d_w_up = torch.randn(rows, hidden, generator=g, device=DEV), torch.empty_like(w_gate), torch.empty_like(w_up)
    gated_backward(d, x, w_gate, w_up, None, d_w_gate, d_w_up, 1.0)
    want = d.double().t() @ x.double()
    root_mean_square(d_w_gate, want, rows)
    root_mean_square(d_w_up, 64 * want, rows)
    rows, dim, hidden = 2100, 2100, 129
    x, w = torch.zeros(rows, dim, device=DEV), torch.randn(hidden, dim, generator=g, device=DEV)
    d, d_x = torch.randn(rows, hidden, generator=g, device=DEV), torch.empty(rows, dim, device=DEV)
    gated_backward(d, x, w, w, d_x, None, None, 0.0)
    root_mean_square(d_x, 64 * (d.double() @ w.double()), hidden)


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


def test_rows_that_are_no_numbers_stay_by_themselves_in_parts():
    """fp32 operands in parts: a row of x with an infinity, a NaN, or products beyond the range changes no other row."""
    rows, vocab, dim = 200, 2700, 1001
    g = gen(9)
    x, w = torch.randn(rows, dim, generator=g, device=DEV), torch.randn(vocab, dim, generator=g, device=DEV) * 0.03
    t = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    odd = x.clone()
    odd[3, 7], odd[4, 1000], odd[70, 0], odd[199] = math.inf, -math.inf, math.nan, 3e38
    bad = torch.zeros(rows, dtype=torch.bool, device=DEV)
    bad[[3, 4, 70, 199]] = True
    d = torch.where(bad, 0.0, 1.0)
    results = []
    for a in (x, odd):
        logprob, stats, d_x, d_w = torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV), torch.empty_like(x), torch.empty_like(w)
        B.adagc_linear_logprobs(a, w, t, logprob, stats, workspace=workspace(B.adagc_linear_logprobs_workspace_bytes(rows, vocab, dim, B.ADAGC_F32)))
        B.adagc_linear_logprobs_backward(a, w, t, stats, d, d_x, None, workspace=workspace(B.adagc_linear_logprobs_backward_workspace_bytes(rows, vocab, dim, B.ADAGC_F32)))
        results.append((logprob, stats, d_x))
    for plain, now in zip(*results):
        assert torch.equal(plain[~bad], now[~bad])
    assert torch.isnan(results[1][0][bad][:3]).all() and (results[1][2][bad] == 0).all()


def test_statistics_that_start_at_any_number():
    """Pairs of fp32 numbers 4 bytes from a multiple of 8."""
    rows, vocab, dim = 21, 300, 40
    g = gen(10)
    x, w, t = torch.randn(rows, dim, generator=g, device=DEV), torch.randn(vocab, dim, generator=g, device=DEV), torch.arange(rows, device=DEV)
    space = workspace(max(B.adagc_linear_logprobs_workspace_bytes(rows, vocab, dim, B.ADAGC_F32), B.adagc_linear_logprobs_backward_workspace_bytes(rows, vocab, dim, B.ADAGC_F32)))
    results = []
    for offset in (0, 1):
        buffer = torch.full((2 * rows + 2,), 77.0, device=DEV)
        stats, d_w = buffer[offset:offset + 2 * rows].view(rows, 2), torch.empty_like(w)
        B.adagc_linear_logprobs(x, w, t, None, stats, workspace=space)
        B.adagc_linear_logprobs_backward(x, w, t, stats, torch.ones(rows, device=DEV), None, d_w, workspace=space)
        assert (buffer[:offset] == 77).all() and (buffer[offset + 2 * rows:] == 77).all()
        results.append((stats.clone(), d_w))
    assert all(torch.equal(a, b) for a, b in zip(*results))
