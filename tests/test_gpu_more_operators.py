"""The operators that keep nothing between the passes on the GPU against the 64-bit oracle: types, lengths from one, odd sizes, strides, tiles
and splits of every kind, rows that are masked out, special values."""
import math

import pytest
import torch

import more_operators_oracle as O
from paper_2502_11034_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODES = {torch.float32: B.ADAGC_F32, torch.bfloat16: B.ADAGC_BF16}
FILL = 77.0                    # what lies around outputs, and has to stay


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


class Framed:
    """A matrix inside a larger buffer: `offset` elements in, `ld` from row to row, FILL around it."""

    def __init__(self, rows, cols, dtype, ld=None, offset=0, data=None, fill=FILL):
        ld = ld or cols
        self.fill = fill
        self.flat = torch.full((offset + rows * ld + 64,), fill, dtype=dtype, device=DEV)
        self.t = self.flat[offset:offset + rows * ld].view(rows, ld)[:, :cols]
        if data is not None:
            self.t.copy_(data)
        self.outside = torch.ones_like(self.flat, dtype=torch.bool)
        self.outside[offset:offset + rows * ld].view(rows, ld)[:, :cols] = False

    def result(self):
        """The matrix; nothing around it was touched."""
        around = self.flat[self.outside]
        assert torch.isnan(around).all() if math.isnan(self.fill) else (around == self.fill).all()
        return self.t


def workspace(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)          # NaN in both types: its contents must not matter


def near(got, want, off, dtype=torch.float32):
    """|got - want| <= off + half a step of dtype, NaN and infinities in the same places."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    same = (got == want) | torch.isnan(want)
    bound = off + O.half_step(dtype) * (want.abs() + off)
    bad = ~same & ~((got - want).abs() <= bound)
    assert not bad.any(), "%d of %d values off, worst %.3g times the bound" % (int(bad.sum()), bad.numel(), float(((got - want).abs() / bound)[bad].max()))


def matrix(rows, cols, dtype, seed, size=1.0, ld=None, offset=0):
    """Inputs lie between NaN: what is read beyond their rows must not count."""
    return Framed(rows, cols, dtype, ld, offset, torch.randn(rows, cols, generator=gen(seed), device=DEV) * size, fill=math.nan)


def some_targets(rows, vocab, seed):
    t = torch.randint(0, vocab, (rows,), generator=gen(seed), device=DEV)
    none = torch.tensor([-1, -100, vocab, 2 ** 40], device=DEV)
    t[1::3] = none[torch.arange(len(t[1::3]), device=DEV) % 4]
    return t


# ------------------------------------------------------------------------------------------------ log-probabilities from the head's input

def run_linear(x, w, t, scale=1.0, stream=None):
    rows, vocab, dim = x.shape[0], w.shape[0], x.shape[1]
    logprob, stats = torch.full((rows,), FILL, device=DEV), torch.full((rows, 2), FILL, device=DEV)
    B.adagc_linear_logprobs(x, w, t, logprob, stats, scale=scale, stream=stream,
                            workspace=workspace(B.adagc_linear_logprobs_workspace_bytes(rows, vocab, dim, CODES[x.dtype])))
    return logprob, stats


def check_linear(x, w, t, scale=1.0):
    logprob, stats = run_linear(x, w, t, scale)
    want = O.linear_logprobs(x, w, t, scale)
    near(logprob, want["logprob"], want["logprob_off"])
    near(stats[:, 0], want["most"], want["most_off"])
    near(stats[:, 1], want["log_sum"], want["log_sum_off"])
    return stats


def run_linear_backward(x, w, t, stats, d, scale, d_x, d_w, accumulate=False):
    rows, vocab, dim = x.shape[0], w.shape[0], x.shape[1]
    B.adagc_linear_logprobs_backward(x, w, t, stats, d, d_x, d_w, scale=scale, accumulate=accumulate,
                                     workspace=workspace(B.adagc_linear_logprobs_backward_workspace_bytes(rows, vocab, dim, CODES[x.dtype])))


def check_linear_backward(x, w, t, stats, scale=1.0, weight_dtype=None, accumulate=False, ld=None, offset=0, seed=9):
    rows, vocab, dim = x.shape[0], w.shape[0], x.shape[1]
    weight_dtype = weight_dtype or x.dtype
    d = torch.randn(rows, generator=gen(seed), device=DEV)
    old = torch.randn(vocab, dim, generator=gen(seed + 1), device=DEV).to(weight_dtype)
    d_x, d_w = Framed(rows, dim, x.dtype, ld, offset), Framed(vocab, dim, weight_dtype, ld, offset, old if accumulate else None)
    run_linear_backward(x, w, t, stats, d, scale, d_x.t, d_w.t, accumulate)
    want_x, off_x, want_w, off_w = O.linear_logprobs_backward(x, w, t, scale, d, x.dtype)
    near(d_x.result(), want_x, off_x, x.dtype)
    if accumulate:
        want_w, off_w = want_w + old.double(), off_w + O.U32 * (want_w.abs() + old.double().abs())
    near(d_w.result(), want_w, off_w, weight_dtype)


LINEAR_SIZES = [               # rows, vocab, dim, leading dimension and offset beyond the least, scale
    (1, 1, 1, 0, 0, 1.0),
    (2, 3, 5, 1, 1, 0.5),
    (1, 257, 64, 0, 0, 1.0),
    (17, 300, 32, 0, 0, 2.0),
    (16, 1000, 33, 3, 3, 1.0),
    (33, 129, 100, 4, 8, 1.3),
    (130, 127, 72, 8, 8, 1.0),
    (127, 259, 765, 0, 0, 1.0),
    (200, 515, 264, 0, 0, 0.1),
    (64, 5003, 40, 0, 0, 1.0),
    (5, 20011, 136, 0, 0, 1.0),
    (300, 1024, 1000, 0, 0, 1.0),
    (4097, 2051, 72, 0, 0, 1.0),
    (2100, 4100, 264, 0, 0, 1.0),
    (8, 700, 768, 0, 0, 1.0),
    (9, 700, 61, 0, 0, 1.0),
    (16, 17000, 200, 0, 0, 1.0),
    (150, 400, 135, 2, 1, 1.0),
    (128, 128, 128, 0, 0, 1.0),
    (191, 129, 191, 0, 0, 1.25),
    (200, 300, 136, 1, 1, 1.0),
    (200, 300, 200, 8, 4, 1.0),
    (4100, 5000, 136, 0, 0, 1.0),
    (300, 9000, 2100, 0, 0, 1.0),
    (4100, 300, 4200, 0, 0, 1.0),
    (300, 2111, 1001, 3, 1, 1.0),
    (333, 1700, 1000, 0, 0, 1.0),
    (40, 300, 2051, 1, 1, 1.0),
    (130, 200, 4104, 0, 0, 1.0),
    (300, 515, 2090, 0, 0, 1.0),
    (17, 600, 4100, 4, 8, 0.7),
    (600, 700, 4128, 0, 0, 1.0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, dim, more, offset, scale", LINEAR_SIZES)
def test_linear_logprobs_forward_and_backward(dtype, rows, vocab, dim, more, offset, scale):
    dtype = TYPES[dtype]
    x, w = matrix(rows, dim, dtype, 1, 1.5, dim + more, offset).t, matrix(vocab, dim, dtype, 2, dim ** -0.5, dim + more, offset).t
    t = some_targets(rows, vocab, 3)
    stats = check_linear(x, w, t, scale)
    check_linear_backward(x, w, t, stats, scale, ld=dim + more, offset=offset)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weight_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, dim", [(70, 333, 96), (300, 700, 265)])
def test_linear_logprobs_accumulates_and_converts(dtype, weight_dtype, rows, vocab, dim):
    dtype = TYPES[dtype]
    x, w, t = matrix(rows, dim, dtype, 4).t, matrix(vocab, dim, dtype, 5, dim ** -0.5).t, some_targets(rows, vocab, 6)
    stats = check_linear(x, w, t)
    for accumulate in (False, True):
        check_linear_backward(x, w, t, stats, weight_dtype=TYPES[weight_dtype], accumulate=accumulate)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, dim", [(16500, 3900, 24), (33000, 2049, 16), (16500, 3900, 130), (130, 9000, 4001)])
def test_linear_logprobs_in_pieces_of_the_vocabulary(dtype, rows, vocab, dim):
    dtype = TYPES[dtype]
    x, w, t = matrix(rows, dim, dtype, 4).t, matrix(vocab, dim, dtype, 5, 0.3).t, some_targets(rows, vocab, 6)
    stats = check_linear(x, w, t)
    check_linear_backward(x, w, t, stats)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, dim", [(513, 22116, 64), (513, 22116, 130), (1000, 33000, 1032)])
def test_linear_logprobs_of_rounds_that_are_not_full(dtype, rows, vocab, dim):
    """A last round of smaller tiles; few tiles that share a long sum out."""
    dtype = TYPES[dtype]
    x, w, t = matrix(rows, dim, dtype, 4).t, matrix(vocab, dim, dtype, 5, dim ** -0.5).t, some_targets(rows, vocab, 6)
    t[0], t[2], t[3] = vocab - 1, vocab - 200, vocab - 360          # on both sides of where the smaller tiles begin
    stats = check_linear(x, w, t)
    check_linear_backward(x, w, t, stats)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, wide, dim", [(40, 300, 2051), (17, 600, 4100), (300, 2111, 1001), (513, 22116, 64), (70, 300, 136), (9, 70, 33)])
def test_nothing_is_written_beyond_a_workspace(dtype, rows, wide, dim, monkeypatch):
    guard, spaces = 1 << 16, []

    def guarded(n):
        space = torch.full((n + guard,), 0xFF, dtype=torch.uint8, device=DEV)
        space[n:] = 0x5A
        spaces.append(space[n:])
        return space[:n]

    monkeypatch.setitem(globals(), "workspace", guarded)
    dtype = TYPES[dtype]
    x, w, t = matrix(rows, dim, dtype, 4).t, matrix(wide, dim, dtype, 5, dim ** -0.5).t, some_targets(rows, wide, 6)
    stats = check_linear(x, w, t)
    check_linear_backward(x, w, t, stats)
    d_x, d_w = torch.empty_like(x.contiguous()), [torch.empty(wide, dim, device=DEV) for _ in range(2)]
    out, gate, up = run_gated(x, w, w, kept=True)
    run_gated_backward(out, x, w, w, d_x, *d_w)
    run_gated_backward(out, x, w, w, d_x, *d_w, gate=gate, up=up)
    assert all(bool((space == 0x5A).all()) for space in spaces) and len(spaces) >= 4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, dim", [(19, 70, 40), (140, 900, 264), (4096, 2048, 64)])
def test_products_of_whole_numbers_are_exact(dtype, rows, vocab, dim):
    """Small whole numbers: every sum is exact, whatever its order, and a place that is missed or counted twice shows."""
    dtype = TYPES[dtype]
    x = torch.randint(-3, 4, (rows, dim), generator=gen(1), device=DEV).to(dtype)
    w = torch.randint(-3, 4, (vocab, dim), generator=gen(2), device=DEV).to(dtype)
    t = torch.arange(rows, device=DEV) * 7 % vocab
    logprob, stats = run_linear(x, w, t)
    z = x.double() @ w.double().t()
    assert torch.equal(stats[:, 0].double(), z.amax(1))
    # log p + L + M is the target's logit, but for the roundings of three sums
    back = logprob.double() + stats[:, 1].double() + stats[:, 0].double()
    own = z.gather(1, t[:, None])[:, 0]
    assert ((back - own).abs() <= 4 * O.U32 * (logprob.double().abs() + own.abs() + stats[:, 1].double().abs())).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_logprobs_special_rows(dtype):
    dtype = TYPES[dtype]
    rows, vocab, dim = 140, 300, 48
    x, w = torch.rand(rows, dim, generator=gen(1), device=DEV) + 0.1, torch.randn(vocab, dim, generator=gen(2), device=DEV)
    w[:, 0], x[:, 0] = 0.0, 0.0
    w[:, 0] = 1.0
    x[3, 0] = -math.inf                                   # all logits -inf
    x[4, 0] = math.inf                                    # all +inf
    x[5, 7] = math.nan
    x[6] = 0                                              # all logits equal
    x, w = x.to(dtype), w.to(dtype)
    t = torch.arange(rows, device=DEV) % vocab
    t[7:20] = -1
    logprob, stats = run_linear(x, w, t)
    want = O.linear_logprobs(x, w, t, 1.0)
    plain = torch.tensor([i for i in range(rows) if i not in (3, 4, 5)], device=DEV)
    near(logprob[plain], want["logprob"][plain], want["logprob_off"][plain])
    assert logprob[3] == -math.inf and stats[3, 0] == -math.inf and stats[3, 1] == 0
    assert torch.isnan(logprob[4]) and torch.isnan(logprob[5])
    assert abs(float(logprob[6]) + math.log(vocab)) < 1e-5
    # the rows without a number: 0 for the one of -inf, NaN for the others, and only there
    d = torch.ones(rows, device=DEV)
    d_x, d_w = torch.full_like(x, FILL), torch.full_like(w, FILL)
    run_linear_backward(x, w, t, stats, d, 1.0, d_x, d_w)
    assert (d_x[3] == 0).all() and torch.isnan(d_x[4]).all() and torch.isnan(d_x[5]).all()
    want_x, off_x, _, _ = O.linear_logprobs_backward(x[plain], w, t[plain], 1.0, d[plain], dtype)
    near(d_x[plain], want_x, off_x, dtype)
    assert (d_x[7:20] == 0).all()


@pytest.mark.parametrize("scale, size, d", [(2.0 ** -100, 1e30, 1.0), (2.0 ** 100, 1e-30, 1e3), (1.0, 1e18, 1.0), (2.0 ** 100, 1e-30, 1e9)])
def test_linear_logprobs_far_scales(scale, size, d):
    """Logits near fp32's ends with a scale that brings them back; a gradient whose product with the scale leaves the range."""
    rows, vocab, dim = 9, 40, 4
    x = torch.randn(rows, dim, generator=gen(1), device=DEV)
    w = torch.randn(vocab, dim, generator=gen(2), device=DEV) * size
    t = some_targets(rows, vocab, 3)
    stats = check_linear(x, w, t, scale)
    d = torch.full((rows,), d, device=DEV)
    d_x, d_w = torch.empty_like(x), torch.empty_like(w)
    run_linear_backward(x, w, t, stats, d, scale, d_x, d_w)
    want_x, off_x, want_w, off_w = O.linear_logprobs_backward(x, w, t, scale, d, x.dtype)
    for got, want, off in ((d_x, want_x, off_x), (d_w, want_w, off_w)):
        inside = want.abs() + off < 1e38
        near(torch.where(inside, got, 0.0), torch.where(inside, want, 0.0), off)


def test_linear_logprobs_single_outputs_and_no_rows():
    x, w, t = matrix(6, 40, torch.bfloat16, 1).t, matrix(90, 40, torch.bfloat16, 2, 0.2).t, some_targets(6, 90, 3)
    logprob, stats = run_linear(x, w, t)
    ws = workspace(B.adagc_linear_logprobs_workspace_bytes(6, 90, 40, B.ADAGC_BF16))
    alone, alone_stats = torch.empty(6, device=DEV), torch.empty(6, 2, device=DEV)
    B.adagc_linear_logprobs(x, w, t, alone, workspace=ws)
    B.adagc_linear_logprobs(x, w, None, None, alone_stats, workspace=ws)
    assert torch.equal(alone, logprob) and torch.equal(alone_stats, stats)
    d = torch.ones(6, device=DEV)
    d_x, d_w = torch.empty_like(x), torch.empty_like(w)
    run_linear_backward(x, w, t, stats, d, 1.0, d_x, d_w)
    for only_x in (True, False):
        a, b = torch.full_like(x, FILL), torch.full_like(w, FILL)
        run_linear_backward(x, w, t, stats, d, 1.0, a if only_x else None, None if only_x else b)
        assert torch.equal(a, d_x) if only_x else torch.equal(b, d_w)
    none = torch.empty(0, 40, device=DEV, dtype=torch.bfloat16)
    B.adagc_linear_logprobs(none, w, t[:0], alone[:0], alone_stats[:0])
    for accumulate in (True, False):
        d_w = torch.full_like(w, 3.0)
        run_linear_backward(none, w, t[:0], alone_stats[:0], d[:0], 1.0, None, d_w, accumulate)
        assert (d_w == (3.0 if accumulate else 0.0)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [5, 20])
def test_rows_far_apart(dtype, rows):
    """Offsets within a tile, and of 32 rows, beyond 32 bits of bytes."""
    dtype = TYPES[dtype]
    vocab, dim, ld = 24, 40, 2 ** 25 + 8
    x, w = matrix(rows, dim, dtype, 1).t, matrix(vocab, dim, dtype, 2, 0.3, ld).t
    t = some_targets(rows, vocab, 3)
    stats = check_linear(x, w, t)
    check_linear_backward(x, w, t, stats)
    far = matrix(rows, dim, dtype, 1, 1.0, ld).t
    assert torch.equal(far, x)
    for a, b in zip(run_linear(far, w, t), run_linear(x, w, t)):
        assert torch.equal(a, b)
    check_linear_backward(far, w, t, stats)


def test_linear_logprobs_gradient_against_differences():
    """The loss sum(d log p) along a direction in x and W: differences of the forward pass in fp32."""
    rows, vocab, dim = 12, 50, 24
    x, w, t = matrix(rows, dim, torch.float32, 1).t.clone(), matrix(vocab, dim, torch.float32, 2, 0.4).t.clone(), some_targets(rows, vocab, 3)
    d = torch.randn(rows, generator=gen(4), device=DEV)
    _, stats = run_linear(x, w, t, 1.25)
    d_x, d_w = torch.empty_like(x), torch.empty_like(w)
    run_linear_backward(x, w, t, stats, d, 1.25, d_x, d_w)
    to_x, to_w = torch.randn(x.shape, generator=gen(5), device=DEV), torch.randn(w.shape, generator=gen(6), device=DEV)
    h = 2.0 ** -9

    def loss(s):
        return float((run_linear(x + s * h * to_x, w + s * h * to_w, t, 1.25)[0].double() * d.double()).sum())

    slope = (loss(1) - loss(-1)) / (2 * h)
    want = float((d_x.double() * to_x).sum() + (d_w.double() * to_w).sum())
    # a difference of sums of 8 log-probabilities below 2^4 in fp32, each off by some 2^-19, over 2^-8; the third derivative over six by h^2
    assert abs(slope - want) <= 0.02 * (1 + abs(want))


# ------------------------------------------------------------------------------------------------ gated projections

def run_gated(x, w_gate, w_up, ld=None, offset=0, kept=False, stream=None):
    rows, hidden, dim = x.shape[0], w_gate.shape[0], x.shape[1]
    out, gate, up = (Framed(rows, hidden, x.dtype, ld, offset) for _ in range(3))
    n = B.adagc_gated_linear_workspace_bytes(rows, dim, hidden, CODES[x.dtype])
    B.adagc_gated_linear(x, w_gate, w_up, out.t, gate.t if kept else None, up.t if kept else None, workspace=workspace(n) if n else None, stream=stream)
    return out.result(), gate.result(), up.result()


def run_gated_backward(d_out, x, w_gate, w_up, d_x, d_w_gate, d_w_up, **how):
    rows, hidden, dim = x.shape[0], w_gate.shape[0], x.shape[1]
    ws = workspace(B.adagc_gated_linear_backward_workspace_bytes(rows, dim, hidden, CODES[x.dtype]))
    B.adagc_gated_linear_backward(d_out, x, w_gate, w_up, d_x, d_w_gate, d_w_up, workspace=ws, **how)


GATED_SIZES = [                # rows, dim, hidden, more, offset
    (1, 1, 1, 0, 0),
    (2, 5, 3, 1, 1),
    (1, 64, 257, 0, 0),
    (15, 100, 16, 0, 0),
    (24, 264, 96, 8, 8),
    (33, 40, 130, 3, 5),
    (64, 768, 200, 0, 0),
    (129, 765, 333, 0, 0),
    (200, 136, 519, 0, 0),
    (300, 1000, 264, 0, 0),
    (4097, 72, 1031, 0, 0),
    (2060, 264, 2056, 0, 0),
    (3, 40, 9001, 0, 0),
    (8, 768, 512, 0, 0),
    (16, 61, 700, 0, 0),
    (150, 135, 400, 1, 1),
    (128, 128, 128, 0, 0),
    (191, 191, 129, 0, 0),
    (200, 136, 300, 1, 1),
    (200, 200, 304, 8, 4),
    (4100, 136, 2600, 0, 0),
    (300, 2100, 4500, 0, 0),
    (400, 1001, 1403, 3, 1),
    (50, 2051, 130, 1, 1),
    (200, 4104, 77, 0, 0),
    (130, 4100, 260, 4, 8),
    (600, 4128, 300, 0, 0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, dim, hidden, more, offset", GATED_SIZES)
def test_gated_linear_forward_and_backward(dtype, rows, dim, hidden, more, offset):
    dtype = TYPES[dtype]
    x = matrix(rows, dim, dtype, 1, 1.0, dim + more, offset).t
    w_gate, w_up = (matrix(hidden, dim, dtype, s, dim ** -0.5, dim + more, offset).t for s in (2, 3))
    want = O.gated_linear(x, w_gate, w_up)
    out, _, _ = run_gated(x, w_gate, w_up, hidden + more, offset)
    near(out, want["out"], want["out_off"], dtype)
    out_too, gate, up = run_gated(x, w_gate, w_up, hidden + more, offset, kept=True)
    assert torch.equal(out, out_too)
    near(gate, want["g"], want["g_off"], dtype)
    near(up, want["u"], want["u_off"], dtype)
    d_out = matrix(rows, hidden, dtype, 4, 1.0, hidden + more, offset).t
    for kept in (False, True):
        g, g_off, u, u_off = (gate.double(), 0.0, up.double(), 0.0) if kept else (want["g"], want["g_off"], want["u"], want["u_off"])
        d_x, d_w_gate, d_w_up = (Framed(r, dim, dtype, dim + more, offset) for r in (rows, hidden, hidden))
        again = Framed(rows, hidden, dtype, hidden + more, offset)
        run_gated_backward(d_out, x, w_gate, w_up, d_x.t, d_w_gate.t, d_w_up.t, gate=gate if kept else None, up=up if kept else None, out=again.t)
        back = O.gated_linear_backward(g, torch.as_tensor(g_off, device=DEV), u, torch.as_tensor(u_off, device=DEV), x, w_gate, w_up, d_out, dtype)
        near(d_x.result(), back["d_x"], back["d_x_off"], dtype)
        near(d_w_gate.result(), back["d_w_gate"], back["d_w_gate_off"], dtype)
        near(d_w_up.result(), back["d_w_up"], back["d_w_up_off"], dtype)
        few = (14 + 3 * g.abs()) * O.U32
        silu = g * torch.sigmoid(g)
        near(again.result(), silu * u, (silu * u).abs() * few + 1.1 * g_off * (u.abs() + u_off) + silu.abs() * u_off, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weight_dtype", ["f32", "bf16"])
def test_gated_linear_accumulates_and_takes_halves_of_one_matrix(dtype, weight_dtype):
    dtype, weight_dtype = TYPES[dtype], TYPES[weight_dtype]
    rows, dim, hidden = 90, 136, 200
    x, d_out = matrix(rows, dim, dtype, 1).t, matrix(rows, hidden, dtype, 4).t
    both = matrix(2 * hidden, dim, dtype, 2, dim ** -0.5).t
    w_gate, w_up = both[:hidden], both[hidden:]
    want = O.gated_linear(x, w_gate, w_up)
    back = O.gated_linear_backward(want["g"], want["g_off"], want["u"], want["u_off"], x, w_gate, w_up, d_out, dtype)
    for accumulate in (False, True):
        grads = torch.randn(2 * hidden, dim, generator=gen(7), device=DEV).to(weight_dtype)
        old = grads.double() if accumulate else torch.zeros_like(grads, dtype=torch.float64)
        run_gated_backward(d_out, x, w_gate, w_up, None, grads[:hidden], grads[hidden:], accumulate=accumulate)
        for got, name, o in ((grads[:hidden], "d_w_gate", old[:hidden]), (grads[hidden:], "d_w_up", old[hidden:])):
            near(got, back[name] + o, back[name + "_off"] + O.U32 * (back[name].abs() + o.abs()), weight_dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gated_linear_special_gates(dtype):
    """Gates from -inf to inf, at and beyond where the sigmoid is 0 or 1; the other products stay what they are."""
    dtype = TYPES[dtype]
    values = [-math.inf, -1e30, -200.0, -120.0, -88.0, -80.0, -20.0, -1.0, -0.0, 0.0, 1e-30, 1.0, 20.0, 88.0, 120.0, 1e30, math.inf, math.nan]
    rows = len(values)
    x = torch.zeros(rows, 8, device=DEV)
    x[:, 0], x[:, 1] = torch.tensor(values, device=DEV), 0.5
    x = x.to(dtype)
    w_gate, w_up, d_out = torch.zeros(5, 8, device=DEV, dtype=dtype), torch.zeros(5, 8, device=DEV, dtype=dtype), torch.ones(rows, 5, device=DEV, dtype=dtype)
    w_gate[2, 0] = 1.0                                    # (0 times an infinity is no number: only column 2 is looked at for those)
    w_up[:, 1] = 3.0
    finite = torch.isfinite(x[:, 0])
    g = x[:, 0].double()
    t = torch.sigmoid(g)
    small = g < -87.0                                     # counted as 0, or as it is
    off = 1.5 * 90 * math.exp(-87.0)
    out, _, _ = run_gated(x, w_gate, w_up)
    want = g * t * 1.5
    near(out[finite, 2], want[finite], want[finite].abs() * (14 + 3 * g[finite].abs().clamp(max=90)) * O.U32 + torch.where(small[finite], off, 0.0), dtype)
    d_x = torch.empty_like(x)
    again = torch.empty_like(d_out)
    x2 = torch.where(torch.isfinite(x), x, 0.0)           # (the weights' gradients would be 0 times inf)
    for gate in (None, True):
        kept = {} if gate is None else {"gate": x[:, :1].expand(rows, 5).contiguous(), "up": torch.full_like(d_out, 1.5)}
        run_gated_backward(d_out, x2 if gate else x, w_gate, w_up, d_x, None, None, out=again, **kept)
        assert torch.isnan(again[-1, 2])
        if gate:
            # every column has the gate: -inf and below -88 give 0, inf gives inf
            assert (again[:4] == 0).all() and (again[-2] == math.inf).all()
            # d_x[:, 1] = 3 sum over 5 columns of d_u = 15 g t
            near(d_x[4:-2, 1], 15 * (g * t)[4:-2], 15 * (g * t)[4:-2].abs() * (O.half_step(dtype) + 300 * O.U32) + 10 * off, dtype)
            assert (d_x[:4, 1] == 0).all() and d_x[-2, 1] == math.inf and torch.isnan(d_x[-1, 1])


def test_gated_linear_no_rows():
    none, w = torch.empty(0, 24, device=DEV), torch.randn(40, 24, device=DEV)
    B.adagc_gated_linear(none, w, w, torch.empty(0, 40, device=DEV))
    for accumulate in (True, False):
        a, b = torch.full_like(w, 3.0), torch.full_like(w, 3.0)
        run_gated_backward(torch.empty(0, 40, device=DEV), none, w, w, None, a, b, accumulate=accumulate)
        assert (a == (3.0 if accumulate else 0.0)).all() and (b == a).all()


def test_gated_linear_gradient_against_differences():
    rows, dim, hidden = 11, 20, 30
    x, d_out = matrix(rows, dim, torch.float32, 1).t.clone(), matrix(rows, hidden, torch.float32, 4).t.clone()
    weights = [matrix(hidden, dim, torch.float32, s, 0.4).t.clone() for s in (2, 3)]
    grads = [torch.empty_like(x)] + [torch.empty_like(w) for w in weights]
    run_gated_backward(d_out, x, *weights, *grads)
    to = [torch.randn(g.shape, generator=gen(5 + i), device=DEV) for i, g in enumerate(grads)]
    h = 2.0 ** -9

    def loss(s):
        a = [v + s * h * d for v, d in zip([x] + weights, to)]
        return float((run_gated(*a)[0].double() * d_out.double()).sum())

    slope, want = (loss(1) - loss(-1)) / (2 * h), float(sum((g.double() * d).sum() for g, d in zip(grads, to)))
    # a difference of 330 products of some 2^3 in fp32, each off by 2^-20, over 2^-8, and the third derivative over six by h^2
    assert abs(slope - want) <= 0.02 * (1 + abs(want))


# ------------------------------------------------------------------------------------------------ dropout

def state(seed, offset):
    signed = [v - 2 ** 64 if v >= 2 ** 63 else v for v in (seed, offset)]
    return torch.tensor(signed, dtype=torch.int64, device=DEV)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols, more, offset", [(1, 1, 0, 0), (3, 2, 1, 1), (5, 7, 2, 3), (2, 8, 0, 0), (9, 33, 0, 1), (4, 131, 5, 0), (17, 256, 8, 8), (3, 1027, 0, 0)])
@pytest.mark.parametrize("p, seed, first", [(0.1, 1, 0), (0.5, 2 ** 63 + 12345678901, 2 ** 32 - 3), (0.0, 5, 2 ** 64 - 2), (1.0, 7, 9), (2.0 ** -32, 3, 2 ** 63)])
def test_dropout(dtype, rows, cols, more, offset, p, seed, first):
    dtype = TYPES[dtype]
    x, residual = matrix(rows, cols, dtype, 1, 1.0, cols + more, offset).t, matrix(rows, cols, dtype, 2, 2.0, cols + more, offset).t
    for r in (None, residual):
        out = Framed(rows, cols, dtype, cols + more, offset)
        B.adagc_dropout(x, out.t, state(seed, first), p, residual=r)
        want = O.dropout(x.cpu(), p, seed, first, None if r is None else r.cpu()).to(DEV)
        # rounded once in fp32 and once in its type; 64 bits hold the sum but for 2^-53 of its parts
        off = O.U32 * want.abs() + 2.0 ** -52 * (want.abs() + 4)
        near(out.result(), want, off if dtype == torch.bfloat16 else 2.0 ** -52 * (want.abs() + 4), dtype)


def test_dropout_in_place_and_dropped_values_that_are_no_numbers():
    rows, cols = 6, 50
    x = torch.full((rows, cols), math.nan, device=DEV)
    residual = torch.randn(rows, cols, generator=gen(1), device=DEV)
    kept = O.keep(rows, cols, 0.5, 11, 3).to(DEV)
    x[kept] = 2.0
    want = residual + torch.where(kept, 4.0, 0.0)
    for where in ("apart", "x", "residual"):
        a, r = x.clone(), residual.clone()
        out = {"apart": torch.empty_like(a), "x": a, "residual": r}[where]
        B.adagc_dropout(a, out, state(11, 3), 0.5, residual=r)
        assert torch.equal(out, want)


def test_dropout_keeps_as_many_as_it_should():
    rows, cols, p = 512, 4096, 0.3
    out = torch.empty(rows, cols, device=DEV)
    B.adagc_dropout(torch.ones(rows, cols, device=DEV), out, state(1234, 0), p)
    n = rows * cols
    kept = int((out > 0).sum())
    assert abs(kept - n * (1 - p)) < 6 * math.sqrt(n * p * (1 - p))          # six standard deviations
    assert ((out == 0) | (out == torch.tensor(1 / (1 - p)))).all()


# ------------------------------------------------------------------------------------------------ how calls are made

def test_calls_on_a_stream_and_replayed_graphs():
    """All operators in one graph on a stream of its own: replays with new data and a new offset give what eager calls give, with eager work
    in between."""
    rows, dim, hidden, vocab, dtype = 70, 72, 200, 600, torch.bfloat16
    g = gen(1)
    x, wg, wu, wd, wo = (torch.randn(*s, generator=g, device=DEV).to(dtype) for s in ((rows, dim), (hidden, dim), (hidden, dim), (dim, hidden), (vocab, dim)))
    t = some_targets(rows, vocab, 3)
    rng = state(5, 0)
    d = torch.randn(rows, generator=g, device=DEV)
    ws = workspace(max(B.adagc_linear_logprobs_workspace_bytes(rows, vocab, dim, B.ADAGC_BF16),
                       B.adagc_linear_logprobs_backward_workspace_bytes(rows, vocab, dim, B.ADAGC_BF16),
                       B.adagc_gated_linear_workspace_bytes(rows, dim, hidden, B.ADAGC_BF16),
                       B.adagc_gated_linear_backward_workspace_bytes(rows, dim, hidden, B.ADAGC_BF16)))

    def buffers():
        return {"a": torch.empty(rows, hidden, device=DEV, dtype=dtype), "y": torch.empty_like(x), "logprob": torch.empty(rows, device=DEV),
                "stats": torch.empty(rows, 2, device=DEV), "d_y": torch.empty_like(x), "d_wo": torch.empty_like(wo), "d_a": torch.empty(rows, hidden, device=DEV, dtype=dtype),
                "d_x": torch.empty_like(x), "d_wg": torch.empty_like(wg), "d_wu": torch.empty_like(wu)}

    def run(b, stream):
        B.adagc_gated_linear(x, wg, wu, b["a"], workspace=ws, stream=stream)
        B.adagc_dropout(x, b["y"], rng, 0.2, residual=x, stream=stream)
        B.adagc_linear_logprobs(b["y"], wo, t, b["logprob"], b["stats"], scale=0.1, workspace=ws, stream=stream)
        B.adagc_linear_logprobs_backward(b["y"], wo, t, b["stats"], d, b["d_y"], b["d_wo"], scale=0.1, workspace=ws, stream=stream)
        B.adagc_dropout(b["a"], b["d_a"], rng, 0.2, stream=stream)
        B.adagc_gated_linear_backward(b["d_a"], x, wg, wu, b["d_x"], b["d_wg"], b["d_wu"], workspace=ws, stream=stream)

    stream = torch.cuda.Stream()
    captured, eager = buffers(), buffers()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        run(captured, stream.cuda_stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run(captured, stream.cuda_stream)
    for i in range(4):
        x.copy_(torch.randn(rows, dim, generator=g, device=DEV).to(dtype))
        rng[1] = 1000 * i
        for b in captured.values():
            b.fill_(FILL)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        run(eager, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for name in captured:
            assert torch.equal(captured[name], eager[name]), (i, name)


def test_results_repeat_bit_for_bit():
    rows, vocab, dim = 700, 3000, 264
    x, w, t = matrix(rows, dim, torch.bfloat16, 1).t, matrix(vocab, dim, torch.bfloat16, 2, 0.1).t, some_targets(rows, vocab, 3)
    d = torch.randn(rows, generator=gen(4), device=DEV)
    first = None
    for _ in range(3):
        logprob, stats = run_linear(x, w, t)
        d_x, d_w = torch.empty_like(x), torch.empty_like(w)
        run_linear_backward(x, w, t, stats, d, 1.0, d_x, d_w)
        now = [logprob, stats, d_x, d_w]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
        first = now


# ------------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_training_step_with_all_of_them(dtype):
    """x -> gated projections -> down product -> dropout and residual -> log-probabilities, back, and the AdaGC step on the gradients:
    against 64-bit automatic differentiation on the same data, with a run of the step's gradients in the Frobenius norm."""
    dtype = TYPES[dtype]
    rows, dim, hidden, vocab, p = 150, 136, 200, 700, 0.2
    code = CODES[dtype]
    x, wg, wu, wd, wo = (matrix(r, c, dtype, i, c ** -0.5 if i else 1.0).t for i, (r, c) in
                         enumerate(((rows, dim), (hidden, dim), (hidden, dim), (dim, hidden), (vocab, dim))))
    t, rng = some_targets(rows, vocab, 8), state(77, 5)
    d_logprob = torch.full((rows,), -1.0 / rows, device=DEV)
    ws = workspace(max(B.adagc_linear_logprobs_workspace_bytes(rows, vocab, dim, code), B.adagc_linear_logprobs_backward_workspace_bytes(rows, vocab, dim, code),
                       B.adagc_gated_linear_workspace_bytes(rows, dim, hidden, code), B.adagc_gated_linear_backward_workspace_bytes(rows, dim, hidden, code)))
    a, h1, dh1, dy, dx = torch.empty(rows, hidden, device=DEV, dtype=dtype), *(torch.empty(rows, dim, device=DEV, dtype=dtype) for _ in range(4))
    logprob, stats = torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
    grads = [torch.empty(w.shape, device=DEV) for w in (wg, wu, wd, wo)]
    B.adagc_gated_linear(x, wg, wu, a, workspace=ws)
    y = a @ wd.t()
    B.adagc_dropout(y, h1, rng, p, residual=x)
    B.adagc_linear_logprobs(h1, wo, t, logprob, stats, workspace=ws)
    B.adagc_linear_logprobs_backward(h1, wo, t, stats, d_logprob, dh1, grads[3], workspace=ws)
    B.adagc_dropout(dh1, dy, rng, p)
    da = dy @ wd
    again = torch.empty_like(a)
    B.adagc_gated_linear_backward(da, x, wg, wu, dx, grads[0], grads[1], out=again, workspace=ws)
    grads[2].copy_(dy.t().float() @ a.float())
    assert torch.equal(again, a)
    leaves = [v.cpu().double().requires_grad_() for v in (x, wg, wu, wd, wo)]
    kept = O.keep(rows, dim, p, 77, 5)
    hidden64 = torch.nn.functional.silu(leaves[0] @ leaves[1].t()) * (leaves[0] @ leaves[2].t())
    h = leaves[0] + torch.where(kept, hidden64 @ leaves[3].t() / (1 - p), 0.0)
    logp = torch.log_softmax(h @ leaves[4].t(), 1)
    has = (t >= 0) & (t < vocab)
    at = torch.where(has, t, 0).cpu()[:, None]
    own = torch.where(has.cpu(), logp.gather(1, at)[:, 0], 0.0)
    (-own.sum() / rows).backward()
    # a handful of roundings to the type, each half a step of values of size up to 5, and what fp32 adds
    u = O.half_step(dtype)
    assert (logprob.cpu().double() - own).abs().max() < 40 * u + 300 * O.U32 * 8
    for got, leaf in zip(grads, leaves[1:]):
        assert (got.cpu().double() - leaf.grad).norm() <= (10 * u + 600 * O.U32) * leaf.grad.norm()
    assert ((dx.cpu().double() + dh1.cpu().double()) - leaves[0].grad).norm() <= (10 * u + 600 * O.U32) * leaves[0].grad.norm()
    # the step takes them
    params = [w.float().clone() for w in (wg, wu, wd, wo)]
    before = [q.clone() for q in params]
    m, v = ([torch.zeros_like(q) for q in params] for _ in range(2))
    opt = B.AdaGC([q.numel() for q in params], B.ADAGC_OPT_ADAMW, B.ADAGC_GRAD_F32)
    opt.step(params, grads, m, v, torch.zeros(4, device=DEV), B.make_hyper(lr=1e-3, weight_decay=0.0), 1)
    norms, _, _ = opt.get_norms()
    for q, b, g, n in zip(params, before, grads, norms):
        assert abs(float(g.double().norm()) - n) <= 1e-5 * n
        moved = (b - q)[g.abs() > 1e-6]
        assert (moved.sign() == g[g.abs() > 1e-6].sign()).all()


def test_gradients_of_the_example_that_makes_everything_again():
    """Relative bounds in the Frobenius norm: a bf16 value is off by u = 2^-8 of itself at most and half of that in the root of the mean square
    (u / sqrt 3 of a power of two, less above it), and on the way to a gradient lie at most ten of them (a, y, h1, d_z, d_h1, its dropout,
    d_a, d_g or d_u, the result), two of which (h1 and a) enter twice: 6 u if all of them pointed the same way."""
    from paper_2502_11034_amd.example_training import Chain, Model
    p = 0.25
    model, chain = Model(300, 96, 160, 777, seed=3, again=True, dropout=p), Chain(300)
    model.rng[1] = 12
    t, target = chain.pairs(777)
    target[::50] = -1
    logprob = model.gradients(t, target).cpu().double()
    w = [c.cpu().double().requires_grad_() for c in model.copies]
    t, target = t.cpu(), target.cpu()
    h0 = w[0][t]
    kept = O.keep(777, 96, p, 3, 12)
    a = torch.nn.functional.silu(h0 @ w[1].t()) * (h0 @ w[2].t())
    logp = torch.log_softmax((h0 + torch.where(kept, a @ w[3].t() / (1 - p), 0.0)) @ w[4].t(), 1)
    lp = torch.where(target >= 0, logp.gather(1, target.clamp(min=0)[:, None])[:, 0], 0.0)
    (-lp.mean()).backward()
    u = 2.0 ** -8
    assert (logprob - lp).abs().max() < 30 * u           # four roundings of values of size up to 5, summed over a row of weights
    for got, want in zip(model.grads, w):
        got, want = got.cpu().double(), want.grad
        assert (got - want).norm() <= 6 * u * want.norm()


def test_the_example_runs_with_everything_made_again():
    from paper_2502_11034_amd.example_training import Chain, Model, main
    loss = main(["--steps", "5", "--vocab", "128", "--dim", "64", "--hidden", "96", "--tokens", "256", "--again", "--dropout", "0.1"])
    assert math.isfinite(loss)
    with pytest.raises(ValueError):
        Model(128, 64, 96, 256, entropy_weight=0.1, again=True)
    with pytest.raises(ValueError):
        Model(128, 64, 96, 256, dropout=0.1)
