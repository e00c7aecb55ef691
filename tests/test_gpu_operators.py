"""The operators around the step on the GPU against the 64-bit oracle: types, lengths, odd sizes, strides, masks, special values."""
import math

import pytest
import torch

import operators_oracle as O
from paper_2502_11034_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FILL = 77.0                    # what lies around outputs, and has to stay


def gen(seed):
    return torch.Generator().manual_seed(seed)


class Framed:
    """A matrix inside a larger buffer: `offset` elements in, `ld` from row to row, FILL around it."""

    def __init__(self, rows, cols, dtype, ld=None, offset=0, data=None):
        self.ld = ld or cols
        self.flat = torch.full((offset + rows * self.ld + 64,), FILL, dtype=dtype, device=DEV)
        self.t = self.flat[offset:offset + rows * self.ld].view(rows, self.ld)[:, :cols]
        if data is not None:
            self.t.copy_(data)
        self.inside = torch.zeros_like(self.flat, dtype=torch.bool)
        self.inside[offset:offset + rows * self.ld].view(rows, self.ld)[:, :cols] = True

    def result(self):
        """The matrix on the CPU; nothing around it was touched."""
        assert (self.flat[~self.inside] == FILL).all()
        return self.t.cpu()


def workspace(n):
    return torch.full((n,), 0xAB, dtype=torch.uint8, device=DEV)          # its contents must not matter


def near(got, want, off, dtype=torch.float32):
    """|got - want| <= off + half a step of dtype, NaN and infinities in the same places."""
    got, want = got.cpu().double(), want.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    same = (got == want) | torch.isnan(want)
    bound = off + O.half_step(dtype) * (want.abs() + off)
    bad = ~same & ~((got - want).abs() <= bound)
    assert not bad.any(), "%d values off, worst %.3g times the bound" % (int(bad.sum()), float(((got - want).abs() / bound)[bad].max()))


# ------------------------------------------------------------------------------------------------ token log-probabilities

def make_logits(rows, vocab, dtype, seed, size=3.0):
    g = gen(seed)
    z = (torch.randn(rows, vocab, generator=g) * size).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g)
    return z, t


def run_logprobs(z, t, scale=1.0, k=0, ld=None, offset=0, entropy=True, stream=None):
    rows, vocab = z.shape
    zd = Framed(rows, vocab, z.dtype, ld, offset, z)
    out = {"logprob": torch.full((rows,), FILL, device=DEV), "stats": torch.full((rows, 2), FILL, device=DEV)}
    if entropy:
        out["entropy"] = torch.full((rows,), FILL, device=DEV)
    if k:
        out["top_logprob"] = torch.full((rows, k), FILL, device=DEV)
        out["top_index"] = torch.full((rows, k), 7777777, dtype=torch.int32, device=DEV)
    B.adagc_token_logprobs(zd.t, t.to(DEV), scale=scale, workspace=workspace(B.adagc_token_logprobs_workspace_bytes(rows, vocab, k)),
                           stream=stream, **out)
    zd.result()
    return zd, out


def check_logprobs(z, t, scale=1.0, k=0, **how):
    zd, out = run_logprobs(z, t, scale, k, **how)
    want = O.logprobs(z, t, scale)
    near(out["logprob"], want["logprob"], want["logprob_off"])
    near(out["stats"][:, 0], want["most"], 0.0)
    near(out["stats"][:, 1], want["log_sum"], want["log_sum_off"])
    if "entropy" in out:
        near(out["entropy"], want["entropy"], want["entropy_off"])
    if k:
        index = O.top(z, k)
        assert torch.equal(out["top_index"].cpu().long(), index)
        near(out["top_logprob"], want["logp"].gather(1, index), want["logp_off"].gather(1, index))
    return zd, out


def check_backward(z, t, scale, zd, out, ld=None, offset=0, in_place=False, seed=9, d_logprob=True, d_entropy=True):
    rows, vocab = z.shape
    g = gen(seed)
    dl, dh = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    target = zd if in_place else Framed(rows, vocab, z.dtype, ld, offset)
    B.adagc_token_logprobs_backward(zd.t, t.to(DEV) if d_logprob else None, out["stats"], out["entropy"] if d_entropy else None,
                                    dl.to(DEV) if d_logprob else None, dh.to(DEV) if d_entropy else None, target.t, scale=scale)
    zero = torch.zeros(rows)
    want, off = O.logprobs_backward(z, t, scale, dl if d_logprob else zero, dh if d_entropy else zero)
    near(target.result(), want, off, z.dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, k, scale, ld, offset", [
    (1, 1, 1, 1.0, None, 0),
    (3, 2, 2, 0.5, None, 1),
    (5, 7, 3, 1.0, 9, 3),
    (2, 8, 8, 1.0, None, 0),
    (64, 63, 5, 2.0, 64, 1),
    (7, 1023, 20, 1.0, None, 0),
    (33, 1025, 64, 1.3, 1027, 5),
    (4, 8191, 0, 1.0, None, 0),
    (3, 8192, 1, 0.1, None, 0),
    (1, 50257, 5, 1.0, None, 1),
    (9, 50257, 8, 1.25, None, 0),
    (2, 128256, 64, 1.0, None, 0),
    (1030, 4099, 4, 1.0, None, 0),
])
def test_logprobs_forward_and_backward(dtype, rows, vocab, k, scale, ld, offset):
    z, t = make_logits(rows, vocab, TYPES[dtype], rows + vocab)
    t[::3] = torch.tensor([-1, -100, vocab, 2 ** 40])[torch.arange(len(t[::3])) % 4]
    zd, out = check_logprobs(z, t, scale, k, ld=ld, offset=offset)
    check_backward(z, t, scale, zd, out, ld, offset)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab", [(6, 300), (6, 20011)])        # a row in one part and in several
def test_logprobs_masks_and_special_values(dtype, rows, vocab):
    dtype = TYPES[dtype]
    lowest = torch.finfo(dtype).min
    z, t = make_logits(8, vocab, dtype, 4)
    z[0] = -math.inf                                   # nothing left
    z[1, 3:] = -math.inf                               # three left, target masked
    t[1] = vocab - 1
    z[2] = lowest                                      # masks of the type's lowest value: everywhere ...
    z[3, 5:] = lowest                                  # ... and in all but five places
    z[4] = -math.inf
    z[4, vocab - 2] = lowest                           # one left, and it is the lowest
    z[5] = 1.5                                         # ties
    z[6, 17] = torch.finfo(dtype).max
    z[7, ::2] = -math.inf
    zd, out = check_logprobs(z, t, 1.0, 6)
    check_backward(z, t, 1.0, zd, out)
    check_backward(z, t, 1.0, zd, out, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 20011])
def test_logprobs_nan_and_inf(dtype, vocab):
    z, t = make_logits(5, vocab, TYPES[dtype], 5)
    z[0, 7] = math.nan
    z[1, vocab - 1] = math.inf
    z[2] = math.nan
    z[3, 11] = math.nan
    z[3, 12] = -math.inf
    zd, out = run_logprobs(z, t, 1.0, 4)
    for name in ("logprob", "entropy"):
        assert torch.isnan(out[name][:4]).all() and torch.isfinite(out[name][4]), name
    assert torch.isnan(out["top_logprob"][:4]).all()
    index = out["top_index"].cpu().long()
    assert torch.equal(index, O.top(z, 4))
    d = Framed(5, vocab, z.dtype)
    one = torch.ones(5, device=DEV)
    B.adagc_token_logprobs_backward(zd.t, t.to(DEV), out["stats"], out["entropy"], one, one, d.t)
    got = d.result()
    assert torch.isfinite(got[4]).all()
    assert torch.isnan(got[:4]).any(1).all()


def test_logprobs_ties_and_order():
    """Equal values come in index order, whichever lane, vector or part they lie in; ascending rows put every value into the list."""
    vocab = 40007
    z = torch.zeros(4, vocab)
    z[1] = torch.arange(vocab) / 7
    z[2] = -torch.arange(vocab) / 7
    z[3, torch.randperm(vocab, generator=gen(6))[:200]] = 3.0
    z[0, 5] = -0.0
    for rows in (z, z.repeat(300, 1)):
        t = torch.zeros(len(rows), dtype=torch.int64)
        for dtype in (torch.float32, torch.bfloat16):
            _, out = run_logprobs(rows.to(dtype), t, 1.0, 64)
            assert torch.equal(out["top_index"].cpu().long(), O.top(rows.to(dtype), 64))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [7, 1100])                            # rows in several parts and in one
def test_logprobs_top_of_mostly_masked_rows(dtype, rows):
    """Fewer tokens than alternatives asked for, parts without any, ones of the type's lowest value, and masks in front of the rest."""
    dtype, vocab, k = TYPES[dtype], 40007, 20
    g = gen(17)
    z = torch.full((7, vocab), -math.inf, dtype=dtype)
    z[1, torch.randperm(vocab, generator=g)[:5]] = torch.randn(5, generator=g).to(dtype)
    z[2, torch.randperm(vocab, generator=g)[:19]] = torch.finfo(dtype).min
    z[3, 7000:] = torch.randn(vocab - 7000, generator=g).to(dtype)
    z[4, :30000] = torch.randn(30000, generator=g).to(dtype)
    z[5, vocab - 3:] = 1.0
    z[6, ::2] = torch.finfo(dtype).min
    z[6, 3] = math.nan
    z = z.repeat(-(-rows // 7), 1)[:rows]
    _, out = run_logprobs(z, torch.zeros(rows, dtype=torch.int64), 1.0, k)
    assert torch.equal(out["top_index"].cpu().long(), O.top(z[:7], k).repeat(-(-rows // 7), 1)[:rows])
    logp = out["top_logprob"].cpu()
    assert (logp[0] == -math.inf).all() and torch.isnan(logp[6]).all()
    assert (logp[1, 5:] == -math.inf).all() and torch.isfinite(logp[1, :5]).all()


@pytest.mark.parametrize("scale", [1e-3, 50.0])
def test_logprobs_scales(scale):
    z, t = make_logits(6, 5003, torch.float32, 7, size=4.0)
    zd, out = check_logprobs(z, t, scale, 3)
    check_backward(z, t, scale, zd, out)


def test_logprobs_partial_outputs_and_gradients():
    z, t = make_logits(11, 999, torch.bfloat16, 8)
    zd, out = check_logprobs(z, t, 1.0, 0)
    _, without = run_logprobs(z, t, 1.0, 5, entropy=False)
    for name in ("logprob", "stats"):
        near(without[name], out[name].cpu(), 1e-5)                   # another order of moving the reference
    check_backward(z, t, 1.0, zd, out, d_entropy=False)
    check_backward(z, t, 1.0, zd, out, d_logprob=False)
    alone = torch.full((11,), FILL, device=DEV)
    B.adagc_token_logprobs(zd.t, entropy=alone)
    assert torch.equal(alone, out["entropy"])


def test_logprobs_offsets_beyond_32_bits():
    rows, vocab, ld = 3, 301, 2 ** 31 - 1024
    z, t = make_logits(rows, vocab, torch.bfloat16, 10)
    flat = torch.empty((rows - 1) * ld + vocab, dtype=torch.bfloat16, device=DEV)
    zd = flat.as_strided((rows, vocab), (ld, 1))
    zd.copy_(z)
    logprob, entropy, stats = (torch.empty(s, device=DEV) for s in ((rows,), (rows,), (rows, 2)))
    B.adagc_token_logprobs(zd, t.to(DEV), logprob, entropy, stats)
    want = O.logprobs(z, t, 1.0)
    near(logprob, want["logprob"], want["logprob_off"])
    one = torch.ones(rows)
    B.adagc_token_logprobs_backward(zd, t.to(DEV), stats, entropy, one.to(DEV), one.to(DEV), zd)
    grad, off = O.logprobs_backward(z, t, 1.0, one, one)
    near(zd.cpu(), grad, off, torch.bfloat16)


def test_logprobs_rows_of_the_largest_length():
    """A row of 2^31 - 1024 tokens, all but some at its ends masked: the same as a row of those."""
    vocab = 2 ** 31 - 1024
    places = torch.tensor([0, 5, 2 ** 30 + 1, vocab - 7168, vocab - 7167, vocab - 2, vocab - 1])
    z = torch.randn(1, len(places), generator=gen(14)).to(torch.bfloat16)
    zd = torch.full((1, vocab), -math.inf, dtype=torch.bfloat16, device=DEV)
    zd[0, places.to(DEV)] = z[0].to(DEV)
    t = places[-2:-1].to(DEV)
    logprob, entropy, stats = (torch.empty(s, device=DEV) for s in ((1,), (1,), (1, 2)))
    top, index = torch.empty(1, 4, device=DEV), torch.empty(1, 4, dtype=torch.int32, device=DEV)
    B.adagc_token_logprobs(zd, t, logprob, entropy, stats, top, index, workspace=workspace(B.adagc_token_logprobs_workspace_bytes(1, vocab, 4)))
    small = torch.tensor([len(places) - 2])
    want = O.logprobs(z, small, 1.0)
    near(logprob, want["logprob"], want["logprob_off"])
    near(entropy, want["entropy"], want["entropy_off"])
    at = O.top(z, 4)
    assert torch.equal(index.cpu().long(), places[at])
    near(top, want["logp"].gather(1, at), want["logp_off"].gather(1, at))
    one = torch.ones(1)
    B.adagc_token_logprobs_backward(zd, t, stats, entropy, one.to(DEV), one.to(DEV), zd)
    grad, off = O.logprobs_backward(z, small, 1.0, one, one)
    near(zd[0, places.to(DEV)].cpu()[None], grad, off, torch.bfloat16)
    assert sum(int(part.count_nonzero()) for part in zd[0].split(2 ** 28)) <= len(places)


@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** 100])
def test_logprobs_extreme_scales(scale):
    """At the least every token is as likely but masked ones; at the most only the largest."""
    z, t = make_logits(4, 5003, torch.float32, 15)
    z[0, 7] = z[1, 9] = torch.finfo(torch.float32).min
    z[1, ::2] = -math.inf
    z[2, 8] = 1e8
    zd, out = check_logprobs(z, t, scale, 3)
    assert all(torch.isfinite(out["entropy"]))


def test_logprobs_gradient_against_differences():
    """Central differences of the forward kernel's own sum in fp32: a step h gives h^2 |f'''| / 6 and rounding / h."""
    z, t = make_logits(4, 40, torch.float32, 11, size=1.0)
    t[3] = -1
    zd, out = run_logprobs(z, t, 1.0, 0)
    d = Framed(4, 40, torch.float32)
    one = torch.ones(4, device=DEV)
    B.adagc_token_logprobs_backward(zd.t, t.to(DEV), out["stats"], out["entropy"], one, 0.5 * one, d.t)
    grad = d.result().double()

    def total(j, h):
        moved = z.clone()
        moved[:, j] += h
        _, o = run_logprobs(moved, t, 1.0, 0)
        return (o["logprob"].double() + 0.5 * o["entropy"].double()).cpu(), moved[:, j].double()

    h, off = 2.0 ** -5, O.logprobs(z, t, 1.0)
    for j in range(0, 40, 3):
        up, at_up = total(j, h)
        down, at_down = total(j, -h)
        bound = 4 * h * h / 6 + 2 * (off["logprob_off"] + off["entropy_off"]) / h      # third derivatives are below 4
        assert ((up - down) / (at_up - at_down) - grad[:, j]).abs().le(bound).all()


# ------------------------------------------------------------------------------------------------ checkpoints

def make_activations(rows, cols, dtype, seed):
    g = gen(seed)
    return (torch.randn(rows, cols, generator=g) * torch.exp(4 * torch.randn(rows, 1, generator=g)) *
            torch.exp(torch.randn(1, cols, generator=g))).to(dtype)


def packed(x, ld=None, offset=0):
    rows, cols = x.shape
    xd = Framed(rows, cols, x.dtype, ld, offset, x)
    n = B.adagc_act8_bytes(rows, cols)
    buffer = torch.full((n + 64,), 0xCD, dtype=torch.uint8, device=DEV)
    B.adagc_act8_pack(xd.t, buffer)
    assert (buffer[n:] == 0xCD).all()
    return buffer[:n]


SHAPES = [(1, 1, None, 0), (3, 31, None, 1), (2, 32, None, 0), (5, 33, 40, 3), (7, 768, None, 0), (129, 100, 101, 7), (64, 257, None, 1),
          (1, 8193, None, 0), (300, 1000, 1008, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols, ld, offset", SHAPES)
def test_checkpoint(dtype, rows, cols, ld, offset):
    x = make_activations(rows, cols, TYPES[dtype], rows + cols)
    ckpt = packed(x, ld, offset)
    want = O.pack_bytes(x)
    assert torch.equal(ckpt.cpu(), want)
    for kind in (torch.float32, torch.bfloat16):                     # what a code stands for is exact in both
        back = Framed(rows, cols, kind, ld, offset)
        B.adagc_act8_unpack(ckpt, back.t)
        assert torch.equal(back.result().double(), O.values(want, rows, cols))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_checkpoint_every_rounding(dtype):
    """Every 16-bit pattern as the upper half of a value, in blocks whose largest value is 1.75 or a step above it."""
    bits = torch.arange(65536, dtype=torch.int32) << 16
    x = bits.view(torch.float32).clone()
    x[x.abs() > 1.75] = 0.0
    x = x.view(-1, 31)[:2114].contiguous() if 65536 % 31 == 0 else torch.cat([x, torch.zeros(-len(x) % 31)]).view(-1, 31)
    x = torch.cat([x, torch.full((len(x), 1), 1.75)], 1)
    high = x.clone()
    high[:, 31] = 1.7578125
    special = torch.randn(40, 64, generator=gen(1))
    special[3, 5], special[4, 40], special[5, :32], special[6] = math.nan, -math.inf, math.inf, 0.0
    special[7] *= 2.0 ** -120
    special[8] *= 2.0 ** -100
    special[9] = special[9].clamp(-1, 1) * 3e38
    special[10, 0] = 3.3895e38
    special[11] = 0.0
    special[11, 9] = 2.0 ** -126
    if dtype == "f32":
        special[11, 10] = 2.0 ** -140
    for m in (x, high, special):
        m = m.to(TYPES[dtype])
        want = O.pack_bytes(m)
        ckpt = packed(m)
        assert torch.equal(ckpt.cpu(), want)
        back = Framed(*m.shape, torch.float32)
        B.adagc_act8_unpack(ckpt, back.t)
        near(back.result(), O.values(want, *m.shape), 0.0)


def test_checkpoint_offsets_beyond_32_bits():
    rows, cols = 2 ** 27 + 77, 32
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    x[-100:] = make_activations(100, cols, torch.bfloat16, 12).to(DEV)
    ckpt = torch.empty(B.adagc_act8_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    B.adagc_act8_pack(x, ckpt)
    want = O.pack_bytes(x[-100:].cpu())
    assert torch.equal(ckpt[(rows - 100) * 32:rows * 32].cpu(), want[:3200])
    assert torch.equal(ckpt[rows * 33 - 100:].cpu(), want[3200:])
    x[-100:] = 5
    B.adagc_act8_unpack(ckpt, x)
    assert torch.equal(x[-100:].cpu().double(), O.values(want, 100, cols))
    assert not x[:-100].any()


@pytest.mark.parametrize("dtype, cols", [("f32", 2 ** 29 + 40), ("bf16", 2 ** 30 + 40)])
def test_checkpoint_of_a_long_row(dtype, cols):
    x = torch.zeros(1, cols, dtype=TYPES[dtype], device=DEV)
    end = make_activations(1, 104, TYPES[dtype], 16)
    x[:, -104:] = end.to(DEV)                                        # from a block's first column on
    ckpt = torch.empty(B.adagc_act8_bytes(1, cols), dtype=torch.uint8, device=DEV)
    B.adagc_act8_pack(x, ckpt)
    want = O.pack_bytes(end)
    ld = O.ld8(cols)
    assert torch.equal(ckpt[ld - 128:ld].cpu(), want[:128]) and torch.equal(ckpt[-4:].cpu(), want[128:])
    x.fill_(5)
    B.adagc_act8_unpack(ckpt, x)
    assert torch.equal(x[:, -104:].cpu().double(), O.values(want, 1, 104)) and not x[:, :-104].any()


# ------------------------------------------------------------------------------------------------ gated activation

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols, ld, offset", SHAPES)
def test_swiglu(dtype, rows, cols, ld, offset):
    dtype, g = TYPES[dtype], gen(rows * cols)
    gate, up = (3 * torch.randn(rows, cols, generator=g)).to(dtype), make_activations(rows, cols, dtype, 3).clamp(-1e4, 1e4)
    d_out = torch.randn(rows, cols, generator=g).to(dtype)
    gd, ud = Framed(rows, cols, dtype, ld, offset, gate), Framed(rows, cols, dtype, None, 0, up)
    out = Framed(rows, cols, dtype, ld, offset)
    n = B.adagc_act8_bytes(rows, cols)
    ckpts = [torch.full((n + 64,), 0xCD, dtype=torch.uint8, device=DEV) for _ in range(2)]
    B.adagc_swiglu(gd.t, ud.t, out.t, *ckpts)
    want, off = O.swiglu(gate, up)
    near(out.result(), want, off, dtype)
    for c, x in zip(ckpts, (gate, up)):
        assert (c[n:] == 0xCD).all() and torch.equal(c[:n].cpu(), O.pack_bytes(x))
    plain = Framed(rows, cols, dtype, None, 1)
    B.adagc_swiglu(gd.t, ud.t, plain.t)
    assert torch.equal(plain.result(), out.result())

    dd = Framed(rows, cols, dtype, ld, offset, d_out)
    d_gate, d_up, again = Framed(rows, cols, dtype, ld, offset), Framed(rows, cols, dtype), Framed(rows, cols, dtype, ld, offset)
    held = [O.values(c[:n].cpu(), rows, cols) for c in ckpts]
    wants = O.swiglu_backward(d_out, *held)
    B.adagc_swiglu_backward(dd.t, *ckpts, d_gate.t, d_up.t, again.t)
    for got, (w, o) in zip((d_gate, d_up, again), wants):
        near(got.result(), w, o, dtype)
    # in place, without the output
    first = d_gate.result()
    d_gate2 = Framed(rows, cols, dtype, ld, offset)
    B.adagc_swiglu_backward(dd.t, *ckpts, d_gate2.t, dd.t)
    assert torch.equal(d_gate2.result(), first) and torch.equal(dd.result(), d_up.result())
    B.adagc_swiglu(gd.t, ud.t, gd.t)
    assert torch.equal(gd.result(), out.result())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_swiglu_extremes(dtype):
    dtype = TYPES[dtype]
    gate = torch.tensor([[0.0, -0.0, 1e-30, 88.0, -88.0, 104.0, -104.0, 1e4, -1e4, 30.0, -30.0, -89.0]]).to(dtype)
    up = torch.full_like(gate, 1.5)
    out = Framed(1, 12, dtype)
    ckpts = [torch.empty(B.adagc_act8_bytes(1, 12), dtype=torch.uint8, device=DEV) for _ in range(2)]
    B.adagc_swiglu(gate.to(DEV), up.to(DEV), out.t, *ckpts)
    want, off = O.swiglu(gate, up)
    near(out.result(), want, off, dtype)
    held = [O.values(c.cpu(), 1, 12) for c in ckpts]
    one = torch.ones_like(gate)
    d_gate, d_up = Framed(1, 12, dtype), Framed(1, 12, dtype)
    B.adagc_swiglu_backward(one.to(DEV), *ckpts, d_gate.t, d_up.t)
    for got, (w, o) in zip((d_gate, d_up), O.swiglu_backward(one, *held)):
        near(got.result(), w, o, dtype)
    gate[0, 2] = math.nan
    B.adagc_swiglu(gate.to(DEV), up.to(DEV), out.t, *ckpts)
    assert torch.isnan(out.result()).sum() == 1
    B.adagc_swiglu_backward(one.to(DEV), *ckpts, d_gate.t, d_up.t)
    assert torch.isnan(d_gate.result()).sum() == 1 and torch.isnan(d_up.result()).sum() == 1


def test_swiglu_gradient_against_differences():
    """Values that a checkpoint holds exactly, so that the forward kernel moves along the same function."""
    g = gen(13)
    gate, up = (torch.randint(-15, 16, (3, 32), generator=g) / 8 for _ in range(2))
    gate[:, 0] = up[:, 0] = 1.875
    d = torch.randn(3, 32, generator=g)
    ckpts = [torch.empty(B.adagc_act8_bytes(3, 32), dtype=torch.uint8, device=DEV) for _ in range(2)]
    out, d_gate, d_up = (Framed(3, 32, torch.float32) for _ in range(3))
    B.adagc_swiglu(gate.to(DEV), up.to(DEV), out.t, *ckpts)
    assert torch.equal(O.values(ckpts[0].cpu(), 3, 32), gate.double())
    B.adagc_swiglu_backward(d.to(DEV), *ckpts, d_gate.t, d_up.t)

    def forward(a, b):
        B.adagc_swiglu(a.to(DEV), b.to(DEV), out.t)
        return out.result().double()

    h = 2.0 ** -6
    # silu's third derivative is below 1; a value of the forward pass is off by 2^-22 of itself at most
    bound = d.double().abs() * (h * h / 6 * 2 + 2.0 ** -22 * 4 / h)
    assert (((forward(gate + h, up) - forward(gate - h, up)) / (2 * h) * d - d_gate.result()).abs() <= bound).all()
    assert (((forward(gate, up + h) - forward(gate, up - h)) / (2 * h) * d - d_up.result()).abs() <= bound).all()


# ------------------------------------------------------------------------------------------------ weight gradient

def run_wgrad(d_out, x, dw, ld_d=None, offset=0, ld_w=None, start=None):
    """(result, the checkpoint's values) of x's checkpoint; start: what d_weight holds, added to."""
    rows, n_out = d_out.shape
    n_in = x.shape[1]
    ckpt = packed(x)
    dd = Framed(rows, n_out, d_out.dtype, ld_d, offset, d_out)
    w = Framed(n_out, n_in, dw, ld_w, offset, start)
    code = B.ADAGC_F32 if d_out.dtype == torch.float32 else B.ADAGC_BF16
    B.adagc_act8_wgrad(dd.t, ckpt, w.t, accumulate=start is not None, workspace=workspace(B.adagc_act8_wgrad_workspace_bytes(rows, n_out, n_in, code)))
    return w.result(), O.values(ckpt.cpu(), rows, n_in)


@pytest.mark.parametrize("dtype, dw", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("rows, n_out, n_in, ld_d, offset, ld_w, accumulate", [
    (1, 1, 1, None, 0, None, False),
    (1, 64, 64, None, 0, None, True),
    (2, 5, 33, 7, 1, 40, False),
    (31, 130, 127, None, 0, None, True),
    (64, 128, 128, None, 0, None, False),
    (65, 257, 96, 259, 3, 97, True),
    (100, 50, 300, None, 0, None, False),
    (333, 256, 512, None, 0, None, False),
    (1000, 129, 65, None, 1, None, True),
    (4097, 64, 40, None, 0, None, False),
    (515, 511, 769, 513, 0, None, True),
    (128, 1024, 1024, 1032, 8, 1030, False),
])
def test_wgrad(dtype, dw, rows, n_out, n_in, ld_d, offset, ld_w, accumulate):
    g = gen(rows + n_out + n_in)
    d_out = (torch.randn(rows, n_out, generator=g) * torch.exp(2 * torch.randn(rows, 1, generator=g))).to(TYPES[dtype])
    x = make_activations(rows, n_in, torch.bfloat16, 5)
    start = torch.randn(n_out, n_in, generator=g).to(TYPES[dw]) if accumulate else None
    got, held = run_wgrad(d_out, x, TYPES[dw], ld_d, offset, ld_w, start)
    want, off = O.wgrad(d_out, held)
    if accumulate:
        want = want + start.double()
        off = off + 2 * O.U32 * (want.abs() + off)
    near(got, want, off, TYPES[dw])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, n_out, n_in, ld_d, offset, accumulate", [
    (700, 2048, 4096, None, 0, False),                 # tiles that are all split along the tokens
    (1027, 2901, 2999, 2903, 1, True),                 # odd everything: the last tiles begin inside others
    (97, 5003, 4100, None, 0, True),
    (31, 4096, 4096, None, 0, False),                  # less than a step
    (2500, 12345, 1500, None, 0, False),               # whole tiles and split ones
    (40, 3000, 3000, 2 ** 24, 0, False),               # rows far apart
])
def test_wgrad_large_tiles(dtype, rows, n_out, n_in, ld_d, offset, accumulate):
    """The oracle's formulas with the product on the GPU, in 64 bits."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)
    flat = torch.full((offset + (rows - 1) * (ld_d or n_out) + n_out,), math.nan, dtype=TYPES[dtype], device=DEV)
    d_out = flat[offset:].as_strided((rows, n_out), (ld_d or n_out, 1), offset)
    d_out.copy_(rand(rows, n_out))
    x = (rand(rows, n_in) * torch.exp(rand(1, n_in))).bfloat16()
    ckpt = torch.empty(B.adagc_act8_bytes(rows, n_in), dtype=torch.uint8, device=DEV)
    B.adagc_act8_pack(x, ckpt)
    held = torch.empty(rows, n_in, device=DEV)
    B.adagc_act8_unpack(ckpt, held)
    w = Framed(n_out, n_in, torch.float32, n_in + 1, 1)
    start = rand(n_out, n_in) if accumulate else torch.zeros(n_out, n_in, device=DEV)
    w.t.copy_(start)
    code = B.ADAGC_F32 if dtype == "f32" else B.ADAGC_BF16
    B.adagc_act8_wgrad(d_out, ckpt, w.t, accumulate=accumulate, workspace=workspace(B.adagc_act8_wgrad_workspace_bytes(rows, n_out, n_in, code)))
    y, held = d_out.double(), held.double()
    want = y.t().contiguous() @ held + start
    off = (rows + 8) * 2 * O.U32 * (y.abs().t().contiguous() @ held.abs()) + 2 * O.U32 * want.abs()
    assert ((w.t.double() - want).abs() <= off).all()
    assert (w.flat[~w.inside] == FILL).all()


@pytest.mark.parametrize("dw", ["f32", "bf16"])
def test_wgrad_no_rows(dw):
    d_out, x = torch.zeros(0, 70), torch.zeros(0, 45, dtype=torch.bfloat16)
    got, _ = run_wgrad(d_out, x, TYPES[dw])
    assert got.shape == (70, 45) and not got.any()
    start = torch.randn(70, 45, generator=gen(1)).to(TYPES[dw])
    got, _ = run_wgrad(d_out, x, TYPES[dw], start=start)
    assert torch.equal(got, start)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_wgrad_is_exact_where_sums_are(dtype):
    """Small whole numbers: every product and sum is exact in fp32, so the order and the tiles cannot matter."""
    g = gen(21)
    for rows, n_out, n_in in ((200, 300, 290), (1500, 60, 70), (70, 1000, 30)):
        d_out = torch.randint(-8, 9, (rows, n_out), generator=g).to(TYPES[dtype])
        x = torch.randint(-8, 9, (rows, n_in), generator=g).to(torch.bfloat16)
        x[:, ::32] = 8                                             # blocks of one scale hold these exactly
        got, held = run_wgrad(d_out, x, torch.float32)
        assert torch.equal(held, x.double())
        assert torch.equal(got.double(), d_out.double().t() @ x.double())


def test_wgrad_fp32_gradient_keeps_all_its_bits():
    """One token: the result is the product itself, all 24 bits of d_out in it."""
    g = gen(22)
    d_out = torch.randn(1, 333, generator=g) * torch.exp2(torch.randint(-60, 60, (1, 333), generator=g).float())
    x = torch.ones(1, 65, dtype=torch.bfloat16)
    got, _ = run_wgrad(d_out, x, torch.float32)
    assert torch.equal(got, d_out.t().expand(333, 65))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_wgrad_special_values_stay_in_their_row_and_column(dtype):
    rows, n_out, n_in = 70, 140, 150
    g = gen(23)
    d_out, x = torch.randn(rows, n_out, generator=g).to(TYPES[dtype]), torch.randn(rows, n_in, generator=g).to(torch.bfloat16)
    d_out[3, 7], d_out[60, 130] = math.nan, math.inf
    x[5, 9], x[69, 149] = math.nan, -math.inf
    got, held = run_wgrad(d_out, x, torch.float32)
    bad = torch.zeros(n_out, n_in, dtype=torch.bool)
    bad[7], bad[130], bad[:, 9], bad[:, 149] = True, True, True, True
    assert (~torch.isfinite(got[bad])).all() and torch.isfinite(got[~bad]).all()


def test_wgrad_tail_of_a_checkpoint_of_nan_codes_is_not_read():
    """Bytes after the buffer, and columns of d_out beyond n_out, may hold anything."""
    rows, n_out, n_in = 37, 100, 100
    g = gen(24)
    d_out, x = torch.randn(rows, n_out, generator=g).to(torch.bfloat16), torch.randn(rows, n_in, generator=g).to(torch.bfloat16)
    ckpt = packed(x)
    n = ckpt.numel()
    buffer = torch.full((n + 8192,), 0x7F, dtype=torch.uint8, device=DEV)
    buffer[:n] = ckpt
    dd = torch.full((rows + 100, 128), math.nan, dtype=torch.bfloat16, device=DEV)
    dd[:rows, :n_out] = d_out.to(DEV)
    w = Framed(n_out, n_in, torch.float32)
    B.adagc_act8_wgrad(dd[:rows, :n_out], buffer[:n], w.t, workspace=workspace(B.adagc_act8_wgrad_workspace_bytes(rows, n_out, n_in, B.ADAGC_BF16)))
    want, off = O.wgrad(d_out, O.values(ckpt.cpu(), rows, n_in))
    near(w.result(), want, off)


def test_wgrad_offsets_beyond_32_bits():
    rows, n_out, n_in, ld = 3, 70, 64, 2 ** 31 - 1024
    g = gen(25)
    d_out, x = torch.randn(rows, n_out, generator=g).to(torch.bfloat16), torch.randn(rows, n_in, generator=g).to(torch.bfloat16)
    flat = torch.empty((rows - 1) * ld + n_out, dtype=torch.bfloat16, device=DEV)
    dd = flat.as_strided((rows, n_out), (ld, 1))
    dd.copy_(d_out)
    ckpt = packed(x)
    w = Framed(n_out, n_in, torch.float32)
    B.adagc_act8_wgrad(dd, ckpt, w.t, workspace=workspace(B.adagc_act8_wgrad_workspace_bytes(rows, n_out, n_in, B.ADAGC_BF16)))
    want, off = O.wgrad(d_out, O.values(ckpt.cpu(), rows, n_in))
    near(w.result(), want, off)


def test_wgrad_offsets_within_a_step_beyond_32_bits():
    """33 rows of 2^27 columns, zero but for the last row of the first step, the row after it and the last columns."""
    rows, n_out, n_in = 33, 128, 2 ** 27
    ckpt = torch.zeros(B.adagc_act8_bytes(rows, n_in), dtype=torch.uint8, device=DEV)
    ckpt[rows * n_in:] = 127
    x = torch.zeros(rows, 64, dtype=torch.bfloat16)
    x[31], x[32] = 2.0, 0.5
    x[:, 32:] = torch.randn(rows, 32, generator=gen(26)).sign()
    codes = O.pack_bytes(x)
    for columns, from_ in ((slice(0, 32), 0), (slice(n_in - 32, n_in), 32)):
        ckpt[:rows * n_in].view(rows, n_in)[:, columns] = codes[:rows * 64].view(rows, 64)[:, from_:from_ + 32].to(DEV)
        ckpt[rows * n_in:].view(rows, n_in // 32)[:, columns.start // 32] = codes[rows * 64:].view(rows, 2)[:, from_ // 32].to(DEV)
    d_out = torch.randint(-8, 9, (rows, n_out), generator=gen(27)).to(torch.bfloat16)
    w = torch.full((n_out, n_in), FILL, dtype=torch.bfloat16, device=DEV)
    B.adagc_act8_wgrad(d_out.to(DEV), ckpt, w, workspace=workspace(max(1, B.adagc_act8_wgrad_workspace_bytes(rows, n_out, n_in, B.ADAGC_BF16))))
    want = (d_out.double().t() @ x.double()).to(torch.bfloat16)      # sums of halves below 2^10: exact before the rounding
    assert torch.equal(w[:, :32].cpu(), want[:, :32]) and torch.equal(w[:, -32:].cpu(), want[:, 32:])
    assert not any(bool(part.any()) for part in w[:, 32:-32].split(2 ** 24, 1))


# ------------------------------------------------------------------------------------------------ streams and graphs

def chain(z, t, x, stream):
    """One call of every operator, on outputs made here."""
    rows, vocab = z.shape
    cols = x.shape[1]
    new = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device=DEV)
    out = {"logprob": new(rows), "entropy": new(rows), "stats": new(rows, 2), "top_logprob": new(rows, 3), "top_index": new(rows, 3, dtype=torch.int32)}
    bufs = dict(ws=workspace(B.adagc_token_logprobs_workspace_bytes(rows, vocab, 3)), d_z=torch.zeros_like(z),
                a=new(B.adagc_act8_bytes(rows, cols), dtype=torch.uint8), b=new(B.adagc_act8_bytes(rows, cols), dtype=torch.uint8),
                h=torch.zeros_like(x), dg=torch.zeros_like(x), du=torch.zeros_like(x), w=new(vocab, cols),
                ws2=workspace(B.adagc_act8_wgrad_workspace_bytes(rows, vocab, cols, B.ADAGC_BF16)), dl=torch.full((rows,), -0.1, device=DEV))

    def call():
        s = stream()
        B.adagc_token_logprobs(z, t, workspace=bufs["ws"], stream=s, **out)
        B.adagc_token_logprobs_backward(z, t, out["stats"], out["entropy"], bufs["dl"], bufs["dl"], bufs["d_z"], stream=s)
        B.adagc_swiglu(x, x, bufs["h"], bufs["a"], bufs["b"], stream=s)
        B.adagc_act8_pack(bufs["h"], bufs["b"], stream=s)
        B.adagc_act8_unpack(bufs["b"], bufs["h"], stream=s)
        B.adagc_swiglu_backward(x, bufs["a"], bufs["b"], bufs["dg"], bufs["du"], stream=s)
        B.adagc_act8_wgrad(bufs["d_z"], bufs["a"], bufs["w"], workspace=bufs["ws2"], stream=s)
        return [out[k] for k in out] + [bufs[k] for k in ("d_z", "a", "b", "h", "dg", "du", "w")]
    return call


def current():
    return torch.cuda.current_stream().cuda_stream


def test_graph_and_other_streams():
    rows, vocab, cols = 20, 9001, 130
    z, t = make_logits(rows, vocab, torch.bfloat16, 30)
    x = make_activations(rows, cols, torch.bfloat16, 31)
    z, t, x = z.to(DEV), t.to(DEV), x.to(DEV)
    want = [r.clone() for r in chain(z, t, x, current)()]
    assert all(torch.equal(a, b) for a, b in zip(want, chain(z, t, x, current)()))       # the same every time
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = chain(z, t, x, current)()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))

    call = chain(z, t, x, current)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = call()
    for seed in (40, 41, 42):
        z2, t2 = make_logits(rows, vocab, torch.bfloat16, seed)
        x2 = make_activations(rows, cols, torch.bfloat16, seed)
        z.copy_(z2)
        t.copy_(t2)
        x.copy_(x2)
        for r in recorded:
            r.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = chain(z, t, x, current)()
        assert all(torch.equal(a, b) for a, b in zip(recorded, eager))
