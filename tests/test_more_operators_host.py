"""Without a GPU: sizes of workspaces and what the operators that keep nothing between the passes refuse, before anything is enqueued."""
import ctypes
import functools

import pytest
import torch

import more_operators_oracle as O
from paper_2502_11034_amd import binding as B

INVALID, LARGE = B.ADAGC_ERR_INVALID_ARG, B.ADAGC_ERR_TOO_LARGE
A = 4096                       # an aligned address that a refused call never reaches
BIG = 2 ** 31 - 1023           # the first length that is too large


def test_published_words_of_the_generator():
    """Known answers of Philox4x32-10, as its authors distribute them."""
    assert O.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert O.philox((2 ** 32 - 1,) * 4, (2 ** 32 - 1,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert O.philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


@pytest.mark.parametrize("f, sizes", [
    ("adagc_linear_logprobs_workspace_bytes", (100, 1000, 64, 0)), ("adagc_linear_logprobs_backward_workspace_bytes", (100, 1000, 64, 1)),
    ("adagc_gated_linear_workspace_bytes", (100, 64, 1000, 0)), ("adagc_gated_linear_backward_workspace_bytes", (100, 64, 1000, 1))])
def test_workspace_sizes(f, sizes):
    size = getattr(B.lib(), f)
    assert size(*sizes) >= 0
    for at in range(4):
        for value in (-1, 0) if at not in (0, 3) else (-1,):
            assert size(*sizes[:at], value, *sizes[at + 1:]) == INVALID
    assert size(*sizes[:3], 2) == INVALID
    assert size(2 ** 24, *sizes[1:]) == LARGE and size(2 ** 62, *sizes[1:]) == LARGE
    for at in (1, 2):
        assert size(*sizes[:at], BIG, *sizes[at + 1:]) == LARGE
        assert size(*sizes[:at], 2 ** 63 - 1, *sizes[at + 1:]) == LARGE
    assert size(2 ** 24 - 1, 2 ** 20, 2 ** 20, 0) == LARGE           # too many tiles
    with pytest.raises(B.AdagcError):
        getattr(B, f)(2 ** 64 + 1, *sizes[1:])
    assert size(0, *sizes[1:]) >= 0


def test_workspaces_are_bounded():
    """The gradients of a piece of the vocabulary, not of all of it."""
    one = B.adagc_linear_logprobs_backward_workspace_bytes(4096, 128256, 4096, B.ADAGC_BF16)
    assert one < 4096 * 128256 * 2 / 3
    assert B.adagc_linear_logprobs_workspace_bytes(4096, 128256, 4096, B.ADAGC_BF16) < 4096 * 128256 * 2 / 25


def call(f, defaults, **change):
    args = dict(defaults, **change)
    return getattr(B.lib(), f)(*args.values())


forward = functools.partial(call, "adagc_linear_logprobs", dict(x=A, ld_x=64, w=A, ld_w=64, dtype=1, rows=10, vocab=100, dim=64, t=A, scale=1.0, logprob=A,
                                                                stats=A, ws=A, ws_bytes=2 ** 30, stream=None))
backward = functools.partial(call, "adagc_linear_logprobs_backward", dict(
    x=A, ld_x=64, w=A, ld_w=64, dtype=1, rows=10, vocab=100, dim=64, t=A, scale=1.0, stats=A, d=A, d_x=A, ld_d_x=64, d_w=A, weight_dtype=0, ld_d_w=64,
    accumulate=0, ws=A, ws_bytes=2 ** 30, stream=None))
gated = functools.partial(call, "adagc_gated_linear", dict(x=A, ld_x=64, wg=A, ld_wg=64, wu=A, ld_wu=64, dtype=1, rows=10, dim=64, hidden=100, out=A, ld_out=100,
                                                           gate=A, ld_gate=100, up=A, ld_up=100, ws=A, ws_bytes=2 ** 30, stream=None))
gated_backward = functools.partial(call, "adagc_gated_linear_backward", dict(
    d_out=A, ld_d_out=100, x=A, ld_x=64, wg=A, ld_wg=64, wu=A, ld_wu=64, dtype=1, rows=10, dim=64, hidden=100, gate=A, ld_gate=100, up=A, ld_up=100, d_x=A,
    ld_d_x=64, d_wg=A, ld_d_wg=64, d_wu=A, ld_d_wu=64, weight_dtype=0, accumulate=0, out=A, ld_out=100, ws=A, ws_bytes=2 ** 30, stream=None))
dropout = functools.partial(call, "adagc_dropout", dict(x=A, ld_x=64, r=A, ld_r=64, dtype=1, rows=10, cols=64, p=0.5, rng=A, out=A, ld_out=64, stream=None))

COMMON = [(dict(rows=-1), INVALID), (dict(dtype=2), INVALID), (dict(x=None), INVALID), (dict(x=A + 1), INVALID), (dict(ld_x=63), INVALID),
          (dict(ld_x=2 ** 31), LARGE)]
LOSS = COMMON + [(dict(vocab=0), INVALID), (dict(dim=0), INVALID), (dict(w=None), INVALID), (dict(w=A + 1), INVALID), (dict(ld_w=63), INVALID),
                 (dict(ld_w=2 ** 31), LARGE), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=2.0 ** 101), INVALID),
                 (dict(scale=float("nan")), INVALID), (dict(t=None), INVALID), (dict(t=A + 4), INVALID), (dict(ws=None), INVALID), (dict(ws=A + 8), INVALID),
                 (dict(ws_bytes=100), INVALID), (dict(ws_bytes=-1), INVALID), (dict(rows=2 ** 24), LARGE), (dict(vocab=BIG), LARGE), (dict(dim=BIG), LARGE),
                 (dict(rows=2 ** 23, vocab=2 ** 22), LARGE), (dict(dtype=0, x=A + 2), INVALID)]
GATED = COMMON + [(dict(hidden=0), INVALID), (dict(dim=0), INVALID), (dict(wg=None), INVALID), (dict(wu=None), INVALID), (dict(wg=A + 1), INVALID),
                  (dict(wu=A + 1), INVALID), (dict(ld_wg=63), INVALID), (dict(ld_wu=63), INVALID), (dict(ld_wg=2 ** 31), LARGE), (dict(ld_wu=2 ** 31), LARGE),
                  (dict(gate=None), INVALID), (dict(up=None), INVALID), (dict(gate=A + 1), INVALID), (dict(up=A + 1), INVALID), (dict(ld_gate=99), INVALID),
                  (dict(ld_up=99), INVALID), (dict(ld_gate=2 ** 31), LARGE), (dict(out=A + 1), INVALID), (dict(ld_out=99), INVALID), (dict(ld_out=2 ** 31), LARGE),
                  (dict(ws_bytes=-1), INVALID), (dict(rows=2 ** 24), LARGE), (dict(hidden=BIG), LARGE), (dict(dim=BIG), LARGE),
                  (dict(rows=2 ** 23, hidden=2 ** 22), LARGE)]


@pytest.mark.parametrize("f, change, code", [
    *[(forward, c, e) for c, e in LOSS + [(dict(logprob=None, stats=None), INVALID), (dict(logprob=A + 2), INVALID), (dict(stats=A + 2), INVALID)]],
    *[(backward, c, e) for c, e in LOSS + [(dict(d_x=None, d_w=None), INVALID), (dict(d_x=A + 1), INVALID), (dict(d_w=A + 1), INVALID), (dict(d_w=A + 2), INVALID),
                                           (dict(stats=None), INVALID), (dict(stats=A + 1), INVALID), (dict(d=None), INVALID), (dict(d=A + 1), INVALID),
                                           (dict(ld_d_x=63), INVALID), (dict(ld_d_w=63), INVALID), (dict(ld_d_x=2 ** 31), LARGE), (dict(ld_d_w=2 ** 31), LARGE),
                                           (dict(weight_dtype=2), INVALID), (dict(accumulate=2), INVALID), (dict(accumulate=-1), INVALID)]],
    *[(gated, c, e) for c, e in GATED + [(dict(out=None), INVALID)]],
    *[(gated_backward, c, e) for c, e in GATED + [(dict(d_out=None), INVALID), (dict(d_out=A + 1), INVALID), (dict(ld_d_out=99), INVALID),
                                                  (dict(ld_d_out=2 ** 31), LARGE), (dict(d_x=None, d_wg=None, d_wu=None), INVALID), (dict(d_wg=None), INVALID),
                                                  (dict(d_wu=None), INVALID), (dict(d_x=A + 1), INVALID), (dict(d_wg=A + 2), INVALID), (dict(d_wu=A + 2), INVALID),
                                                  (dict(ld_d_x=63), INVALID), (dict(ld_d_wg=63), INVALID), (dict(ld_d_wu=63), INVALID), (dict(ld_d_x=2 ** 31), LARGE),
                                                  (dict(ld_d_wg=2 ** 31), LARGE), (dict(ld_d_wu=2 ** 31), LARGE), (dict(weight_dtype=2), INVALID),
                                                  (dict(accumulate=2), INVALID), (dict(ws=None), INVALID), (dict(ws=A + 8), INVALID), (dict(ws_bytes=100), INVALID)]],
    *[(dropout, c, e) for c, e in COMMON + [(dict(cols=0), INVALID), (dict(p=-0.1), INVALID), (dict(p=1.1), INVALID), (dict(p=float("nan")), INVALID),
                                            (dict(rng=None), INVALID), (dict(rng=A + 4), INVALID), (dict(out=None), INVALID), (dict(out=A + 1), INVALID),
                                            (dict(ld_out=63), INVALID), (dict(r=A + 1), INVALID), (dict(ld_r=63), INVALID), (dict(ld_r=2 ** 31), LARGE),
                                            (dict(ld_out=2 ** 31), LARGE), (dict(rows=2 ** 31), LARGE), (dict(cols=BIG), LARGE),
                                            (dict(rows=2 ** 31 - 1, cols=2 ** 20, ld_x=2 ** 20, ld_out=2 ** 20, ld_r=2 ** 20), LARGE)]],
])
def test_refusals(f, change, code):
    assert f(**change) == code


def test_no_rows_are_a_valid_call_without_data():
    assert forward(rows=0, x=None, w=None, t=None, logprob=None, stats=None, ws=None, ws_bytes=0) == B.ADAGC_OK
    assert gated(rows=0, x=None, out=None, gate=None, up=None, ws=None, ws_bytes=0) == B.ADAGC_OK
    assert dropout(rows=0, x=None, r=None, out=None, rng=None) == B.ADAGC_OK


def test_the_binding_refuses_before_the_library():
    x, w, t = torch.zeros(4, 8), torch.zeros(20, 8), torch.zeros(4, dtype=torch.int64)
    one, two, buffer, out = torch.zeros(4), torch.zeros(4, 2), torch.zeros(2 ** 20, dtype=torch.uint8), torch.zeros(4, 20)
    rng = torch.zeros(2, dtype=torch.int64)
    for wrong in (lambda: B.adagc_linear_logprobs(x, w[:, :7], t, one, workspace=buffer), lambda: B.adagc_linear_logprobs(x, w, t[:3], one, workspace=buffer),
                  lambda: B.adagc_linear_logprobs(x, w, t, one, one, workspace=buffer), lambda: B.adagc_linear_logprobs(x, w, t, one),
                  lambda: B.adagc_linear_logprobs(x, w, t, one, workspace=buffer[:16]), lambda: B.adagc_linear_logprobs(x.t(), w, t, one, workspace=buffer),
                  lambda: B.adagc_linear_logprobs_backward(x, w, t, two, one, out, None, workspace=buffer),
                  lambda: B.adagc_linear_logprobs_backward(x, w, t, two, one, None, x, workspace=buffer),
                  lambda: B.adagc_gated_linear(x, w, w[:10], out, workspace=buffer), lambda: B.adagc_gated_linear(x, w[:, :7], w, out, workspace=buffer),
                  lambda: B.adagc_gated_linear(x, w, w, x, workspace=buffer), lambda: B.adagc_gated_linear(x, w, w, out, x, out, workspace=buffer),
                  lambda: B.adagc_gated_linear_backward(out, x, w, w, x, None, x, workspace=buffer),
                  lambda: B.adagc_gated_linear_backward(x, x, w, w, x, workspace=buffer), lambda: B.adagc_gated_linear_backward(out, x, w, w, x),
                  lambda: B.adagc_dropout(x, out, rng, 0.1), lambda: B.adagc_dropout(x, x, rng[:1], 0.1), lambda: B.adagc_dropout(x, x, rng, 0.1, residual=out)):
        with pytest.raises(ValueError):
            wrong()
    for wrong in (lambda: B.adagc_linear_logprobs(x.double(), w, t, one, workspace=buffer), lambda: B.adagc_linear_logprobs(x, w.bfloat16(), t, one, workspace=buffer),
                  lambda: B.adagc_linear_logprobs(x, w, t.int(), one, workspace=buffer), lambda: B.adagc_gated_linear(x, w.bfloat16(), w, out, workspace=buffer),
                  lambda: B.adagc_gated_linear_backward(out, x, w, w, None, w.clone(), w.bfloat16(), workspace=buffer),
                  lambda: B.adagc_dropout(x, x, rng.int(), 0.1), lambda: B.adagc_dropout(x, x.bfloat16(), rng, 0.1), lambda: B.adagc_dropout(x.half(), x, rng, 0.1)):
        with pytest.raises(TypeError):
            wrong()
    # right in all but that it is host memory
    for host in (lambda: B.adagc_linear_logprobs(x, w, t, one, two, workspace=buffer),
                 lambda: B.adagc_linear_logprobs_backward(x, w, t, two, one, x.clone(), w.clone(), workspace=torch.zeros(2 ** 22, dtype=torch.uint8)),
                 lambda: B.adagc_gated_linear(x, w, w, out, workspace=buffer),
                 lambda: B.adagc_gated_linear_backward(out, x, w, w, x.clone(), workspace=torch.zeros(2 ** 22, dtype=torch.uint8)),
                 lambda: B.adagc_dropout(x, x.clone(), rng, 0.1)):
        with pytest.raises(B.AdagcError) as e:
            host()
        assert "device" in str(e.value)
