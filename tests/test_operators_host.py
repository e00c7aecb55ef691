"""The operators around the step without a GPU: sizes, refusals before anything is enqueued, and the 64-bit oracle's own pins."""
import ctypes
import math

import pytest
import torch

import operators_oracle as O
from paper_2502_11034_amd import binding as B

P = 1 << 20                    # a pointer that is never read: every call below is refused before that, or has no rows
BAD, LARGE, OK = B.ADAGC_ERR_INVALID_ARG, B.ADAGC_ERR_TOO_LARGE, B.ADAGC_OK


def forward(logits=P, dtype=1, rows=4, vocab=100, ld=100, targets=P, scale=1.0, top_k=0, logprob=P, entropy=P, stats=P, top_logprob=None,
            top_index=None, workspace=P, workspace_bytes=1 << 20):
    return B.lib().adagc_token_logprobs(logits, dtype, rows, vocab, ld, targets, scale, top_k, logprob, entropy, stats, top_logprob,
                                        top_index, workspace, workspace_bytes, None)


def backward(logits=P, dtype=1, rows=4, vocab=100, ld=100, targets=P, scale=1.0, stats=P, entropy=P, d_logprob=P, d_entropy=P, d_logits=2 * P,
             ld_d=100):
    return B.lib().adagc_token_logprobs_backward(logits, dtype, rows, vocab, ld, targets, scale, stats, entropy, d_logprob, d_entropy,
                                                 d_logits, ld_d, None)


def pack(x=P, dtype=1, rows=4, cols=100, ld=100, ckpt=P):
    return B.lib().adagc_act8_pack(x, dtype, rows, cols, ld, ckpt, None)


def unpack(x=P, dtype=1, rows=4, cols=100, ld=100, ckpt=P):
    return B.lib().adagc_act8_unpack(ckpt, rows, cols, x, dtype, ld, None)


def swiglu(gate=P, ld_gate=100, up=2 * P, ld_up=100, dtype=1, rows=4, cols=100, out=3 * P, ld_out=100, gate_ckpt=4 * P, up_ckpt=5 * P):
    return B.lib().adagc_swiglu(gate, ld_gate, up, ld_up, dtype, rows, cols, out, ld_out, gate_ckpt, up_ckpt, None)


def swiglu_backward(d_out=P, ld_d_out=100, dtype=1, gate_ckpt=2 * P, up_ckpt=3 * P, rows=4, cols=100, d_gate=4 * P, ld_d_gate=100, d_up=5 * P,
                    ld_d_up=100, out=None, ld_out=0):
    return B.lib().adagc_swiglu_backward(d_out, ld_d_out, dtype, gate_ckpt, up_ckpt, rows, cols, d_gate, ld_d_gate, d_up, ld_d_up, out,
                                         ld_out, None)


def wgrad(d_out=P, dtype=1, ld_d_out=100, ckpt=P, rows=4, n_out=100, n_in=64, d_weight=2 * P, weight_dtype=0, ld_weight=64, accumulate=0,
          workspace=4 * P, workspace_bytes=1 << 40):
    return B.lib().adagc_act8_wgrad(d_out, dtype, ld_d_out, ckpt, rows, n_out, n_in, d_weight, weight_dtype, ld_weight, accumulate, workspace,
                                    workspace_bytes, None)


HUGE = 1 << 40
REFUSED = [
    (forward, BAD, [dict(logits=None), dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(vocab=0), dict(ld=99), dict(scale=0.0),
                    dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(targets=None), dict(top_k=-1),
                    dict(top_k=65, top_logprob=P, top_index=P), dict(vocab=4, top_k=5, top_logprob=P, top_index=P), dict(top_k=3),
                    dict(top_k=3, top_logprob=P), dict(top_logprob=P), dict(top_index=P), dict(logprob=None, entropy=None, stats=None),
                    dict(logits=P + 1), dict(dtype=0, logits=P + 2), dict(targets=P + 4), dict(stats=P + 2), dict(workspace_bytes=-1),
                    dict(rows=1, vocab=128256, ld=128256, workspace=None), dict(rows=1, vocab=128256, ld=128256, workspace_bytes=15),
                    dict(rows=1, vocab=128256, ld=128256, workspace=P + 8)]),
    (forward, LARGE, [dict(rows=1 << 24), dict(vocab=1 << 31, ld=1 << 31), dict(ld=HUGE)]),
    (backward, BAD, [dict(logits=None), dict(dtype=2), dict(rows=-1), dict(vocab=0), dict(ld=99), dict(ld_d=99), dict(scale=0.0),
                     dict(stats=None), dict(targets=None), dict(entropy=None), dict(d_logits=None), dict(d_logits=2 * P + 1),
                     dict(d_logits=P, ld=100, ld_d=101), dict(d_entropy=P + 2)]),
    (backward, LARGE, [dict(rows=1 << 24), dict(ld_d=HUGE)]),
    (pack, BAD, [dict(x=None), dict(dtype=2), dict(rows=-1), dict(cols=0), dict(ld=99), dict(x=P + 1), dict(ckpt=None), dict(ckpt=P + 8)]),
    (pack, LARGE, [dict(rows=1 << 31), dict(cols=1 << 31, ld=1 << 31), dict(ld=HUGE)]),
    (unpack, BAD, [dict(x=None), dict(dtype=3), dict(rows=-1), dict(cols=0), dict(ld=99), dict(x=P + 1), dict(ckpt=None), dict(ckpt=P + 8)]),
    (swiglu, BAD, [dict(gate=None), dict(up=None), dict(out=None), dict(dtype=2), dict(ld_gate=99), dict(ld_up=99), dict(ld_out=99),
                   dict(gate_ckpt=None), dict(up_ckpt=None), dict(up_ckpt=4 * P), dict(gate_ckpt=4 * P + 4), dict(out=P, ld_out=101),
                   dict(out=2 * P, ld_out=200), dict(rows=-1), dict(cols=0)]),
    (swiglu, LARGE, [dict(ld_up=HUGE)]),
    (swiglu_backward, BAD, [dict(d_out=None), dict(gate_ckpt=None), dict(up_ckpt=None), dict(d_gate=None), dict(d_up=None),
                            dict(d_up=4 * P), dict(out=4 * P, ld_out=100), dict(out=5 * P, ld_out=100), dict(out=P, ld_out=100),
                            dict(out=6 * P, ld_out=99), dict(d_gate=P, ld_d_gate=128), dict(d_up=P, ld_d_up=128), dict(dtype=7),
                            dict(gate_ckpt=2 * P + 8)]),
    (wgrad, BAD, [dict(d_out=None), dict(ckpt=None), dict(d_weight=None), dict(dtype=2), dict(weight_dtype=2), dict(ld_d_out=99),
                  dict(ld_weight=63), dict(accumulate=2), dict(accumulate=-1), dict(rows=-1), dict(n_out=0), dict(n_in=0),
                  dict(ckpt=P + 8), dict(d_weight=2 * P + 2), dict(d_out=P + 1), dict(workspace_bytes=-1)]),
    (wgrad, LARGE, [dict(rows=1 << 31), dict(n_out=1 << 31, ld_d_out=1 << 31), dict(ld_weight=HUGE), dict(ld_d_out=HUGE)]),
]


@pytest.mark.parametrize("call, code, arguments", [(c, code, a) for c, code, many in REFUSED for a in many],
                         ids=lambda v: v.__name__ if callable(v) else str(v))
def test_refused(call, code, arguments):
    assert call(**arguments) == code


@pytest.mark.parametrize("call", [forward, backward])
def test_scales_out_of_range_are_refused(call):
    for scale in (2.0 ** -101, 2.0 ** 101, 1e-45, 3e38):
        assert call(scale=scale) == BAD


def test_no_rows_is_a_valid_call_with_nothing_to_do():
    assert forward(rows=0, logits=None, targets=None, logprob=None, entropy=None, stats=None) == OK
    assert backward(rows=0, logits=None, targets=None, stats=None, d_logits=None) == OK
    assert pack(rows=0, x=None, ckpt=None) == OK and unpack(rows=0, x=None, ckpt=None) == OK
    assert swiglu(rows=0, gate=None, up=None, out=None) == OK
    assert swiglu_backward(rows=0, d_out=None, d_gate=None, d_up=None, gate_ckpt=None, up_ckpt=None) == OK


def test_sizes():
    assert B.adagc_act8_bytes(3, 32) == 3 * 33
    assert B.adagc_act8_bytes(3, 33) == 3 * 66
    assert B.adagc_act8_bytes(0, 5) == 0
    assert B.adagc_act8_bytes(1 << 30, 1 << 20) == (1 << 30) * ((1 << 20) + (1 << 15))
    assert B.adagc_token_logprobs_workspace_bytes(4096, 128256, 5) == 0
    assert B.adagc_token_logprobs_workspace_bytes(1, 128256, 0) < B.adagc_token_logprobs_workspace_bytes(1, 128256, 5) < 1 << 16
    for bad in ((-1, 5), (1, 0)):
        with pytest.raises(B.AdagcError):
            B.adagc_act8_bytes(*bad)
    with pytest.raises(B.AdagcError):
        B.adagc_token_logprobs_workspace_bytes(1, 4, 5)
    with pytest.raises(B.AdagcError):
        B.adagc_act8_wgrad_workspace_bytes(1, 4, 5, 2)
    for rows, n_out, n_in in ((1, 1, 1), (8192, 64, 64), (8192, 14336, 4096), (0, 5, 5)):
        assert 0 <= B.adagc_act8_wgrad_workspace_bytes(rows, n_out, n_in, B.ADAGC_BF16) <= 1 << 31


def test_sizes_take_numpy_integers():
    np = pytest.importorskip("numpy")
    assert B.adagc_act8_bytes(np.int64(3), np.int32(33)) == 3 * 66
    assert B.adagc_token_logprobs_workspace_bytes(np.int64(4096), np.int64(128256), np.int64(5)) == 0
    assert B.adagc_act8_wgrad_workspace_bytes(np.int64(0), np.int64(5), np.int64(5), np.int64(1)) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    f = lambda *s: torch.zeros(*s)
    ckpt = torch.zeros(B.adagc_act8_bytes(4, 64), dtype=torch.uint8)
    for error, call in [
        (TypeError, lambda: B.adagc_act8_pack(torch.zeros(4, 64, dtype=torch.float16), ckpt)),
        (ValueError, lambda: B.adagc_act8_pack(bf(4, 128)[:, ::2], ckpt)),
        (ValueError, lambda: B.adagc_act8_pack(bf(4, 65), ckpt)),
        (ValueError, lambda: B.adagc_act8_pack(bf(4, 64), None)),
        (ValueError, lambda: B.adagc_act8_pack(bf(64), ckpt)),
        (ValueError, lambda: B.adagc_act8_unpack(ckpt, bf(5, 64))),
        (ValueError, lambda: B.adagc_swiglu(bf(4, 64), bf(4, 63), bf(4, 64))),
        (TypeError, lambda: B.adagc_swiglu(bf(4, 64), f(4, 64), bf(4, 64))),
        (ValueError, lambda: B.adagc_swiglu(bf(4, 64), bf(4, 64), bf(4, 64), ckpt, ckpt[1:])),
        (B.AdagcError, lambda: B.adagc_swiglu(bf(4, 64), bf(1, 64).expand(4, 64), bf(4, 64))),
        (TypeError, lambda: B.adagc_swiglu_backward(bf(4, 64), ckpt, ckpt, bf(4, 64), f(4, 64))),
        (ValueError, lambda: B.adagc_act8_wgrad(bf(4, 10), ckpt, f(11, 64))),
        (ValueError, lambda: B.adagc_act8_wgrad(bf(5, 10), ckpt, f(10, 64))),
        (ValueError, lambda: B.adagc_token_logprobs(f(4, 10), torch.zeros(5, dtype=torch.int64), f(4))),
        (TypeError, lambda: B.adagc_token_logprobs(f(4, 10), torch.zeros(4, dtype=torch.int32), f(4))),
        (TypeError, lambda: B.adagc_token_logprobs(f(4, 10), torch.zeros(4, dtype=torch.int64), f(4).double())),
        (ValueError, lambda: B.adagc_token_logprobs(f(4, 10), stats=f(4, 4)[:, ::2])),
        (ValueError, lambda: B.adagc_token_logprobs(f(4, 10), top_logprob=f(4, 3), top_index=torch.zeros(4, 2, dtype=torch.int32))),
        (ValueError, lambda: B.adagc_token_logprobs(f(1, 128256), entropy=f(1))),
        (TypeError, lambda: B.adagc_token_logprobs_backward(f(4, 10), None, f(4, 2), None, None, None, bf(4, 10))),
        (ValueError, lambda: B.adagc_token_logprobs_backward(f(4, 10), None, f(4, 2), None, None, None, f(4, 11))),
    ]:
        with pytest.raises(error):
            call()


def test_binding_refuses_host_memory():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    f = lambda *s: torch.zeros(*s)
    ckpt = torch.zeros(B.adagc_act8_bytes(4, 64), dtype=torch.uint8)
    for call in (lambda: B.adagc_act8_pack(bf(4, 64), ckpt), lambda: B.adagc_act8_unpack(ckpt, bf(4, 64)),
                 lambda: B.adagc_swiglu(bf(4, 64), bf(4, 64), bf(4, 64)),
                 lambda: B.adagc_swiglu_backward(bf(4, 64), ckpt, ckpt.clone(), bf(4, 64), bf(4, 64)),
                 lambda: B.adagc_act8_wgrad(bf(4, 10), ckpt, f(10, 64)), lambda: B.adagc_token_logprobs(f(4, 10), entropy=f(4)),
                 lambda: B.adagc_token_logprobs_backward(f(4, 10), None, f(4, 2), f(4), None, f(4), f(4, 10))):
        with pytest.raises(B.AdagcError, match="not in device memory"):
            call()


# ---- the oracle: hand-worked values and torch's own routines

def test_oracle_pack():
    x = torch.zeros(1, 40, dtype=torch.float64)
    x[0, :6] = torch.tensor([448.0, -1.0625, 1.1875, 2.0 ** -9, 2.0 ** -10, -0.0])
    x[0, 32:36] = torch.tensor([449.0, math.inf, math.nan, 1.0])
    codes, e = O.pack(x)
    assert e.tolist() == [[0, 1]]
    # 1.0625 and 1.1875 lie halfway: to 1.0 and 1.25, the even ones; 2^-9 is the least number, half of it goes to 0
    assert codes[0, :6].tolist() == [0x7E, 0xB8, 0x3A, 0x01, 0x00, 0x80]
    assert codes[0, 32:36].tolist() == [0x76, 0x7F, 0x7F, 0x30]        # 449 / 2 = 224.5 -> 224
    assert (codes[0, 36:] == 0).all() and codes.shape == (1, 64)
    assert O.pack(torch.zeros(1, 1))[1].tolist() == [[-100]]
    y = torch.randn(50, 70, generator=torch.Generator().manual_seed(1)) * 100
    codes, e = O.pack(y)
    scaled = torch.nn.functional.pad(y, (0, 26)).view(50, 3, 32).double() * O.pow2(-e)[:, :, None]
    assert torch.equal(codes.view(50, 3, 32), scaled.float().to(torch.float8_e4m3fn).view(torch.uint8))
    held = O.values(O.pack_bytes(y), 50, 70)
    assert ((held - y.double()).abs() <= y.double().abs() / 16 + 2.0 ** -10 * 4).all()


def test_oracle_logprobs_and_gradient():
    g = torch.Generator().manual_seed(2)
    z = torch.randn(5, 11, generator=g, dtype=torch.float64, requires_grad=True)
    t = torch.tensor([0, 10, -1, 3, -100])
    f = O.logprobs(z.detach(), t, 0.7)
    dist = torch.distributions.Categorical(logits=0.7 * z)
    assert torch.allclose(f["logp"], torch.log_softmax(0.7 * z, 1).detach(), rtol=1e-13)
    assert torch.allclose(f["entropy"], dist.entropy().detach(), rtol=1e-13)
    dl, dh = torch.randn(5, generator=g, dtype=torch.float64), torch.randn(5, generator=g, dtype=torch.float64)
    loss = (dl * torch.where(t >= 0, torch.log_softmax(0.7 * z, 1).gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)).sum() + (dh * dist.entropy()).sum()
    loss.backward()
    grad, _ = O.logprobs_backward(z.detach(), t, 0.7, dl, dh)
    assert torch.allclose(grad, z.grad, rtol=1e-11, atol=1e-14)


def test_oracle_swiglu_gradient():
    g = torch.Generator().manual_seed(3)
    gate, up, d = (torch.randn(4, 6, generator=g, dtype=torch.float64) for _ in range(3))
    gate.requires_grad_()
    up.requires_grad_()
    out = torch.nn.functional.silu(gate) * up
    out.backward(d)
    (dg, _), (du, _), (again, _) = O.swiglu_backward(d, gate.detach(), up.detach())
    assert torch.allclose(dg, gate.grad, rtol=1e-12) and torch.allclose(du, up.grad, rtol=1e-12) and torch.allclose(again, out.detach(), rtol=1e-13)
