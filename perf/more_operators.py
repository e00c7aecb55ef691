"""Timed cases of the operators that make the gradients the optimizer step takes without keeping what they make on the way: token
log-probabilities straight from the head's input and weights (no logits are kept), the gated projections of a feed-forward layer
(both products and the activation in one pass), and dropout whose mask is made again where it is needed.

A case names an operator and its sizes.  ``prepare`` makes what a training program holds before the call, ``run`` is one pass (a
training pass forward and backward), ``exact`` the same from the definitions in 64 bits.  With ``own`` false ``run`` is
elementary torch in 32 bits, with ``own`` true the library's kernels.

Dropout's random words: value j of row i of a rows x cols matrix takes word j mod 4 of block number offset + i ceil(cols / 4) + j / 4
(modulo 2^64) of Philox4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011), with the block number in the
counter's first two words, zeros in its others, and the seed as key.  It is kept if the word is at least p 2^32, rounded to whole.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # scoring a single sampled token with Llama-3-8B's head: every weight is read for one row
        dict(name="score_one_token_llama3_8b", op="loss", rows=1, vocab=128256, dim=4096, dtype="bf16", scale=1.0, backward=False),
        # scoring a prompt's tokens with GPT-2's head at another temperature
        dict(name="score_prompt_gpt2", op="loss", rows=1024, vocab=50257, dim=768, dtype="bf16", scale=1.25, backward=False),
        # a training step of a small fp32 model, odd numbers of everything
        dict(name="loss_fp32_odd", op="loss", rows=333, vocab=8191, dim=765, dtype="f32", scale=1.0, backward=True),
        # a training step of GPT-2's head: loss and both gradients
        dict(name="loss_gpt2", op="loss", rows=4096, vocab=50257, dim=768, dtype="bf16", scale=1.0, backward=True),
        # a training step of Llama-3-8B's head: the large end
        dict(name="loss_llama3_8b", op="loss", rows=4096, vocab=128256, dim=4096, dtype="bf16", scale=1.0, backward=True),
        # one token through a GPT-2-sized gated layer: latency
        dict(name="gated_one_token", op="gated", rows=1, dim=768, hidden=2048, dtype="bf16", kept=False, backward=False),
        # a few sequences' tokens through Llama-3-8B's gated layer: every weight is read for them
        dict(name="gated_few_tokens_llama3_8b", op="gated", rows=24, dim=4096, hidden=14336, dtype="bf16", kept=False, backward=False),
        # a training step of a small fp32 model's gated layer, odd numbers of everything, nothing kept between the passes
        dict(name="gated_fp32_odd", op="gated", rows=333, dim=765, hidden=2731, dtype="f32", kept=False, backward=True),
        # a training step of Llama-3-8B's gated layer on 8192 tokens, both products kept for the backward pass
        dict(name="gated_llama3_8b", op="gated", rows=8192, dim=4096, hidden=14336, dtype="bf16", kept=True, backward=True),
        # dropout and residual of a few tokens: latency
        dict(name="dropout_few_tokens", op="dropout", rows=7, cols=768, dtype="bf16", p=0.1, residual=True, backward=False),
        # dropout of a small fp32 model's activation, odd numbers of rows and columns, both ways
        dict(name="dropout_fp32_odd", op="dropout", rows=333, cols=2731, dtype="f32", p=0.25, residual=False, backward=True),
        # dropout before the residual sum of 16384 tokens of Llama-3-8B, both ways
        dict(name="dropout_llama3_8b", op="dropout", rows=16384, cols=4096, dtype="bf16", p=0.1, residual=True, backward=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case of the listed ranges: sizes over their logarithm, odd ones among them."""
    op = rng.choice(["loss", "loss", "gated", "gated", "dropout"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op == "dropout":
        return dict(op=op, rows=_log_uniform(rng, 1, 16384), cols=_log_uniform(rng, 32, 4096), dtype=dtype,
                    p=rng.choice([0.0, 0.05, 0.1, 0.25, 0.5]), residual=rng.random() < 0.5, backward=rng.random() < 0.5)
    backward = rng.random() < 0.6
    most = 2 ** 41 if dtype == "bf16" else 2 ** 36                         # multiplications of one product
    if op == "loss":
        vocab = rng.choice([_log_uniform(rng, 257, 128256), 32000, 50257, 128256])
        dim = rng.choice([_log_uniform(rng, 64, 4096), 768, 1024, 4096])
        rows = _log_uniform(rng, 1, min(4096, most // (vocab * dim)))
        return dict(op=op, rows=rows, vocab=vocab, dim=dim, dtype=dtype, scale=rng.choice([1.0, 1.0, 0.7, 1.25]), backward=backward)
    dim = rng.choice([_log_uniform(rng, 64, 4096), 768, 1024, 4096])
    hidden = _log_uniform(rng, 64, 14336)
    rows = _log_uniform(rng, 1, min(8192, most // (2 * hidden * dim)))
    return dict(op=op, rows=rows, dim=dim, hidden=hidden, dtype=dtype, kept=backward and rng.random() < 0.5, backward=backward)


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dtype, rows = TYPES[case["dtype"]], case["rows"]

    def normal(r, c, size):
        return torch.randn(r, c, generator=g, device=DEV).mul_(size)

    state = {"case": case, "dtype": dtype, "buffers": {}}
    if case["op"] == "loss":
        vocab, dim = case["vocab"], case["dim"]
        weight = normal(vocab, dim, dim ** -0.5)
        targets = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
        x = normal(rows, dim, 2.0)
        x += weight[targets] * (8 * torch.rand(rows, 1, generator=g, device=DEV))                  # a model that has learned something
        targets[torch.rand(rows, generator=g, device=DEV) < 0.03] = -1                             # padding
        state.update(x=x.to(dtype), weight=weight.to(dtype), targets=targets)
        if case["backward"]:
            state["d_logprob"] = (torch.rand(rows, generator=g, device=DEV) - 1.5) / rows
    elif case["op"] == "gated":
        dim, hidden = case["dim"], case["hidden"]
        state["x"] = normal(rows, dim, 1.0).to(dtype)
        state["w_gate"], state["w_up"] = (normal(hidden, dim, dim ** -0.5).to(dtype) for _ in range(2))
        if case["backward"]:
            state["d_out"] = normal(rows, hidden, 1e-3).to(dtype)
    else:
        state["x"] = normal(rows, case["cols"], 1.0).to(dtype)
        if case["residual"]:
            state["residual"] = normal(rows, case["cols"], 2.0).to(dtype)
        if case["backward"]:
            state["d_out"] = normal(rows, case["cols"], 1e-3).to(dtype)
        state["rng"] = torch.randint(-2 ** 63, 2 ** 63 - 1, (2,), generator=g, device=DEV)          # seed and offset
    return state


# ------------------------------------------------------------------------------------------------ one pass, plain

def _plain_loss(state):
    case, x, w, targets = state["case"], state["x"].float(), state["weight"].float(), state["targets"]
    s, has = case["scale"], targets >= 0
    at = targets.clamp(min=0)[:, None]
    z = torch.mm(x, w.t())
    most = z.amax(1, keepdim=True)
    logp = (z - most).mul_(s)
    log_sum = logp.exp().sum(1, keepdim=True).log()
    logp -= log_sum
    out = {"logprob": torch.where(has, logp.gather(1, at)[:, 0], torch.zeros_like(most[:, 0])), "stats": torch.cat([most, log_sum], 1)}
    if case["backward"]:
        d_logprob = torch.where(has, state["d_logprob"], torch.zeros_like(state["d_logprob"]))[:, None]
        d_z = logp.exp_().mul_(-d_logprob)
        d_z.scatter_add_(1, at, d_logprob)
        d_z *= s
        out["d_x"] = torch.mm(d_z, w).to(state["dtype"])
        out["d_weight"] = torch.mm(d_z.t(), x).to(state["dtype"])
    return out


def _plain_gated(state):
    case, dtype = state["case"], state["dtype"]
    x, w_gate, w_up = (state[name].float() for name in ("x", "w_gate", "w_up"))
    gate, up = torch.mm(x, w_gate.t()), torch.mm(x, w_up.t())
    t = 1 / (1 + torch.exp(-gate))
    out = {"out": (gate * t * up).to(dtype)}
    if case["kept"]:
        out["gate"], out["up"] = gate.to(dtype), up.to(dtype)
    if case["backward"]:
        d_out = state["d_out"].float()
        d_gate = d_out * up * t * (1 + gate * (1 - t))
        d_up = d_out * gate * t
        out["d_x"] = (torch.mm(d_gate, w_gate) + torch.mm(d_up, w_up)).to(dtype)
        out["d_w_gate"], out["d_w_up"] = torch.mm(d_gate.t(), x).to(dtype), torch.mm(d_up.t(), x).to(dtype)
    return out


def _keep(case, rng):
    """Truth values [rows][cols]: the words of the module's description, in whole numbers of 64 bits that wrap around."""
    rows, cols = case["rows"], case["cols"]
    blocks = -(-cols // 4)
    low = 0xFFFFFFFF
    n = torch.arange(rows * blocks, device=DEV) + rng[1]
    c0, c1 = n & low, (n >> 32) & low
    c2, c3 = torch.zeros_like(n), torch.zeros_like(n)
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 1).view(rows, 4 * blocks)[:, :cols]
    return words >= round(case["p"] * 2 ** 32)


def _plain_dropout(state):
    case, dtype = state["case"], state["dtype"]
    keep, factor = _keep(case, state["rng"]), 1 / (1 - case["p"])
    y = torch.where(keep, state["x"].float() * factor, 0.0)
    if case["residual"]:
        y += state["residual"].float()
    out = {"out": y.to(dtype)}
    if case["backward"]:
        out["d_x"] = torch.where(keep, state["d_out"].float() * factor, 0.0).to(dtype)
    return out


# ------------------------------------------------------------------------------------------------ one pass, the library's

def _buffers(state):
    """Outputs and workspaces, which a training loop allocates once."""
    from paper_2502_11034_amd import binding as B
    case, b = state["case"], state["buffers"]
    if b:
        return B, b
    rows, dtype = case["rows"], state["dtype"]
    code = B.ADAGC_F32 if case["dtype"] == "f32" else B.ADAGC_BF16

    def new(*shape, dtype=dtype):
        return torch.empty(shape, dtype=dtype, device=DEV)

    need = 0
    if case["op"] == "loss":
        vocab, dim = case["vocab"], case["dim"]
        b.update(logprob=new(rows, dtype=torch.float32), stats=new(rows, 2, dtype=torch.float32))
        need = B.adagc_linear_logprobs_workspace_bytes(rows, vocab, dim, code)
        if case["backward"]:
            b.update(d_x=new(rows, dim), d_weight=new(vocab, dim))
            need = max(need, B.adagc_linear_logprobs_backward_workspace_bytes(rows, vocab, dim, code))
    elif case["op"] == "gated":
        dim, hidden = case["dim"], case["hidden"]
        b["out"] = new(rows, hidden)
        if case["kept"]:
            b.update(gate=new(rows, hidden), up=new(rows, hidden))
        need = B.adagc_gated_linear_workspace_bytes(rows, dim, hidden, code)
        if case["backward"]:
            b.update(d_x=new(rows, dim), d_w_gate=new(hidden, dim), d_w_up=new(hidden, dim))
            need = max(need, B.adagc_gated_linear_backward_workspace_bytes(rows, dim, hidden, code))
    else:
        b["out"] = new(rows, case["cols"])
        if case["backward"]:
            b["d_x"] = new(rows, case["cols"])
    b["workspace"] = new(need, dtype=torch.uint8)
    return B, b


def run(state):
    case = state["case"]
    if not own:
        return {"loss": _plain_loss, "gated": _plain_gated, "dropout": _plain_dropout}[case["op"]](state)
    B, b = _buffers(state)
    stream = torch.cuda.current_stream().cuda_stream
    if case["op"] == "loss":
        x, w, t = state["x"], state["weight"], state["targets"]
        B.adagc_linear_logprobs(x, w, t, b["logprob"], b["stats"], scale=case["scale"], workspace=b["workspace"], stream=stream)
        if case["backward"]:
            B.adagc_linear_logprobs_backward(x, w, t, b["stats"], state["d_logprob"], b["d_x"], b["d_weight"], scale=case["scale"],
                                             workspace=b["workspace"], stream=stream)
    elif case["op"] == "gated":
        x, w_gate, w_up = state["x"], state["w_gate"], state["w_up"]
        B.adagc_gated_linear(x, w_gate, w_up, b["out"], b.get("gate"), b.get("up"), workspace=b["workspace"], stream=stream)
        if case["backward"]:
            B.adagc_gated_linear_backward(state["d_out"], x, w_gate, w_up, b["d_x"], b["d_w_gate"], b["d_w_up"], gate=b.get("gate"),
                                          up=b.get("up"), workspace=b["workspace"], stream=stream)
    else:
        B.adagc_dropout(state["x"], b["out"], state["rng"], case["p"], residual=state.get("residual"), stream=stream)
        if case["backward"]:
            B.adagc_dropout(state["d_out"], b["d_x"], state["rng"], case["p"], stream=stream)
    return {name: value for name, value in b.items() if name != "workspace"}


# ------------------------------------------------------------------------------------------------ work

def work(case):
    """Inputs once in, outputs once out; the products of the formulas once each, also where nothing is kept between the passes."""
    rows, size = case["rows"], 4 if case["dtype"] == "f32" else 2
    if case["op"] == "loss":
        vocab, dim = case["vocab"], case["dim"]
        n, product = (rows + vocab) * dim * size, 2.0 * rows * vocab * dim
        if case["backward"]:
            return {"bytes": float(2 * n + 24 * rows), "flops": 3 * product + 8.0 * rows * vocab}
        return {"bytes": float(n + 20 * rows), "flops": product + 4.0 * rows * vocab}
    if case["op"] == "gated":
        dim, hidden = case["dim"], case["hidden"]
        outer, inner, weights, product = rows * dim, rows * hidden, 2 * hidden * dim, 4.0 * rows * hidden * dim
        n = outer + weights + inner * (3 if case["kept"] else 1)
        if case["backward"]:
            return {"bytes": float((n + outer + weights + inner) * size), "flops": 3 * product + 20.0 * inner}
        return {"bytes": float(n * size), "flops": product + 8.0 * inner}
    n = rows * case["cols"]
    arrays = 2 + (1 if case["residual"] else 0) + (2 if case["backward"] else 0)
    return {"bytes": float(arrays * n * size + 16), "flops": 2.0 * n * (2 if case["backward"] else 1)}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits

def _exact_loss(case, state):
    s, w = case["scale"], state["weight"].double()
    parts, d_weight = [], torch.zeros_like(w) if case["backward"] else None
    step = max(1, 2 ** 27 // case["vocab"])
    for r in range(0, case["rows"], step):
        x, t = state["x"][r:r + step].double(), state["targets"][r:r + step]
        z = x @ w.t()
        total = torch.logsumexp(s * z, 1)
        most = z.max(1).values
        has = torch.nonzero(t >= 0)[:, 0]
        logprob = torch.zeros_like(total)
        logprob[has] = s * z[has, t[has]] - total[has]
        part = {"logprob": logprob, "stats": torch.stack([most, total - s * most], 1)}
        if case["backward"]:
            d = torch.where(t >= 0, state["d_logprob"][r:r + step].double(), 0.0)
            z = torch.softmax(s * z, 1)
            z[has, t[has]] -= 1.0
            z *= (-s * d)[:, None]
            part["d_x"] = z @ w
            d_weight += z.t() @ x
        parts.append(part)
    out = {name: torch.cat([part[name] for part in parts]) for name in parts[0]}
    if case["backward"]:
        out["d_weight"] = d_weight
    return out


def _exact_gated(case, state):
    x, w_gate, w_up = (state[name].double() for name in ("x", "w_gate", "w_up"))
    gate, up = x @ w_gate.t(), x @ w_up.t()
    out = {"out": torch.nn.functional.silu(gate) * up}
    if case["kept"]:
        out["gate"], out["up"] = gate, up
    if case["backward"]:
        d_out, t = state["d_out"].double(), torch.sigmoid(gate)
        d_gate, d_up = d_out * up * (t + gate * t * torch.sigmoid(-gate)), d_out * gate * t
        out["d_x"] = d_gate @ w_gate + d_up @ w_up
        out["d_w_gate"], out["d_w_up"] = d_gate.t() @ x, d_up.t() @ x
    return out


def _times(a, m):
    """High and low half of the 64-bit product of whole numbers a below 2^32 with the constant m, by halves of 16 bits."""
    a0, a1, m0, m1 = a % 65536, a // 65536, m % 65536, m // 65536
    mid = a1 * m0 + a0 * m0 // 65536
    other = a0 * m1 + mid % 65536
    return a1 * m1 + mid // 65536 + other // 65536, other % 65536 * 65536 + a0 * m0 % 65536


def _exact_dropout(case, state):
    rows, cols = case["rows"], case["cols"]
    seed, offset = (int(v) % 2 ** 64 for v in state["rng"].tolist())
    blocks = (cols + 3) // 4
    first = torch.arange(rows * blocks, device=DEV).view(rows, blocks) + offset % 2 ** 32
    counter = [first % 2 ** 32, (first // 2 ** 32 + offset // 2 ** 32) % 2 ** 32, torch.zeros_like(first), torch.zeros_like(first)]
    key = [seed % 2 ** 32, seed // 2 ** 32]
    for i in range(10):
        high0, low0 = _times(counter[0], 0xD2511F53)
        high1, low1 = _times(counter[2], 0xCD9E8D57)
        k0, k1 = (key[0] + i * 0x9E3779B9) % 2 ** 32, (key[1] + i * 0xBB67AE85) % 2 ** 32
        counter = [high1 ^ counter[1] ^ k0, low1, high0 ^ counter[3] ^ k1, low0]
    word = torch.stack(counter, 2).reshape(rows, 4 * blocks)[:, :cols]
    kept = (word.double() / 2 ** 32 >= round(case["p"] * 2 ** 32) / 2 ** 32).double()
    out = {"out": state["x"].double() * kept / (1 - case["p"])}
    if case["residual"]:
        out["out"] = out["out"] + state["residual"].double()
    if case["backward"]:
        out["d_x"] = state["d_out"].double() * kept / (1 - case["p"])
    return out


def exact(case, seed):
    return {"loss": _exact_loss, "gated": _exact_gated, "dropout": _exact_dropout}[case["op"]](case, prepare(case, seed))
