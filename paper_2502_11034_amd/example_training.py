"""A small language model trained with this library: forward and backward pass with activations kept in 8 bits, then the AdaGC step.

    python -m paper_2502_11034_amd.example_training [--steps 200] [--vocab 512] [--dim 256] [--hidden 512] [--tokens 2048]

One gated layer between an embedding and a head, predicting the next token of a synthetic Markov chain.  Matrix products with the weights
are torch's; everything else on the way from the logits to the new weights is the library's:

    h0 = E[t]                                 adagc_act8_pack(h0)
    a = silu(h0 Wg^T) * (h0 Wu^T)             adagc_swiglu, which leaves both factors in checkpoints
    h1 = h0 + a Wd^T                          adagc_act8_pack(h1)
    log p(t') of softmax(h1 Wo^T)             adagc_token_logprobs, and its gradient
    dWo, dWd, dWg, dWu                        adagc_act8_wgrad; a for dWd is made again by adagc_swiglu_backward
    E, Wg, Wu, Wd, Wo                         adagc_step (AdamW on fp32 weights, with the bf16 copies that the next step reads)

What is kept of a token between the passes is 33/32 bytes for each value of h0, gate, up and h1, beside the logits.
"""
import argparse

import torch

from . import binding as B

DEV = "cuda:0"


class Model:
    """Weights, optimizer state and all buffers of a step on a fixed number of tokens; nothing is allocated by step() but by torch."""

    def __init__(self, vocab, dim, hidden, tokens, entropy_weight=0.0, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def weight(rows, cols, size):
            return torch.randn(rows, cols, generator=g, device=DEV).mul_(size)

        self.vocab, self.tokens, self.entropy_weight = vocab, tokens, entropy_weight
        self.weights = [weight(vocab, dim, 1.0), weight(hidden, dim, dim ** -0.5), weight(hidden, dim, dim ** -0.5),
                        weight(dim, hidden, hidden ** -0.5), weight(vocab, dim, dim ** -0.5)]
        self.copies = [w.bfloat16() for w in self.weights]
        self.grads = [torch.zeros_like(w) for w in self.weights]
        self.m = [torch.zeros_like(w) for w in self.weights]
        self.v = [torch.zeros_like(w) for w in self.weights]
        self.gamma = torch.zeros(len(self.weights), device=DEV)
        self.opt = B.AdaGC([w.numel() for w in self.weights], B.ADAGC_OPT_ADAMW, B.ADAGC_GRAD_F32, has_bf16_param_copy=True)
        self.opt.set_param_copies(self.copies)
        self.hyper = B.make_hyper(lr=3e-3, lambda_rel=1.05, ema_beta=0.98, lambda_abs=1.0, t_start=20)
        self.t = 0

        def new(*shape, dtype=torch.bfloat16):
            return torch.empty(shape, dtype=dtype, device=DEV)

        def checkpoint(cols):
            return new(B.adagc_act8_bytes(tokens, cols), dtype=torch.uint8)

        self.c_h0, self.c_h1, self.c_a = checkpoint(dim), checkpoint(dim), checkpoint(hidden)
        self.c_gate, self.c_up = checkpoint(hidden), checkpoint(hidden)
        self.a, self.d_gate, self.d_up = new(tokens, hidden), new(tokens, hidden), new(tokens, hidden)
        self.logprob, self.entropy, self.stats = (new(*s, dtype=torch.float32) for s in ((tokens,), (tokens,), (tokens, 2)))
        self.d_logprob = torch.full((tokens,), -1.0 / tokens, device=DEV)                    # the loss is the mean of -log p ...
        self.d_entropy = torch.full((tokens,), -entropy_weight / tokens, device=DEV)         # ... less a bonus for entropy
        sizes = [(vocab, dim), (hidden, dim), (dim, hidden)]
        self.workspace = new(max([B.adagc_token_logprobs_workspace_bytes(tokens, vocab, 0)] +
                                 [B.adagc_act8_wgrad_workspace_bytes(tokens, o, i, B.ADAGC_BF16) for o, i in sizes]), dtype=torch.uint8)

    def logits(self, t, keep=True):
        e, wg, wu, wd, wo = self.copies
        s = torch.cuda.current_stream().cuda_stream
        h0 = e[t]
        gate, up = h0 @ wg.t(), h0 @ wu.t()
        a = self.a if keep else torch.empty_like(gate)
        if keep:
            B.adagc_act8_pack(h0, self.c_h0, stream=s)
            B.adagc_swiglu(gate, up, a, self.c_gate, self.c_up, stream=s)
        else:
            B.adagc_swiglu(gate, up, a, stream=s)
        h1 = torch.addmm(h0, a, wd.t())
        if keep:
            B.adagc_act8_pack(h1, self.c_h1, stream=s)
        return h1 @ wo.t()

    def gradients(self, t, target):
        """Log-probabilities of the targets (below 0: none), with the gradients in self.grads."""
        _, wg, wu, wd, wo = self.copies
        d_e, d_wg, d_wu, d_wd, d_wo = self.grads
        s = torch.cuda.current_stream().cuda_stream
        z = self.logits(t)
        B.adagc_token_logprobs(z, target, self.logprob, self.entropy, self.stats, workspace=self.workspace, stream=s)
        B.adagc_token_logprobs_backward(z, target, self.stats, self.entropy, self.d_logprob, self.d_entropy if self.entropy_weight else None, z,
                                        stream=s)
        B.adagc_act8_wgrad(z, self.c_h1, d_wo, workspace=self.workspace, stream=s)
        d_h1 = z @ wo
        d_a = d_h1 @ wd
        B.adagc_swiglu_backward(d_a, self.c_gate, self.c_up, self.d_gate, self.d_up, self.a, stream=s)
        B.adagc_act8_pack(self.a, self.c_a, stream=s)
        B.adagc_act8_wgrad(d_h1, self.c_a, d_wd, workspace=self.workspace, stream=s)
        B.adagc_act8_wgrad(self.d_gate, self.c_h0, d_wg, workspace=self.workspace, stream=s)
        B.adagc_act8_wgrad(self.d_up, self.c_h0, d_wu, workspace=self.workspace, stream=s)
        d_h0 = torch.addmm(torch.addmm(d_h1, self.d_gate, wg), self.d_up, wu)
        d_e.zero_().index_add_(0, t, d_h0.float())
        return self.logprob

    def step(self, t, target):
        logprob = self.gradients(t, target)
        self.t += 1
        self.opt.step(self.weights, self.grads, self.m, self.v, self.gamma, self.hyper, self.t, stream=torch.cuda.current_stream().cuda_stream)
        return logprob

    def most_likely(self, t, k):
        """(log-probabilities, tokens) of the k most likely next tokens after each of t."""
        z = self.logits(t, keep=False)
        n = len(t)
        logp, index = torch.empty(n, k, device=DEV), torch.empty(n, k, dtype=torch.int32, device=DEV)
        ws = torch.empty(B.adagc_token_logprobs_workspace_bytes(n, self.vocab, k), dtype=torch.uint8, device=DEV)
        B.adagc_token_logprobs(z, top_logprob=logp, top_index=index, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)
        return logp, index


class Chain:
    """Tokens of which each is followed by one of four, with probabilities 0.6, 0.2, 0.15 and 0.05."""
    P = (0.6, 0.2, 0.15, 0.05)

    def __init__(self, vocab, seed=1):
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        self.vocab = vocab
        self.next = torch.stack([torch.randperm(vocab, generator=self.g, device=DEV) for _ in self.P], 1)

    def pairs(self, n):
        t = torch.randint(0, self.vocab, (n,), generator=self.g, device=DEV)
        which = torch.multinomial(torch.tensor(self.P, device=DEV), n, replacement=True, generator=self.g)
        return t, self.next[t, which]


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("steps", 200), ("vocab", 512), ("dim", 256), ("hidden", 512), ("tokens", 2048)):
        parser.add_argument("--" + name, type=int, default=value)
    args = parser.parse_args(argv)
    model, chain = Model(args.vocab, args.dim, args.hidden, args.tokens), Chain(args.vocab)
    loss = 0.0
    for step in range(args.steps):
        logprob = model.step(*chain.pairs(args.tokens))
        if step % 20 == 0 or step == args.steps - 1:
            loss = -logprob.mean().item()
            print("step %4d  loss %.4f  entropy %.4f" % (step, loss, model.entropy.mean().item()), flush=True)
    t = torch.arange(min(4, args.vocab), device=DEV)
    logp, index = model.most_likely(t, 4)
    for i in range(len(t)):
        print("after %d: %s (drawn with 0.6, 0.2, 0.15, 0.05: %s)" % (
            i, ", ".join("%d %.2f" % (j, p) for j, p in zip(index[i].tolist(), logp[i].exp().tolist())), chain.next[i].tolist()))
    return loss


if __name__ == "__main__":
    main()
