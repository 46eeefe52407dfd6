"""Arithmetic sampling from a small model of one's own, with what serving puts on its logits: a runnable example.

    python -m paper_2210_15458_amd.shaped_decode [--prompts 4] [--codes 16] [--steps 24]

The model is an embedding, one feed-forward block on a residual stream and a head, all of it layers of this library; each
prompt is decoded by N lattice codes (Sec. 4.2 of the paper), with penalties for repeated tokens, a request's token biases and a
grammar of its own per code.  One step is five calls, on one stream, without a host round trip, captured once in a graph:

    as_history_add     the token of the step before joins each sequence's record
    as_linear  x 2     h = x + W2 silu(W1 x + b1) + b2
    as_linear          logits = 30 tanh(W h / 30), shaped and rounded in the same pass
    as_step_ex         the token whose interval holds the code, and the code in it
"""
import argparse

import torch

from . import binding as B


class Grammar:
    """A finite automaton over classes of tokens: allowed [states, V] truth values, follows [states, classes] the next state."""

    def __init__(self, allowed, token_class, follows):
        states, V = allowed.shape
        words = (V + 31) // 32
        bits = torch.zeros(states, words * 32, dtype=torch.bool, device=allowed.device)
        bits[:, :V] = allowed
        weight = torch.bitwise_left_shift(torch.ones(32, dtype=torch.int32, device=allowed.device),
                                          torch.arange(32, dtype=torch.int32, device=allowed.device))
        self.allowed, self.token_class, self.follows = allowed, token_class.long(), follows.int()
        self.mask = (bits.view(states, words, 32) * weight).sum(dim=2, dtype=torch.int32)


class ShapedDecoder:
    """Decodes B prompts by N codes each, one token a step."""

    def __init__(self, E, W1, b1, W2, b2, head, B_, N, grammar=None, bias=None, repetition=1.2, presence=0.2, frequency=0.1,
                 temp=0.8, top_k=0, top_p=0.95, eos_id=1, cap=30.0, stream=None):
        V, d = E.shape
        self.E, self.V, self.N, self.rows = E, V, N, B_ * N
        self.temp, self.top_k, self.top_p, self.eos_id, self.grammar = temp, top_k, top_p, eos_id, grammar
        self.ctx = B.Ctx(self.rows, V, torch.bfloat16, stream=stream)
        self.up, self.down = B.Layer(W1, bias=b1, act="silu"), B.Layer(W2, bias=b2)
        self.head = B.Layer(head, act="softcap", act_arg=cap)
        new = lambda *shape, **kw: torch.zeros(*shape, device="cuda", **kw)  # noqa: E731
        self.seen, self.counts = new(self.rows, (V + 31) // 32, dtype=torch.int32), new(self.rows, V, dtype=torch.int32)
        self.tokens, self.codes = new(self.rows, dtype=torch.int32), new(self.rows)
        self.finished, self.state = new(self.rows, dtype=torch.uint8), new(self.rows, dtype=torch.int32)
        self.hidden, self.h = new(self.rows, W1.shape[0], dtype=torch.bfloat16), new(self.rows, d, dtype=torch.bfloat16)
        self.logits = new(self.rows, V, dtype=torch.bfloat16)
        strength = lambda v: torch.full((self.rows,), v, device="cuda")  # noqa: E731
        self.shaping = B.Shaping(self.rows, V, seen=self.seen, counts=self.counts, repetition=strength(repetition),
                                 presence=strength(presence), frequency=strength(frequency), bias=bias,
                                 mask=None if grammar is None else grammar.mask, mask_ids=None if grammar is None else self.state,
                                 finished=self.finished)

    def start(self, prompts, u):
        """prompts: lists of token ids, one each; u: a shift of the lattice each."""
        offsets = torch.tensor([0] + [len(p) for p in prompts]).cumsum(0).cuda()
        flat = torch.tensor([t for p in prompts for t in p], dtype=torch.int32, device="cuda")
        B.as_history_set(self.ctx, self.seen, self.counts, flat, offsets, self.N)
        B.as_lattice(self.ctx, u, self.N, self.codes)
        self.tokens.copy_(torch.tensor([p[-1] for p in prompts], dtype=torch.int32, device="cuda").repeat_interleave(self.N))
        self.finished.zero_()
        self.state.zero_()

    def forward(self):
        """The shaped logits that follow self.tokens."""
        x = self.E[self.tokens.long()]
        B.as_linear(self.ctx, self.up, x, self.hidden)
        B.as_linear(self.ctx, self.down, self.hidden, self.h, residual=x)
        B.as_linear(self.ctx, self.head, self.h, self.logits, shaping=self.shaping)

    def step(self):
        self.forward()
        B.as_step_ex(self.ctx, self.logits, self.codes, self.temp, self.top_k, self.top_p, self.tokens, self.codes,
                     finished_in=self.finished, eos_id=self.eos_id, finished_out=self.finished)
        if self.grammar is not None:
            self.state.copy_(self.grammar.follows[self.state.long(), self.grammar.token_class[self.tokens.long()]])
        B.as_history_add(self.ctx, self.seen, self.counts, self.tokens, self.finished)


def example_model(V=4000, d=256, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = lambda *s: (torch.randn(*s, device="cuda", generator=g) * s[-1] ** -0.5).to(torch.bfloat16)  # noqa: E731
    return {"E": torch.randn(V, d, device="cuda", generator=g).to(torch.bfloat16), "W1": w(4 * d, d), "b1": w(4 * d),
            "W2": w(d, 4 * d), "b2": w(d), "head": (3 * w(V, d).float()).to(torch.bfloat16)}


def example_grammar(V, eos_id=1):
    """Words (ids from 100 on) and digits (10 .. 19): a digit after every third word, then the end or a word."""
    ids = torch.arange(V, device="cuda")
    word, digit, end = ids >= 100, (ids >= 10) & (ids < 20), ids == eos_id
    allowed = torch.stack([word, word, word, digit, word | end])
    follows = torch.tensor([[1, 0, 0], [2, 0, 0], [3, 0, 0], [0, 4, 0], [1, 0, 4]], device="cuda")      # by word, digit, other
    return Grammar(allowed, torch.where(word, 0, torch.where(digit, 1, 2)), follows)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--prompts", type=int, default=4)
    ap.add_argument("--codes", type=int, default=16)
    ap.add_argument("--steps", type=int, default=24)
    a = ap.parse_args()
    model = example_model()
    V = model["E"].shape[0]
    bias = torch.zeros(1, V, device="cuda")
    bias[0, 100:110] = -float("inf")                     # words that this request forbids
    g = torch.Generator().manual_seed(3)
    prompts = [torch.randint(100, V, (int(n),), generator=g).tolist() for n in torch.randint(1, 20, (a.prompts,), generator=g)]
    u = torch.rand(a.prompts, generator=g).cuda()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        d = ShapedDecoder(**model, B_=a.prompts, N=a.codes, grammar=example_grammar(V), bias=bias, stream=side)
        d.start(prompts, u)
        d.step()                                         # (the first call of a size may allocate: not under capture)
        side.synchronize()
        d.start(prompts, u)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            d.step()
        out = []
        for _ in range(a.steps):
            graph.replay()
            out.append(d.tokens.clone())
        side.synchronize()
    tokens = torch.stack(out, dim=1).view(a.prompts, a.codes, a.steps).cpu()
    for b, p in enumerate(prompts):
        print(f"prompt of {len(p)} tokens: {len({tuple(s) for s in tokens[b].tolist()})} different continuations of {a.codes} codes")
        for s in tokens[b, :2].tolist():
            print("   ", *(t for i, t in enumerate(s) if 1 not in s[:i]))


if __name__ == "__main__":
    main()
