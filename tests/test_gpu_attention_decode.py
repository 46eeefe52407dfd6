"""Layers, cache, attention, shaped head, histories and the sampling step run together, as the example runs them: its logits against the
model's formula in 64 bits on the tokens that it emitted, and a captured step against the calls one by one."""
import numpy as np
import pytest
import torch

from paper_2210_15458_amd import shaped_decode as S

pytestmark = pytest.mark.gpu

PROMPTS = [[150, 151, 150, 900, 300], [333], [101 + i for i in range(60)]]
N, STEPS = 5, 12
HEADS, KV_HEADS = 4, 2


def decoder(model, stream=None, **more):
    torch.cuda.synchronize()
    attention = S.example_attention(model, heads=HEADS, kv_heads=KV_HEADS, prompt_room=60, room=STEPS + 1, **more)
    d = S.ShapedDecoder(**model, B_=len(PROMPTS), N=N, grammar=S.example_grammar(model["E"].shape[0]), stream=stream, attention=attention)
    d.start(PROMPTS, torch.tensor([0.1, 0.5, 0.9], device="cuda"))
    return d, attention


def formula(model, attention, tokens, window, sinks):
    """float64 hidden state of the last of a sequence's tokens behind the blocks and the feed-forward block, and the head's logits."""
    w = {k: v.double().cpu().numpy() for k, v in model.items()}
    x = w["E"][np.array(tokens)]
    n, d = x.shape
    dim = d // HEADS
    at = np.arange(n)
    see = (at[None] <= at[:, None]) & ((window <= 0) | (at[None] > at[:, None] - window) | (at[None] < sinks))
    for qkv, o in attention["blocks"]:
        y = x @ qkv.double().cpu().numpy().T
        q = y[:, :HEADS * dim].reshape(n, HEADS, dim)
        k = y[:, HEADS * dim:(HEADS + KV_HEADS) * dim].reshape(n, KV_HEADS, dim).repeat(HEADS // KV_HEADS, 1)
        v = y[:, (HEADS + KV_HEADS) * dim:].reshape(n, KV_HEADS, dim).repeat(HEADS // KV_HEADS, 1)
        s = np.einsum("ihd,jhd->hij", q, k) / np.sqrt(dim)
        s = np.where(see[None], s, -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        x = x + np.einsum("hij,jhd->ihd", p, v).reshape(n, -1) @ o.double().cpu().numpy().T
    x = x[-1]
    z = w["W1"] @ x + w["b1"]
    h = x + w["W2"] @ (z / (1 + np.exp(-z))) + w["b2"]
    return 30 * np.tanh(w["head"] @ h / 30)


@pytest.mark.parametrize("window,sinks", [(0, 0), (9, 2)])
def test_logits_follow_the_formula(window, sinks):
    model = S.example_model(V=1500, d=128)
    d, attention = decoder(model, window=window, sinks=sinks)
    # no penalties: the logits are the head's, where the grammar leaves them
    for t in (d.shaping._tensors[2], d.shaping._tensors[3], d.shaping._tensors[4]):
        t.fill_(1.0 if t is d.shaping._tensors[2] else 0.0)
    rows = len(PROMPTS) * N
    seqs = [list(PROMPTS[r // N]) for r in range(rows)]
    ended = np.zeros(rows, dtype=bool)
    for t in range(STEPS):
        d.step()
        torch.cuda.synchronize()
        logits, tokens = d.logits.float().cpu().numpy(), d.tokens.cpu().numpy()
        for r in range(rows):
            if ended[r]:
                continue
            want = formula(model, attention, seqs[r], window, sinks)
            free = np.isfinite(logits[r])
            # roundings to bf16 of nine tensors on the way (values up to about 4, half a step 2^-8 each) and of the logits
            assert np.abs(logits[r][free] - want[free]).max() < 0.3, (t, r)
            ended[r] = tokens[r] == 1
            seqs[r].append(int(tokens[r]))
    own = d.attention.lens.cpu().numpy()
    for r in range(rows):
        fed = len(seqs[r]) - len(PROMPTS[r // N])
        assert own[r] == (fed if ended[r] else STEPS)


def test_graph_replays_equal_the_calls():
    model = S.example_model(V=2100, d=128, seed=4)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        one, _ = decoder(model, side)
        two, _ = decoder(model, side)
        two.step()                                        # (the first call of a size may allocate: not under capture)
        side.synchronize()
        two.start(PROMPTS, torch.tensor([0.1, 0.5, 0.9], device="cuda"))
        want = []
        for _ in range(STEPS):
            one.step()
            want.append((one.tokens.clone(), one.codes.clone(), one.attention.lens.clone(), one.attention.x.clone()))
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            two.step()
        for t in range(STEPS):
            graph.replay()
            side.synchronize()
            for a, b in zip(want[t], (two.tokens, two.codes, two.attention.lens, two.attention.x)):
                assert torch.equal(a, b), t
            torch.randn(1000, device="cuda").sort()
    torch.cuda.synchronize()


def test_the_example_runs(capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["shaped_decode", "--prompts", "2", "--codes", "4", "--steps", "8", "--attention"])
    S.main()
    out = capsys.readouterr().out
    assert out.count("different continuations") == 2
