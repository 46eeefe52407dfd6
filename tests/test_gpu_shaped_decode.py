"""The example that runs the layers, the shaped head, the histories and the sampling step together: its logits against the model's
formula in 64 bits on the tokens that it emitted, its grammar and biases, and a graph against the calls one by one."""
import numpy as np
import pytest
import torch

from paper_2210_15458_amd import shaped_decode as S

pytestmark = pytest.mark.gpu

PROMPTS = [[150, 151, 150, 900], [333], [101 + i for i in range(60)]]
N, STEPS = 5, 10


def decoder(model, stream=None):
    V = model["E"].shape[0]
    bias = torch.zeros(1, V, device="cuda")
    bias[0, 100:110] = -float("inf")
    bias[0, 200:260] = 1.5
    torch.cuda.synchronize()
    d = S.ShapedDecoder(**model, B_=len(PROMPTS), N=N, grammar=S.example_grammar(V), bias=bias, stream=stream)
    d.start(PROMPTS, torch.tensor([0.1, 0.5, 0.9], device="cuda"))
    return d, bias


def formula(model, d, bias, tokens, history):
    """float64 logits of a row whose last token is tokens[-1]; history: (prompt, own tokens)."""
    w = {k: v.double().cpu().numpy() for k, v in model.items()}
    x = w["E"][tokens]
    z = w["W1"] @ x + w["b1"]
    hidden = z / (1 + np.exp(-z))
    h = x + w["W2"] @ hidden + w["b2"]
    y = 30 * np.tanh(w["head"] @ h / 30)
    prompt, own = history
    n = np.bincount(own, minlength=len(y))
    seen = n > 0
    seen[prompt] = True
    y = np.where(seen, np.where(y > 0, y / 1.2, y * 1.2), y) - 0.1 * n - 0.2 * (n > 0)
    return y + bias[0].double().cpu().numpy()


def test_logits_tokens_and_grammar():
    model = S.example_model(V=1500, d=128)
    d, bias = decoder(model)
    V, rows = 1500, len(PROMPTS) * N
    own = [[] for _ in range(rows)]
    state = np.zeros(rows, dtype=int)
    allowed, cls, follows = (t.cpu().numpy() for t in (d.grammar.allowed, d.grammar.token_class, d.grammar.follows))
    last = np.array([PROMPTS[r // N][-1] for r in range(rows)])
    ended = np.zeros(rows, dtype=bool)
    for t in range(STEPS):
        d.step()
        torch.cuda.synchronize()
        logits, tokens = d.logits.float().cpu().numpy(), d.tokens.cpu().numpy()
        for r in range(rows):
            if ended[r]:
                assert tokens[r] == 1
                continue
            want = formula(model, d, bias, last[r], (PROMPTS[r // N], np.array(own[r], dtype=int)))
            free = allowed[state[r]] & np.isfinite(want)
            assert np.array_equal(np.isfinite(logits[r]), free)
            # two roundings to bf16 inside (the hidden layer, the residual stream) and one at the end, each 2^-8 of what it rounds
            assert np.abs(logits[r][free] - want[free]).max() < 0.15, (t, r)
            assert free[tokens[r]], "a token that the grammar or the biases forbid"
            state[r] = follows[state[r], cls[tokens[r]]]
            ended[r] = tokens[r] == 1
            if not ended[r]:
                own[r].append(int(tokens[r]))
        last = tokens
    counts = d.counts.cpu().numpy()
    for r in range(rows):
        assert np.array_equal(counts[r], np.bincount(np.array(own[r], dtype=int), minlength=V))
    assert len({tuple(o) for o in own[:N]}) > 1


def test_graph_replays_equal_the_calls():
    model = S.example_model(V=2100, d=128, seed=4)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        one, _ = decoder(model, side)
        two, _ = decoder(model, side)
        want = []
        for _ in range(STEPS):
            one.step()
            want.append((one.tokens.clone(), one.codes.clone(), one.seen.clone(), one.state.clone()))
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            two.step()
        for t in range(STEPS):
            graph.replay()
            side.synchronize()
            for a, b in zip(want[t], (two.tokens, two.codes, two.seen, two.state)):
                assert torch.equal(a, b), t
            torch.randn(1000, device="cuda").sort()
    torch.cuda.synchronize()


def test_the_example_runs(capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["shaped_decode", "--prompts", "2", "--codes", "4", "--steps", "8"])
    S.main()
    out = capsys.readouterr().out
    assert out.count("different continuations") == 2
