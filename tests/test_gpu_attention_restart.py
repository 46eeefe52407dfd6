"""The example's decoder taken up again with other prompts, its step captured once: the prompts' calls leave the step's workspace
where the graph has it."""
import pytest
import torch

from paper_2210_15458_amd import binding as B
from paper_2210_15458_amd import shaped_decode as S

pytestmark = pytest.mark.gpu

ROOM, STEPS, N = 4096, 6, 4
LONG, SHORT = [100 + i % 900 for i in range(4000)], [100 + i % 77 for i in range(41)]


def decoder(model, side):
    attention = S.example_attention(model, heads=4, kv_heads=2, prompt_room=ROOM, room=STEPS)
    return S.ShapedDecoder(**model, B_=1, N=N, stream=side, attention=attention)


def u():
    return torch.tensor([0.3], device="cuda")


def test_prompts_and_steps_have_contexts_of_their_own(monkeypatch):
    """The workspaces are a context's, and grow by what is called on it."""
    used = {}
    for name in ("as_linear", "as_cache_add", "as_attend", "as_attend_prompts"):
        def call(ctx, *a, name=name, own=getattr(B, name), **kw):
            used.setdefault((phase, name), set()).add(id(ctx))
            return own(ctx, *a, **kw)
        monkeypatch.setattr(B, name, call)
    d = decoder(S.example_model(V=1500, d=128), torch.cuda.current_stream())
    phase = "start"
    d.start([SHORT], u())
    phase = "step"
    d.step()
    torch.cuda.synchronize()
    of = lambda phase: set.union(*(ids for (p, _), ids in used.items() if p == phase))  # noqa: E731
    assert ("start", "as_attend_prompts") in used and ("step", "as_attend") in used
    assert not of("start") & of("step")


def test_replays_after_other_prompts():
    model = S.example_model(V=1500, d=128)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        d, eager = decoder(model, side), decoder(model, side)
        d.start([LONG], u())
        d.step()
        side.synchronize()
        d.start([LONG], u())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            d.step()
        for prompt in (LONG, SHORT, LONG[:2000], [333], SHORT[:7], LONG):
            d.start([prompt], u())
            eager.start([prompt], u())
            for t in range(STEPS):
                graph.replay()
                side.synchronize()
                eager.step()
                side.synchronize()
                for a, b in ((d.tokens, eager.tokens), (d.codes, eager.codes), (d.attention.x, eager.attention.x), (d.logits, eager.logits)):
                    assert torch.equal(a, b), (len(prompt), t)
    torch.cuda.synchronize()


def test_prompts_that_do_not_fit_are_refused():
    model = S.example_model(V=1500, d=128)
    d = S.ShapedDecoder(**model, B_=2, N=3, attention=S.example_attention(model, heads=4, kv_heads=2, prompt_room=20, room=4))
    two = torch.tensor([0.3, 0.6], device="cuda")
    d.start([SHORT[:21], SHORT[:3]], two)
    d.step()
    before = d.tokens.clone()
    with pytest.raises(ValueError, match="more than 21 tokens"):
        d.start([SHORT[:22], SHORT[:3]], two)
    with pytest.raises(ValueError, match="1 prompts, not 2"):
        d.start([SHORT[:2]], two)
    torch.cuda.synchronize()
    assert torch.equal(d.tokens, before)
