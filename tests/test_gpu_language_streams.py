"""The operators at the ends of a language model on streams whose work overlaps, and replayed from graphs beside eager calls: bit for bit the
results of the same calls one after another."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _calls(seed):
    from paper_1911_04070_b200 import binding, layer
    g = torch.Generator("cuda").manual_seed(seed)
    ids = torch.randint(0, 3000, (4, 6000 + seed), generator=g, device="cuda")
    w = torch.randn(3000, 136 + seed, generator=g, device="cuda").bfloat16()
    d = torch.randn(4, 6000 + seed, 136 + seed, generator=g, device="cuda").bfloat16()
    many = torch.randint(0, 50, (150000 + seed,), generator=g, device="cuda")           # beyond the sort in one launch
    dm = torch.randn(150000 + seed, 24, generator=g, device="cuda")
    grads = [torch.randn(300 + seed, 400, generator=g, device="cuda") for _ in range(9)]
    x = torch.randn(200, 33000 + seed, generator=g, device="cuda").bfloat16()
    h = torch.randint(0, 33000, (200, 500), generator=g, device="cuda")
    few = x[:3]
    return [lambda: layer.token_states(ids, w, 2.0, 5), lambda: binding.bpt_embed_bwd(ids, d, 3000, torch.bfloat16), lambda: binding.bpt_embed_bwd(many, dm, 50, torch.float32),
            lambda: torch.cat([t.view(-1) for t in (lambda o: (layer.clip_gradients(grads, 0.5, out=o), *o))([torch.empty_like(t) for t in grads])]),
            lambda: layer.gradient_norm(grads), lambda: layer.adjust_logits(x, h, repetition=1.5, frequency=0.25),
            lambda: layer.adjust_logits(few, h[:3], presence=0.5)]


def test_overlapping_streams():
    sets = [_calls(s) for s in range(3)]
    want = [[f() for f in calls] for calls in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(6):
        got = [[] for _ in sets]
        for i in range(len(sets[0])):
            for s, calls, out in zip(streams, sets, got):
                with torch.cuda.stream(s):
                    out.append(calls[(i + len(out)) % len(calls)]())
        torch.cuda.synchronize()
        for calls, out, ref in zip(sets, got, want):
            for i, v in enumerate(out):
                assert torch.equal(v, ref[2 * i % len(ref)]), i


def test_graphs_beside_eager_calls():
    calls = _calls(7)
    want = [f() for f in calls]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for f in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(f())
        graphs.append(graph)
    side = torch.cuda.Stream()
    for _ in range(4):
        for o in outs:
            o.zero_()
        side.wait_stream(torch.cuda.current_stream())
        eager = []
        for graph, f in zip(graphs, reversed(calls)):
            graph.replay()
            with torch.cuda.stream(side):
                eager.append(f())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)) and all(torch.equal(a, b) for a, b in zip(reversed(eager), want))
