"""Token-gate calls captured into graphs: each graph has scratch of its own, for as long as it lives."""
import gc

import pytest
import torch

from paper_2308_10037_b200 import api
from test_gpu_gate import ctx, gen, rnd   # noqa: F401 (ctx is a fixture)

pytestmark = pytest.mark.gpu


def problem(i, T=20000, V=3000, n=128, C=40):
    ids, dout = torch.randint(0, V, (T,), generator=gen(i), device="cuda"), rnd(T, n, seed=i + 2)
    q, s = api.lr_ckpt8_save(dout)
    return ids, dout, V, q, s, rnd(T, C, seed=i + 4)


def calls(ids, dout, V, q, s, dz, c=None):
    return (api.lr_embed_grad(ids, dout, V, ctx=c), *api.lr_ckpt8_grad(q, s, dz, ctx=c), api.lr_route(dz, 2, ctx=c)[2])


@pytest.mark.parametrize("shared", [False, True])
def test_graphs_replayed_beside_one_another_and_beside_calls(ctx, shared):
    c = ctx if shared else None                     # one context for all of them, or those of the module's functions
    work = [problem(i) for i in range(3)]
    want = [[t.clone() for t in calls(*w, c)] for w in work]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for w in work[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(calls(*w, c))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for st, g in zip(streams, graphs):
            with torch.cuda.stream(st):
                g.replay()
        eager = calls(*work[2], c)                  # on the default stream
    torch.cuda.synchronize()
    for got, exp in zip((*outs, eager), want):
        assert all(torch.equal(a, b) for a, b in zip(got, exp))
    assert ctx.check_guards() == 0


def test_branches_of_one_graph_do_not_meet(ctx):
    work = [problem(i) for i in range(2)]
    want = [[t.clone() for t in calls(*w, ctx)] for w in work]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            one = calls(*work[0], ctx)
        two = calls(*work[1], ctx)
        main.wait_stream(side)
    for _ in range(10):
        g.replay()
    torch.cuda.synchronize()
    for got, exp in zip((one, two), want):
        assert all(torch.equal(a, b) for a, b in zip(got, exp))


def test_the_first_call_of_a_context_may_be_a_captured_one():
    w = problem(7)
    want = [t.clone() for t in calls(*w)]
    torch.cuda.synchronize()
    c = api.Context(n_max=1, device=0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = calls(*w, c)
    stream = torch.cuda.Stream()
    g2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g2, stream=stream):       # a stream that no default context has served
        got2 = calls(*w)
    g.replay(), g2.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, b2) for a, b, b2 in zip(want, got, got2))
    assert c.check_guards() == 0
    del g
    c.close()


def free_bytes():
    gc.collect()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    return torch.cuda.mem_get_info()[0]


def test_scratch_is_given_back():
    T, n = 400_000, 512                             # pieces of 2 * T / 32 rows: about 50 MB, 100 MB and 200 MB
    c = api.Context(n_max=1, device=0)
    ids, out = torch.zeros(4 * T, dtype=torch.int32, device="cuda"), torch.zeros(1, n, device="cuda")
    dout = torch.zeros(4 * T, n, dtype=torch.bfloat16, device="cuda")
    c.embed_grad(ids[:4], dout[:4], 1, out=out)
    used = []
    start = free_bytes()
    for rows in (T, 2 * T, 4 * T):
        c.embed_grad(ids[:rows], dout[:rows], 1, out=out)
        used.append(start - free_bytes())
    assert used[2] < 4.5 * used[0]                  # what it outgrew is gone: 200 MB, not 350
    before = free_bytes()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.embed_grad(ids, dout, 1, out=out)
        c.embed_grad(ids[:T], dout[:T], 1, out=out)         # in the same scratch
    held = before - free_bytes()
    assert 0.5 * used[2] < held < 1.5 * used[2]
    g.replay()
    torch.cuda.synchronize()
    del g
    free_bytes()
    c.embed_grad(ids[:4], dout[:4], 1, out=out)     # a later call gives the graph's scratch back
    assert before - free_bytes() < 0.1 * held
    c.close()
