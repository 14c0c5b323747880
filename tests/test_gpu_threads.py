"""Calls from host threads: the first CUDA call of a thread, and threads that share a stream."""
import ctypes
import threading

import pytest
import torch

from paper_2308_10037_b200 import api
from test_gpu_gate import ctx, gen, rnd   # noqa: F401 (ctx is a fixture)

pytestmark = pytest.mark.gpu


def in_a_new_thread(f):
    got = []

    def run():
        try:
            got.append(f())
        except Exception as e:                      # noqa: BLE001 (raised again in the test's thread)
            got.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    if isinstance(got[0], Exception):
        raise got[0]
    return got[0]


def test_a_tensor_map_is_made_in_a_thread_that_has_made_no_cuda_call():
    # the encoder of tensor maps is a driver call: it needs the thread's context, which a runtime call before it would have set
    c = api.Context(n_max=2048, device=0)
    q, s = c.ckpt8_save(rnd(500, 256))
    dz, gw, gb = rnd(500, 8, seed=1), torch.zeros(8, 256, device="cuda"), torch.zeros(8, device="cuda")
    want = [t.clone() for t in c.ckpt8_grad(q, s, dz)]
    torch.cuda.synchronize()
    in_a_new_thread(lambda: c.ckpt8_grad(q, s, dz, gw, gb))
    torch.cuda.synchronize()
    assert torch.equal(gw, want[0]) and torch.equal(gb, want[1])
    # rows of the binary model that are copied through a tensor map
    X, y = rnd(300, 2048, seed=2), (rnd(300, seed=3) < 0).float()
    assert api.plan_query(300, 2048)["variant"] == 1
    w, b = torch.zeros(2048, device="cuda"), torch.zeros(1, device="cuda")
    want = [t.clone() for t in c.loss_grad(X, y, w, b)]
    torch.cuda.synchronize()
    got = in_a_new_thread(lambda: c.loss_grad(X, y, w, b))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    c.close()


def test_a_new_context_is_ready_when_it_is_there(ctx):
    # its words are cleared when the call returns, not when the default stream gets to it: that one is busy here, and the stream in use
    # does not wait for it.  Memory of that size that was freed with other contents makes the difference visible.
    rt = ctypes.CDLL(next(p for p in map(str.strip, open("/proc/self/maps").read().split()) if "libcudart.so" in p))
    blocks = [ctypes.c_void_p() for _ in range(512)]
    for p in blocks:
        assert rt.cudaMalloc(ctypes.byref(p), ctypes.c_size_t(8192)) == 0
        assert rt.cudaMemset(p, 0xFF, ctypes.c_size_t(8192)) == 0
    torch.cuda.synchronize()
    for p in blocks:
        assert rt.cudaFree(p) == 0
    x = rnd(30001, 64, seed=5)
    want = ctx.route(x, 4)[2]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(600_000_000)                  # the default stream, a third of a second
    c = api.Context(n_max=1, device=0)
    with torch.cuda.stream(side):
        got = [c.route(x, 4)[2] for _ in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    c.close()


def test_two_threads_on_one_stream(ctx):
    # calls of several kernels that hand data on through one scratch: each thread's results are those of its calls alone
    work = []
    for i, (T, V, n, C) in enumerate([(20000, 3000, 128, 40), (700, 50, 96, 5)]):
        ids, dout = torch.randint(0, V, (T,), generator=gen(i), device="cuda"), rnd(T, n, seed=i + 2)
        dz = rnd(T, C, seed=i + 4)
        q, s = ctx.ckpt8_save(dout)
        work.append((ids, dout, V, q, s, dz, (ctx.embed_grad(ids, dout, V), *ctx.ckpt8_grad(q, s, dz), ctx.route(dz, 2)[2])))
    torch.cuda.synchronize()
    start, wrong = threading.Barrier(2), [None, None]

    def run(i):
        ids, dout, V, q, s, dz, want = work[i]
        start.wait()
        got = [(api.lr_embed_grad(ids, dout, V), *api.lr_ckpt8_grad(q, s, dz), api.lr_route(dz, 2)[2]) for _ in range(150)]
        torch.cuda.synchronize()
        wrong[i] = sum(not torch.equal(a, b) for one in got for a, b in zip(one, want))

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == [0, 0]


def test_released_contexts_give_their_memory_back_and_come_again():
    x, y = rnd(2000, 64, seed=6), (rnd(2000, seed=7) < 0).float()
    ids = torch.randint(0, 50, (200_000,), generator=gen(8), device="cuda")
    dout = rnd(200_000, 256, seed=9)
    want = [t.clone() for t in (api.lr_fit(x, y, 0.5, 3)[0], api.lr_embed_grad(ids, dout, 50))]
    torch.cuda.synchronize()
    held = torch.cuda.mem_get_info()[0]
    api.release_contexts()
    assert torch.cuda.mem_get_info()[0] > held
    got = (api.lr_fit(x, y, 0.5, 3)[0], api.lr_embed_grad(ids, dout, 50))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
