"""Calls from host threads: the first CUDA call of a thread, and threads that share a stream."""
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
