"""Which context the token-gate functions take when they are given none.  CPU only: contexts and streams are imitated."""
import threading
import time

import pytest

from paper_2308_10037_b200 import api
from test_gate_validation import fake


@pytest.fixture
def made(monkeypatch):
    """The contexts that were made, in order; making one takes a while, as in earnest."""
    got = []

    class Slow:
        def __init__(self, n_max, device):
            time.sleep(0.05)
            self.device, self.open = device, True
            got.append(self)

        def close(self):
            self.open = False

    monkeypatch.setattr(api, "Context", Slow)
    monkeypatch.setattr(api, "_gate_ctx", {})
    monkeypatch.setattr(api, "_default_ctx", {})
    monkeypatch.setattr(api, "_raw_stream", lambda device: 7)
    return got


def test_threads_that_come_first_together_share_one_context(made):
    x, seen, start = fake((2, 2)), [], threading.Barrier(8)

    def call():
        start.wait()
        seen.append(api._ctx_of(x, None))

    threads = [threading.Thread(target=call) for _ in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(made) == 1 and len(seen) == 8 and all(c is made[0] for c in seen)


def test_contexts_can_be_released(made, monkeypatch):
    x = fake((2, 2))
    first = api._ctx_of(x, None)
    monkeypatch.setattr(api, "_raw_stream", lambda device: 8)
    assert api._ctx_of(x, None) is not first and api._ctx_of(x, None) is made[1] and len(made) == 2
    api.release_contexts()
    assert not any(c.open for c in made)
    assert api._ctx_of(x, None) is made[2] and made[2].open
