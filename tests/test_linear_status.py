"""The status word of the binding's linear() calls, with host threads: on the CPU, over stand-ins for the GPU's part."""
import threading
import time

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2507_22424_b200.build import build
    build()
    from paper_2507_22424_b200 import binding
    return binding


@pytest.fixture
def fake(B, monkeypatch):
    """No words yet; a word is made in host memory, slowly."""
    zeros = torch.zeros

    def slow_zeros(*shape, device=None, **kw):
        time.sleep(0.05)
        return zeros(*shape, **kw)
    monkeypatch.setattr(B, "_status_words", {})
    monkeypatch.setattr(torch, "zeros", slow_zeros)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return B


def in_threads(n, work):
    out, errors, start = [None] * n, [], threading.Barrier(n)

    def run(k):
        try:
            start.wait()
            out[k] = work(k)
        except Exception as e:                                        # reported by the main thread
            errors.append(e)
    threads = [threading.Thread(target=run, args=(k,)) for k in range(n)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    return out


def test_threads_first_calls_share_one_word(fake):
    words = in_threads(8, lambda k: fake._status_word(0))
    assert all(w is words[0] for w in words) and fake._status_words[0] is words[0]
