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
    monkeypatch.setattr(B, "_status_told", {})
    monkeypatch.setattr(B, "_status_seen", type(B._status_seen)())
    monkeypatch.setattr(torch, "zeros", slow_zeros)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return B


def in_threads(n, work):
    out, errors, start = [None] * n, [], threading.Barrier(n, timeout=20)

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


@pytest.fixture
def fake_calls(fake, monkeypatch):
    """linear() whose launches only say whether a wait gave up: fails = {thread name: calls that do}."""
    B, fails = fake, {}

    class Lib:
        @staticmethod
        def specvla_linear(args, stream):
            if fails.get(threading.current_thread().name, 0):
                fails[threading.current_thread().name] -= 1
                B._status_words[0] += 1
            return 0

        @staticmethod
        def specvla_gemm_status(word, stream):
            return -6 if int(B._status_words[0]) else 0

        @staticmethod
        def specvla_strerror(code):
            return b"device-side wait timed out"
    monkeypatch.setattr(B, "lib", Lib)
    monkeypatch.setattr(B, "_device", lambda *t: 0)
    monkeypatch.setattr(B, "_stream", lambda: None)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    return B, fails


def calls(B):
    B.linear(torch.zeros(2, 8, dtype=torch.float16), torch.zeros(3, 8, dtype=torch.float16))


def told(B):
    try:
        B.linear_status()
    except B.SpecVLAError as e:
        assert e.code == -6
        return True
    return False


def test_a_failure_is_told_to_every_thread_that_was_calling(fake_calls):
    B, fails = fake_calls
    both, first, second = (threading.Barrier(2, timeout=20) for _ in range(3))

    def work(k):
        calls(B)
        assert not told(B)
        both.wait()
        if k == 0:
            fails[threading.current_thread().name] = 1
            calls(B)
        first.wait()
        out = []
        if k == 1:                                                    # the other thread asks first
            out = [told(B), told(B)]
        second.wait()
        if k == 0:
            out = [told(B), told(B)]
            calls(B)
            out.append(told(B))
        return out
    assert in_threads(2, work) == [[True, False, False], [True, False]]
    assert in_threads(1, lambda k: told(B)) == [False]                # a thread that comes later


def test_a_failure_is_told_to_a_thread_that_only_asks(fake_calls):
    B, fails = fake_calls

    def failing(k):
        fails[threading.current_thread().name] = 1
        calls(B)
    in_threads(1, failing)
    assert told(B) and not told(B)


def test_failures_while_the_status_is_read_are_not_lost(fake_calls, monkeypatch):
    """A wait of another stream gives up between the status that this thread reads and its end."""
    B, fails = fake_calls
    calls(B)
    read = B.lib.specvla_gemm_status

    def then_fails(word, stream):
        rc = read(word, stream)
        if rc:
            B._status_words[0] += 1
            monkeypatch.setattr(B.lib, "specvla_gemm_status", read)
        return rc
    B._status_words[0] += 1
    monkeypatch.setattr(B.lib, "specvla_gemm_status", then_fails)
    assert in_threads(1, lambda k: (calls(B), told(B))[1]) == [True]
    assert told(B)
