"""A linear() call whose wait gives up, seen from other streams, threads and graphs."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def _b():
    from paper_2507_22424_b200 import binding
    return binding


def told(B):
    try:
        B.linear_status()
    except B.SpecVLAError as e:
        assert e.code == -6
        return True
    return False


@pytest.mark.parametrize("T", [5, 400])
def test_other_threads_status_does_not_take_a_failure_away(T):
    B = _b()
    x, w = torch.randn(T, 1024, device="cuda").half(), torch.randn(512, 1024, device="cuda").half()
    want = B.linear(x, w)
    told(B)
    torch.cuda.synchronize()
    failed, asked = (threading.Barrier(2, timeout=60) for _ in range(2))
    out, errors = [None, None], []

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                B.linear(x, w)
                assert not told(B)
                if k == 0:
                    assert B.lib.specvla_linear_fault_test(2_000_000, 1) == 0
                    B.linear(x, w)
                    torch.cuda.current_stream().synchronize()
                failed.wait()
                if k == 1:
                    out[1] = [told(B), told(B)]
                asked.wait()
                if k == 0:
                    out[0] = [told(B), told(B)]
                assert torch.equal(B.linear(x, w), want) and not told(B)
        except Exception as e:                                        # reported by the main thread
            errors.append(e)
    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    assert out == [[True, False], [True, False]]
    assert told(B) and not told(B)                                    # this thread had called before


def test_a_captured_call_that_gives_up_is_told_on_the_stream_that_replays_it():
    B = _b()
    x, w = torch.randn(5, 1024, device="cuda").half(), torch.randn(512, 1024, device="cuda").half()
    want = B.linear(x, w)
    told(B)
    bad, good = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    assert B.lib.specvla_linear_fault_test(2_000_000, 1) == 0
    with torch.cuda.graph(bad):
        B.linear(x, w)
    with torch.cuda.graph(good):
        y = B.linear(x, w)
    for _ in range(2):
        bad.replay()
        assert told(B)
        good.replay()
        assert not told(B) and torch.equal(y, want)
