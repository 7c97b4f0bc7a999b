"""Waits that ran out, as Python learns of them.  They are made to run out by the library's self-test, which gives up in good order."""
import subprocess
import sys
from pathlib import Path

import pytest
import torch

from paper_2411_17887_b200 import api
from paper_2411_17887_b200 import binding as B
from tests.test_gpu_linattn import draw
from tests.test_gpu_linattn_ends import raw

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def give_up():
    """A call that gives up a wait and records it where api's own calls do."""
    q, k, v, _, decay, _, _ = draw(1, 1, 200, 2, 64, 64, torch.bfloat16)
    args, held, _ = raw(q, k, v, decay)
    B.check(B.tcu_linattn_selftest_timeout(args, 0, 0, 5, api._status[torch.cuda.current_device()].ptr, 256, torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()


FIRST_CALL_CAPTURED = """
import gc, sys, torch
sys.path.insert(0, {root!r})
from paper_2411_17887_b200 import api
from tests.test_gpu_linattn import draw
from tests.test_gpu_lm_status import give_up
q, k, v, _, decay, _, _ = draw(1, 1, 200, 2, 64, 64, torch.bfloat16)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    o, _ = api.linear_attention(q, k, v, decay)
assert api.linear_attention_status() == 0          # before the first replay
graph.replay()
torch.cuda.synchronize()
want = o.clone()
assert api.linear_attention_status() == 0
give_up()
graph.replay()                                     # does not wipe out what was recorded
torch.cuda.synchronize()
assert api._status[0].error.value == 5
assert api.linear_attention_status() == 5
api._status[0].error.value = 0
del graph, o
gc.collect()
torch.cuda.empty_cache()
others = [torch.full((512,), 255, dtype=torch.uint8, pin_memory=True) for _ in range(50)]      # the graph is gone, the status is not
assert torch.equal(api.linear_attention(q, k, v, decay)[0], want)
assert api.linear_attention_status() == 0
"""


def test_first_call_in_a_capture():
    root = str(Path(__file__).resolve().parents[1])
    done = subprocess.run([sys.executable, "-c", FIRST_CALL_CAPTURED.format(root=root)], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def test_threads_share_one_status(monkeypatch):
    """Threads whose first calls come at the same time get the same memory: kernels write to it."""
    import threading
    monkeypatch.setattr(api, "_status", {})
    start, got = threading.Barrier(8), []

    def first():
        start.wait()
        got.append(api._status_of(0))

    threads = [threading.Thread(target=first) for _ in range(8)]
    for one in threads:
        one.start()
    for one in threads:
        one.join()
    assert len(got) == 8 and all(one is got[0] for one in got) and api._status == {0: got[0]}


def test_the_next_call_raises():
    """A loop that never asks for the status does not go on with invalid tensors."""
    q, k, v, d_o, decay, _, _ = draw(2, 1, 200, 2, 64, 64, torch.bfloat16)
    want = api.linear_attention(q, k, v, decay)[0]
    for call in (lambda: api.linear_attention(q, k, v, decay), lambda: api.linear_attention_backward(d_o, q, k, v, decay),
                 lambda: api.linear_attention(q.clone().requires_grad_(), k, v, decay)):
        give_up()
        with pytest.raises(RuntimeError, match="gave up a wait"):
            call()
        call()                                          # it is said once
        assert api.linear_attention_status() == B.TCU_OK
        give_up()
        assert api.linear_attention_status("cuda") == B.TCU_ERR_TIMEOUT
        call()
    assert torch.equal(api.linear_attention(q, k, v, decay)[0], want)
