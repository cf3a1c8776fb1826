"""The first call of a thread under capture: contexts allocate, which a captured stream does not allow."""
import threading

import pytest
import torch

from layer_cases import Layer, draw
from paper_2312_07759_amd import autograd, binding


def in_a_thread(body):
    """body() in a new thread; what it raises is raised here."""
    raised = []

    def run():
        try:
            body()
        except BaseException as e:  # noqa: BLE001
            raised.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    if raised:
        raise raised[0]


def test_no_context_is_made_under_capture(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    monkeypatch.setattr(binding, "Context", lambda device: pytest.fail("made"))
    with pytest.raises(RuntimeError, match="first call"):
        in_a_thread(lambda: autograd._context(0))


@pytest.mark.gpu
def test_a_module_can_be_captured_at_once():
    stored = Layer(48, 192, 16, 1, 64, torch.bfloat16, seed=1).on_gpu(binding)
    X = draw((5, 192), torch.bfloat16, 1).cuda()

    def body():
        m = autograd.CodesLinear(stored)
        graph = torch.cuda.CUDAGraph()
        with torch.no_grad(), torch.cuda.graph(graph):
            Y = m(X)
        for i in range(3):
            X.copy_(draw((5, 192), torch.bfloat16, 2 + i).cuda())
            graph.replay()
            with torch.no_grad():
                ref = m(X)
            torch.cuda.synchronize()
            assert bool(torch.equal(Y, ref))

    in_a_thread(body)
