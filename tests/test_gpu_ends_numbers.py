"""Learning rate and step in tensors of a subclass: addresses for the GPU to read, as in plain tensors and parameters, never numbers that the host waits for."""
import pytest
import torch

import ends_util as V
from paper_2410_08661_amd import binding as B

pytestmark = pytest.mark.gpu
READ = []


class Watched(torch.Tensor):
    """Notes whoever asks for its value."""

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        if getattr(func, "__name__", "") in ("item", "__float__", "__index__", "__int__", "tolist"):
            READ.append(func.__name__)
        return super().__torch_function__(func, types, args, kwargs or {})


KINDS = [lambda t: t, lambda t: torch.nn.Parameter(t, requires_grad=False), lambda t: t.as_subclass(Watched)]


def a_list(seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    g, w = (torch.randn(1000, generator=gen, device="cuda") for _ in range(2))
    return g, w, B.TensorList([g], masters=[w], **B.make_adamw_states([w], 32))


def test_the_value_is_not_asked_for():
    assert float(torch.ones(1, device="cuda").as_subclass(Watched)) == 1 and READ
    READ.clear()
    _, _, plan = a_list()
    lr, step = torch.tensor([1e-2], device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda")
    for native in (True, False):
        with pytest.MonkeyPatch.context() as mp:
            if not native:
                mp.setattr(B, "_native", V.NONE)
            B.qeft_adamw_step(plan, lr.as_subclass(Watched), 3)
            B.qeft_adamw_step(plan, 1e-2, step.as_subclass(Watched))
            B.qeft_adamw_step(plan, lr.as_subclass(Watched), step.as_subclass(Watched))
    assert READ == []


@pytest.mark.parametrize("kind", KINDS)
def test_replays_read_what_the_tensor_holds_then(kind):
    (g, w, plan), (_, v, other) = a_list(), a_list()
    lr, step = torch.tensor([1e-2], device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        B.qeft_adamw_step(plan, kind(lr), kind(step))
    for i in range(4):
        lr.fill_(1e-2 / (i + 1))
        step.fill_(i + 1)
        graph.replay()
        torch.cuda.synchronize()
        B.qeft_adamw_step(other, lr, step)
        assert torch.equal(w, v)
