"""What making a step of the block does on the device, without a GPU: nothing. A step may run on another stream than the
one that was current when it was made, and no work of the making is ordered before it there."""
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2608_09160_amd import _serve, block


class Recorded(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.ops = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        self.ops.append(func.overloadpacket.__name__)
        return func(*args, **(kwargs or {}))


class Call:
    """Stands for a prepared call: makes the outputs that it would."""

    def __init__(self, x=None, segs=(), *args, **kw):
        for s in segs if isinstance(segs, list) else []:
            if s.y is None:
                s.y = torch.empty(x.shape[0], s.w.shape[0], dtype=x.dtype)
        self.out = x


def test_making_a_step_writes_nothing(monkeypatch):
    for name in ("PreparedProj", "PreparedAdapters", "PreparedRopeCache", "PreparedAttn"):
        monkeypatch.setattr(block, name, Call)
    def mat(*shape):
        return torch.empty(*shape, dtype=torch.bfloat16)
    w = block.Weights(mat(64, 32), mat(32, 32), mat(32, 32), mat(32, 64), torch.empty(64), torch.empty(32),
                      tuple((mat(2, 8, 32), mat(2, d, 8)) for d in (64, 32, 32)))
    index = torch.empty(5, dtype=torch.int32)
    batch = block.Batch(mat(5, 32), index, torch.empty(5, dtype=torch.int64), index, index, index.view(5, 1), 1, 16, index)
    cache = _serve.KVCache(mat(4, 1, 16, 32), mat(4, 1, 16, 32))
    for tp in (1, 4):
        with Recorded() as seen:
            step = block.Step(w, cache, torch.empty(16, 16, 2), batch, tp=tp, rank=tp - 1, exchange=lambda *a: None)
        assert step.stat_q.shape == step.stat_k.shape == (tp, 5)
        assert set(seen.ops) <= {"empty", "select", "view", "slice"}, seen.ops
