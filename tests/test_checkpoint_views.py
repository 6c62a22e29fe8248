"""The tensors of a Checkpoint that was made as one room, asked for by two threads at once (no GPU needed)."""
import threading

import pytest
import torch

import paper_2311_12862_amd as sp


class _Room(torch.Tensor):
    """Host memory that passes for a device's; `between` runs, once, in the middle of a view's making."""
    is_cuda = True
    between = None

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        if func is torch.Tensor.view and cls.between is not None:
            between, cls.between = cls.between, None
            between()
        return super().__torch_function__(func, types, args, kwargs or {})


@pytest.mark.parametrize("after", [0, 1, 2, 3])
@pytest.mark.parametrize("first", ["data", "exps"])
def test_two_threads(monkeypatch, after, first):
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: empty(*a, **k).as_subclass(_Room))
    kept = sp.Checkpoint.empty(4, 40)
    seen = []

    def other():
        for name in ("data", "exps", "data"):
            t = getattr(kept, name)
            seen.append((name, tuple(t.shape), t.dtype))

    def between(left):
        if left:
            _Room.between = lambda: between(left - 1)     # a later view
            return
        t = threading.Thread(target=other)
        t.start()
        t.join()

    _Room.between = lambda: between(after)
    getattr(kept, first)
    _Room.between = None
    other()
    want = {"data": ((4, 40), torch.int8), "exps": ((4, 2), torch.uint8)}
    assert len(seen) in (3, 6)
    for name, shape, dtype in seen:
        assert (shape, dtype) == want[name]
    assert kept.data.data_ptr() + 160 == kept.exps.data_ptr()
