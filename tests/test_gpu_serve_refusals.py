"""The serving example refuses a step that does not fit, and is then as it was before (GPU)."""
import importlib.util
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu


def _example():
    spec = importlib.util.spec_from_file_location("serve", Path(__file__).resolve().parent.parent / "examples" / "serve.py")
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_steps_that_do_not_fit():
    server = _example().Server(1, 2, 40)
    x = torch.randn(120, 768, generator=torch.Generator().manual_seed(3)).cuda()
    server.step(x[:25], [20, 5])
    state = lambda: (list(server.past), server.free.tolist(), server.table.tolist(), [c.clone() for c in server.layers[0].cache])   # noqa: E731
    before = state()
    server.free, blocks = server.free[:0], server.free
    for fresh, what in (([21, 1], "longer than 40"), ([1], "requests bring"), ([2, -1], "requests bring"), ([1, 1], "requests bring"), ([13, 0], "too few blocks")):
        n = 13 if what == "too few blocks" else 22
        with pytest.raises(ValueError, match=what):
            server.step(x[:n], fresh)
    server.free = blocks
    after = state()
    assert before[:3] == after[:3] and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before[3], after[3]))
    assert server.step(x[:20], [20, 0]).isfinite().all() and server.past == [40, 5]
