"""What the operators write counts as a change to the tensors that hold it, so that automatic differentiation notices when a value
that it has saved is overwritten; results themselves carry no history."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))
from _gpu import DEV, GPU_MARKS, say  # noqa: E402

pytestmark = GPU_MARKS


def test_written_tensors_change_their_version():
    import paper_2402_11857_amd as pkg

    say("case versions of written tensors")
    x, w = torch.ones(2, 3, 16, device=DEV), torch.ones(2, 16, device=DEV)
    dy, out, dx, dw, db = (torch.zeros_like(t) for t in (x, x, x, w, w))
    grads, rows, norms = [torch.ones(2, 5, device=DEV), torch.ones(2, 3, device=DEV)], torch.empty(2, 8, device=DEV), torch.empty(2, device=DEV)

    def changed(tensors, call):
        before = [t._version for t in tensors]
        call()
        return [t._version > b for t, b in zip(tensors, before)]

    _, mean, rstd = pkg.liec_layer_norm(x, w)
    assert changed([out, x, w], lambda: pkg.liec_layer_norm(x, w, out=out)) == [True, False, False]
    assert changed([dx, dw, db, x, dy, mean], lambda: pkg.liec_layer_norm_backward(dy, x, mean, rstd, w, dx=dx, dweight=dw, dbias=db)) == [True] * 3 + [False] * 3
    assert changed([norms, *grads], lambda: pkg.liec_grad_norm(grads, norms)) == [True, False, False]
    assert changed([rows, norms, *grads], lambda: pkg.liec_gather_grads(grads, rows, 1.0, norms)) == [True, True, False, False]
    assert changed([norms, *grads], lambda: pkg.liec_clip_grads(grads, 1.0, norms)) == [True] * 3
    with torch.inference_mode():                             # tensors without a counter
        inside = torch.ones(2, 3, 16, device=DEV)
        pkg.liec_layer_norm(inside, out=inside)
    with torch.inference_mode():
        pkg.liec_clip_grads([inside], 1.0)


def test_a_saved_value_that_is_overwritten_is_noticed():
    import paper_2402_11857_amd as pkg

    say("case a saved value that is overwritten")
    a = torch.ones(2, 16, device=DEV, requires_grad=True)
    b = a * 2.0
    loss = b.square().sum()                                  # keeps b
    pkg.liec_clip_grads([b.detach()], 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_results_carry_no_history():
    import paper_2402_11857_amd as pkg

    say("case results without history")
    x = torch.ones(2, 3, 16, device=DEV, requires_grad=True)
    y, mean, rstd = pkg.liec_layer_norm(x)
    assert not (y.requires_grad or mean.requires_grad or rstd.requires_grad)
