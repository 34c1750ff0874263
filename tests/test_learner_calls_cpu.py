"""The native calls of the learner operators on the host: what they do not take (host
tensors, other objects) they leave to the binding, whose checks name the error."""
import pytest
import torch

import paper_2106_07551_amd as M
from paper_2106_07551_amd import binding as B

X, W = torch.ones(3, 4), torch.ones(2, 4)
A, F = torch.zeros(3, dtype=torch.int32), torch.zeros(3)


@pytest.mark.parametrize("name, args", [
    ("linear", (X, W, None, 0, None, None, None, None, 0)),
    ("linear", ("x", W, None, 0, None, None, None, None, 0)),
    ("linear", (None, None, None, None, None, None, None, None, None)),
    ("linear_backward", (torch.ones(3, 2), X, W, 0, None, (True,) * 3, None, None, None, None, 0)),
    ("linear_backward", (X, X, W, 0, None, 7, None, None, None, None, 0)),
    ("policy_loss", (X, A, F, F, 0.2, 0.2, 0.0, 0.0, None, None, None, None, True, None, None,
                     None, None, 0)),
    ("policy_loss", (X, A, F, F, "a") + (None,) * 13),
    ("distill_loss", (X, A[:, None], F[:, None], 1.0, None, None, True, None, None, None, None,
                      0)),
])
def test_left_to_the_binding(name, args):
    assert getattr(B._native(), name)(*args) is None


def test_wrong_number_of_arguments():
    for name in ("linear", "linear_backward", "policy_loss", "distill_loss"):
        with pytest.raises(TypeError):
            getattr(B._native(), name)(X)


def test_another_library_is_refused(tmp_path):
    with pytest.raises(ImportError):
        B._native().load(str(tmp_path / "none.so"))
    B._native().load(B.LIB_PATH)


def test_host_tensors_are_named():
    with pytest.raises(M.ArgumentError, match="x: expected a device tensor"):
        M.linear(X, W)
    with pytest.raises(M.ArgumentError, match="logits: expected a device tensor"):
        M.policy_loss(X, A, F, F)
