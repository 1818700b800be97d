"""Pins of oracle/train_oracle.py where a value lies at the edge of what can occur, against torch's double-precision autograd."""
import numpy as np
import torch

from oracle import train_oracle as R


def test_gradient_of_a_label_that_cannot_occur_is_autograds():
    """The given label's logit is -inf, others are possible: dlogp at that label, -dlogp p elsewhere, 0 at other impossible ones."""
    x = np.random.default_rng(8).standard_normal((2, 2, 7))
    x[:, :, [1, 4]] = -np.inf
    label, w = np.array([[1, 2], [4, 1]]), np.array([[0.5, -1.0], [2.0, 0.25]])
    leaf = torch.tensor(x, requires_grad=True)
    q = torch.log_softmax(leaf, -1).gather(2, torch.tensor(label)[:, :, None])[:, :, 0]
    q.backward(torch.tensor(w))
    d = R.label_score_bwd(x, label, w)
    np.testing.assert_allclose(d, leaf.grad.numpy(), atol=1e-15)
    np.testing.assert_allclose(R.label_score_fwd(x, label)["logp"], q.detach().numpy(), atol=1e-14)
    assert d[0, 0, 1] == 0.5 and d[1, 0, 4] == 2.0 and d[0, 0, 4] == 0
