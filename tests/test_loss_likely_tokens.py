"""What test_gpu_loss_values would notice, without a GPU: a gradient by h from which any one of the likely tokens is left out is further off than the bound allows."""
import pytest
import torch

import loss_plain as plain
from test_gpu_loss import check
from test_gpu_loss_values import LIKELY, likely_tokens


@pytest.mark.parametrize("T,V,K", [c for c in LIKELY if c[0] * c[1] < 1 << 22])
def test_each_likely_token_shows(T, V, K):
    h, w, target, dloss, hot = likely_tokens(T, V, K)
    value, bound = plain.softmax_loss(h, w, target, dloss)["dh"]
    z = h.double() @ w.double().t()
    p = torch.softmax(z, 1)
    assert (p[:, hot].sum(1) > 0.98).all() and (p[:, hot] > 0.02).all()
    check({"dh": value.float()}, {"dh": (value, bound)})
    for token in hot.tolist():
        got = value - (dloss.double() * p[:, token])[:, None] * w[token].double()
        with pytest.raises(AssertionError):
            check({"dh": got.float()}, {"dh": (value, bound)})
