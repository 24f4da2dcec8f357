"""Flags that have no truth value are refused with the error that says so, before anything is queued."""
import pytest
import torch

import paper_2501_16385_b200 as fbq

BOTH = torch.tensor([True, False])


def test_flags():
    x, layer = torch.zeros((1, 128), dtype=torch.float16), (torch.zeros(512, dtype=torch.int32), *(torch.zeros((32, 1), dtype=torch.float16) for _ in range(2)), None, None)
    dy = torch.zeros((1, 32), dtype=torch.float16)
    for call in (lambda: fbq.gated(x, *layer, 32, 128, 4, save=BOTH), lambda: fbq.linear_backward(dy, x, *layer, 128, 4, want_dx=BOTH),
                 lambda: fbq.linear_backward(dy, x, *layer, 128, 4, want_factors=BOTH)):
        with pytest.raises(RuntimeError, match="ambiguous"):
            call()
