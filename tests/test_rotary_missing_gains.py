"""The gains' own check refuses a call without them, whatever else is given: no GPU needed."""
import types

import pytest
import torch

from paper_2509_22323_b200 import binding


@pytest.mark.parametrize("with_k", [False, True])
def test_gradients_without_a_gain_are_refused(monkeypatch, with_k):
    monkeypatch.setattr(binding, "_device", lambda what, like: -1)   # as if host tensors were on the current device
    q = torch.zeros(1, 2, 4, 64)
    k = q if with_k else None
    rotary = types.SimpleNamespace(check=lambda *_: None)
    with pytest.raises(ValueError, match="q_gain"):
        binding.rapid3_norm_rotary_backward(q, k, q, k, None, torch.ones(64), 1e-6, rotary)
    with pytest.raises(ValueError, match="q_gain"):
        binding.rapid3_norm_rotary(q, k, None, torch.ones(64), 1e-6, rotary)
    if with_k:
        for call in (lambda *a: binding.rapid3_norm_rotary_backward(q, k, *a), binding.rapid3_norm_rotary):
            with pytest.raises(ValueError, match="k_gain"):
                call(q, k, torch.ones(64), None, 1e-6, rotary)
