"""What the binding of the operators around attention refuses, on host tensors, with a stand-in
for the current device."""
import pytest
import torch

import paper_2404_08763_amd as P
from paper_2404_08763_amd import _lib


@pytest.mark.parametrize("shape", [(), (2, 16)])
def test_frequencies_have_one_dimension(monkeypatch, shape):
    monkeypatch.setattr(_lib, "_device", lambda: -1)  # (what host tensors call theirs)
    out = (torch.zeros(2, 2, 64), torch.zeros(2, 1, 64))
    with pytest.raises(ValueError, match="freq must have one dimension"):
        P.qk_norm_rope(torch.zeros(2, 192), 2, 1, 64, torch.zeros(2, dtype=torch.int32), torch.zeros(shape), out=out)
