"""Refusals of the paged cache's binding that need no GPU."""
import types

import pytest
import torch

from paper_2609_12075_amd import paged


def test_q_out_without_q_is_refused():
    """Nothing would be written to it, and it would be returned as if."""
    pool, batch = types.SimpleNamespace(index=0, n_kv=2), types.SimpleNamespace(index=0)
    k = torch.zeros(3, 2, 64)
    with pytest.raises(ValueError, match="q_out without q"):
        paged.append(pool, batch, k, k, q_out=torch.zeros(3, 4, 64))
