"""Norms after the sub-layers that are named but not given, on the CPU: as if they were
not named, for weights of every kind."""
import pytest
import torch

from paper_2608_02474_amd import api


def test_a_16_bit_block_without_norms_is_not_refused_for_their_names():
    """What refuses the call here is the host tensor, not the names."""
    x, idx = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int32)
    p = {n: torch.zeros(2, 2) for n in api.WEIGHT_NAMES}
    with pytest.raises(ValueError, match="x must be a device tensor"):
        api.block_partial({**p, "after1": None, "after2": None}, x, idx, 4, 2)
    for n in ("after1", "after2"):
        with pytest.raises(ValueError, match="8 or 4 bits"):
            api.block_partial({**p, n: torch.zeros(64)}, x, idx, 4, 2)
