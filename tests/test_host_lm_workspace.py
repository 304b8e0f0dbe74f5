"""A workspace that kernels could not write is refused before anything is launched."""
import pytest
import torch

import paper_2105_00053_amd as pn
from paper_2105_00053_amd import lm


@pytest.mark.parametrize("workspace", [torch.empty(4096, dtype=torch.uint8), torch.empty(0), torch.empty(4096, dtype=torch.uint8)[::2], [0] * 4096, 4096])
def test_a_workspace_is_a_dense_device_tensor(workspace):
    with pytest.raises(pn.PositError):
        lm._work(1024, torch.device("cuda"), workspace)
