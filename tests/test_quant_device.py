"""A QuantCache is made on a GPU: another device is refused before anything is allocated."""
import pytest
import torch

import paper_2607_00760_amd as M


@pytest.mark.parametrize("device", ["cpu", "meta", torch.device("cpu")])
def test_device_that_is_no_gpu(device):
    with pytest.raises(ValueError, match="device"):
        M.QuantCache(M.QuantParams(), 1, 64, device=device)
