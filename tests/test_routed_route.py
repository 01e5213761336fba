"""What a Route checks by itself, without a device."""
import pytest
import torch

import paper_2607_22866_b200 as gm


def test_arrays_that_were_replaced_are_noticed():
    R = gm.DeviceCSR(3, 2, torch.tensor([0, 1, 1, 2]), torch.tensor([0, 1], dtype=torch.int32), torch.ones(2))
    route = gm.Route(None, R, 0, torch.zeros(6 + 3 * 2, dtype=torch.int32))
    row_ptr, val = R.row_ptr, R.val

    def refused(val):
        with pytest.raises(gm.GmError) as e:
            route._reads("here", val)
        assert e.value.status == -1

    R.val.mul_(2)
    route._reads("here", True)
    R.val = val.clone()
    route._reads("here", False)
    refused(True)
    R.val, R.row_ptr = val, row_ptr.clone()
    refused(False)
    refused(True)
    R.row_ptr = row_ptr
    route._reads("here", True)
    R.val.data = torch.zeros(2)
    refused(True)
