"""Updates whose small matrices' products are launches of their own (the shorter side above 1024), masked, both orientations."""
import pytest
import torch

from test_ortho_gpu import check_update, state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,k", [(1100, 1200), (1300, 1030)])
@pytest.mark.parametrize("masked,dtype", [(True, torch.float32), (False, torch.bfloat16)])
def test_updates(m, k, masked, dtype):
    check_update(*state(m, k, masked, dtype, m + k))
