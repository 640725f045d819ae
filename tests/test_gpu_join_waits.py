"""The waits of a join's thread blocks for each other: one that runs out ends the call, is not taken up again, and leaves the device as it was."""
import numpy as np
import pytest
import torch

from paper_2608_16308_b200 import binding as B
from rows_util import DEV, Join


def test_refused():
    a = np.zeros(2, np.int32)
    for bad in (dict(max_tries=0), dict(max_tries=5000), dict(silent=2), dict(silent=-2), dict(gave_up=None)):
        with pytest.raises(B.DbSpmspvError) as e:
            B.dbspmspv_test_cluster_wait(**{**dict(max_tries=64, silent=-1, gave_up=a, stream=0), **bad})
        assert e.value.status == B.ERR_INVALID_ARG


@pytest.mark.gpu
def test_a_silent_block():
    n = torch.full((2,), 77, dtype=torch.int32, device=DEV)
    for silent, want in ((-1, [0, 0]), (1, [4, 4]), (0, [4, 4]), (-1, [0, 0])):
        B.dbspmspv_test_cluster_wait(64, silent, n)
        torch.cuda.synchronize()
        assert n.tolist() == want
    j = Join(50, 8192, gate="shared", drop=0.1)
    j.forward()
    j.backward()
    torch.cuda.synchronize()
    j.check(), j.check_back()
