"""gcn_sample_labels at T = 0 does not read u and takes none.  (No GPU is
touched: the argument checked next is a bad one.)"""
import os

import pytest

from paper_2010_12635_amd import gcn as G
from tests.test_abi_scores import INVALID, WORKSPACE, sample

pytestmark = pytest.mark.skipif(not os.path.exists(G.LIB_PATH), reason="libgcn.so not built")


def test_u_is_needed_above_0_only():
    assert sample(u=None, T=0.0, ws=None) == WORKSPACE
    assert sample(u=None, T=1.0, ws=None) == INVALID
    assert sample(u=None, T=-0.0, ws=None) == WORKSPACE
    assert sample(u=None, T=0.0, y=None) == INVALID
