"""Leading dimensions that no address space holds are refused by every call on
rows in 8 bits before sizes are computed from them (no GPU is touched)."""
import os

import pytest

from paper_2010_12635_amd import gcn as G
from tests.test_abi_q8 import UNSUPPORTED, backward, dequantize, layer, product, quantize, weights

pytestmark = pytest.mark.skipif(not os.path.exists(G.LIB_PATH), reason="libgcn.so not built")

OPERANDS = [(quantize, ("ld", "ldq")), (dequantize, ("ld", "ldq")), (weights, ("ld", "ldq")),
            (product, ("ldq", "ldw", "ld")), (backward, ("ldq", "ldw", "ldg", "ldz")), (layer, ("ldq", "ldi", "ldo"))]


@pytest.mark.parametrize("rows", [1, 10])
# just past the largest; where 64 rows' bytes pass 63 and 64 bits; the largest multiple of 16 there is
@pytest.mark.parametrize("ld", [(1 << 48) + 16, 1 << 55, 1 << 57, 1 << 58, 1 << 61, (1 << 63) - 16])
@pytest.mark.parametrize("call,name", [(c, n) for c, names in OPERANDS for n in names])
def test_refused(call, name, ld, rows):
    assert call(**{"n": rows, name: ld}) == UNSUPPORTED
