"""The operators beside the decoder at the edges of what they take: every tile that wfst_linear chooses from, the numbers of classes at
which wfst_loglikes changes its tiles, as many named tokens as there may be; against the definitions in 64 bits.

Tolerances as derived in test_gpu_outputs.py."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2311_04996_amd import linear  # noqa: E402
from test_gpu_outputs import DT, check_linear, gen, randn  # noqa: E402


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("stride", [65, 64 + 8, 1 << 40])
def test_linear_of_one_row_whatever_its_stride(stride, dt):
    """What a tile reads behind the only row of x or w does not depend on the row's stride.  (More than 256 tiles of 16 x 16.)"""
    g = gen(90)
    k = 64
    one = lambda t: t.as_strided((1, k), (stride, 1))
    flat = randn(g, k + 8).to(DT[dt])
    check_linear(one(flat[:k]), (randn(g, 4200, k) / 8).to(DT[dt]), randn(g, 4200), "silu")
    check_linear(randn(g, 4200, k).to(DT[dt]), one(flat[8:]), randn(g, 1), "relu")
