"""fb_mx4_linear at the edges of the form that keeps x in registers: two row tiles whose
chunks leave waves without work take it from longer outputs on.  Tolerances as in
test_gpu_mx4.py."""
import pytest

from tail_harness import Batch
from test_gpu_mx4 import check_device, long_call, long_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [16, 17, 31, 32])
@pytest.mark.parametrize("N,K", [(65536, 1568), (98288, 1536), (98305, 1536), (98323, 1568), (98304, 1792),
                                 (65555, 1920), (98288, 2176), (98309, 2080), (98304, 2304), (98310, 2816),
                                 (65541, 2944), (98304, 2912)])
def test_two_row_tiles(rows, N, K):
    bt = Batch(w=[1], o=[3], bl=rows, W_max=1).cuda()
    case = long_inputs(bt, N, K, seed=rows + K)
    out = "bf16" if rows % 16 else "f32"
    check_device(bt, *case, long_call(bt, *case, out), out)
