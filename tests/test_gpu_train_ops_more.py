"""More calls of the operators for training other models: many records of several tiles, strided narrow rows."""
import numpy as np
import pytest

import test_gpu_rmsnorm
from test_gpu_attention_packed import U, Call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,most,H,Hk,D,causal,window", [(65, 300, 2, 1, 64, 1, 0), (70, 400, 2, 2, 128, 1, 0), (129, 200, 1, 1, 64, 0, 0),
                                                         (80, 390, 3, 1, 64, 1, 150)])
def test_more_than_64_records_of_several_tiles(n, most, H, Hk, D, causal, window):
    lens = np.random.default_rng(n).integers(0, most, n)
    lens[:4] = (0, 128, 129, 256)
    starts = np.concatenate([[5], 5 + np.cumsum(lens)])
    T, scale = int(starts[-1]) + 9, D ** -0.5
    q, k, v, do = make(T, H, Hk, D, n)
    for layout, with_lo in (("packed", True), ("strided", False)):
        c = Call(q, k, v, do, starts, scale, causal, window, layout, with_lo)
        c.fwd()
        c.bwd()
        check(c, q, k, v, do, starts, scale, causal, window, 2.0 ** -16 if with_lo else U, "%d records, %s" % (n, layout))


@pytest.mark.parametrize("T,d,res,codes", [(1, 64, None, True), (47, 64, None, True), (35, 128, "fp32", True), (50, 136, "bf16", False),
                                           (19, 24, None, False), (9, 8, "fp32", False)])
def test_norm_of_narrow_rows_apart(T, d, res, codes):
    test_gpu_rmsnorm.run(T, d, res, codes, extra=72)
