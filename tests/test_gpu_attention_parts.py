"""The heads of a group dealt over several blocks, whose number follows from the rows of the call: a record among more rows."""
import numpy as np
import pytest

from oracle import train_ops as to
from gpu_util import say
from test_gpu_attention_packed import Call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,rows", [(64, 8400), (64, 40000), (128, 8400)])
def test_one_record_among_more_rows(D, rows):
    """300 tokens, 16 heads on 2: eight blocks share a key head in a call of 300 rows, four in one of 8400, one in one of 40000.  o, lse and
    dq are sums of one block and keep their bits; dk and dv are added up in another order and keep their bounds."""
    n, H, Hk = 300, 16, 2
    starts = np.array([0, n])
    q, k, v, do = make(n, H, Hk, D, 31)
    got = []
    for T in (n, rows):
        more = [np.concatenate([t, np.full((T - n,) + t.shape[1:], np.nan, np.float32)]) for t in (q, k, v, do)]
        c = Call(*more, starts, D ** -0.5, 1, 0, "dense")
        c.fwd()
        c.bwd()
        check(c, *more, starts, D ** -0.5, 1, 0, 2.0 ** -16, "%d rows" % T)
        got.append(c.results())
    for name, axis in (("o", 0), ("dq", 0), ("lse", 1)):
        assert np.array_equal(*(np.take(g[name], range(n), axis) for g in got)), name
    say("   elements of dk, dv that differ: %.1e" % np.mean([(got[0][x] != got[1][x][:n]).mean() for x in ("dk", "dv")]))
