"""Attention with a scale of 0 and with very small ones: scores that are huge
before they are scaled still weigh what the scaled ones say."""
import numpy as np
import pytest

from attn_util import Case
from oracle import attention as O
from test_attn_gpu import check_verify, run_verify

pytestmark = pytest.mark.gpu


def big(dtype, D, product):
    """A batch whose products of queries and keys are about `product`."""
    c = Case([0, 70, 300], 5, 4, 2, D, 16, dtype, seed=D)
    to = lambda x: c.values(x.shape, 1.0) * np.float32(2.0 ** round(np.log2((product / D ** 0.5) ** 0.5)))
    c.k, c.q = to(c.k), to(c.q)
    return c


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("scale,product", [(0.0, 1e32), (0.0, 3e36), (1e-33, 1e33), (-1e-36, 1e36), (4e-39, 3e37)])
def test_small_scales(dtype, D, scale, product):
    c = big(dtype, D, product)
    check_verify(c, run_verify(c, scale=scale), float(np.float32(scale)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_scale_of_0_keeps_what_is_not_a_number(dtype):
    """0 times an infinity or a NaN is a NaN; all other queries weigh their keys equally."""
    c = Case([40, 9], 3, 4, 2, 128, 16, dtype)
    c.parent[:] = [-1, 0, 0]
    want = run_verify(c, scale=0.0)
    c.q[0, 1, 2, 5], c.q[0, 2, 0, 77] = np.inf, np.nan
    pg, row = O.row_of(c.table[1], 10, 16)  # the second sequence's node 1, first kv head
    c.k[pg, 0, row, 3] = -np.inf
    got = run_verify(c, scale=0.0)
    bad = np.zeros(got.shape[:3], bool)
    bad[0, 1, 2] = bad[0, 2, 0] = bad[1, 1, :2] = True
    assert np.isnan(got[bad]).all()
    np.testing.assert_array_equal(got[~bad], want[~bad])
