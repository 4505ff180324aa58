"""The example's session when its pool runs out in the middle of a batch: the
error leaves every branch's rows in place, and a later try gives the logits that
a session with room for all gives."""
import numpy as np
import pytest
import torch

from test_hybrid_round_gpu import E  # noqa: F401  (the example, as a fixture)

pytestmark = pytest.mark.gpu


def test_a_pool_that_runs_out_loses_nothing(E):
    target = E.Target()
    tokens = np.random.default_rng(3).integers(0, E.VOCAB, 72).tolist()  # four pages and a half
    step = np.array([[5], [6], [7]], np.int32), np.full((3, 1), -1, np.int32)
    logits = []
    for pages in (40, 7):
        s = E.Session(target, pages=pages)
        s.prompt(tokens)
        other = s.pool.new()
        s.pool.reserve(other, 16)  # one page of seven is left: two of the branches need one
        b = s.fork(3)
        s.close()
        if pages == 7:
            with pytest.raises(MemoryError):
                b.verify(*step)
            s.pool.free(other)
        logits.append(b.verify(*step))
    assert torch.equal(*logits)
