"""The size of sla_prefill's workspace, on the CPU: a serving loop sizes one for its
largest call, and every smaller call has to take it."""
import ctypes
import random

import pytest

from paper_2607_16673_amd import binding as B


def need(tokens, batch, heads=4, k_heads=None, d_k=128, d_v=64, dtype=B.SLA_DTYPE_BF16, family=B.SLA_FAMILY_GDN):
    s = B.SlaPrefillShape(tokens, batch, heads, k_heads or heads, d_k, d_v, dtype, family)
    return B.lib().sla_prefill_workspace_bytes(ctypes.byref(s))


@pytest.mark.parametrize("heads,d_v", [(1, 16), (4, 64), (16, 128), (65, 16), (1100, 64)])
@pytest.mark.parametrize("dtype", [B.SLA_DTYPE_BF16, B.SLA_DTYPE_F32])
def test_it_grows_with_tokens_and_sequences(heads, d_v, dtype):
    """Both limits of the division (how many workgroups, how many tokens to a sequence) lie in these ranges."""
    tokens = sorted({0, 1, *range(5, 30), 63, 64, 65, 127, 200, 400, 1000, 2000, 16384, 16385, 20000, 100000})
    batch = sorted({*range(1, 34), 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 300, 1023, 1024, 1025, 5000, 65535})
    table = [[need(t, b, heads=heads, d_v=d_v, dtype=dtype) for b in batch] for t in tokens]
    for row in table:
        assert all(x <= y for x, y in zip(row, row[1:]))
    for a, b in zip(table, table[1:]):
        assert all(x <= y for x, y in zip(a, b))
    assert not any(table[tokens.index(6)]) and table[-1][0] > 0


def test_it_grows_in_random_shapes():
    rng = random.Random(1)
    for _ in range(3000):
        kh, d_k, d_v = rng.choice([1, 2, 4, 16]), rng.choice([64, 128, 256]), 16 * rng.randint(1, 16)
        shape = dict(heads=kh * rng.choice([1, 2, 3]), k_heads=kh, d_k=d_k, d_v=d_v, dtype=rng.randint(0, 1),
                     family=rng.randint(0, 2))
        t, b = int(2 ** rng.uniform(0, 21)), int(2 ** rng.uniform(0, 15.99))
        whole = need(t, b, **shape)
        assert need(rng.randint(0, t), rng.randint(1, b), **shape) <= whole


def test_it_is_refused_when_too_small():
    """A call takes what the size of its own shape says, whichever way its sequences go."""
    L = B.lib()
    for tokens, batch in ((20, 256), (20, 2), (2000, 255), (2000, 256), (40, 40)):
        s = B.SlaPrefillShape(tokens, batch, 4, 4, 128, 64, B.SLA_DTYPE_BF16, B.SLA_FAMILY_GDN)
        n = need(tokens, batch)
        at = [(i + 1) << 36 for i in range(10)]
        call = lambda ws, size, out: L.sla_prefill(ctypes.byref(s), at[0], at[1], 512, at[2], 512, at[3], 256, at[4], at[5],
                                                   at[6], out, at[8], ws, size, None, None)
        assert n > 0
        assert call(None, n, at[7]) == B.SLA_ERR_NULL and call(at[9], n - 1, at[7]) == B.SLA_ERR_SHAPE
        assert call(at[9], n, at[7] + 4) == B.SLA_ERR_UNSUPPORTED  # in order but for a misaligned output


@pytest.mark.gpu
def test_one_workspace_for_a_loop_whose_sequences_leave():
    from prompt_util import Prompt

    largest = Prompt([7] * 255 + [215], heads=4, dk=64, dv=32)
    ws = largest.workspace()
    largest.check(largest.run(workspace=ws))
    for lens in ([7] * 254 + [215], [7] * 30 + [215], [215], [1900], [3] * 200, [20], [1] * 256):
        p = Prompt(lens, heads=4, dk=64, dv=32, seed=len(lens))
        p.check(p.run(workspace=ws))
