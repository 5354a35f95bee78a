"""The 8-bit KV cache on the device at the edges of its numbers: values below fp32's normal range, scales of zero and
below it, scores beyond it; against the restatement in 64 bits (oracle/cache_q8.py)."""
import numpy as np
import pytest

from oracle import cache_q8 as oq
from test_gpu_q8 import B, Cache, _bf16, _i32, _values  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _steps(c, rng, what, kv=1.0):
    """A decode and two fused steps, each against the oracle."""
    n, hq = len(c.lens0), c.heads * c.group
    o, qf = c.decode(rng.standard_normal((n, hq, c.d)))
    c.check_rows(o, qf, what=f"{what} decode")
    for t in range(2):
        o, qf = c.step(rng.standard_normal((n, hq, c.d)), *(_values(rng, n, c.heads, c.d) * kv for _ in range(2)))
        c.check_rows(o, qf, what=f"{what} step {t}")
    c.check_pool(what)
    assert c.status() == c.B.CPA_OK


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("num_sms", [0, 1])
def test_rows_below_the_normal_range_keep_their_values(B, d, num_sms):
    # V of 2^-131 .. 2^-127: bf16 holds them (down to 2^-133), and so has the output; one block is joined across CTAs
    lens = [3000, 20, 1]
    c = Cache(B, lens, 2, 2, d, seed=d, num_sms=num_sms)
    rng = np.random.default_rng(31)
    k, v = (_values(rng, sum(lens), 2, d) for _ in range(2))
    c.append(k, v * 2.0 ** -129, lens)
    q = rng.standard_normal((3, 8, d))
    o, qf = c.decode(q)
    c.check_rows(o, qf)
    assert (o[1:] != 0).any()
    o, qf = c.step(q, _values(rng, 3, 2, d), _values(rng, 3, 2, d) * 2.0 ** -129)
    c.check_rows(o, qf, what="step")
    c.check_pool()
