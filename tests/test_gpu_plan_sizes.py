"""The cache plan at the largest sizes its arguments allow."""

import numpy as np
import pytest

import paper_2607_16190_amd as fva
from test_gpu_cache import DEV, i32

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [2**31 - 1, 2**31 - 1000, 2**31 - 65536, 2**31 - 65537])
def test_as_many_rows_as_there_can_be(tokens):
    """Buffers of up to 2^31 - 1 rows: the step past their end is no index."""
    table, ring = i32([[-1, -1, -1, -1], [2, -1, -1, -1]]), i32([5, 6, 7, 8])
    # the rows stand in one buffer between others, which stay
    guard = 1 << 20
    rows = [torch.full((tokens + 2 * guard,), 77, dtype=torch.int32, device=DEV) for _ in range(2)]
    out = (*(i32(np.zeros(n)) for n in (2, 3)), *(r[guard: guard + tokens] for r in rows), i32([0, 0, 0]))
    kv_len, q_start, slots, ids, state = fva.fva_cache_plan(i32([0, 3]), i32([20, 14]), i32([1, 4, 0]), ring, table, 16, tokens, out=out)
    assert kv_len.tolist() == [20, 17] and q_start.tolist() == [0, 20, 34] and state.tolist() == [0, 1, 0]
    assert ids[:34].tolist() == [*range(20), *range(3, 17)]
    assert slots[:34].tolist() == [*range(96, 112), *range(112, 116), *range(35, 48), 128]
    for x in (slots, ids):
        assert int(x[34:].max()) == int(x[34:].min()) == -1
    for r in rows:
        assert bool((r[:guard] == 77).all()) and bool((r[guard + tokens:] == 77).all())
