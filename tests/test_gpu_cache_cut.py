"""Streams that pass the end of Q: the plan gives such tokens pages but no slot, and attention leaves their rows out."""

import numpy as np
import pytest

import paper_2607_16190_amd as fva
from oracle.stream import attn_ref, attn_tolerance, cached
from test_gpu_cache import DEV, Video, attn_case, bits, i32

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("frame,window", [(0, 0), (1, 0), (1, 100), (7, 50), (0, 60)])
@pytest.mark.parametrize("lens,rows,H,KH", [([300, 90, 200], [20, 30, 9], 4, 2), ([100, 4500], [20, 150], 16, 8)])
def test_rows_that_are_left_keep_their_positions(lens, rows, H, KH, frame, window):
    c = attn_case(lens, rows, 64, H, KH, seed=frame + window)
    cut = rows[0] + rows[1] // 2
    q = c["q"][:, :, :cut]
    (kc, ke), (vc, ve) = c["k"], c["v"]
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    start = np.concatenate([[0], np.cumsum(rows)])
    got = fva.fva_attn_cache(q, d(kc), d(vc), d(ke), d(ve), i32(c["table"]), i32(lens), i32(start), max(rows), frame=frame, window=window)
    got = bits(got)[0].transpose(1, 0, 2)
    x = bits(c["q"])[0].transpose(1, 0, 2)
    for s in (0, 1):
        k, v = (cached(*c[t], c["table"][s], lens[s]) for t in "kv")
        O, mass, reach = attn_ref(x[start[s]: start[s + 1]], k, v, frame, window)
        n = min(start[s + 1], cut) - start[s]
        err = np.abs(got[start[s]: start[s] + n] - O[:n])
        assert (err <= attn_tolerance(O, mass, reach)[:n]).all(), s


def test_a_step_whose_buffers_are_too_short():
    """Causal by token, the rows that fit are those of a step with room for all."""
    a, b = Video(), Video()
    outs = []
    q, k, v = a.inputs(67, 3)
    for video, n in ((a, 67), (b, 45)):
        o, q_start, held = video.step(*(t[:, :, :n].contiguous() for t in (q, k, v)), i32([20, 40, 7]), 1)
        assert q_start.tolist() == [0, 20, 60, 67] and held.tolist() == [20, 40, 7]
        outs.append(o)
    assert torch.equal(outs[0][:, :, :45], outs[1])
