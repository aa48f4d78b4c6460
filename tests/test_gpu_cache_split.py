"""Large tiles of attention over the cache: calls whose tiles leave most of the device idle split their keys.

A call that splits leaves partial results in its workspace, one that does not leaves the chunk length alone.
"""

import numpy as np
import pytest

import paper_2607_16190_amd as fva
from oracle.stream import attn_ref, attn_tolerance, cached
from test_gpu_cache import DEV, bits, i32

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def run(lens, rows, H, KH, frame, window=0, page=64, seed=0):
    """One call with a cleared workspace: whether it split any keys; its output is compared at some rows."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 1
    order = np.random.default_rng(seed).permutation(pages)
    table, at = np.full((len(lens), max(need) + 1), -1), 0
    for s, n in enumerate(need):
        table[s, :n] = order[at: at + n]
        at += n
    code = lambda: (torch.randn((pages, KH, page, 128), generator=g, device=DEV, dtype=torch.bfloat16) * 60).clamp(-448, 448).to(  # noqa: E731
        torch.float8_e4m3fn).view(torch.uint8)
    k8, v8 = code(), code()
    ke, ve = (torch.randint(-7, -4, (pages, KH), generator=g, device=DEV, dtype=torch.int32) for _ in range(2))
    q = torch.randn((1, sum(rows), H, 128), generator=g, device=DEV).to(torch.bfloat16).transpose(1, 2)
    start = np.concatenate([[0], np.cumsum(rows)])
    cache = fva._cache_of(k8, v8, ke, ve)
    nbytes = fva.fva_attn_cache_workspace_size(fva._rows_of(q), cache, table.shape[1], len(lens), max(rows))
    ws = torch.zeros(max(nbytes, 256) // 4, dtype=torch.int32, device=DEV)
    out = fva.fva_attn_cache(q, k8, v8, ke, ve, i32(table), i32(lens), i32(start), max(rows), frame=frame, window=window, workspace=ws)
    assert out.isfinite().all()
    host = {}
    longest = int(np.argmax(lens))
    for s in {0, longest, len(lens) - 1}:
        n, m = lens[s], rows[s]
        if not n or not m:
            continue
        mine = torch.from_numpy(table[s, : need[s]]).to(DEV)
        for h in {0, KH - 1}:
            kk, vv = (cached(c[mine][:, h: h + 1].cpu().numpy(), e[mine][:, h: h + 1].cpu().numpy(), np.arange(need[s]), n)
                      for c, e in ((k8, ke), (v8, ve)))
            heads = slice(h * (H // KH), (h + 1) * (H // KH))
            for i in {0, m // 2, m - 1}:
                p = n - m + i
                end = min(n, (p // frame + 1) * frame) if frame else n
                lo = max(0, ((p // frame + 1) * frame if frame else n) - window) if window else 0
                a = start[s] + i
                O, mass, reach = attn_ref(bits(q[0, heads, a: a + 1]).transpose(1, 0, 2), kk[lo:end], vv[lo:end])
                err = np.abs(bits(out[0, heads, a: a + 1]).transpose(1, 0, 2) - O)
                assert (err <= attn_tolerance(O, mass, reach)).all(), (s, h, i)
    return int((ws != 0).sum().item()) > 128


@pytest.mark.parametrize("frame", [1, 1560])
@pytest.mark.parametrize("H,rows,keys", [(5, 4680, 15600), (5, 4680, 32760), (8, 1560, 61560), (40, 1560, 34320)])
def test_causal_chunks_are_split(H, rows, keys, frame):
    """185, 185, 104 and 520 tiles for the 512 workgroups that run at once."""
    assert run([keys], [rows], H, H, frame)


@pytest.mark.parametrize("keys", range(6000, 33000, 2700))
def test_a_share_of_heads_is_split_at_every_length(keys):
    assert run([keys], [4680], 5, 5, 1560)


@pytest.mark.parametrize("frame", [0, 1])
@pytest.mark.parametrize("streams,H,keys,at", [(100, 8, 100000, 0), (100, 8, 100000, 57), (30, 40, 30000, 11), (64, 8, 60000, 63), (65, 8, 60000, 64)])
def test_a_long_stream_among_many_short_ones_is_split(streams, H, keys, at, frame):
    """More tiles than there are places for partial results, or streams than a wave has lanes: the short ones leave none."""
    lens = [300 + (7 * s) % 50 for s in range(streams)]
    lens[at] = keys
    assert run(lens, [32 - s % 3 for s in range(streams)], H, H, frame, seed=at)


@pytest.mark.parametrize("frame", [0, 1, 450])
def test_many_streams_that_one_round_has_no_room_for(frame):
    """The mean of causal rows is half of their widest: twice as many chunks as estimated."""
    run([900] * 66, [900] * 66, 1, 1, frame, page=16)
    lens, rows = [900] * 66, [900] * 66
    lens[40] = 20000
    assert run(lens, rows, 1, 1, frame, page=16)


def test_long_and_short_streams_in_turn():
    """Partial results of split streams with unsplit ones between them, on both sides of the 64th."""
    lens = [9000 if s % 9 == 4 else 200 + 3 * s for s in range(100)]
    assert run(lens, [33] * 100, 16, 4, 1)
    assert run(lens[:60], [33] * 60, 16, 4, 1)
