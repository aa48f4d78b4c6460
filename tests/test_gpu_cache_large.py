"""Attention over the cache in large tiles of 128 rows, on calls that are shown to take them.

The estimate of the longest stream's rows chooses the kernel: with 0 every call takes tiles of 16 rows, whose sums are in
another order, so that some of the output's bits differ where the call itself takes the large ones.
"""

import numpy as np
import pytest

import paper_2607_16190_amd as fva
from oracle.stream import attn_ref, attn_tolerance, cached
from test_gpu_cache import DEV, attn_case, bits, check_attn, i32

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def upload(c):
    """The case's cache on the device once."""
    (kc, ke), (vc, ve) = c["k"], c["v"]
    c["dev"] = [torch.from_numpy(np.ascontiguousarray(a)).to(DEV) for a in (kc, vc, ke, ve)] + [i32(c["table"])]
    return c


def attend(c, frame=0, window=0, max_q=None, lens=None, start=None, q=None, **kw):
    start = np.concatenate([[0], np.cumsum(c["rows"])]) if start is None else start
    return fva.fva_attn_cache(c["q"] if q is None else q, *c["dev"], i32(c["lens"] if lens is None else lens), i32(start),
                              max(c["rows"]) if max_q is None else max_q, frame=frame, window=window, **kw)


def takes_large(c, frame=0, window=0):
    return not torch.equal(attend(c, frame, window), attend(c, frame, window, max_q=0))


@pytest.mark.parametrize("frame,window", [(1, 700), (100, 333), (0, 900), (1000, 600), (2000, 600)])
@pytest.mark.parametrize("page", [16, 64])
def test_short_windows(frame, window, page):
    c = upload(attn_case([2601, 150, 0, 1300, 129], [150, 150, 3, 257, 0], page, 48, 16, seed=page + window))
    if frame < 2000:  # no row sees a key of a frame that is cached to less than its last 600
        assert takes_large(c, frame, window)
    check_attn(c, frame, window)


@pytest.mark.parametrize("lens,H,frame,window,split", [
    ([1500], 40, 1, 1000, False), ([1500], 40, 0, 1300, False), ([1500], 40, 50, 700, False),  # 200 workgroups: either way
    ([2600], 20, 1, 1500, True), ([2600], 20, 0, 1300, True), ([2600], 20, 50, 1700, True),
])
@pytest.mark.parametrize("page", [32, 128])
def test_windows_of_up_to_2048_keys(lens, H, frame, window, split, page):
    c = upload(attn_case(lens, [600], page, H, H, seed=window))
    assert takes_large(c, frame, window)
    cache = fva._cache_of(*c["dev"][:4])
    nbytes = fva.fva_attn_cache_workspace_size(fva._rows_of(c["q"]), cache, c["table"].shape[1], 1, 600)
    ws = torch.zeros(nbytes // 4 + 1, dtype=torch.int32, device=DEV)
    out = attend(c, frame, window, workspace=ws)
    if split:
        assert int((ws != 0).sum()) > 128  # partial results
    assert torch.equal(out, attend(c, frame, window))
    check_attn(c, frame, window)


def test_uneven_rows():
    """Q rows of very different size, a few large channels, zeros, tiny elements, and a NaN row that stays alone."""
    c = attn_case([4500], [150], 64, 8, 8, seed=2)
    g = torch.Generator().manual_seed(3)
    q = c["q"].float().cpu() * torch.exp(1.5 * torch.randn((1, 8, 150, 1), generator=g).clamp(-2, 1))
    q[..., 5] *= 12
    q[0, 3, 7] = 0
    q[0, 2, 9, 1:] *= 2.0**-20
    q[0, 4, 11] *= 2.0**-60
    q[0, 5, 13] *= 2.0**-126  # below what the codes of Q hold: scores of nearly zero
    c["q"] = q.to(torch.bfloat16).to(DEV)
    upload(c)
    for frame in (0, 1):
        assert takes_large(c, frame)
        check_attn(c, frame)
    want = attend(c, 1)
    c["q"][0, 1, 2, 77] = float("nan")
    c["q"][0, 6, 140, 3] = float("inf")
    got = attend(c, 1)
    for h, i in ((1, 2), (6, 140)):
        assert got[0, h, i].isnan().all()
        got[0, h, i] = want[0, h, i]
    assert torch.equal(got, want)


@pytest.mark.parametrize("frame", [0, 1])
def test_estimates_of_the_longest_stream(frame):
    """max_q chooses the kernel and nothing else: either one is within its tolerance."""
    c = upload(attn_case([4500, 40], [120, 2], 64, 8, 8, seed=4))
    large = attend(c, frame)
    start = np.concatenate([[0], np.cumsum(c["rows"])])
    q = bits(c["q"])[0].transpose(1, 0, 2)
    for estimate in (0, 1, 17, 120, 5000):
        got = attend(c, frame, max_q=estimate)
        assert torch.equal(got, large) == (estimate > 16)
        for s, (n, m) in enumerate(zip(c["lens"], c["rows"])):
            k, v = (cached(*c[x], c["table"][s], n) for x in "kv")
            O, mass, reach = attn_ref(q[start[s]: start[s + 1]], k, v, frame)
            err = np.abs(bits(got)[0].transpose(1, 0, 2)[start[s]: start[s + 1]] - O)
            assert (err <= attn_tolerance(O, mass, reach)).all()


def test_small_tiles_keep_the_bits_of_q():
    """Q of widely different elements: small tiles round none of them, so the bound has no part for that."""
    c = attn_case([700, 90], [2, 5], 64, 4, 2, seed=6)
    g = torch.Generator().manual_seed(5)
    q = c["q"].float().cpu() * torch.exp2(torch.randint(-16, 3, c["q"].shape, generator=g).float())
    q[..., 7] = 200.0
    # the large channel meets keys of zero: the small ones decide
    for side in (c["k"][0],):
        side[..., 7] = 0
    c["q"] = q.to(torch.bfloat16).to(DEV)
    upload(c)
    got = bits(attend(c, 1))[0].transpose(1, 0, 2)
    x = bits(c["q"])[0].transpose(1, 0, 2)
    at = 0
    for s, (n, m) in enumerate(zip(c["lens"], c["rows"])):
        k, v = (cached(*c[t], c["table"][s], n) for t in "kv")
        O, mass, _ = attn_ref(x[at: at + m], k, v, 1)
        kk = np.repeat(k, 2, axis=1)  # heads of a group
        reach = np.einsum("ihd,jhd->ihj", np.abs(x[at: at + m]), np.abs(kk)).max(-1) / 128**0.5
        assert (np.abs(got[at: at + m] - O) <= attn_tolerance(O, mass, reach)).all()
        at += m


def test_starts_that_are_not_ascending_stay_in_bounds():
    """Rows of such streams are of no meaning; the call returns, and rows of no stream, in or around the tensor, stay."""
    c = upload(attn_case([4500, 700, 800], [80, 40, 40], 64, 8, 8, seed=7))
    assert takes_large(c, 1)
    around = torch.full((160 + 64, 8, 128), 5.0, dtype=torch.bfloat16, device=DEV)
    out = around[32:192].transpose(0, 1)[None]
    assert out.stride() == c["q"].stride()
    cache = fva._cache_of(*c["dev"][:4])
    nbytes = fva.fva_attn_cache_workspace_size(fva._rows_of(c["q"]), cache, c["table"].shape[1], 3, 80)
    guard = 1 << 20
    ws = torch.full((nbytes + 2 * guard,), 7, dtype=torch.uint8, device=DEV)
    for start in ([0, 160, 0, 160], [-5, 2**31 - 1, -7, 30], [100, 50, 20, 0], [0, 40, 80, 2**31 - 1], [160, 0, 160, 0], [40, 80, 80, 120]):
        for frame in (0, 1):
            attend(c, frame, lens=[2**31 - 1, -4, 800], start=start, out=out, workspace=ws[guard: guard + nbytes])
    assert bool((around[:32] == 5).all()) and bool((around[192:] == 5).all())
    assert bool((ws[:guard] == 7).all()) and bool((ws[guard + nbytes:] == 7).all())
    around.fill_(5.0)
    attend(c, 1, start=[40, 80, 80, 120], out=out)
    assert bool((out[:, :, :40] == 5).all()) and bool((out[:, :, 120:] == 5).all()) and bool(out[:, :, 40:120].isfinite().all())


def test_captured_call_on_new_lengths():
    """A captured call of large tiles, split and whole by the lengths of the moment, against eager calls."""
    c = upload(attn_case([9000, 4000], [300, 200], 64, 16, 8, seed=8))
    lens, start = i32(c["lens"]), i32([0, 300, 500])
    call = lambda: fva.fva_attn_cache(c["q"], *c["dev"], lens, start, 300, frame=1)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for n in ([9000, 4000], [300, 200], [9000, 0], [1200, 3999], [0, 0], [8999, 250], [9000, 4000]):
        lens.copy_(i32(n))
        graph.replay()
        want = call()
        torch.cuda.synchronize()
        assert torch.equal(out, want), n


def test_two_streams_at_once():
    cases = [upload(attn_case([5000 + 300 * i], [200], 64, 16, 8, seed=i)) for i in (0, 1)]
    want = [attend(c, 1) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                got.append(attend(c, 1))
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))
