"""Rotary positions and the paged cache, on the host: refusals of the C ABI and the binding, and pins of the oracle.

The refused calls never reach a kernel, so fake device addresses are safe.
"""

import ctypes

import numpy as np
import pytest
import torch

import paper_2607_16190_amd as fva
from oracle.fp8 import e4m3_decode
from oracle.stream import attn_ref, cached, page_exponent, plan_ref, rope_angles, rope_ref, store_ref, visible_keys

A = 0x7F0000001000  # 4 KiB aligned, never dereferenced


def desc(B=1, H=4, N=10, D=128, sb=None, sh=None, sn=None):
    return fva._Desc(B, H, N, D, H * N * D if sb is None else sb, N * D if sh is None else sh, D if sn is None else sn)


def params(**kw):
    p = dict(H=5, W=6, dim_t=32, dim_y=48, dim_x=48, t0=0, y0=0, x0=0, pairing=0, inverse=0, theta=1e4)
    p.update(kw)
    return fva._RopeParams(*(p[n] for n, _ in fva._RopeParams._fields_))


def rope(q=A, qo=A + 0x100000, qd=None, k=None, ko=None, kd=None, dtype=0, p=None, ids=None, stride=0):
    r = ctypes.byref
    qd = desc() if qd is None else qd
    return fva.lib.fva_rope(q, qo, r(qd) if qd else None, k, ko, r(kd) if kd else None, dtype, r(p or params()), ids, stride, None)


def test_rope_refusals():
    INV, SHAPE, UNS = fva.FVA_ERR_INVALID_ARG, fva.FVA_ERR_SHAPE, fva.FVA_ERR_UNSUPPORTED
    for want, kw in [
        (INV, dict(q=None)), (INV, dict(qo=None)), (INV, dict(q=A + 8)), (INV, dict(dtype=3)), (INV, dict(dtype=-1)),
        (INV, dict(k=A)), (INV, dict(kd=desc())), (INV, dict(k=A, kd=desc())), (INV, dict(k=A + 2, ko=A, kd=desc())),
        (INV, dict(p=params(pairing=2))), (INV, dict(p=params(inverse=2))), (INV, dict(p=params(theta=0.0))),
        (INV, dict(p=params(theta=float("nan")))), (INV, dict(p=params(theta=float("inf")))), (INV, dict(ids=A + 2)),
        (INV, dict(ids=A, stride=-1)),
        (SHAPE, dict(p=params(dim_t=34))), (SHAPE, dict(p=params(dim_t=31, dim_y=49))), (SHAPE, dict(p=params(dim_t=-2))),
        (SHAPE, dict(p=params(H=0))), (SHAPE, dict(p=params(H=1 << 20, W=1 << 20))), (SHAPE, dict(qd=desc(N=-1))),
        (SHAPE, dict(qd=desc(sn=132))), (SHAPE, dict(qd=desc(sh=0))), (SHAPE, dict(qd=desc(sn=0))), (SHAPE, dict(qd=desc(sn=120))),
        (SHAPE, dict(qd=desc(H=4, N=10, sn=256, sh=128))),  # rows of heads 2 and 3 lie on the next token's
        (SHAPE, dict(k=A, ko=A, kd=desc(N=11))), (SHAPE, dict(k=A, ko=A, kd=desc(B=2))),
        (UNS, dict(qd=desc(D=64))), (UNS, dict(qd=desc(H=65536))), (UNS, dict(qd=desc(B=65536, N=1))),
        (UNS, dict(p=params(dim_t=30, pairing=1))),
    ]:
        assert rope(**kw) == want, kw
    # nothing to turn: no pointers needed, nothing launched
    assert rope(q=None, qo=None, qd=desc(N=0)) == fva.FVA_OK


def plan(**kw):
    a = dict(held=A, fresh=A + 0x1000, streams=3, page=64, state=A + 0x2000, ring=A + 0x3000, ring_size=9, table=A + 0x4000,
             width=5, tokens=7, kv_len=A + 0x5000, q_start=A + 0x6000, slots=A + 0x7000, ids=A + 0x8000, state_out=A + 0x9000)
    a.update(kw)
    return fva.lib.fva_cache_plan(*a.values(), None)


def test_plan_refusals():
    for name in ("held", "fresh", "state", "ring", "table", "kv_len", "q_start", "slots", "ids", "state_out"):
        assert plan(**{name: None}) == fva.FVA_ERR_INVALID_ARG, name
        assert plan(**{name: A + 2}) == fva.FVA_ERR_INVALID_ARG, name
    assert plan(kv_len=A) == plan(kv_len=A + 0x1000) == plan(state_out=A + 0x2000) == fva.FVA_ERR_INVALID_ARG
    for kw in (dict(streams=0), dict(ring_size=0), dict(width=0), dict(tokens=-1)):
        assert plan(**kw) == fva.FVA_ERR_SHAPE, kw
    for kw in (dict(page=48), dict(page=0), dict(page=256), dict(streams=2049), dict(width=1 << 28, page=16)):
        assert plan(**kw) == fva.FVA_ERR_UNSUPPORTED, kw


def cache(**kw):
    a = dict(pages=20, heads=2, page=64, head_dim=128, k8=A, v8=A + 0x100000, k_exp=A + 0x200000, v_exp=A + 0x300000)
    a.update(kw)
    return fva._Cache(*a.values())


def bad_caches():
    INV, SHAPE, UNS = fva.FVA_ERR_INVALID_ARG, fva.FVA_ERR_SHAPE, fva.FVA_ERR_UNSUPPORTED
    return [(INV, cache(k8=None)), (INV, cache(v8=None)), (INV, cache(k_exp=None)), (INV, cache(v_exp=None)), (INV, cache(k8=A + 8)),
            (INV, cache(v_exp=A + 1)), (SHAPE, cache(pages=0)), (SHAPE, cache(heads=0)), (UNS, cache(head_dim=64)), (UNS, cache(page=8)),
            (UNS, cache(page=100)), (UNS, cache(pages=1 << 25))]


def store(k=A, v=A, d=None, slots=A, c=None):
    return fva.lib.fva_cache_store(k, v, ctypes.byref(d or desc(H=2)), slots, ctypes.byref(c or cache()), None)


def test_store_refusals():
    INV, SHAPE, UNS = fva.FVA_ERR_INVALID_ARG, fva.FVA_ERR_SHAPE, fva.FVA_ERR_UNSUPPORTED
    for want, c in bad_caches():
        assert store(c=c) == want
    for want, kw in [(INV, dict(k=None)), (INV, dict(v=None)), (INV, dict(slots=None)), (INV, dict(k=A + 8)), (INV, dict(slots=A + 2)),
                     (SHAPE, dict(d=desc(H=3))), (SHAPE, dict(d=desc(H=2, sn=4))), (SHAPE, dict(d=desc(H=2, N=-1))),
                     (UNS, dict(d=desc(H=2, D=64))), (UNS, dict(d=desc(B=1 << 16, H=2, N=1 << 14)))]:
        assert store(**kw) == want, kw
    assert store(k=None, v=None, slots=None, d=desc(H=2, N=0)) == fva.FVA_OK


def attn(q=A, d=None, c=None, table=A, width=5, kv_len=A, q_start=A, streams=3, max_q=4, frame=0, window=0, scale=0.0, o=A,
         ws=A, nbytes=1 << 40):
    return fva.lib.fva_attn_cache(q, ctypes.byref(d or desc()), ctypes.byref(c or cache()), table, width, kv_len, q_start, streams,
                                  max_q, frame, window, ctypes.c_float(scale), o, ws, nbytes, None)


def test_attn_refusals():
    INV, SHAPE, UNS, WS = fva.FVA_ERR_INVALID_ARG, fva.FVA_ERR_SHAPE, fva.FVA_ERR_UNSUPPORTED, fva.FVA_ERR_WORKSPACE
    for want, c in bad_caches():
        assert attn(c=c) == want
    for want, kw in [
        (INV, dict(q=None)), (INV, dict(o=None)), (INV, dict(table=None)), (INV, dict(kv_len=None)), (INV, dict(q_start=None)),
        (INV, dict(q=A + 8)), (INV, dict(o=A + 8)), (INV, dict(table=A + 2)), (INV, dict(max_q=-1)), (INV, dict(frame=-1)),
        (INV, dict(window=-1)), (INV, dict(scale=float("nan"))), (INV, dict(scale=float("inf"))),
        (SHAPE, dict(d=desc(B=2))), (SHAPE, dict(d=desc(H=3))), (SHAPE, dict(d=desc(sn=0))), (SHAPE, dict(width=0)),
        (SHAPE, dict(streams=-1)), (UNS, dict(d=desc(D=64))), (UNS, dict(width=1 << 24)),
        (WS, dict(width=100, ws=None)), (WS, dict(width=100, nbytes=100)), (WS, dict(width=100, ws=A + 128)),
    ]:
        assert attn(**kw) == want, kw
    assert attn(q=None, o=None, d=desc(N=0)) == fva.FVA_OK
    assert attn(streams=0) == fva.FVA_OK


@pytest.mark.parametrize("pages, heads", [((1 << 27) + 1, 2), (1 << 28, 2), (1 << 14, 1 << 15), (1, 1 << 29)])
def test_pools_of_too_many_page_heads(pages, heads):
    """Pages times heads, and slots, past what the kernels index with 32 bits: refused by every call that takes a pool."""
    for page in (16, 128):
        c = cache(pages=pages, heads=heads, page=page)
        assert store(d=desc(H=heads), c=c) == fva.FVA_ERR_UNSUPPORTED
        assert attn(d=desc(H=heads), c=c) == fva.FVA_ERR_UNSUPPORTED
        with pytest.raises(fva.FvaError):
            fva.fva_attn_cache_workspace_size(desc(H=heads), c, 1, 1, 1)


def test_attn_workspace_size():
    n = fva.fva_attn_cache_workspace_size(desc(N=1), cache(), 100, 1, 1)
    assert n > 0 and n % 4 == 0
    # one page of keys is never split, nor are rows that fill the device by themselves
    assert fva.fva_attn_cache_workspace_size(desc(N=1), cache(), 1, 1, 1) == 0
    assert fva.fva_attn_cache_workspace_size(desc(N=1 << 20), cache(), 100, 1, 1 << 20) == 0
    with pytest.raises(fva.FvaError):
        fva.fva_attn_cache_workspace_size(desc(H=3), cache(), 100, 1, 1)


def test_binding_refuses_host_tensors_and_wrong_types():
    x = torch.zeros((1, 2, 4, 128), dtype=torch.bfloat16)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        fva.fva_rope(x, None, (2, 2), (32, 48, 48))
    with pytest.raises(ValueError):
        fva.fva_rope(x.double(), None, (2, 2), (32, 48, 48))
    with pytest.raises(ValueError):
        fva.fva_rope(x, x.float(), (2, 2), (32, 48, 48))
    with pytest.raises(ValueError):
        fva.fva_cache_store(x.float(), x, None, None, None, None, None)
    with pytest.raises(ValueError):
        fva.fva_cache_store(x, x[:, :1], None, None, None, None, None)
    with pytest.raises(ValueError):
        fva.fva_attn_cache(x.half(), None, None, None, None, None, None, None, 1)


# ---- the oracle -------------------------------------------------------------


def test_rope_closed_forms():
    # position 0 turns nothing; one full turn neither; a quarter turn moves u to v and v to -u
    x = np.random.default_rng(0).standard_normal((2, 3, 128))
    zero = rope_angles([0, 0, 0], 4, 4, (32, 48, 48), (0, 0, 0), 1e4)
    assert np.array_equal(rope_ref(x, zero, False), x)
    quarter = np.full((3, 64), np.pi / 2)
    y = rope_ref(x, quarter, False)
    assert np.allclose(y[..., 1::2], x[..., 0::2]) and np.allclose(y[..., 0::2], -x[..., 1::2])
    y = rope_ref(x, quarter, True)
    assert np.allclose(y[..., 64:], x[..., :64]) and np.allclose(y[..., :64], -x[..., 64:])
    # axis and channel of an angle: id 4 * 4 + 2 * 4 + 3 is (1, 2, 3)
    a = rope_angles([27], 4, 4, (4, 6, 8), (0, 0, 0), 100.0)[0]
    want = [1, 1 / 10] + [2 * 100 ** (-2 * i / 6) for i in range(3)] + [3 * 100 ** (-2 * i / 8) for i in range(4)]
    assert np.allclose(a, want)


def test_rope_scores_depend_on_differences():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 128))
    dots = []
    for origin in ((0, 0, 0), (5, 2, 9)):
        a, b = (rope_angles([n], 8, 9, (44, 42, 42), origin, 1e4) for n in (101, 17))
        dots.append(rope_ref(q, a, False)[0] @ rope_ref(k, b, False)[0])
    assert np.allclose(*dots)


def test_plan_by_hand():
    kv, qs, slots, ids, st, table, ring = plan_ref([10, 0, 33], [8, 20, -1], [3, 2, 0], [7, 8, 9, 4, 5], [[2, -1], [-1, -1], [0, 1]], 16, 30)
    assert kv.tolist() == [18, 0, 0] and qs.tolist() == [0, 8, 28, 28]
    # stream 0 takes page 4; stream 1 needs two of the one that is left: refused; stream 2 gives its three pages back
    assert table.tolist()[0] == [2, 4] and st.tolist()[2] == 1
    assert slots[:8].tolist() == [2 * 16 + 10 + i for i in range(6)] + [64, 65] and (slots[8:] == -1).all()
    assert ids[:8].tolist() == list(range(10, 18))


def test_store_and_cached():
    assert page_exponent(448.0) == 0 and page_exponent(449.0) == 1 and page_exponent(0.0) == -100 and page_exponent(2.0**-126) == -100
    x = np.zeros((3, 1, 128))
    x[0], x[1], x[2] = 448, 1, 1000
    codes, exps = store_ref(x[:2], [5 * 16, 5 * 16 + 1], np.zeros((6, 1, 16, 128), np.uint8), np.zeros((6, 1), int))
    assert exps[5, 0] == 0 and e4m3_decode(codes[5, 0, 1, 0]) == 1
    codes, exps = store_ref(x[2:], [5 * 16 + 2], codes, exps)  # the scale grows: 448 -> 224 * 2^... , 1 -> 0.5 ...
    assert exps[5, 0] == 2
    assert cached(codes, exps, [5], 3)[:, 0, 0].tolist() == [448, 1, 1024]


def test_visible_keys_and_attention():
    assert visible_keys(10, 10, 3, 1, 0) == (0, 4) and visible_keys(10, 2, 0, 0, 0) == (0, 10)
    assert visible_keys(100, 10, 0, 32, 40) == (56, 96) and visible_keys(100, 10, 9, 32, 40) == (88, 100)
    assert visible_keys(3, 5, 0, 4, 0) == (0, 0)
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((3, 6, 2, 128))
    O, _, _ = attn_ref(q, k, v, 1, 0)
    assert np.allclose(O[0], v[0])  # the first token sees itself
    s = np.einsum("ihd,jhd->hij", q, k) / 128**0.5
    s[:, ~np.tri(6, dtype=bool)] = -np.inf
    w = np.exp(s - s.max(-1, keepdims=True))
    assert np.allclose(O, np.einsum("hij,jhd->ihd", w / w.sum(-1, keepdims=True), v))
