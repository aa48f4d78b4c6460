"""Index tensors of the cache calls and the rotary positions laid out the other way round are refused, not read as if
they lay right. Host tensors: every check here comes before the call."""

import pytest
import torch

import paper_2607_16190_amd as fva

PAGES, HEADS, PAGE, B, N, S, W = 6, 2, 16, 2, 5, 3, 4


@pytest.fixture(autouse=True)
def _host(monkeypatch):
    monkeypatch.setattr(fva, "_same_device", lambda *tensors: 0)

    class NoCall:
        def __getattr__(self, name):
            raise AssertionError(f"{name} was called")

    monkeypatch.setattr(fva, "lib", NoCall())


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def rows(heads, batch=B, tokens=N):
    return torch.zeros((batch, heads, tokens, 128), dtype=torch.bfloat16)


def codes():
    return torch.zeros((PAGES, HEADS, PAGE, 128), dtype=torch.uint8)


def refused(what, call, *args, **kw):
    with pytest.raises(ValueError, match=f"^{what} must be a contiguous int32 tensor of shape"):
        call(*args, **kw)


def rope(ids):
    return fva.fva_rope(rows(1), None, (3, 3), (32, 48, 48), ids=ids)


def store(slots=None, k_exp=None, v_exp=None):
    e = ints(PAGES, HEADS)
    return fva.fva_cache_store(rows(HEADS), rows(HEADS), ints(B * N) if slots is None else slots, codes(), codes(),
                               e if k_exp is None else k_exp, e if v_exp is None else v_exp)


def attn(kv_len=None, q_start=None, table=None, k_exp=None, v_exp=None):
    e = ints(PAGES, HEADS)
    return fva.fva_attn_cache(rows(HEADS, 1), codes(), codes(), e if k_exp is None else k_exp, e if v_exp is None else v_exp,
                              ints(S, W) if table is None else table, ints(S) if kv_len is None else kv_len,
                              ints(S + 1) if q_start is None else q_start, N)


def plan(**kw):
    a = dict(held=ints(S), fresh=ints(S), state=ints(3), ring=ints(9), block_table=ints(S, W))
    a.update(kw)
    return fva.fva_cache_plan(*a.values(), PAGE, N)


def test_documented_shapes_reach_the_call():
    for call in (lambda: rope(ints(N)), lambda: rope(ints(B, N)), store, lambda: store(ints(B, N)), attn, plan):
        with pytest.raises(AssertionError, match="was called"):
            call()


@pytest.mark.parametrize("shape", [(N, B), (1, B * N), (B, N, 1), ()])
def test_ids(shape):
    refused("ids", rope, ints(*shape))


@pytest.mark.parametrize("shape", [(HEADS, PAGES), (PAGES * HEADS,), (PAGES, HEADS, 1)])
def test_exponents(shape):
    for call in (store, attn):
        refused("k_exp", call, k_exp=ints(*shape))
        refused("v_exp", call, v_exp=ints(*shape))
    refused("k_exp", store, k_exp=ints(HEADS, PAGES).t())  # right shape, other order in memory


@pytest.mark.parametrize("shape", [(N, B), (1, B * N), (B, N, 1)])
def test_slots(shape):
    refused("slots", store, ints(*shape))


def test_lengths_and_tables():
    for shape in ((W, S), (S * W,), (1, S, W), ()):
        refused("block_table", attn, table=ints(*shape))
        refused("block_table", plan, block_table=ints(*shape))
    refused("kv_len", attn, kv_len=ints(S, 1))
    refused("q_start", attn, q_start=ints(1, S + 1))
    for name in ("held", "fresh", "state"):
        refused(name, plan, **{name: ints(1, S)})
    refused("ring", plan, ring=ints(3, 3))
