"""fva_rope on more tokens than one launch has threads for."""

import pytest

import paper_2607_16190_amd as fva

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [2**29 - 32, 2**29 - 31, 2**29 + 5])
def test_more_rows_than_a_launch(tokens):
    """137 GB in place: rows at both ends and around the middle against a call on those rows alone."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 256 * tokens + (8 << 30):
        pytest.skip("needs 145 GB of free device memory")
    x = torch.empty((1, 1, tokens, 128), dtype=torch.bfloat16, device="cuda:0")
    at = torch.tensor([0, 1, 31, 32, 33, 2**28 - 1, 2**28, 2**28 + 1, 2**28 + 40, tokens - 40, tokens - 2, tokens - 1])
    rows = torch.randn((1, 1, len(at), 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to("cuda:0")
    x[:, :, at.to("cuda:0")] = rows
    fva.fva_rope(x, None, (1000, 1000), (32, 48, 48), out=x)
    want = fva.fva_rope(rows, None, (1000, 1000), (32, 48, 48), ids=at.to(torch.int32).to("cuda:0"))
    got = x[:, :, at.to("cuda:0")]
    del x
    torch.cuda.empty_cache()
    assert torch.equal(got, want)
