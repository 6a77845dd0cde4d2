"""Decoding operators on arguments and timings at the edge of what they take."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g

    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("tokens,row", [(1, 1), (1, 9), (7, 7), (37, 40), (2500, 2500)])
def test_mrope_of_positions_expanded_over_the_axes(tokens, row, adjacent):
    """Text tokens have equal positions on all axes: one row expanded gives what its
    copies give, bit for bit."""
    from paper_2605_31598_gb300 import mrope, mrope_frequencies

    freq, axis = mrope_frequencies((8, 12, 12), 1e4)
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    q, k = (torch.randn((tokens, h, 64), generator=gen, device="cuda").to(torch.bfloat16) for h in (6, 2))
    at = torch.arange(1000, 1000 + row, dtype=torch.int32, device="cuda").expand(3, row)[:, row - tokens:]
    want = mrope(q, k, at.contiguous(), freq, axis, adjacent=adjacent)
    got = mrope(q, k, at, freq, axis, adjacent=adjacent)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
