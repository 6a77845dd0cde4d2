"""Attention over the 8-bit cache on values at the edge: against the definition in
64 bits.  The tolerance of an output element is 2^-8 |o| for its rounding to bf16 and
(2^-11 + 2 eps) sum p |v| for fp16 weights and scores off by eps, as in
``test_gpu_qcache.py``; what a test adds to it is derived in its docstring."""
import pytest
import torch

from .test_gpu_decoding_edges import definition, dequantised, noise

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g

    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def wide_capacity(n_rows, H=1):
    """A capacity at which even one unit's call goes to the tcgen05 kernel."""
    return -(-25 * 160 * 32 // (H * -(-n_rows // 24) * 128)) * 128


@pytest.mark.parametrize("rows", [1, 40, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_zero_queries_and_zero_keys(d, rows):
    """Padding: queries that are zero (or tiny) over blocks of keys that are zero, in
    steps where some keys are masked (by the diagonal, `first`, the end of the rows).
    Their scores are 0 whatever the scales, so the row is the mean of V: weights are
    equal, and eps is 2^-20 (exponentials and sums)."""
    from paper_2605_31598_gb300 import QCache

    held, block = 500, 16
    c = QCache(1, 1, 1, d, wide_capacity(rows), block_tokens=block)
    k, v = noise((1, 1, held, 1, d), 1), noise((1, 1, held, 1, d), 2)
    k[:, :, 32:64] = 0
    k[:, :, 192:] = 0
    k[:, :, 176:192] *= 2.0 ** -40
    k = k.masked_fill((torch.arange(held, device="cuda") < 16)[:, None, None], 0)
    zero = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    assert c.append(k, v, zero) == 0 and c.sync() == 0
    n = min(rows, held)
    q = torch.zeros((1, 1, n, 1, d), dtype=torch.bfloat16, device="cuda")
    q[:, :, 1::4] = 2.0 ** -120
    q[:, :, 2::4] = noise(q[:, :, 2::4].shape, 3) * 2.0 ** -30
    start = zero + held - n
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:4], float("nan"), device="cuda")
    kk, vv = dequantised(c, held)
    for first in (None, zero + 3, zero + 197):
        assert c.attend(q, start, out, lse=lse, first=first) == 0 and c.sync() == 0
        f = 0 if first is None else int(first)
        want, size = definition(q, kk[:, :, :, f:], vv[:, :, :, f:], start - f)
        seen = (held - n - f + 1 + torch.arange(n, device="cuda")).clamp_min(0)
        some = seen > 0  # a query before `first` sees nothing
        tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2.0 ** -19) * size
        assert ((out.double() - want).abs() <= tol)[:, :, some].all()
        assert not out[:, :, ~some].any()
        z = torch.where(some, seen.double().log(), float("-inf"))[None, None, :, None]
        assert torch.equal(lse.isinf(), z.isinf().expand(lse.shape))
        assert ((lse.double() - z).abs()[:, :, some] <= 2.0 ** -19 * z[:, :, some] + 2.0 ** -19).all()
