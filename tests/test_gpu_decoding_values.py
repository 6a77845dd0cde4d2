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


def outlier_queries(n, d, kind):
    """Rows with one element far above the others."""
    g = torch.Generator(device="cuda").manual_seed(n + d)
    u = torch.rand((1, 1, n, 1, d), generator=g, device="cuda")
    if kind == "small":    # all others at 2^-18 to 2^-17 of the largest's power of two, of one sign
        q = (0.5 + 0.49 * u) * 2.0 ** -10
        q[..., 0] = 192.0
    else:                  # a thousand among 0.02 to 0.1
        q = (0.02 + 0.08 * u) * torch.where(torch.rand(u.shape, generator=g, device="cuda") < 0.5, -1.0, 1.0)
        q[..., 0] = 1000.0
    return (q * torch.exp2(torch.arange(n, device="cuda") % 9 - 4.0)[:, None, None]).to(torch.bfloat16)


@pytest.mark.parametrize("kind", ["small", "mixed"])
@pytest.mark.parametrize("d,rows", [(64, 1), (128, 1), (64, 40), (128, 40), (128, 300)])
def test_queries_with_an_outlier(d, rows, kind):
    """A query's small elements count beside a large one.  At d = 128 the tcgen05 kernel
    takes Q as two 8-bit parts, off by 2^-21 of the row's largest element at most, so a
    score is off by that times scale sum |k|: eps = 2^-20 + scale (d 2^-24 max sum |q k| +
    2^-21 max |q| max sum |k|).  Keys have nothing at the outlier's place."""
    from paper_2605_31598_gb300 import QCache

    held = 400
    c = QCache(1, 1, 1, d, wide_capacity(rows), block_tokens=16)
    size = torch.linspace(0.5, 2.0, held, device="cuda")[:, None, None]
    sign = torch.ones(d, device="cuda") if kind == "small" else torch.where(torch.arange(d, device="cuda") % 3 == 0, -1.0, 1.0)
    k = (size * sign).expand(1, 1, held, 1, d).clone()
    k[..., 0] = 0
    v = torch.where(size > 1.25, 1.0, -1.0) * (1 + torch.arange(d, device="cuda") / d)
    zero = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    assert c.append(k.to(torch.bfloat16), v.expand(1, 1, held, 1, d).to(torch.bfloat16), zero) == 0 and c.sync() == 0
    q = outlier_queries(rows, d, kind)
    kk, vv = dequantised(c, held)
    start = zero + held - rows
    out, lse = torch.empty_like(q), torch.empty(q.shape[:4], device="cuda")
    # a scale at which the small elements alone make scores of about one for the middle rows
    scale = 2.0 ** 10 / d if kind == "small" else 0.25
    assert c.attend(q, start, out, lse=lse, softmax_scale=scale) == 0 and c.sync() == 0
    want, mag = definition(q, kk, vv, start, scale)
    qq = q.double()[0, 0, :, 0]
    z = qq @ kk[0, 0, 0].T * scale
    lim = held - rows + torch.arange(rows, device="cuda")
    hidden = torch.arange(held, device="cuda") > lim[:, None]
    z = torch.logsumexp(z.masked_fill(hidden, float("-inf")), -1)
    total = (qq.abs() @ kk[0, 0, 0].abs().T).amax(-1)
    eps = 2.0 ** -20 + scale * (d * 2.0 ** -24 * total + 2.0 ** -21 * qq.abs().amax(-1) * kk.abs().sum(-1).max())
    assert ((lse[0, 0, :, 0].double() - z).abs() <= eps + 2.0 ** -20 * z.abs()).all()
    tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * eps[:, None, None]) * mag
    assert ((out.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("rows", [1, 30, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_that_are_not_finite(d, rows):
    """A query with an infinity or a NaN has no softmax, whatever the keys: its output
    and lse are NaN, and its neighbours' are within their own bounds."""
    from paper_2605_31598_gb300 import QCache

    held = 300
    c = QCache(1, 1, 1, d, wide_capacity(rows), block_tokens=16)
    k, v = noise((1, 1, held, 1, d), 1), noise((1, 1, held, 1, d), 2)
    k[..., 3] = -k[..., 3].abs() - 0.5  # an infinity there makes every score -inf
    k[..., 4] = k[..., 4].abs() + 0.5
    zero = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    assert c.append(k, v, zero) == 0 and c.sync() == 0
    q = noise((1, 1, rows, 2, d), 3)
    start = zero + held - rows
    kk, vv = dequantised(c, held)
    want, size = definition(q, kk, vv, start)
    total = torch.einsum("slnhd,slgjd->slnhj", q.double().abs(), kk.abs()).amax(-1)
    tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * (2.0 ** -20 + d ** 0.5 * 2.0 ** -24 * total[..., None])) * size
    inf = float("inf")
    for place, value in ((3, inf), (3, -inf), (4, inf), (4, -inf), (9, inf), (9, float("nan"))):
        bad = q.clone()
        bad[0, 0, ::5, 1, place] = value
        hit = torch.isnan(bad).any(-1) | torch.isinf(bad).any(-1)
        out, z = torch.zeros_like(q), torch.zeros(q.shape[:4], device="cuda")
        assert c.attend(bad, start, out, lse=z) == 0 and c.sync() == 0
        assert torch.isnan(out[hit]).all() and torch.isnan(z[hit]).all(), (place, value)
        assert ((out.double() - want).abs() <= tol)[~hit].all() and torch.isfinite(z[~hit]).all()
