"""Gradients of ``mrope`` through autograd."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g

    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def inputs(tokens=37, hq=6, hk=2, d=64):
    from paper_2605_31598_gb300 import mrope_frequencies

    gen = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.randn((tokens, hq + 2 * hk, d), generator=gen, device="cuda").to(torch.bfloat16)
    at = torch.randint(0, 5000, (3, tokens), generator=gen, device="cuda", dtype=torch.int32)
    return qkv, hq, hk, at, *mrope_frequencies((8, 12, 8), 1e4)


def plain(x, at, freq, axis, scale, adjacent):
    """The definition in 64-bit torch operations, which autograd differentiates."""
    P = len(freq)
    ang = (at.double()[axis.long().cuda()] * freq.cuda()[:, None]).T[:, None]
    c, s = scale * torch.cos(ang), scale * torch.sin(ang)
    a, b = (x[..., 0:2 * P:2], x[..., 1:2 * P:2]) if adjacent else (x[..., :P], x[..., P:2 * P])
    y = [a * c - b * s, b * c + a * s]
    y = torch.stack(y, -1).flatten(-2) if adjacent else torch.cat(y, -1)
    return torch.cat((y, x[..., 2 * P:]), -1)


@pytest.mark.parametrize("adjacent", [False, True])
def test_gradients_reach_the_projection(adjacent):
    """d loss / d qkv of a loss over the turned q and k, which are slices of one
    tensor: each element within its rounding to bf16 (2^-8), the loss's gradient being
    given in bf16, and 2^-20 of its pair in fp32."""
    from paper_2605_31598_gb300 import mrope

    qkv, hq, hk, at, freq, axis = inputs()
    kw = dict(scale=1.25, adjacent=adjacent)
    gq = torch.randn_like(qkv[:, :hq]).transpose(0, 1).contiguous().transpose(0, 1)  # heads first
    gk = torch.randn((1, 1, 64), device="cuda").to(torch.bfloat16).expand(37, hk, 64)
    x = qkv.clone().requires_grad_()
    q, k = mrope(x[:, :hq], x[:, hq:hq + hk], at, freq, axis, **kw)
    assert q.requires_grad and k.requires_grad
    torch.autograd.backward((q, k), (gq, gk))
    y = qkv.double().requires_grad_()
    torch.autograd.backward([plain(z, at, freq, axis, **kw) for z in (y[:, :hq], y[:, hq:hq + hk])], (gq.double(), gk.double()))
    assert torch.equal(x.grad[:, hq + hk:], torch.zeros_like(x.grad[:, hq + hk:]))
    pair = 2.0 ** -20 * 1.25 * 2 * max(float(gq.abs().max()), float(gk.abs().max()))
    assert ((x.grad.double() - y.grad).abs() <= 2.0 ** -8 * y.grad.abs() + pair).all()


def test_one_tensor_with_a_gradient_and_none():
    from paper_2605_31598_gb300 import mrope

    qkv, hq, hk, at, freq, axis = inputs()
    q, k = qkv[:, :hq].clone().requires_grad_(), qkv[:, hq:hq + hk].clone()
    want = mrope(q.detach(), k, at, freq, axis)
    got = mrope(q, k, at, freq, axis)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got[0].sum().backward()  # the gradient comes expanded from one element
    one = torch.ones_like(want[0])
    assert torch.equal(q.grad, mrope(one, None, at, freq, axis, transpose=True)[0])
    q.grad = None
    turned, none = mrope(q, None, at, freq, axis, transpose=True)
    assert none is None
    turned.backward(one)
    assert torch.equal(q.grad, mrope(one, None, at, freq, axis)[0])
    q.grad = None
    mrope(None, k.requires_grad_(), at, freq, axis)[1].sum().backward()
    assert q.grad is None and torch.equal(k.grad, mrope(None, torch.ones_like(k), at, freq, axis, transpose=True)[1].detach())
    with torch.no_grad():
        assert not mrope(q, k, at, freq, axis)[0].requires_grad


def test_what_autograd_cannot_follow_is_refused():
    from paper_2605_31598_gb300 import mrope

    qkv, hq, hk, at, freq, axis = inputs()
    q = qkv[:, :hq].clone().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        mrope(q, None, at, freq, axis, q_out=torch.empty_like(q))
    with torch.no_grad():
        mrope(q, None, at, freq, axis, q_out=torch.empty_like(q))
    turned = mrope(q, None, at, freq, axis)[0]
    at.add_(1)  # the positions that the gradient needs are gone
    with pytest.raises(RuntimeError, match="inplace"):
        turned.sum().backward()
