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


def filled_cache(S, L, H, d, capacity, block, held, seed):
    """A cache with ``held`` rows of noise in every unit."""
    from paper_2605_31598_gb300 import QCache

    c = QCache(S, L, H, d, capacity, block_tokens=block)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((S, L, held, H, d), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    assert c.append(k, v, torch.zeros((S, L), dtype=torch.int32, device="cuda")) == 0 and c.sync() == 0
    return c


def noise(shape, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(torch.bfloat16)


def dequantised(c, held):
    """K and V of the first ``held`` rows in 64 bits: [S][L][H][held][d]."""
    return [getattr(c, x + "_codes").view(torch.float8_e4m3fn)[:, :, :, :held].double()
            * getattr(c, x + "_scale").double().repeat_interleave(c.block_tokens, -1)[:, :, :, :held, None] for x in "kv"]


def definition(q, k, v, start, scale=None):
    """Causal attention in 64 bits of q [S][L][n][Hq][d] at rows start + i, and sum p |v|."""
    S, L, n, Hq, d = q.shape
    H, held = k.shape[2:4]
    qq = q.double().view(S, L, n, H, Hq // H, d)
    z = torch.einsum("slnhgd,slhjd->slnhgj", qq, k) * (d ** -0.5 if scale is None else scale)
    lim = start.long()[:, :, None] + torch.arange(n, device=q.device)
    z = z.masked_fill((torch.arange(held, device=q.device) > lim[..., None])[:, :, :, None, None], float("-inf"))
    p = torch.softmax(z, -1)
    return [torch.einsum("slnhgj,slhjd->slnhgd", p, x).reshape(q.shape) for x in (v, v.abs())]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L,capacity", [(1, 20_480), (60, 3_072)])
def test_calls_of_other_lengths_in_turn(d, L, capacity):
    """160 query rows of a KV head over the same cache at lengths that change from call
    to call, so the tiles that CTAs share change too, on one workspace and without a
    wait between the calls: each gives what the definition says (one rounding to bf16,
    weights in fp16), and the same bits every time."""
    n, Hq, held = 40, 4, 3_000
    c = filled_cache(1, L, 1, d, capacity, 64, held, seed=d + L)
    q = noise((1, L, n, Hq, d), 5)
    lengths = [held, 257, 1_500, 700, n]
    starts = [torch.full((1, L), m - n, dtype=torch.int32, device="cuda") for m in lengths]
    if L > 1:  # and lengths that differ between the units
        starts.append((torch.arange(L, device="cuda", dtype=torch.int32) * 49)[None].contiguous())
    outs = [[torch.zeros_like(q) for _ in range(12)] for _ in starts]
    for i in range(12):
        for st, out in zip(starts, outs):
            assert c.attend(q, st, out[i]) == 0
    assert c.sync() == 0
    k, v = dequantised(c, held)
    for st, out in zip(starts, outs):
        for x in out[1:]:
            assert torch.equal(x.view(torch.int16), out[0].view(torch.int16))
        for l in range(0, L, 20):
            want, size = definition(q[:, l:l + 1], k[:, l:l + 1], v[:, l:l + 1], st[:, l:l + 1])
            assert ((out[0][:, l:l + 1].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * size).all()


@pytest.mark.parametrize("d", [64, 128])
def test_a_nan_row_reaches_its_queries_in_many_short_units(d):
    """40 queries of one KV head in each of 400 units of 110 keys (a tile of one step
    each), every unit with a NaN code in one of the rows that some queries see: exactly
    those queries have it, in every call."""
    L, n, held = 400, 40, 110
    c = filled_cache(1, L, 1, d, 128, 16, held, seed=d)
    unit = torch.arange(L, device="cuda")
    row, place = held - n + 1 + unit % (n - 1), unit * 7 % d  # rows 71 .. 109
    c.v_codes[0, unit, 0, row, place] = 0x7F
    q = noise((1, L, n, 1, d), 3)
    start = torch.full((1, L), held - n, dtype=torch.int32, device="cuda")
    want = torch.zeros((1, L, n, 1, d), dtype=torch.bool, device="cuda")
    sees = held - n + torch.arange(n, device="cuda")[None] >= row[:, None]
    want[0, :, :, 0].scatter_(2, place[:, None, None].expand(L, n, 1), sees[..., None])
    out = torch.empty_like(q)
    for _ in range(20):
        out.zero_()
        assert c.attend(q, start, out) == 0 and c.sync() == 0
        assert torch.equal(torch.isnan(out), want)


def test_a_captured_step_outlives_a_larger_call():
    """A token step captured with the cache's own workspace, then a prompt that needs a
    larger one: the graph still has its memory, and writes to nobody else's."""
    L, H, Hq, d, held = 4, 4, 28, 128, 3_000
    c = filled_cache(1, L, H, d, 16_384, 64, held, seed=9)
    small = c.workspace.numel()
    q, start = noise((1, L, 1, Hq, d), 1), torch.full((1, L), held - 1, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    assert c.attend(q, start, out) == 0 and c.sync() == 0
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert c.attend(q, start, out) == 0
    prompt = noise((1, L, 60, Hq, d), 2)
    begin = start - 59
    first = torch.zeros_like(prompt)
    assert c.attend(prompt, begin, first) == 0 and c.sync() == 0
    assert c.workspace.numel() > small
    mine = [torch.full((small,), 7, dtype=torch.uint8, device="cuda") for _ in range(4)]
    for _ in range(3):
        out.zero_()
        graph.replay()
        again = torch.zeros_like(prompt)
        assert c.attend(prompt, begin, again) == 0 and c.sync() == 0
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        assert torch.equal(again.view(torch.int16), first.view(torch.int16))
    assert all(bool((x == 7).all()) for x in mine)


def test_a_prompt_whose_first_call_is_captured():
    """Two layers' attention captured before any call of their size; an eager call comes
    before the first replay, and others between the replays."""
    L, H, Hq, d, held, n = 2, 2, 14, 128, 3_000, 60
    c = filled_cache(1, L, H, d, 65_536, 64, held, seed=19)
    assert c.workspace_bytes(n, Hq, 1, 1) > c.workspace.numel()
    q = noise((1, L, n, Hq, d), 1)
    parts = [q[:, l:l + 1].contiguous() for l in range(L)]
    outs = [torch.zeros_like(x) for x in parts]
    start = torch.full((1, L), held - n, dtype=torch.int32, device="cuda")
    k, v = dequantised(c, held)
    want, size = definition(q, k, v, start)
    dirty = [torch.full((c.workspace_bytes(n, Hq, 1, 1),), 0x55, dtype=torch.uint8, device="cuda") for _ in range(3)]
    del dirty  # what the allocator hands out next is not zero
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for l in range(L):
            assert c.attend(parts[l], start, outs[l], layer_begin=l, layer_count=1) == 0
    for turn in range(3):
        eager = torch.zeros_like(q)
        assert c.attend(q, start, eager) == 0 and c.sync() == 0
        for x in outs:
            x.zero_()
        graph.replay()
        assert c.sync() == 0
        for got in (eager, torch.cat(outs, 1)):
            assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * size).all(), turn


def test_after_an_expired_wait_the_workspaces_are_usable_on_the_stream_given(monkeypatch):
    """``sync`` of a stream that reports an expired wait zeroes the counters before
    that stream's next call, whatever the current stream is doing."""
    from paper_2605_31598_gb300 import qcache

    c = filled_cache(1, 1, 4, 128, 16_384, 64, 3_000, seed=29)
    side = torch.cuda.Stream()
    token, prompt = noise((1, 1, 1, 28, 128), 1), noise((1, 1, 60, 28, 128), 2)
    start = torch.full((1, 1), 2_940, dtype=torch.int32, device="cuda")
    calls = [(x, start + 60 - x.shape[2]) for x in (token, prompt)]
    want = [torch.zeros_like(x) for x, _ in calls]
    spaces = []
    for (x, st), out in zip(calls, want):
        assert c.attend(x, st, out) == 0 and c.sync() == 0
        spaces.append(c.workspace)
    assert spaces[0] is not spaces[1]
    real = qcache.statekv_qcache_sync
    monkeypatch.setattr(qcache, "statekv_qcache_sync", lambda *a: real(*a) or 5)  # DEVICE_TIMEOUT
    got = [torch.zeros_like(x) for x, _ in calls]
    for ws in spaces:
        ws[:4096] = 1  # as a call that stopped halfway may leave it
    torch.cuda.synchronize()
    torch.cuda._sleep(400_000_000)
    assert c.sync(side) == 5
    with torch.cuda.stream(side):
        seen = [ws[:4096].cpu() for ws in spaces]
    assert not any(x.any() for x in seen)
    monkeypatch.undo()
    for (x, st), out in zip(calls, got):
        assert c.attend(x, st, out, stream=side) == 0
    assert c.sync(side) == 0
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_a_new_cache_is_ready_for_every_stream():
    """The counters and the status word of a cache made while its stream is busy are zero
    for a stream that does not wait for it."""
    from paper_2605_31598_gb300 import QCache

    side = torch.cuda.Stream()
    sizes = [(1, 1, 1, 64, 64), (1, 1, 4, 128, 256)]
    for S, L, H, d, cap in sizes:
        nbytes = QCache(S, L, H, d, cap).workspace.numel()
        dirty = [torch.full((nbytes,), 0x55, dtype=torch.uint8, device="cuda") for _ in range(3)]
        word = [torch.full((1,), 3, dtype=torch.int32, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        del dirty, word
        torch.cuda._sleep(400_000_000)  # a fifth of a second
        c = QCache(S, L, H, d, cap)
        with torch.cuda.stream(side):
            seen = c.workspace[:4096].cpu(), c.status.cpu()
        assert not seen[0].any() and not seen[1].any()
        torch.cuda.synchronize()


def test_a_step_of_no_tokens_does_nothing():
    """As for ``mrope``: an empty call is no error, with or without a workspace."""
    L, H, Hq, d, held = 2, 2, 4, 64, 100
    c = filled_cache(1, L, H, d, 128, 32, held, seed=39)
    before = [getattr(c, x).clone() for x in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail")]
    start = torch.full((1, L), held, dtype=torch.int32, device="cuda")
    kv = torch.empty((1, L, 0, H, d), dtype=torch.bfloat16, device="cuda")
    q = torch.empty((1, L, 0, Hq, d), dtype=torch.bfloat16, device="cuda")
    assert c.workspace_bytes(0, Hq) == c.workspace_bytes(1, Hq)
    ws = torch.zeros(c.workspace_bytes(0, Hq), dtype=torch.uint8, device="cuda")
    assert c.append(kv, kv, start) == 0
    assert c.attend(q, start, torch.empty_like(q)) == 0
    assert c.attend(q, start, torch.empty_like(q), lse=torch.empty((1, L, 0, Hq), device="cuda"), workspace=ws) == 0
    assert c.append(kv[:, :1], kv[:, :1], start, layer_begin=2, layer_count=1) == 1  # a range that is not there
    assert c.sync() == 0
    for x, y in zip(before, ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail")):
        assert torch.equal(x.view(torch.uint8), getattr(c, y).view(torch.uint8))
