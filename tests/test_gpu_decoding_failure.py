"""What follows an expired wait in the attention over the 8-bit cache.

The debug library takes one wait of the first CTA as run out, in half the lanes of its
warp, when STATEKV_QCACHE_EXPIRE_MS is set (its value is the limit of all other waits,
which then run out in turn); every copy has landed by then and nothing waits without
a limit.  Every warp leaves, the launch completes, the call reports DEVICE_TIMEOUT,
and after ``sync`` the same cache gives the right results again.  In a child process:
STATEKV_DEBUG=1 selects the library when the binding loads."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r'''
import os, sys, time
sys.path.insert(0, ROOT)
from paper_2605_31598_gb300 import build_ext
build_ext.build(debug=True)
import torch
from paper_2605_31598_gb300 import QCache, statekv
assert statekv.LIB_PATH.endswith("libstatekv_debug.so")

gen = torch.Generator(device="cuda").manual_seed(1)
noise = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
L, H, Hq, held = 3, 4, 28, 12_000
for d in (64, 128):
    c = QCache(1, L, H, d, 13_056)
    zero = torch.zeros((1, L), dtype=torch.int32, device="cuda")
    assert c.append(noise(1, L, held, H, d), noise(1, L, held, H, d), zero) == 0 and c.sync() == 0
    for n in (1, 20, 60, 147):  # 7 rows of a KV head, 140 and 420 on tcgen05, 1029: both kernels
        q, start = noise(1, L, n, Hq, d), zero + held - n
        want, got = torch.zeros_like(q), torch.zeros_like(q)
        assert c.attend(q, start, want) == 0 and c.sync() == 0
        os.environ["STATEKV_QCACHE_EXPIRE_MS"] = "100"
        t0 = time.monotonic()
        assert c.attend(q, start, got) == 0
        status = c.sync()
        elapsed = time.monotonic() - t0
        del os.environ["STATEKV_QCACHE_EXPIRE_MS"]
        assert status == 5 and elapsed < 10, (status, elapsed)  # STATEKV_ERR_DEVICE_TIMEOUT
        for _ in range(2):
            got.zero_()
            assert c.attend(q, start, got) == 0 and c.sync() == 0
            assert torch.equal(got.view(torch.int16), want.view(torch.int16)), (d, n)
        print(d, n, "%.2f s" % elapsed)
print("expired waits ok")
'''


@pytest.mark.gpu
def test_an_expired_wait_ends_the_call_and_sync_makes_the_cache_usable():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    env = dict(os.environ, STATEKV_DEBUG="1")
    env.pop("STATEKV_QCACHE_EXPIRE_MS", None)
    r = subprocess.run([sys.executable, "-c", "ROOT = %r\n" % ROOT + CHILD], env=env, cwd=ROOT,
                       capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert "expired waits ok" in r.stdout
    print(r.stdout)
