"""A wait of prompt or draft attention that runs out: reported, not hung, and the context goes on."""
import time

import pytest
import torch

from turn_cases import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,n,p", [
    ("prefill", [40], [0]),                  # one piece per item, no merge
    ("prefill", [200, 33], [900, 300]),      # pairs of row tiles, items cut between CTAs
    ("tree", [16, 7], [2000, 129]),          # one row tile: every other key tile per stream
])
def test_wait_that_runs_out_is_reported(cuda_dev, kind, n, p):
    """The first copy's barrier of one CTA expects 16 bytes more than its copies bring, so its phase never
    completes although every copy lands."""
    from paper_2609_25782_gb300 import kvtier
    c = Call(kind, n, p, seed=29)
    first = c.run().clone()
    assert torch.equal(c.run(), first) and c.pool.check_device() == 0
    kvtier.kv_pool_inject_decode_timeout(c.pool.handle, 1)
    t0 = time.monotonic()
    c.run()
    torch.cuda.synchronize()
    elapsed = time.monotonic() - t0
    assert c.pool.check_device() == kvtier.KV_DEVICE_TIMEOUT
    assert 1.5 < elapsed < 7                 # the wait and the drain's, 2 s each
    c.out.fill_(7.0)
    t0 = time.monotonic()
    assert torch.equal(c.run(), first)       # the hook has disarmed itself, the context is intact
    assert time.monotonic() - t0 < 1.0 and c.pool.check_device() == 0
