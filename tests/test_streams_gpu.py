"""Steps of one cache on many streams: the die that a launch begins on is the hardware queue's, and a process with more
streams than a few has queues that begin on different ones.  The results are those of the default stream."""
import pytest
import torch

from tests import lockstep as ls
from workloads import decode_inputs, get_workload, prompt_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("units", [(1, 8), (2, 8)])
def test_steps_on_many_streams_match_the_default_stream(units):
    from paper_2410_23079_amd import FLAG_AUTO_EVICT, FLAG_DETERMINISTIC, BuzzCache
    wl = get_workload("tiny").scaled(batch=units[0], n_kv_heads=units[1], n_q_heads=4 * units[1], head_dim=128, dtype="bf16", prompt=2600,
               decode_steps=24, sink=4, window=1100, segment=16, keep=3, evict_every=16, n_obs=24)
    p, d = prompt_inputs(wl, device="cuda"), decode_inputs(wl, device="cuda")
    a, b = (BuzzCache(ls.buzz_config(wl, flags=FLAG_AUTO_EVICT | FLAG_DETERMINISTIC)) for _ in range(2))
    for c in (a, b):
        c.prefill(p["K"], p["V"], q_obs=p["q_obs"])
    out_a, out_b = (torch.empty(wl.batch, wl.n_q_heads, wl.head_dim, dtype=torch.float32, device="cuda") for _ in range(2))
    streams = [torch.cuda.Stream() for _ in range(8)]
    for t in range(wl.decode_steps):
        a.decode_step(d["q"][t], d["k"][t], d["v"][t], out_a)
        torch.cuda.synchronize()
        with torch.cuda.stream(streams[t % 8]):
            b.decode_step(d["q"][t], d["k"][t], d["v"][t], out_b)
        torch.cuda.synchronize()
        assert torch.isfinite(out_a).all(), t
        assert torch.equal(out_a, out_b), t
    for x, y in zip(a.export(), b.export()):
        assert torch.equal(x, y)
