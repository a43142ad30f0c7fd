"""What tells a caller that an update could not be computed: the status word, and NaN in the result."""
import time

import pytest
import torch

import paper_2304_14698_b200 as xrl


def test_the_layers_status_word_is_the_calls(monkeypatch):
    from paper_2304_14698_b200 import binding
    seen = {}
    monkeypatch.setattr(binding, "xrl_orthogonalise", lambda *a, **k: seen.update(k))
    m = dict(T=13, S=8, H=64, K=2, L=2, Hm=32, Dg=1, dtype="fp32", A_max=8)
    status = torch.zeros(1, dtype=torch.int32)
    xrl.orthogonalise_layers(m, torch.zeros(50000), device_status=status)
    assert seen["device_status"] is status


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,side,steps", [(torch.bfloat16, 4096, 64), (torch.float32, 2048, 64)])
def test_a_word_that_is_set_while_a_call_runs_leaves_no_update(dtype, side, steps):
    """A wait that runs out sets the word between a call's first launch and its last.  Here a copy from the host does, behind a call
    that takes 7 ms or more, half a millisecond after it began (by a copy engine: no kernel would find room beside the products)."""
    g = torch.randn(side, side, device="cuda").to(dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    good = xrl.xrl_orthogonalise(g, steps=steps, device_status=status)
    code = torch.full((1,), 6, dtype=torch.int32).pin_memory()
    side_stream, out = torch.cuda.Stream(), torch.empty_like(g)
    torch.cuda.synchronize()
    assert int(status) == 0 and bool(torch.isfinite(good).all())
    for _ in range(5):                                            # (again if the host was held up for the whole call)
        for _ in range(6):
            xrl.xrl_orthogonalise(g, steps=steps)
        first, last = torch.cuda.Event(), torch.cuda.Event()
        first.record()
        xrl.xrl_orthogonalise(g, steps=steps, out=out, device_status=status)
        last.record()
        first.synchronize()                                       # the call's first launch is next: microseconds
        time.sleep(5e-4)
        with torch.cuda.stream(side_stream):
            status.copy_(code, non_blocking=True)
        side_stream.synchronize()
        in_time = not last.query()
        torch.cuda.synchronize()
        if in_time:
            break
    assert in_time
    assert int(status) == 6 and bool(torch.isnan(out).all())
    assert torch.equal(xrl.xrl_orthogonalise(g, steps=steps, out=out, device_status=status), good) and int(status) == 0
