"""Edges of the calls that a server makes around the 8-bit cache: what is refused, what is left alone, and what stays the same."""
import time

import numpy as np
import pytest
import torch

from tests.test_kv8_gpu import _B, _ctx

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------- set-up
def test_a_context_pays_for_profiling_only_when_it_is_asked_for():
    """Creating a context is cheaper than the first cod_profile_enable, which makes the events; records work as before."""
    _ctx()[0].close()
    made, enabled = [], []
    for _ in range(5):
        torch.cuda.synchronize()
        t = time.perf_counter()
        ctx, st, cfg = _ctx(W=1, n_pages=4)
        made.append(time.perf_counter() - t)
        assert ctx.profile_read("attn") == (0.0, 0)
        ctx.profile_enable(())
        t = time.perf_counter()
        ctx.profile_enable(("rowops",))
        enabled.append(time.perf_counter() - t)
        J = torch.zeros(1, 3, 2, 2, 128, dtype=torch.bfloat16, device="cuda")
        ctx.kv_append(J, torch.arange(3, dtype=torch.int32, device="cuda"), st)
        ms, n = ctx.profile_read("rowops")
        assert n == 1 and ms > 0
        ctx.profile_enable(())
        ctx.kv_append(J, torch.arange(3, dtype=torch.int32, device="cuda"), st)
        assert ctx.profile_read("rowops") == (0.0, 0)
        ctx.close()
    assert min(made) < min(enabled)
