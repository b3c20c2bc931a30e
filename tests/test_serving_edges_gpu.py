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


# ----------------------------------------------------------------------------- refusals
def test_scales_that_are_not_8_byte_aligned_are_refused():
    """Every call that reads a page's two scales as one word; nothing is launched."""
    B = _B()
    ctx, st, cfg = _ctx(S=2)
    whole = torch.zeros(st.kv_scale.numel() + 1, device="cuda")
    st.kv_scale = whole[1:].view(st.kv_scale.shape)
    assert st.kv_scale.data_ptr() % 8 == 4
    J = torch.ones(1, 8, 2, 2, 128, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(2, 4, 4, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 4, 2, 128, dtype=torch.bfloat16, device="cuda")
    i32 = torch.zeros(2, 5, dtype=torch.int32, device="cuda")
    n = ctx.launch_count()
    for call in (lambda: ctx.kv_append(J, i32[0].repeat(2)[:8].contiguous(), st),
                 lambda: ctx.block_attn(0, q, k, k, st, 2, True, torch.empty_like(q)),
                 lambda: ctx.scatter_kv(J, B.Split(2, 4), 2, B.COD_CARRY, st),
                 lambda: ctx.draft_round(i32[:, :4].contiguous(), i32, q, 2, 1, B.COD_CARRY, st, None, i32)):
        with pytest.raises(B.CodError, match="invalid"):
            call()
    assert ctx.launch_count() == n and not whole.any()
    ctx.close()
