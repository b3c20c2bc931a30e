"""Edges of the calls that a server makes around the 8-bit cache: what is refused, what is left alone, and what stays the same."""
import time

import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests.test_kv8_gpu import _B, _check_bytes, _ctx, _i32, _values

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------- set-up
def test_a_context_pays_for_profiling_only_when_it_is_asked_for():
    """The first cod_profile_enable makes the 8192 events (over a millisecond), the later ones and cod_create do not; records work as before."""
    first, again = [], []
    for _ in range(5):
        ctx, st, cfg = _ctx(W=1, n_pages=4)
        assert ctx.profile_read("attn") == (0.0, 0)
        ctx.profile_enable(())
        for spent in (first, again):
            t = time.perf_counter()
            ctx.profile_enable(("rowops",))
            spent.append(time.perf_counter() - t)
        J = torch.zeros(1, 3, 2, 2, 128, dtype=torch.bfloat16, device="cuda")
        ctx.kv_append(J, torch.arange(3, dtype=torch.int32, device="cuda"), st)
        ms, n = ctx.profile_read("rowops")
        assert n == 1 and ms > 0
        ctx.profile_enable(())
        ctx.kv_append(J, torch.arange(3, dtype=torch.int32, device="cuda"), st)
        assert ctx.profile_read("rowops") == (0.0, 0)
        ctx.close()
    assert min(first) > 10 * min(again)


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


def test_tensors_of_fewer_sequences_pages_or_rows_do_not_reach_the_device():
    B = _B()
    ctx, st, cfg = _ctx(S=4)
    pages, plan, n = B.Pages(cfg, 4), B.RowPlan(4, 16), torch.ones(4, dtype=torch.int32, device="cuda")
    short = _ctx(S=3)[1]
    count = ctx.launch_count()
    for args in ((B.Pages(cfg, 3), n, st, 4, plan), (pages, n, short, 4, plan), (pages, n, st, 4, B.RowPlan(3, 16)), (pages, n.cpu(), st, 4, plan)):
        with pytest.raises(ValueError):
            ctx.pages_reserve(*args)
    for args in ((B.Pages(cfg, 3), n, st, 4), (pages, None, short, 4)):
        with pytest.raises(ValueError):
            ctx.pages_release(*args)
    J, slot = torch.ones(1, 2, 2, 2, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    few = _ctx(S=4, n_pages=8)[1]
    with pytest.raises(ValueError):
        ctx.kv_append(J, slot, few)
    few.kv_pool = st.kv_pool
    with pytest.raises(ValueError):
        ctx.kv_append(J, slot, few)
    assert ctx.launch_count() == count
    ctx.pages_reserve(pages, n, st, 4, plan)                     # and what fits goes through
    assert ctx.poll_status() == 0 and plan.row_off.tolist() == [0, 1, 2, 3, 4]
    ctx.close()


# ----------------------------------------------------------------------------- append
@pytest.mark.parametrize("layers,dtype", [(1, "bf16"), (3, "f32")])
@pytest.mark.parametrize("case", ["hole", "hole_later", "backwards", "start_again", "wide_hole", "far", "farther", "fine"])
def test_append_skips_what_follows_a_hole_in_its_own_page(case, layers, dtype):
    """Rows that go nowhere between two rows of one page: the second part would be a second owner of the page. It is skipped and
    reported; the rest of the map, and the page's first part, are stored as if it were not there."""
    B = _B()
    n = {"far": 300, "farther": 6000, "wide_hole": 33}.get(case, 2)
    one = {"hole": [18, -1, 19], "hole_later": [16, 17, 18, 19, -1, -7, 22, 23], "backwards": [21, -1, 17, 18], "start_again": [21, 22, -1, 16, 17],
           "fine": [18, 19, 20, -1, 48, 49, -1, -1, 33, 34]}.get(case, [18] + [-1] * n + [25, 26])
    keep = {"hole": 1, "hole_later": 6, "backwards": 1, "start_again": 2, "fine": 10}.get(case, 1)
    rng = np.random.default_rng(len(one))
    for lead in (0, 1, 3, 15, 40):                             # where the break lies in the blocks' chunks of rows
        head = list(range(64 + 9, 64 + 9 + lead)) if lead < 40 else list(range(64, 64 + lead))
        bad = head + one + [112, 113, -1, 128]
        good = list(head) + one[:keep] + [-1] * (len(one) - keep) + [112, 113, -1, 128]
        ctx, st, _ = _ctx(S=1, W=1, n_q=2, n_kv=2, hd=64, layers=layers, n_pages=12, dtype=dtype)
        st.kv_pool.view(torch.uint8).copy_(torch.from_numpy(rng.integers(0, 0x7F, size=tuple(st.kv_pool.shape), dtype=np.uint8)))
        st.kv_scale.copy_(torch.from_numpy(2.0 ** rng.integers(-6, 1, size=tuple(st.kv_scale.shape)).astype(np.float64)))
        J = torch.from_numpy(rng.normal(size=(layers, len(bad), 2, 2, 64))).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
        pool, scale = _values(st.kv_pool), _values(st.kv_scale)
        ctx.kv_append(J, _i32(bad), st)
        ref.append(pool, scale, _values(J), np.array(good))
        _check_bytes(st, pool, scale)
        assert ctx.poll_status() == (0 if case == "fine" else B.DEV_BAD_SLOT)
        ctx.close()
