"""Edges of the calls that a server makes around the 8-bit cache: what is refused, what is left alone, and what stays the same."""
import time

import numpy as np
import pytest
import torch

from tests import kv8_ref as ref
from tests.helpers import small_bf16
from tests.test_kv8_gpu import _B, _check_bytes, _ctx, _i32, _values

pytestmark = pytest.mark.gpu


def H_():
    from tests import gpu_harness
    return gpu_harness


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


# ----------------------------------------------------------------------------- page tables
def _held_state(S=4, width=6, n_pages=40, carry_rounds=2, lens=(20, 33, 5, 40)):
    """Four sequences with pages for their tokens and for a block behind them, and carried rows."""
    B = _B()
    ctx, st, cfg = _ctx(S=S, width=width, n_pages=n_pages, carry_rounds=carry_rounds)
    pages = B.Pages(cfg, S)
    t = ref.Tables(n_pages, S, width, [0] * S)
    ctx.pages_reserve(pages, _i32(lens), st, S, advance=True)
    t.reserve(lens, advance=True)
    ctx.pages_reserve(pages, _i32([16] * S), st, S)
    t.reserve([16] * S)
    st.carry_len.fill_(3)
    st.carry_hist.fill_(1)
    assert ctx.poll_status() == 0
    return ctx, st, cfg, pages, t


def _all_of(st, pages):
    return {k: v.clone() for k, v in (("table", st.block_table), ("lens", st.committed_len), ("carry_len", st.carry_len), ("hist", st.carry_hist),
                                      ("free", pages.free_list), ("n_free", pages.n_free), ("held", pages.held))}


@pytest.mark.parametrize("what", ["keep", "held_above", "held_below", "length"])
def test_release_leaves_a_sequence_with_bad_numbers_as_it_was(what):
    """The other sequences are served as ever; of the bad one nothing moves, and only pages that exist are on the free list."""
    B = _B()
    ctx, st, cfg, pages, t = _held_state()
    keep = [0, -1 if what == "keep" else 20, 5, 17]
    if what.startswith("held"):
        pages.held[1] = 99 if what == "held_above" else -2
    if what == "length":
        st.committed_len[1] = -7
    was = _all_of(st, pages)
    ctx.pages_release(pages, _i32(keep), st, 4)
    assert ctx.poll_status() == B.DEV_BAD_LEN
    now = _all_of(st, pages)
    for k in ("table", "lens", "carry_len", "hist", "held"):
        assert torch.equal(now[k][1], was[k][1]), k
    gone = []
    for s, first in ((0, 0), (2, 1), (3, 2)):
        gone += t.table[s][first:t.held[s]]
        assert now["table"][s].tolist() == t.table[s][:first] + [-1] * (6 - first) and now["held"][s] == first
    assert now["lens"].tolist() == [0, int(was["lens"][1]), 5, 17] and now["carry_len"].tolist() == [0, 3, 3, 0]
    assert now["hist"].tolist() == [[0, 0], [1, 1], [1, 1], [0, 0]]
    want = t.free + gone[::-1]
    assert int(now["n_free"]) == len(want) and now["free"][:len(want)].tolist() == want
    ctx.close()


def test_what_is_no_page_does_not_come_onto_the_free_list():
    """Table entries that were overwritten: reported, left out, and the list has no hole; its pages can be handed out again."""
    B = _B()
    ctx, st, cfg, pages, t = _held_state(S=4, width=40, n_pages=200, lens=(600, 33, 500, 40))
    rng = np.random.default_rng(3)
    for s, n in ((0, 5), (2, 30), (3, 1)):
        for j in rng.permutation(t.held[s])[:n]:
            t.table[s][j] = int(rng.choice([-1, -9, 200, 2 ** 31 - 1]))
    st.block_table.copy_(_i32(t.table))
    ctx.pages_release(pages, _i32([0, 33, 0, 0]), st, 4)
    assert ctx.poll_status() == B.DEV_BAD_PAGE
    gone = [p for s, first in ((0, 0), (1, 3), (2, 0), (3, 0)) for p in t.table[s][first:t.held[s]] if 0 <= p < 200]
    want = t.free + gone[::-1]
    assert int(pages.n_free) == len(want) == 200 - 3 - 36
    assert pages.free_list[:len(want)].tolist() == want and pages.held.tolist() == [0, 3, 0, 0]
    ctx.pages_release(pages, None, st, 4)                        # nothing is left over from the report
    assert ctx.poll_status() == 0 and int(pages.n_free) == len(want)
    ctx.pages_reserve(pages, _i32([0, 0, 600, 0]), st, 4)
    assert ctx.poll_status() == 0 and st.block_table[2, :38].tolist() == want[::-1][:38]
    ctx.close()


@pytest.mark.parametrize("n_free", [-1, 41])
def test_a_free_list_of_an_impossible_length_is_left_alone(n_free):
    B = _B()
    ctx, st, cfg, pages, t = _held_state()
    pages.n_free.fill_(n_free)
    was = _all_of(st, pages)
    ctx.pages_release(pages, _i32([0, 0, 0, 0]), st, 4)
    assert ctx.poll_status() == B.DEV_BAD_LEN
    ctx.pages_reserve(pages, _i32([40, 1, 1, 1]), st, 4, advance=False)
    assert ctx.poll_status() == B.DEV_BAD_LEN | B.DEV_NO_PAGES
    for k, v in _all_of(st, pages).items():
        assert torch.equal(v, was[k]), k
    ctx.close()


def test_a_request_that_ends_without_tokens_leaves_no_carried_rows():
    """keep = 0 ends a request at any length, 0 included; a release without keep does not, whatever the length."""
    ctx, st, cfg, pages, t = _held_state(lens=(0, 33, 0, 40))
    ctx.pages_release(pages, None, st, 4)
    assert st.carry_len.tolist() == [3, 3, 3, 3] and st.carry_hist.tolist() == [[1, 1]] * 4
    ctx.pages_release(pages, _i32([0, 33, 5, 0]), st, 4)
    assert st.committed_len.tolist() == [0, 33, 0, 0]
    assert st.carry_len.tolist() == [0, 3, 3, 0] and st.carry_hist.tolist() == [[0, 0], [1, 1], [1, 1], [0, 0]]
    assert ctx.poll_status() == 0
    ctx.close()


@pytest.mark.parametrize("carry_rounds", [1, 2])
def test_the_next_request_in_a_place_does_not_see_the_last_one_s_rows(carry_rounds):
    """An empty request whose window was rejected whole ends; a new one with the same window in its place drafts what a fresh
    state drafts."""
    B = _B()
    wl = small_bf16(S=2, W=8, n_layers=1, ctx=(0, 0), kv8=True, n_rounds=6, carry_rounds=carry_rounds)
    pair = H_().Pair(wl, 6, fill_pool=False)
    st, ctx = pair.st_g, pair.ctx
    pages = B.Pages(pair.cfg_g, 2)
    rd, dev = pair.round_inputs(0)
    other = dev["draft"].clone()
    other[:] = (dev["target"][:, :8] + 1) % wl.shape.vocab       # nothing is accepted
    fresh = [x.clone() for x in (st.kv_pool.view(torch.uint8), st.kv_scale, st.carry_kv)]

    def rounds():
        seen = []
        for draft in (other, dev["draft"]):
            ctx.pages_reserve(pages, _i32([8, 8]), st, 2)
            ctx.draft_round(draft, dev["target"], dev["H"], 2, 0, B.COD_CARRY, st, pair.split, pair.next_draft, pair.taps)
            ctx.pages_release(pages, None, st, 2)
            seen += [pair.taps.x_final.clone(), st.carry_len.clone()]
        return seen

    st.block_table.fill_(-1)
    st.committed_len.zero_()
    want = rounds()
    ctx.pages_release(pages, _i32([0, 0]), st, 2)
    ctx.pages_reserve(pages, _i32([8, 8]), st, 2)
    ctx.draft_round(other, dev["target"], dev["H"].flip(0).contiguous(), 2, 0, B.COD_CARRY, st, pair.split, pair.next_draft, pair.taps)
    assert st.committed_len.tolist() == [0, 0] and (st.carry_len == 8).all()
    ctx.pages_release(pages, _i32([0, 0]), st, 2)                # the request ends; the places are taken again
    for x, y in zip((st.kv_pool.view(torch.uint8), st.kv_scale, st.carry_kv), fresh):
        x.copy_(y)
    got = rounds()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert ctx.poll_status() == 0
    pair.close()
