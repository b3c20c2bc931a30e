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


# ----------------------------------------------------------------------------- rounds without pages
def _serve(kv8, mode, carry_rounds, starve, n_inputs=6, S=3, W=8):
    """Prompts, then one captured step (trim, reserve, round) replayed until every sequence has been through n_inputs windows. In the
    replays that `starve` names nothing is on the free list. Returns the state and what each window of each sequence gave."""
    B, H = _B(), H_()
    wl = small_bf16(S=S, W=W, n_layers=2, ctx=(1, 60), kv8=kv8, n_rounds=16, carry_rounds=carry_rounds)
    pair = H.Pair(wl, 4, fill_pool=False)
    sh, st, ctx = wl.shape, pair.st_g, pair.ctx
    st.block_table.fill_(-1)
    st.committed_len.zero_()
    pages, prompts = B.Pages(pair.cfg_g, S), [37, 0, 50]
    plan = B.RowPlan(S, sum(prompts))
    ctx.pages_reserve(pages, _i32(prompts), st, S, plan, advance=True)
    J = torch.from_numpy(np.random.default_rng(8).normal(size=(2, plan.max_rows, 2, sh.n_kv, 128))).to(torch.bfloat16).cuda()
    ctx.kv_append(J, plan.slot, st)
    room = torch.full((S,), W, dtype=torch.int32, device="cuda")
    inputs = [pair.round_inputs(r)[1] for r in range(n_inputs)]
    dev = {k: v.clone() for k, v in inputs[0].items()}

    def step():
        ctx.pages_release(pages, None, st, S)
        ctx.pages_reserve(pages, room, st, S)
        ctx.draft_round(dev["draft"], dev["target"], dev["H"], S, 1, mode, st, pair.split, pair.next_draft, pair.taps)

    tensors = [t for t in (st.kv_pool.view(torch.uint8), st.kv_scale, st.committed_len, st.carry_kv, st.carry_len, st.carry_hist, st.block_table,
                           pages.free_list, pages.n_free, pages.held) if t is not None]
    saved = [t.clone() for t in tensors]
    step()                                                     # warm-up, taken back
    for t, x in zip(tensors, saved):
        t.copy_(x)
    ctx.poll_status()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    at, gave, sat_out, r = [0] * S, [[] for _ in range(S)], 0, 0
    while min(at) < n_inputs:
        for k, v in dev.items():
            rows = v.shape[0] // S
            for s in range(S):
                v[s * rows:(s + 1) * rows] = inputs[min(at[s], n_inputs - 1)][k][s * rows:(s + 1) * rows]
        hog = []
        if r in starve:
            ctx.pages_release(pages, None, st, S)
            hog = pages.free_list[:int(pages.n_free)].tolist()
            pages.n_free.zero_()
        before = [t.clone() for t in (st.committed_len, st.carry_len, st.carry_kv)] + [st.carry_hist.clone() if st.carry_hist is not None else None]
        mine = [_rows_of(st, s) for s in range(S)]
        g.replay()
        torch.cuda.synchronize()
        flags, m, slots = ctx.poll_status(), pair.split.accept_len.tolist(), pair.split.carry_slot.view(S, W)
        want_flags = 0
        for s in range(S):
            if at[s] >= n_inputs:                              # (a sequence that is through goes on with its last window; it is not looked at)
                want_flags |= flags & (B.DEV_BAD_PAGE | B.DEV_NO_PAGES)
                continue
            if m[s] == 0:                                      # (with a forced first row a round that goes ahead accepts one at least)
                assert r in starve and (slots[s] == -1).all()
                sat_out += 1
                want_flags |= B.DEV_BAD_PAGE
                assert int(pair.split.bonus[s]) == int(dev["draft"][s, 0]) == int(pair.next_draft[s, 0])
                for x, y in zip((st.committed_len, st.carry_len), before):
                    assert torch.equal(x[s], y[s])
                assert torch.equal(st.carry_kv[:, s], before[2][:, s]) and (before[3] is None or torch.equal(st.carry_hist[s], before[3][s]))
                assert all(torch.equal(x, y) for x, y in zip(_rows_of(st, s), mine[s]))
                continue
            gave[s].append((m[s], int(pair.split.bonus[s]), int(st.committed_len[s]), int(st.carry_len[s]),
                            st.carry_kv[:, s, :, :, :int(st.carry_len[s])].clone(), pair.taps.x_final.view(S, W, -1)[s].cpu().numpy()))
            at[s] += 1
        assert flags & ~B.DEV_NO_PAGES == want_flags & ~B.DEV_NO_PAGES and (not want_flags or flags & B.DEV_NO_PAGES)
        if hog:                                                # the pages come back, below those that are free by now
            now = hog + pages.free_list[:int(pages.n_free)].tolist()
            pages.free_list[:len(now)] = _i32(now)
            pages.n_free.fill_(len(now))
        r += 1
        assert r < 40
    del g
    final = [_rows_of(st, s, gave[s][-1][2]) for s in range(S)]
    pair.close()
    return gave, final, sat_out


def _rows_of(st, s, L=None):
    """The bits of a sequence's committed rows, [Ld, n_kv, 2, L, hd], and its pages' scales."""
    L = int(st.committed_len[s]) if L is None else L
    ids = st.block_table[s, :(L + 15) // 16].long()
    bits = st.kv_pool.view(torch.uint8 if st.kv_scale is not None else torch.int16)[:, ids]        # [Ld, pages, n_kv, 2, 16, hd]
    rows = bits.permute(0, 2, 3, 1, 4, 5).flatten(3, 4)[:, :, :, :L]
    return rows.clone(), st.kv_scale[:, ids].clone() if st.kv_scale is not None else torch.zeros(0)


@pytest.mark.parametrize("kv8,mode,carry_rounds", [(True, 0, 1), (True, 0, 2), (True, 1, 1), (False, 0, 1)])
def test_a_sequence_without_pages_waits_and_goes_on_as_if_nothing_had_been(kv8, mode, carry_rounds):
    """The free list runs out inside the captured loop, then pages come back: the sequences that had to wait lose nothing."""
    from tests.helpers import rel_err
    gave, final, waited = _serve(kv8, mode, carry_rounds, starve=range(1, 6))
    want, end, none = _serve(kv8, mode, carry_rounds, starve=())
    assert waited >= 6 and none == 0
    for s in range(3):
        for i, (x, y) in enumerate(zip(gave[s][:6], want[s][:6])):
            assert x[:4] == y[:4] and torch.equal(x[4], y[4]), (s, i)
            assert rel_err(x[5], y[5]) < H_().TOL["bf16"], (s, i)
        L = want[s][5][2]
        assert gave[s][5][2] == L
        if kv8:                                                # whole pages: a sequence that was through first has gone on in its last one
            assert torch.equal(final[s][1][:, :L // 16], end[s][1][:, :L // 16])
            L = L // 16 * 16
        assert torch.equal(final[s][0][:, :, :, :L], end[s][0][:, :, :, :L])


def test_a_round_at_temperature_1_leaves_a_sequence_without_pages_alone():
    """The same in one eager round of the stochastic form and through the parts; a sequence beyond its table's end waits, too."""
    B, H = _B(), H_()
    wl = small_bf16(S=3, W=16, n_layers=1, ctx=(40, 60), kv8=True, n_rounds=4)
    pair = H.Pair(wl, 3, fill_pool=False)
    st, ctx, S, W = pair.st_g, pair.ctx, 3, 16
    rd, dev = pair.round_inputs(0)
    st.committed_len.copy_(_i32([47, 47, pair.cfg_g.max_pages_per_seq * 16 - 3]))
    st.block_table[1, 3:] = -1
    st.carry_len.fill_(5)
    ones, zeros = torch.ones((S, W), device="cuda"), torch.zeros((S, W), device="cuda")
    was = [t.clone() for t in (st.kv_pool.view(torch.uint8), st.kv_scale, st.carry_kv)]
    ctx.draft_round_stochastic(dev["target"], ones, ones, zeros, dev["H"], S, 1, B.COD_CARRY, st, pair.split, pair.next_draft, pair.taps)
    assert ctx.poll_status() == B.DEV_BAD_PAGE | B.DEV_PAGE_OVERFLOW
    assert pair.split.accept_len.tolist() == [16, 0, 0] and pair.split.bonus.tolist()[1:] == [-1, -1] == pair.next_draft[1:, 0].tolist()
    assert pair.split.acc_off.tolist() == [0, 16, 16, 16] and pair.split.rej_off.tolist() == [0, 0, 16, 32]
    assert pair.split.rej_rows.tolist() == list(range(16, 48)) + [-1] * 16 and pair.split.acc_rows.tolist() == list(range(16)) + [-1] * 32
    assert st.committed_len.tolist() == [63, 47, pair.cfg_g.max_pages_per_seq * 16 - 3] and st.carry_len.tolist() == [0, 5, 5]
    changed = [int(p) for p in (st.kv_scale != was[1]).flatten(2).any(-1).any(0).nonzero().flatten()]
    assert set(changed) <= set(st.block_table[0, :4].tolist()) and torch.equal(st.carry_kv, was[2])
    # by parts: rows 0 and 1 of a window that fits are accepted, the others carried
    draft = dev["draft"].clone()
    draft[:, 2] = (dev["target"][:, 2] + 1) % wl.shape.vocab
    draft[:, 1] = dev["target"][:, 1]
    ctx.verify_accept(draft, dev["target"], S, 1, st, pair.split)
    assert pair.split.accept_len.tolist() == [2, 0, 2] and pair.split.bonus[1] == draft[1, 0]
    J = torch.ones((1, S * W, 2, wl.shape.n_kv, 128), dtype=torch.bfloat16, device="cuda")
    ctx.scatter_kv(J, pair.split, S, B.COD_CARRY, st)
    assert st.committed_len.tolist() == [65, 47, pair.cfg_g.max_pages_per_seq * 16 - 1] and st.carry_len.tolist() == [14, 5, 14]
    assert torch.equal(st.carry_kv[:, 1], was[2][:, 1]) and ctx.poll_status() == B.DEV_BAD_PAGE
    pair.close()
