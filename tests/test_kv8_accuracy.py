"""Attention over the 8-bit cache against its error model: rows and carried shares within what the roundings explain, so that a
lost key, a wrong scale or a share that is not computed shows. The checks themselves are tested on the host."""
import numpy as np
import pytest
import torch

from tests import kv8_model as model
from tests import kv8_ref as ref


def _bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def _host_case(S=2, W=4, n_q=4, n_kv=2, hd=64, lens=(900, 33), seed=0):
    rng = np.random.default_rng(seed)
    n = [(L + 15) // 16 for L in lens]
    x = rng.normal(size=(sum(n), n_kv, 2, 16, hd)) * 2.0 ** rng.integers(-1, 2, size=(sum(n), n_kv, 2, 1, 1))
    scale = np.vectorize(ref.scale_for)(np.abs(x).max((-1, -2)))
    pool = ref.e4m3(x / scale[..., None, None])
    table = np.full((S, max(n) + 1), -1)
    order = rng.permutation(sum(n))
    for s in range(S):
        table[s, :n[s]] = order[sum(n[:s]):sum(n[:s + 1])]
    mk = lambda *sh: _bf16(rng.normal(size=sh))  # noqa: E731
    return dict(q=mk(S, W, n_q, hd), kb=mk(S, W, n_kv, hd), vb=mk(S, W, n_kv, hd), pool=pool, scale=scale, table=table, lens=list(lens),
                carry=mk(S, n_kv, 2, W, hd), carry_len=[W, 1], theta=1e6)


def test_the_model_accepts_what_rounded_arithmetic_gives():
    """Rotated q and block keys rounded to bf16, output to bf16."""
    for seed in range(3):
        c = _host_case(seed=seed)
        want = model.attend(**c)
        pos = (np.array(c["lens"])[:, None] + np.arange(4))[:, :, None]
        turn = lambda x: ref.rope(_bf16(ref.rope(x, pos, 1e6)), -pos, 1e6)  # noqa: E731
        got = model.attend(**(c | {"q": turn(c["q"]), "kb": turn(c["kb"])}))
        model.check(_bf16(got[0]), want[0], want[1], got[2], want[2], want[3])


@pytest.mark.parametrize("what", ["zero", "mass_zero", "mass_twice", "lost_key", "scale_k", "scale_v", "rows_swapped", "no_carry", "one_more_token"])
def test_the_checks_refuse_wrong_results(what):
    c = _host_case()
    want = model.attend(**c)
    out, mass = want[0], want[2]
    first = int(c["table"][0, 7])
    if what == "zero":
        out = 0 * out
    elif what == "mass_zero":
        mass = 0 * mass
    elif what == "mass_twice":
        mass = 2 * mass
    elif what == "lost_key":                                    # one of 900
        out = model.attend(**c, drop={(0, 0): 415})[0]
    elif what.startswith("scale"):                              # of one page of 57, one head
        c["scale"] = c["scale"].copy()
        c["scale"][first, 0, int(what == "scale_v")] *= 2
        out = model.attend(**c)[0]
    elif what == "rows_swapped":
        out = out[:, :, [1, 0, 2, 3]]
    elif what == "no_carry":
        out = model.attend(**(c | {"carry_len": [0, 0]}))[0]
    elif what == "one_more_token":
        out = model.attend(**(c | {"lens": [901, 33]}))[0]
    with pytest.raises(AssertionError):
        model.check(_bf16(out), want[0], want[1], mass, want[2], want[3])


# ----------------------------------------------------------------------------- the kernels
def _gpu():
    from tests import test_kv8_gpu
    return test_kv8_gpu


CASES = {
    "token": dict(S=4, W=1, n_q=8, n_kv=2, hd=128, lens=[0, 1, 17, 900], carry=False),
    "token_mqa": dict(S=2, W=1, n_q=16, n_kv=1, hd=128, lens=[1000, 77], carry=True),
    "rows8": dict(S=3, W=2, n_q=8, n_kv=2, hd=128, lens=[45, 1000, 16], carry=True),
    "rows9": dict(S=2, W=9, n_q=2, n_kv=2, hd=128, lens=[500, 31], carry=True),
    "block16": dict(S=3, W=16, n_q=8, n_kv=2, hd=128, lens=[0, 33, 1025], carry=True),
    "rows66": dict(S=2, W=22, n_q=6, n_kv=2, hd=128, lens=[400, 129], carry=True),
    "block32": dict(S=2, W=32, n_q=4, n_kv=1, hd=128, lens=[7, 1100], carry=True),
    "retained": dict(S=2, W=16, n_q=4, n_kv=1, hd=128, lens=[40, 300], carry=True, carry_rounds=4),
    "hd64_token": dict(S=3, W=1, n_q=8, n_kv=2, hd=64, lens=[0, 65, 700], carry=True),
    "hd64_block16": dict(S=2, W=16, n_q=8, n_kv=2, hd=64, lens=[160, 1025], carry=True),
    # row tiles in more than one pass over the keys, the last one not full
    "hd64_rows96": dict(S=2, W=24, n_q=8, n_kv=2, hd=64, lens=[130, 1025], carry=True),
    "hd64_rows100": dict(S=3, W=25, n_q=8, n_kv=2, hd=64, lens=[0, 47, 600], carry=True),
    "hd64_block32": dict(S=2, W=32, n_q=8, n_kv=2, hd=64, lens=[700, 16], carry=True),
}


def _run(case, flags=0, seed=1, **kw):
    T = _gpu()
    ctx, st, args, *_ = T._attn_case(**(CASES[case] if isinstance(case, str) else case), flags=flags, seed=seed)
    return ctx, st, args


def _compare(ctx, st, args):
    T = _gpu()
    layer, q, kb, vb, _, S, use, out, mass = args
    v = T._values
    ctx.block_attn(*args)
    lens, car = st.committed_len.tolist(), [c if use else 0 for c in st.carry_len.tolist()]
    want = model.attend(v(q), v(kb), v(vb), np.nan_to_num(v(st.kv_pool)[layer]), np.nan_to_num(v(st.kv_scale)[layer]), st.block_table.cpu().numpy(),
                        lens, np.nan_to_num(v(st.carry_kv)[layer]), car, 1e6)
    model.check(v(out), want[0], want[1], v(mass), want[2], want[3])


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [0, 2], ids=["", "plain_fma"])
@pytest.mark.parametrize("name", CASES)
def test_rows_are_as_near_as_their_roundings_allow(name, flags):
    ctx, st, args = _run(name, flags)
    _compare(ctx, st, args)
    assert ctx.poll_status() == 0
    ctx.close()


BAD = {
    "token": dict(S=3, W=1, n_q=8, n_kv=2, hd=128, lens=[500, 40, 17], carry=False),
    "rows8": dict(S=2, W=4, n_q=4, n_kv=2, hd=128, lens=[700, 129], carry=True),
    "block16": dict(S=3, W=16, n_q=8, n_kv=2, hd=128, lens=[900, 300, 130], carry=True),
    "block32": dict(S=2, W=32, n_q=4, n_kv=1, hd=128, lens=[600, 700], carry=True),
    "hd64": dict(S=2, W=16, n_q=8, n_kv=2, hd=64, lens=[300, 40], carry=True),
}


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [0, 2], ids=["", "plain_fma"])
@pytest.mark.parametrize("which", ["some", "last", "runs", "all"])
@pytest.mark.parametrize("name", BAD)
def test_keys_of_a_bad_page_do_not_count(name, which, flags):
    """The same in every kernel: whole pages, the last one, runs that fill tiles, all of them. Page 0, which belongs to somebody
    else, is not read in their place."""
    T = _gpu()
    ctx, st, args = _run(BAD[name], flags, seed=3)
    rng = np.random.default_rng(1)
    for s, L in enumerate(st.committed_len.tolist()):
        n = (L + 15) // 16
        at = {"some": rng.permutation(n)[:max(1, n // 3)], "last": [n - 1], "runs": [j for j in range(n) if j // 8 % 2 == s % 2], "all": range(n)}[which]
        for j in at:
            st.block_table[s, int(j)] = int(rng.choice([-1, 10 ** 6, st.kv_pool.shape[1], -2 ** 31]))
    _compare(ctx, st, args)
    assert ctx.poll_status() in ((T._B().DEV_BAD_PAGE,) if which != "runs" else (T._B().DEV_BAD_PAGE, 0))
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [0, 2], ids=["", "plain_fma"])
@pytest.mark.parametrize("W", [1, 16, 32])
def test_low_scores_behind_bad_pages_keep_their_weights(W, flags):
    """Tiles of bad pages first, then keys whose scores lie some 300 log2 units below zero: nothing but their differences counts."""
    ctx, st, args = _run(dict(S=1, W=W, n_q=4, n_kv=1, hd=128, lens=[1200], carry=False), flags, seed=5)
    q, kb = args[1], args[2]
    # a direction that the rotation leaves almost alone (the lowest frequencies): q has 36 there, the keys -16, block keys too
    q[..., 60:64] = 36.0
    kb[..., 60:64] = -16.0
    table = st.block_table[0].long()
    ids = table[:75]
    st.kv_scale[0, ids] = 1.0
    vals = st.kv_pool[0].float()
    vals[ids] = torch.from_numpy(np.random.default_rng(2).normal(size=tuple(vals[ids].shape))).float().cuda()
    vals[ids, :, 0, :, 60:64] = -16.0
    st.kv_pool[0] = vals.to(torch.float8_e4m3fn)
    st.block_table[0, :32] = -1
    _compare(ctx, st, args)
    ctx.close()


# ----------------------------------------------------------------------------- rows of one head group do not touch each other
MIXED = {
    "token": dict(S=2, W=1, n_q=8, n_kv=1, hd=128, lens=[700, 40], carry=True),
    "rows16": dict(S=2, W=4, n_q=8, n_kv=2, hd=128, lens=[700, 129], carry=True),
    "block16": dict(S=2, W=16, n_q=8, n_kv=2, hd=128, lens=[1025, 40], carry=True),
    "block32": dict(S=2, W=32, n_q=4, n_kv=1, hd=128, lens=[700, 300], carry=True),
    "hd64": dict(S=2, W=16, n_q=8, n_kv=2, hd=64, lens=[700, 40], carry=True),
}


def _compare_all_but(ctx, st, args, odd):
    """The rows for which `odd` [S, W, n_q] is false, against the model; returns the others."""
    T = _gpu()
    layer, q, kb, vb, _, S, use, out, mass = args
    v = T._values
    ctx.block_attn(*args)
    calm = np.where(odd[..., None], 0.0, v(q))
    want = model.attend(calm, v(kb), v(vb), np.nan_to_num(v(st.kv_pool)[layer]), np.nan_to_num(v(st.kv_scale)[layer]), st.block_table.cpu().numpy(),
                        st.committed_len.tolist(), np.nan_to_num(v(st.carry_kv)[layer]), st.carry_len.tolist(), 1e6)
    rest = ~odd
    model.check(v(out)[rest], want[0][rest], want[1][rest], v(mass)[rest], want[2][rest], want[3][rest])
    return v(out)[odd]


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [0, 2], ids=["", "plain_fma"])
@pytest.mark.parametrize("k", [10, 14, 18, 24, 40])
@pytest.mark.parametrize("name", MIXED)
def test_a_row_s_precision_does_not_depend_on_a_larger_one(name, k, flags):
    """One row per head group is 2^k larger than the others, the keys by as much larger as the others are smaller."""
    case = MIXED[name]
    ctx, st, args = _run(case, flags, seed=7)
    q, kb = args[1], args[2]
    odd = np.zeros(tuple(q.shape[:3]), bool)
    odd[:, case["W"] // 2, 1::case["n_q"] // case["n_kv"]] = True
    q[torch.from_numpy(~odd).cuda()] *= 2.0 ** -k
    kb *= 2.0 ** k
    st.carry_kv[:, :, :, 0] *= 2.0 ** k
    st.kv_scale[..., 0] *= 2.0 ** k
    _compare_all_but(ctx, st, args, odd)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [0, 2], ids=["", "plain_fma"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), 3e38])
@pytest.mark.parametrize("name", MIXED)
def test_a_row_that_is_not_finite_or_huge_leaves_the_others_alone(name, value, flags):
    case = MIXED[name]
    ctx, st, args = _run(case, flags, seed=8)
    odd = np.zeros(tuple(args[1].shape[:3]), bool)
    odd[0, case["W"] // 2, 1] = True
    args[1][0, case["W"] // 2, 1, 5] = value
    rows = _compare_all_but(ctx, st, args, odd)
    assert value == 3e38 or not np.isfinite(rows).any()          # what has no score has no output, in every kernel
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [0, 2], ids=["", "plain_fma"])
@pytest.mark.parametrize("k", [6, 10, 13, 16, 17, 18, 19, 20, 22, 26, 32, 40, 60])
@pytest.mark.parametrize("name", MIXED)
def test_outputs_of_huge_scores_stay_among_the_values(name, k, flags):
    """Scores of up to 2^60: the weights' differences are lost in their rounding, their sum is not. Every output lies between the
    least and the largest value of its column, but for the weights' and its own rounding, and a row whose largest score leads
    by far is that key's value."""
    T = _gpu()
    case = MIXED[name]
    ctx, st, args = _run(case, flags, seed=9)
    layer, q, kb, vb, _, S, use, out, mass = args
    args[2].mul_(2.0 ** k)
    st.carry_kv[:, :, :, 0] *= 2.0 ** k
    st.kv_scale[..., 0] *= 2.0 ** k
    ctx.block_attn(*args)
    v = T._values
    o, m = v(out), v(mass)
    assert np.isfinite(o).all() and (m >= 0).all() and (m <= 1 + 2.0 ** -10).all()
    rep, W, n_led = case["n_q"] // case["n_kv"], case["W"], 0
    pool, scale, car = np.nan_to_num(v(st.kv_pool)[0]), np.nan_to_num(v(st.kv_scale)[0]), np.nan_to_num(v(st.carry_kv)[0])
    for s in range(S):
        L, c = int(st.committed_len[s]), int(st.carry_len[s])
        ids = st.block_table[s, :(L + 15) // 16].cpu().numpy()
        pos = (L + np.arange(W))[:, None]
        qs, ks = ref.rope(v(q)[s], pos, 1e6), ref.rope(v(kb)[s], pos, 1e6)
        for h in range(case["n_kv"]):
            body = [(pool[ids, h, i] * scale[ids, h, i][:, None, None]).reshape(-1, case["hd"])[:L] for i in range(2)]
            keys = np.concatenate([body[0], car[s, h, 0, :c], ks[:, h]])
            vals = np.concatenate([body[1], car[s, h, 1, :c], v(vb)[s, :, h]])
            # f16 weights: each off by 2^-11, their sum of products by that of the largest |value|; then the output's own rounding
            slack = (2.0 ** -10 + 2.0 ** -8) * np.abs(vals).max(0)
            for g in range(h * rep, (h + 1) * rep):
                assert (o[s, :, g] >= vals.min(0) - slack).all() and (o[s, :, g] <= vals.max(0) + slack).all()
                sc = qs[:, g] @ keys.T / np.sqrt(case["hd"])
                room = 2 * 2.0 ** -7 * (np.abs(qs[:, g]) @ np.abs(keys).T).max(1) / np.sqrt(case["hd"]) + 40      # q's and the key's rounding at two keys
                best = sc.argmax(1)
                lead = sc.max(1) - np.partition(sc, -2, 1)[:, -2] if sc.shape[1] > 1 else np.full(W, np.inf)
                for i in np.nonzero(lead > room)[0]:
                    n_led += 1
                    assert (np.abs(o[s, i, g] - vals[best[i]]) <= slack).all()
    assert n_led > 0 or k < 10 or case["W"] > 1
    ctx.close()
