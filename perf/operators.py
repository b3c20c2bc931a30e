"""Cases and plain forms of the 8-bit KV cache's operators.

Three operators that a server of the drafter uses together:

* ``attn``: block attention over a committed cache held in 8 bits (e4m3) with one power-of-two scale for each page of
  16 tokens, KV head and K | V, followed by the carried rows and the block's own rows in the storage type.
* ``append``: rows of K and V quantised into that cache through a slot map. A page that already holds rows keeps them;
  its scale only grows, and then the rows it holds are rescaled.
* ``pages``: one scheduling step of the page tables: what a sequence reserved and does not need goes back to the free
  list, the next step's pages are taken from it, and every new row gets its slot, position and sequence.

``run`` computes them in elementary torch operations, or, with ``own`` set, calls the library.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
E4M3_MAX = 448.0
MIN_EXP = -100
THETA = 1.0e6


# ------------------------------------------------------------------------------------------------- cases
def _attn(name, S, W, n_q, n_kv, hd, lo, hi, carry, dtype="bf16"):
    return {"name": name, "op": "attn", "S": S, "W": W, "n_q": n_q, "n_kv": n_kv, "hd": hd, "ctx_lo": lo, "ctx_hi": hi,
            "carry": carry, "dtype": dtype}


def _append(name, S, n_kv, hd, layers, ctx_lo, ctx_hi, new_lo, new_hi, dtype="bf16"):
    return {"name": name, "op": "append", "S": S, "n_kv": n_kv, "hd": hd, "layers": layers, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "new_lo": new_lo, "new_hi": new_hi, "dtype": dtype}


def _pages(name, S, ctx_lo, ctx_hi, new_lo, new_hi):
    return {"name": name, "op": "pages", "S": S, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "new_lo": new_lo, "new_hi": new_hi}


def listed():
    return [
        # one token of one request: latency
        _attn("attn_token_b1", 1, 1, 32, 8, 128, 2048, 2048, False),
        # one token of each of 32 requests, ragged contexts: the bytes of the cache
        _attn("attn_token_b32", 32, 1, 32, 8, 128, 512, 8192, False),
        # a drafted block of 16 for one request, with the rows carried from its last round
        _attn("attn_block16_b1", 1, 16, 32, 8, 128, 2048, 2048, True),
        # the same at batch 32, ragged contexts: the drafting round's ordinary load
        _attn("attn_block16_b32", 32, 16, 32, 8, 128, 512, 8192, True),
        # block 32 over long contexts
        _attn("attn_block32_32k", 4, 32, 32, 8, 128, 32768, 32768, True),
        # float storage, head size 64, odd lengths that end inside a page
        _attn("attn_f32_small", 3, 8, 4, 2, 64, 5, 140, True, "f32"),
        # one token of each of 32 requests written to all five layers
        _append("append_token_b32", 32, 8, 128, 5, 512, 8192, 1, 1),
        # the accepted rows of a round at batch 32, and prompts of 64 requests
        _append("append_round_b32", 32, 8, 128, 5, 512, 8192, 1, 16),
        _append("append_prompts", 24, 8, 128, 5, 0, 0, 100, 2048),
        # a drafting round's reservation at batch 32: 16 rows more for each, the unused pages of the last round back
        _pages("pages_round_b32", 32, 512, 8192, 16, 16),
        # admission of 64 prompts
        _pages("pages_prompts_b64", 64, 0, 0, 100, 8192),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "append", "pages"])
    if op == "attn":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        hd = rng.choice([64, 128, 128])
        n_kv, rep, W = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 5, 8, 16, 32])
        while W * rep > 128:
            rep //= 2
        n_kv = max(n_kv, 128 // hd, 1)
        S = _log_int(rng, 1, 48)
        most = (16384 if dtype == "f32" else 140000) * 8 // (n_kv * S)
        hi = min(_log_int(rng, 1, 33000), max(1, most))
        lo = rng.randint(0, hi)
        return _attn("", S, W, n_kv * rep, n_kv, hd, lo, hi, rng.random() < 0.5, dtype) | {"name": "drawn"}
    if op == "append":
        hd, n_kv, layers = rng.choice([64, 128]), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 5])
        n_kv = max(n_kv, 128 // hd, 1)
        S = _log_int(rng, 1, 64)
        hi = min(_log_int(rng, 1, 2048), max(1, 24000 // S))
        ctx = rng.choice([0, _log_int(rng, 1, max(2, 60000 // S))])
        return _append("", S, n_kv, hd, layers, rng.randint(0, ctx), ctx, rng.randint(0, hi), hi,
                       rng.choice(["bf16", "bf16", "f32"])) | {"name": "drawn"}
    S = _log_int(rng, 1, 512)
    hi = min(_log_int(rng, 1, 8192), max(1, 262144 // S))
    ctx = min(_log_int(rng, 1, 8192), max(1, 262144 // S))
    return _pages("", S, rng.randint(0, ctx), ctx, rng.randint(0, hi), hi) | {"name": "drawn"}


# ------------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """Committed lengths, rows to come and carried rows of a case's sequences: part of the case, the same for every seed."""
    rng = np.random.default_rng([case["S"], case["ctx_hi"], case.get("new_hi", 0)])
    lens = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=case["S"])
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, size=case["S"]) if "new_hi" in case else np.zeros_like(lens)
    car = rng.integers(0, case["W"] + 1, size=case["S"]) if case.get("carry") else np.zeros_like(lens)
    new[-1] = case.get("new_hi", 0)                       # some sequence has the longest
    return lens.astype(np.int64), new.astype(np.int64), car.astype(np.int64)


def _pages_of(n):
    return (n + PAGE - 1) // PAGE


def _table(rng, lens, width, n_pages):
    """Distinct physical pages in a random order; entries past a sequence's pages hold -1."""
    order = rng.permutation(n_pages)
    table = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(_pages_of(lens)):
        table[s, :n] = order[at:at + n]
        at += n
    return table, order[at:].astype(np.int32)


def _exponent(amax):
    """The least e with amax <= 448 * 2^e (448 = 0.875 * 2^9), at least MIN_EXP."""
    m, k = torch.frexp(amax)
    e = torch.where(m <= 0.875, k - 9, k - 8)
    return torch.where(amax == 0, torch.full_like(e, MIN_EXP), e).clamp(min=MIN_EXP)


def _pow2(e, dtype=torch.float32):
    """2^e for whole e, exactly (a device's pow() may be an ulp off)."""
    table = torch.tensor([2.0 ** k for k in range(-126, 128)], dtype=dtype, device=e.device)
    return table[e.long() + 126]


def _random_pool(g, shape):
    """8-bit pages of normal rows, a few of their channels larger, with the scales that appending would give them."""
    Ld, n_pages, n_kv, _, _, hd = shape
    pool = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
    scale = torch.empty(shape[:4], dtype=torch.float32, device="cuda")
    gain = 1.0 + 3.0 * (torch.rand(n_kv, 2, 1, hd, generator=g, device="cuda") < 0.03).float()
    for l in range(Ld):
        for p0 in range(0, n_pages, 8192):
            n = min(8192, n_pages - p0)
            x = torch.randn(n, n_kv, 2, PAGE, hd, generator=g, device="cuda") * gain
            sc = _pow2(_exponent(x.abs().amax((-1, -2))))
            pool[l, p0:p0 + n] = (x / sc[..., None, None]).to(torch.float8_e4m3fn)
            scale[l, p0:p0 + n] = sc
    return pool, scale


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(device="cuda", dtype=dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng([seed, 11])
    lens, new, car = _lengths(case)
    S, op = case["S"], case["op"]
    td = torch.float32 if case.get("dtype") == "f32" else torch.bfloat16
    st = {"case": case}
    if op == "pages":
        # the state that the last step left: pages for the committed rows and for the rows reserved behind them
        full = lens + new
        width = int(_pages_of(full).max()) + 2
        n_pages = int(_pages_of(full).sum()) + 64
        table, free = _table(rng, full, width, n_pages)
        free_list = np.zeros(n_pages, dtype=np.int32)
        free_list[:len(free)] = free
        st |= {"table": _dev(table), "lens": _dev(lens), "carry_len": _dev(car), "new": _dev(new), "keep": _dev(lens),
               "free_list": _dev(free_list), "n_free": _dev(np.array([len(free)])), "held": _dev(_pages_of(full)),
               "rows": int(new.sum()) + 16}
        shape = dict(n_layers=1, n_q=1, n_kv=1, hd=64, W=16, dtype="bf16")
    else:
        Ld, n_kv, hd = case.get("layers", 1), case["n_kv"], case["hd"]
        full = lens + new
        width = max(1, int(_pages_of(full).max()) + 4)
        n_pages = int(_pages_of(full).sum()) + 4
        table, _ = _table(rng, full, width, n_pages)
        pool, scale = _random_pool(g, (Ld, n_pages, n_kv, 2, PAGE, hd))
        st |= {"pool": pool, "scale": scale, "table": _dev(table), "lens": _dev(lens)}
        if op == "attn":
            W, n_q = case["W"], case["n_q"]
            mk = lambda *sh: torch.randn(*sh, generator=g, device="cuda").to(td)  # noqa: E731
            st |= {"q": mk(S, W, n_q, hd), "kb": mk(S, W, n_kv, hd), "vb": mk(S, W, n_kv, hd),
                   "carry": mk(1, S, n_kv, 2, W, hd), "carry_len": _dev(car), "out": torch.empty(S, W, n_q, hd, dtype=td, device="cuda"),
                   "most": int(lens.max())}
            shape = dict(n_layers=1, n_q=n_q, n_kv=n_kv, hd=hd, W=W, dtype=case["dtype"])
        else:
            # rows of all sequences one behind the other, and eight more that go nowhere
            R = int(new.sum()) + 8
            slot = np.full(R, -1, dtype=np.int64)
            at = 0
            for s in range(S):
                pos = lens[s] + np.arange(new[s])
                slot[at:at + new[s]] = table[s, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE
                at += int(new[s])
            rows = torch.randn(Ld, R, 2, n_kv, hd, generator=g, device="cuda")
            rows *= torch.exp(0.5 * torch.randn(1, R, 1, 1, 1, generator=g, device="cuda"))
            st |= {"rows": rows.to(td), "slot": _dev(slot)}
            shape = dict(n_layers=Ld, n_q=n_kv, n_kv=n_kv, hd=hd, W=1, dtype=case["dtype"])
    if own:
        from paper_2609_14717_b200 import binding as B, synth
        sh = synth.DrafterShape(d_target=8, n_cap=1, d_model=shape["n_q"] * shape["hd"], vocab=64, rope_theta=THETA,
                                kv8=True, **shape)
        cfg = B.make_config(sh, S, width, n_pages)
        kept = prepare.__dict__.setdefault("contexts", {})            # a program makes a configuration's context once
        if bytes(cfg) not in kept:
            kept[bytes(cfg)] = B.Context(cfg)
        st["ctx"] = kept[bytes(cfg)]
        # the state over the tensors above; a pool that this operator does not touch is there in name only
        pool = st["pool"] if "pool" in st else torch.empty((), dtype=torch.float8_e4m3fn, device="cuda").expand(1, n_pages, 1, 2, PAGE, 64)
        scale = st["scale"] if "scale" in st else torch.empty((), device="cuda").expand(1, n_pages, 1, 2)
        own_state = B.State(cfg, sh.dtype, S, st["table"], st["lens"], kv_pool=pool, kv_scale=scale, carry_kv=st.get("carry"),
                            carry_len=st.get("carry_len"))
        st["state"] = own_state
        if op == "pages":
            st["pages"] = B.Pages(cfg, S, st["free_list"], st["n_free"], st["held"])
            st["plan"] = B.RowPlan(S, st["rows"])
    return st


# ------------------------------------------------------------------------------------------------- plain forms
def _rotate(x, pos):
    """Rotary embedding of x [S, W, heads, hd] at positions pos [S, W]; angles in 64 bits, the rest in 32."""
    half = x.shape[-1] // 2
    freq = THETA ** (-2.0 * torch.arange(half, dtype=torch.float64, device=x.device) / x.shape[-1])
    ang = pos.double()[..., None] * freq
    cos, sin = ang.cos().float()[:, :, None], ang.sin().float()[:, :, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _attn_plain(st):
    c = st["case"]
    S, W, n_kv, hd = c["S"], c["W"], c["n_kv"], c["hd"]
    rep = c["n_q"] // n_kv
    lens, table = st["lens"].long(), st["table"].long().clamp(min=0)
    n_pg = _pages_of(st["most"])
    pos = lens[:, None] + torch.arange(W, device="cuda")
    q = _rotate(st["q"].float(), pos).view(S, W, n_kv, rep, hd)
    kb = _rotate(st["kb"].float(), pos)
    pages = table[:, :n_pg]
    kv = st["pool"][0][pages].float() * st["scale"][0][pages][..., None, None]          # [S, pages, n_kv, 2, 16, hd]
    kv = kv.permute(0, 2, 3, 1, 4, 5).reshape(S, n_kv, 2, n_pg * PAGE, hd)
    blk = torch.stack([kb, st["vb"].float()], 2).permute(0, 3, 2, 1, 4)                 # [S, n_kv, 2, W, hd]
    kv = torch.cat([kv, st["carry"][0].float(), blk], 3)
    t = torch.arange(n_pg * PAGE, device="cuda")
    u = torch.arange(W, device="cuda")
    seen = torch.cat([t < lens[:, None], u < st["carry_len"].long()[:, None], (u >= 0).expand(S, W)], 1)
    kv = torch.where(seen[:, None, None, :, None], kv, torch.zeros((), device="cuda"))
    score = torch.einsum("swhgd,shtd->shgwt", q, kv[:, :, 0]) / math.sqrt(hd)
    score = torch.where(seen[:, None, None, None], score, torch.full((), -math.inf, device="cuda"))
    p = torch.exp(score - score.amax(-1, keepdim=True))
    o = torch.einsum("shgwt,shtd->swhgd", p, kv[:, :, 1]) / p.sum(-1).permute(0, 3, 1, 2)[..., None]
    return o.reshape(S, W, c["n_q"], hd).to(st["q"].dtype)


def _append_plain(st):
    pool, scale, slot = st["pool"], st["scale"], st["slot"].long()
    n_pages = pool.shape[1]
    live = (slot >= 0).nonzero().flatten()
    if live.numel() == 0:
        return {"pool": pool, "scale": scale}
    page, off = slot[live] // PAGE, slot[live] % PAGE
    x = st["rows"][:, live].float()                                                     # [Ld, n, 2, n_kv, hd]
    size = torch.where(x.isfinite(), x.abs(), torch.zeros_like(x)).amax(-1).transpose(2, 3)
    amax = torch.zeros(scale.shape, device="cuda").index_reduce_(1, page, size, "amax")
    first = torch.full((n_pages,), PAGE, device="cuda").scatter_reduce_(0, page, off, "amin")
    touched = torch.unique(page)
    old = scale[:, touched] * (first[touched] > 0)[None, :, None, None]
    grown = torch.maximum(old, _pow2(_exponent(amax[:, touched])))
    raw = pool.view(torch.uint8)
    body = pool[:, touched].float() * (old / grown)[..., None, None]
    stays = torch.arange(PAGE, device="cuda") < first[touched][:, None]
    raw[:, touched] = torch.where(stays[None, :, None, None, :, None], body.to(torch.float8_e4m3fn).view(torch.uint8), raw[:, touched])
    scale[:, touched] = grown
    y = (x / scale[:, page].transpose(2, 3)[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    raw[:, page, :, :, off] = y.view(torch.uint8).permute(1, 0, 3, 2, 4)
    return {"pool": pool, "scale": scale}


def _pages_plain(st):
    table, lens, held, n_free, free = st["table"], st["lens"], st["held"], st["n_free"], st["free_list"]
    width = table.shape[1]
    col = torch.arange(width, device="cuda")
    # back to the free list: what lies behind the kept rows. The first page freed ends up on top.
    keep = st["keep"].long()
    first = torch.minimum(_pages_of(keep), held.long())
    n = held.long() - first
    gone = (col >= first[:, None]) & (col < held.long()[:, None])
    rank = (n.cumsum(0) - n)[:, None] + col - first[:, None]
    top = n_free.long() + n.sum()
    free[(top - 1 - rank)[gone]] = table[gone]
    table[gone] = -1
    n_free.copy_(top)
    held.copy_(first)
    st["carry_len"][keep < lens] = 0
    lens.copy_(torch.minimum(lens.long(), keep))
    # the next step's pages, sequence by sequence from the top of the free list
    L, new = lens.long(), st["new"].long()
    need = (_pages_of(L + new) - held.long()).clamp(min=0)
    upto = need.cumsum(0)
    served = (need == 0) | (upto <= n_free.long())
    take = served[:, None] & (col >= held.long()[:, None]) & (col < (held.long() + need)[:, None])
    rank = (upto - need)[:, None] + col - held.long()[:, None]
    table[take] = free[(n_free.long() - 1 - rank)[take]]
    got = torch.where(served, need, torch.zeros_like(need))
    held.add_(got.to(torch.int32))
    n_free.sub_(got.sum().to(torch.int32))
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), new.cumsum(0)])
    r = torch.arange(st["rows"], device="cuda")
    s = torch.searchsorted(off[1:], r, right=True)
    live = s < len(L)
    s = s.clamp(max=len(L) - 1)
    pos = L[s] + r - off[s]
    slot = table[s, (pos // PAGE).clamp(max=width - 1)].long() * PAGE + pos % PAGE
    none = torch.full_like(r, -1)
    return {"table": table, "held": held, "n_free": n_free, "lens": lens, "row_off": off.int(),
            "slot": torch.where(live & served[s], slot, none).int(), "row_pos": torch.where(live, pos, none).int(),
            "row_seq": torch.where(live, s, none).int()}


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"attn": _attn_plain, "append": _append_plain, "pages": _pages_plain}[op](state)
    ctx, st, S = state["ctx"], state["state"], state["case"]["S"]
    if op == "attn":
        ctx.block_attn(0, state["q"], state["kb"], state["vb"], st, S, True, state["out"])
        return state["out"]
    if op == "append":
        ctx.kv_append(state["rows"], state["slot"], st)
        return {"pool": st.kv_pool, "scale": st.kv_scale}
    pages, plan = state["pages"], state["plan"]
    ctx.pages_release(pages, state["keep"], st, S)
    ctx.pages_reserve(pages, state["new"], st, S, plan)
    return {"table": st.block_table, "held": pages.held, "n_free": pages.n_free, "lens": st.committed_len,
            "row_off": plan.row_off, "slot": plan.slot, "row_pos": plan.row_pos, "row_seq": plan.row_seq}


# ------------------------------------------------------------------------------------------------- sizes, 64-bit forms
def work(case):
    """Bytes each read or written once, and the products' operations."""
    lens, new, car = _lengths(case)
    S = case["S"]
    if case["op"] == "pages":
        moved = int((_pages_of(lens + new) - _pages_of(lens)).sum())
        # a page that goes back and comes again: table read, list written, list read, table written; rows: three words
        return {"bytes": 4.0 * (moved * 4 + int(new.sum()) * 3 + S * 10 + 2), "flops": 0.0}
    es = 4 if case["dtype"] == "f32" else 2
    hd, n_kv = case["hd"], case["n_kv"]
    if case["op"] == "attn":
        W, n_q = case["W"], case["n_q"]
        keys = lens + car + W
        cache = int(lens.sum()) * n_kv * 2 * hd + int(_pages_of(lens).sum()) * (n_kv * 2 * 4 + 4)
        rest = es * hd * (int(car.sum()) * n_kv * 2 + S * W * (2 * n_q + 2 * n_kv))
        return {"bytes": float(cache + rest), "flops": 4.0 * int(keys.sum()) * W * n_q * hd}
    rows, Ld = int(new.sum()), case["layers"]
    return {"bytes": float(Ld * rows * 2 * n_kv * hd * (es + 1) + 4 * rows + 4 * Ld * int(new.astype(bool).sum()) * n_kv * 2), "flops": 0.0}


def _e4m3_round(x):
    """Nearest e4m3 value of float64 x, |x| <= 448, ties to even: a grid of 2^(e - 3) in the binade of 2^e, 2^-9 below 2^-6."""
    _, k = torch.frexp(x)
    step = _pow2((k - 1).clamp(min=-6) - 3, torch.float64)
    return torch.round(x / step) * step


def _attn_exact(case, seed):
    st = prepare(case, seed)
    S, W, n_kv, hd = case["S"], case["W"], case["n_kv"], case["hd"]
    rep = case["n_q"] // n_kv
    out = torch.empty(S, W, case["n_q"], hd, dtype=torch.float64, device="cuda")
    ang = THETA ** (-torch.arange(0, hd, 2, dtype=torch.float64, device="cuda") / hd)

    def turn(x, p):                         # x [W, heads, hd] as complex numbers (first half, second half)
        z = torch.complex(x[..., :hd // 2], x[..., hd // 2:]) * torch.polar(torch.ones_like(ang), p * ang)[:, None]
        return torch.cat([z.real, z.imag], -1)

    for s in range(S):
        L, c = int(st["lens"][s]), int(st["carry_len"][s])
        p = (L + torch.arange(W, device="cuda")).double()[:, None]
        q, kb = turn(st["q"][s].double(), p), turn(st["kb"][s].double(), p)
        ids = st["table"][s, :_pages_of(L)].long()
        kv = st["pool"][0].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() * st["scale"][0][ids].double()[..., None, None]
        for h in range(n_kv):
            k = torch.cat([kv[:, h, 0].reshape(-1, hd)[:L], st["carry"][0, s, h, 0, :c].double(), kb[:, h]])
            v = torch.cat([kv[:, h, 1].reshape(-1, hd)[:L], st["carry"][0, s, h, 1, :c].double(), st["vb"][s, :, h].double()])
            a = torch.softmax(q[:, h * rep:(h + 1) * rep].reshape(-1, hd) @ k.T * hd ** -0.5, -1) @ v
            out[s, :, h * rep:(h + 1) * rep] = a.view(W, rep, hd)
    return out


def _append_exact(case, seed):
    st = prepare(case, seed)
    slot = st["slot"].tolist()
    pool, scale = st["pool"].float().double(), st["scale"].double()
    r = 0
    while r < len(slot):
        if slot[r] < 0:
            r += 1
            continue
        pg, off = divmod(slot[r], PAGE)
        n = 1
        while r + n < len(slot) and slot[r + n] == slot[r] + n and off + n < PAGE:
            n += 1
        x = st["rows"][:, r:r + n].double().permute(0, 3, 2, 1, 4)                      # [Ld, n_kv, 2, n, hd]
        top = x.abs().amax((-1, -2)).clamp(min=2.0 ** -120)
        e = torch.ceil(torch.log2(top / E4M3_MAX) - 1e-9)                               # log2 may miss a whole number
        now = _pow2(torch.where(top > E4M3_MAX * _pow2(e, torch.float64), e + 1, e).clamp(min=MIN_EXP), torch.float64)
        if off:
            old = scale[:, pg].clone()
            now = torch.maximum(old, now)
            pool[:, pg, :, :, :off] = _e4m3_round(pool[:, pg, :, :, :off] * (old / now)[..., None, None])
        pool[:, pg, :, :, off:off + n] = _e4m3_round(x / now[..., None, None])
        scale[:, pg] = now
        r += n
    return {"pool": pool, "scale": scale}


def exact(case, seed):
    if case["op"] == "attn":
        return _attn_exact(case, seed)
    return _append_exact(case, seed) if case["op"] == "append" else None
